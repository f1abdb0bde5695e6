"""HiF4 grouped products with rows behind the last group: what the plan of a batch with dropped assignments gives."""
import pytest
import torch

from tests.test_gpu_experts import gen, hif4  # noqa: F401  (hif4: fixture)

pytestmark = pytest.mark.gpu

COUNTS = [[0, 0, 0], [1, 0, 2], [40, 0, 129, 1, 300], [5] * 40, [600, 1, 64, 65], [0, 17, 31, 32, 33], [256, 512, 0]]


@pytest.fixture(params=["default", "single", "simt", "noalloc"])
def product(request, hif4):  # noqa: F811
    """Each kernel that a grouped product may come from."""
    path = {"single": 2, "simt": 1}.get(request.param, 0)
    hif4.lib.hif4_debug_set_gemm_path(path)
    yield (lambda a, b, off, out: hif4.hif4_grouped_gemm_noalloc(a, b, off, out)) if request.param == "noalloc" else \
        (lambda a, b, off, out: hif4.hif4_grouped_gemm(a, b, off, out=out))
    hif4.lib.hif4_debug_set_gemm_path(0)


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("N,K", [(130, 256), (512, 2816), (100, 192), (64, 64)])
@pytest.mark.parametrize("behind", [1, 19, 300])
def test_rows_behind_the_last_group(hif4, product, counts, N, K, behind):  # noqa: F811
    g = gen(sum(counts) + N + K)
    G, used = len(counts), sum(counts)
    a = hif4.hif4_quantize(torch.randn(used + behind, K, generator=g, device="cuda"))
    b = hif4.hif4_quantize(torch.randn(G * N, K, generator=g, device="cuda")).view(G, N, K // 64, 36)
    a[used:] = 255                                          # NaN units, which no group reads into its rows
    off = torch.tensor([0] + counts, device="cuda").cumsum(0)
    A, B = hif4.hif4_dequantize(a[:used], torch.float32).double(), hif4.hif4_dequantize(b.view(G * N, K // 64, 36), torch.float32).double().view(G, N, K)
    c = torch.full((used + behind, N + 3), 9.0, device="cuda")[:, :N]
    whole = c._base
    product(a, b, off, c)
    for n in range(G):
        x = A[off[n]:off[n + 1]]
        want, size = x @ B[n].t(), x.abs() @ B[n].abs().t()
        assert bool(((c[off[n]:off[n + 1]].double() - want).abs() <= 1e-5 * size + 1e-300).all())
    assert bool((whole[used:] == 9.0).all()) and bool((whole[:, N:] == 9.0).all())
    assert hif4.hif4_last_device_status() == 0


def test_products_of_no_terms(hif4, product):  # noqa: F811
    """K = 0: rows of the groups become zeros, those behind stay."""
    off = torch.tensor([0, 3, 3, 8], device="cuda")
    a, b = torch.empty(12, 0, 36, dtype=torch.uint8, device="cuda"), torch.empty(3, 70, 0, 36, dtype=torch.uint8, device="cuda")
    c = torch.full((12, 70), 9.0, device="cuda")
    product(a, b, off, c)
    assert bool((c[:8] == 0.0).all()) and bool((c[8:] == 9.0).all())


@pytest.mark.parametrize("N,K", [(130, 256), (512, 2816), (100, 192)])
@pytest.mark.parametrize("cap", [1, 100, 257, 599])
def test_fewer_rows_than_assignments(hif4, product, N, K, cap):  # noqa: F811
    """Rows up to a capacity: assignments past it have no row, and the offsets that count them reach no memory behind the rows."""
    g = gen(N + cap)
    G, T, k = 7, 300, 2
    x = torch.randn(T, K, generator=g, device="cuda").to(torch.bfloat16)
    b = hif4.hif4_quantize(torch.randn(G * N, K, generator=g, device="cuda")).view(G, N, K // 64, 36)
    off, row_of = hif4.hif4_expert_plan(torch.randint(0, G, (T, k), generator=g, device="cuda", dtype=torch.int32), G)
    pool = torch.full((cap + 300, K // 64, 36), 255, dtype=torch.uint8, device="cuda")          # NaN units behind the rows
    a = hif4.hif4_dispatch(x, row_of, fmt=hif4.HIF4_FMT_HIF4, out=pool[:cap])
    A, B = hif4.hif4_dequantize(a, torch.float32).double(), hif4.hif4_dequantize(b.view(G * N, K // 64, 36), torch.float32).double().view(G, N, K)
    c = torch.full((cap + 300, N), 9.0, device="cuda")
    for offsets in (off, torch.cat([torch.tensor([-5], device="cuda"), off[1:-1], torch.tensor([2 ** 40], device="cuda")])):
        c.fill_(9.0)
        product(a, b, offsets, c[:cap])
        for n in range(G):
            rows = slice(min(cap, int(off[n])), min(cap, int(off[n + 1])))
            want, size = A[rows] @ B[n].t(), A[rows].abs() @ B[n].abs().t()
            assert bool(((c[rows].double() - want).abs() <= 1e-5 * size + 1e-300).all())
        assert bool((c[cap:] == 9.0).all())
    assert hif4.hif4_last_device_status() == 0


def layer(hif4, x, logits, up, down, k, E, N):  # noqa: F811
    """Routing, HiF4 rows, two grouped products around an activation, their sum: nothing is read back."""
    ids, w = hif4.hif4_route(logits, k)
    off, row_of = hif4.hif4_expert_plan(ids, E)
    h = hif4.hif4_grouped_gemm(hif4.hif4_dispatch(x, row_of, fmt=hif4.HIF4_FMT_HIF4), up, off)
    a = hif4.hif4_quantize((torch.nn.functional.silu(h[:, :N]) * h[:, N:]).to(torch.bfloat16))
    return hif4.hif4_combine(hif4.hif4_grouped_gemm(a, down, off), row_of, w, residual=x, dtype=torch.bfloat16), ids, w, off, row_of, h, a


@pytest.mark.parametrize("T,E,k,K,N", [(1, 8, 2, 256, 128), (20, 12, 3, 256, 128), (300, 16, 4, 512, 256), (64, 40, 6, 192, 192)])
def test_a_layer_with_padded_tokens(hif4, T, E, k, K, N):  # noqa: F811
    """Padded tokens (no expert left by the mask) have no row; each product against 64 bits on its operands, eager and captured."""
    g = gen(T + E)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)      # noqa: E731
    x, logits = rnd(T, K), torch.randn(T, E, generator=g, device="cuda")
    up, down = hif4.hif4_quantize(rnd(E * 2 * N, K) / 16), hif4.hif4_quantize(rnd(E * K, N) / 8)
    U, D = hif4.hif4_dequantize(up, torch.float32).double().view(E, 2 * N, K), hif4.hif4_dequantize(down, torch.float32).double().view(E, K, N)
    up, down = up.view(E, 2 * N, K // 64, 36), down.view(E, K, N // 64, 36)

    def check(padded, y, ids, w, off, row_of, h, a):
        there = ids >= 0
        assert int(off[-1]) == int(there.sum()) and bool((row_of[padded] == -1).all()) and bool(there[~padded].all())
        X = hif4.hif4_dequantize(hif4.hif4_quantize(x), torch.float32).double()
        at, row = ids.long().clamp(min=0), row_of.long().clamp(min=0)
        want, size = torch.einsum("tkno,to->tkn", U[at], X), torch.einsum("tkno,to->tkn", U[at].abs(), X.abs())
        assert bool((((h[row].double() - want).abs() <= 1e-5 * size) | ~there.unsqueeze(-1)).all())
        A = hif4.hif4_dequantize(a, torch.float32).double()[row]
        A = torch.where(there.unsqueeze(-1), A, 0.0)
        W = torch.where(there, w, 0.0).double().unsqueeze(-1)
        want = x.double() + (W * torch.einsum("tkon,tkn->tko", D[at], A)).sum(1)
        size = x.double().abs() + (W * torch.einsum("tkon,tkn->tko", D[at].abs(), A.abs())).sum(1)
        # FP32 sums of a product: 1e-5 of its terms; k + 1 multiply-adds behind them add 7 x 2^-24; one rounding to BF16
        assert bool(((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.1e-5 * size).all())
        assert torch.equal(y[padded], x[padded])

    padded = torch.arange(T, device="cuda") % 3 == 1
    logits[padded] = float("-inf")
    check(padded, *layer(hif4, x, logits, up, down, k, E, N))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(hif4, x, logits, up, down, k, E, N)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = layer(hif4, x, logits, up, down, k, E, N)
    torch.cuda.current_stream().wait_stream(side)
    x.copy_(rnd(T, K))
    logits.copy_(torch.randn(T, E, generator=g, device="cuda"))
    padded = torch.arange(T, device="cuda") % 4 == 0
    logits[padded] = float("-inf")
    for t in out:
        t.fill_(3)
    graph.replay()
    check(padded, *out)
