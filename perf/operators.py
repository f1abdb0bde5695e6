"""The operators around the HiF4 linear layer of a transformer block, as measurable cases.

  norm / norm_grad      norms after and before a block with gate, residual and residual scale
  linear / linear_grad  HiF4 product with bias, activation and residual
  gated / gated_grad    gated feed-forward: two HiF4 projections, activation, product
  block                 norm -> gated feed-forward -> down projection with residual, as a served block runs them

`run` computes a case with elementary torch operations in 32 bits (`own` false) or with this package's calls (`own`
true); `exact` computes it in 64 bits from the definitions.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a served model: the norm in front of a block, latency only
        dict(name="norm one token", op="norm", M=1, K=4096, dtype="bf16", post="none", pre="rms", gate=0, scale=1.0),
        # a prompt through a block with norms on both sides and a gate per sequence
        dict(name="norm prompt", op="norm", M=8192, K=5120, dtype="bf16", post="rms", pre="rms", gate=2048, scale=0.5),
        # rows and width that fill no tile; layer norm in FP16
        dict(name="norm ragged", op="norm", M=777, K=1000, dtype="fp16", post="none", pre="layer", gate=1, scale=1.0),
        # training step of both norms' weights and the gates of four sequences
        dict(name="norm gradient", op="norm_grad", M=4000, K=4096, dtype="bf16", post="rms", pre="rms", gate=1000, scale=1.0),
        # attention output projection of one token with its residual
        dict(name="linear one token", op="linear", M=1, N=4096, K=4096, dtype="bf16", act="none", bias=False, residual=True),
        # down projection of a prompt with its residual
        dict(name="linear prompt", op="linear", M=4096, N=4096, K=14336, dtype="bf16", act="none", bias=False, residual=True),
        # a projection with bias and activation for a few sequences, sizes that fill no tile
        dict(name="linear ragged", op="linear", M=77, N=1001, K=1024, dtype="fp16", act="gelu", bias=True, residual=False),
        # an adapter's training step through a frozen projection
        dict(name="linear gradient", op="linear_grad", M=2048, N=4096, K=4096, dtype="bf16", act="gelu_tanh", bias=True, residual=False),
        # gated feed-forward of one token
        dict(name="gated one token", op="gated", M=1, N=14336, K=4096, dtype="bf16", act="silu", bias=False),
        # of a prompt, the largest product of the layer
        dict(name="gated prompt", op="gated", M=4096, N=14336, K=4096, dtype="bf16", act="silu", bias=False),
        # its gradient with respect to the activations
        dict(name="gated gradient", op="gated_grad", M=1024, N=14336, K=4096, dtype="bf16", act="silu", bias=False),
        # the feed-forward block of a small decoding batch, norm to residual
        dict(name="block of 8 tokens", op="block", M=8, N=14336, K=4096, dtype="bf16", act="silu", bias=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "linear", "linear", "linear_grad", "gated", "gated", "gated_grad", "block"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("norm", "norm_grad"):
        rows = _log_int(rng, 1, 8192)
        width = _log_int(rng, 128, 8192) if rng.random() < 0.25 else 64 * _log_int(rng, 2, 128)
        while rows * width > (8192 * 5120 if op == "norm" else 4096 * 4096):
            rows = max(1, rows // 2)
        gate = rng.choice([0, 0, 1, max(1, rows // 4), rows])
        return dict(op=op, M=rows, K=width, dtype=dtype, post=rng.choice(["none", "rms", "layer"]),
                    pre=rng.choice(["rms", "layer"]), gate=gate, scale=rng.choice([1.0, 0.5, 0.25]))
    act = rng.choice(["silu", "gelu", "gelu_tanh", "relu"])
    # contraction and width: mostly multiples of 256 and 64 as layers have them, odd widths among them
    K = 256 * _log_int(rng, 1, 56) if rng.random() < 0.8 else 64 * _log_int(rng, 1, 200)
    N = 64 * _log_int(rng, 1, 224) if rng.random() < 0.7 else _log_int(rng, 8, 14336)
    M = _log_int(rng, 1, 4096)
    limit = {"linear": 4096 * 4096 * 14336, "linear_grad": 2048 * 4096 * 4096, "gated": 4096 * 14336 * 4096,
             "gated_grad": 1024 * 14336 * 4096, "block": 1024 * 14336 * 4096}[op]
    while M * N * K > limit:
        M = max(1, M // 2)
    case = dict(op=op, M=M, N=N, K=K, dtype=dtype, act=act, bias=rng.random() < 0.5)
    if op == "linear":
        case.update(act=rng.choice(["none", act]), residual=rng.random() < 0.5)
    if op == "linear_grad":
        case.update(residual=False)
    if op in ("linear_grad", "gated_grad"):
        case.update(dtype=rng.choice(["bf16", "bf16", "fp16"]))
    if op == "block":
        case.update(N=max(64, N // 64 * 64), dtype="bf16")
    return case


def work(case):
    M, K = case["M"], case["K"]
    e = 4 if case["dtype"] == "fp32" else 2
    op = case["op"]
    if op == "norm":                                  # x, residual in; h, y out; gates and weights
        gates = -(-M // case["gate"]) if case["gate"] else 0
        return {"bytes": 4 * e * M * K + e * K * (1 + (case["post"] != "none") + gates), "flops": 16 * M * K}
    if op == "norm_grad":                             # dy, dh, h, x in; dx, dresidual out
        return {"bytes": 6 * e * M * K, "flops": 30 * M * K}
    N = case["N"]
    w = N * K * 36 // 64
    if op == "linear":
        return {"bytes": w + e * (M * K + M * N * (2 if case["residual"] else 1)), "flops": 2 * M * N * K}
    if op == "linear_grad":
        return {"bytes": w + e * (2 * M * K + M * N), "flops": 4 * M * N * K}
    if op == "gated":
        return {"bytes": 2 * w + e * (M * K + M * N), "flops": 4 * M * N * K}
    if op == "gated_grad":
        return {"bytes": 2 * w + e * (2 * M * K + M * N), "flops": 8 * M * N * K}
    return {"bytes": 3 * w + e * 4 * M * K, "flops": 6 * M * N * K}


# ------------------------------------------------------------------------------------------------------------- inputs
def _activations(rows, cols, g, dtype):
    """Heavy-tailed activations with a few outlier channels, as hidden states have them."""
    z = torch.randn(rows, cols, generator=g, device="cuda")
    z *= torch.rsqrt(torch.rand(rows, cols, generator=g, device="cuda") + 0.05)
    z[:, torch.randperm(cols, generator=g, device="cuda")[: max(1, cols // 200)]] *= 20.0
    return z.to(dtype)


def _weight_units(rows, cols, g):
    """HiF4 units [rows, cols / 64, 36] of a Gaussian weight matrix, in slabs (the weights that a program loads)."""
    out = torch.empty(rows, cols // 64, 36, dtype=torch.uint8, device="cuda")
    slab = max(1, (1 << 24) // cols)
    for r in range(0, rows, slab):
        n = min(slab, rows - r)
        w = (torch.randn(n, cols, generator=g, device="cuda") / math.sqrt(cols)).to(torch.bfloat16)
        byte, e8, e16, code, sign = _encode(w)
        code = (code | (sign << 3)).view(n, cols // 64, 32, 2)
        out[r:r + n, :, 4:] = (code[..., 0] | (code[..., 1] << 4)).to(torch.uint8)
        out[r:r + n, :, 0] = byte.to(torch.uint8)
        out[r:r + n, :, 1] = (e8 << torch.arange(8, device="cuda", dtype=torch.int32)).sum(-1).to(torch.uint8)
        bits = (e16.view(n, cols // 64, 2, 8) << torch.arange(8, device="cuda", dtype=torch.int32)).sum(-1)
        out[r:r + n, :, 2:4] = bits.to(torch.uint8)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt, M, K, op = DTYPES[case["dtype"]], case["M"], case["K"], case["op"]
    s = {"case": dict(case)}

    def vector(n, mean, std):
        return (torch.randn(n, generator=g, device="cuda") * std + mean).to(dt)

    def gradient(rows, cols):
        return (torch.randn(rows, cols, generator=g, device="cuda") * 0.1).to(dt)

    if op in ("norm", "norm_grad"):
        s["x"] = _activations(M, K, g, dt)
        s["w"] = vector(K, 1.0, 0.2)
        s["b"] = vector(K, 0.0, 0.2) if case["pre"] == "layer" else None
        s["wp"] = vector(K, 1.0, 0.2) if case["post"] != "none" else None
        s["gate"] = None
        if case["gate"]:
            s["gate"] = torch.rand(-(-M // case["gate"]), K, generator=g, device="cuda").to(dt)
        if op == "norm":
            s["r"] = _activations(M, K, g, dt)
        else:
            s["h"], s["dy"], s["dh"] = _activations(M, K, g, dt), gradient(M, K), gradient(M, K)
        return s
    N = case["N"]
    s["x"] = _activations(M, K, g, dt)
    if op == "block":
        s["r"], s["w"] = _activations(M, K, g, dt), vector(K, 1.0, 0.2)
    s["wg"] = _weight_units(N, K, g)
    s["bg"] = vector(N, 0.0, 0.5) if case["bias"] else None
    if op in ("gated", "gated_grad", "block"):
        s["wu"] = _weight_units(N, K, g)
        s["bu"] = vector(N, 0.0, 0.5) if case["bias"] else None
    if op == "block":
        s["wd"] = _weight_units(K, N, g)
    if op == "linear":
        s["r"] = _activations(M, N, g, dt) if case["residual"] else None
    if op in ("linear_grad", "gated_grad"):
        s["dy"] = gradient(M, N)
    return s


# --------------------------------------------------------------------------------------------------------- plain form
def _encode(x):
    """HiF4 units of x [rows, cols]: scale bytes [rows, units], level-2 and level-3 micro-exponents [.., 8] and [.., 16],
    magnitudes and signs [.., 64], by Algorithm 1 in the arithmetic of x (BF16, or FP32 for FP16 and FP32)."""
    wide = torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float32
    v = x.to(wide).view(x.shape[0], -1, 64)
    a = v.abs()
    seventh = torch.full((), 1.0 / 7.0, dtype=torch.float32, device=x.device).to(wide)
    sf = (a.amax(-1) * seventh).float().clamp(2.0 ** -48, 2.0 ** 15 * 1.5)
    bits = sf.view(torch.int32)
    byte = (((bits + 0xFFFFF + ((bits >> 21) & 1)) >> 21) - ((127 - 48) << 2)).clamp(0, 0xFE)
    table = torch.tensor([1.0, 0.8, 2.0 / 3.0, 4.0 / 7.0], device=x.device)
    rec = (table[(byte & 3).long()] * torch.exp2(48.0 - (byte >> 2).float())).to(wide)
    t = a * rec.unsqueeze(-1)
    e8 = (t.view(*t.shape[:2], 8, 8).amax(-1) >= 4.0).int()
    e16 = (t.view(*t.shape[:2], 16, 4).amax(-1) >= torch.exp2(1.0 + e8.repeat_interleave(2, -1).float())).int()
    shift = (e8.repeat_interleave(2, -1) + e16).repeat_interleave(4, -1)
    code = torch.round(t.float() * torch.exp2(2.0 - shift.float())).clamp(max=7.0).int()
    return byte.int(), e8, e16, code, torch.signbit(v).int()


def _scales(byte):
    return torch.exp2((byte >> 2).float() - 48.0) * (1.0 + (byte & 3).float() * 0.25)


def _through_units(x):
    """x converted to HiF4 and back, FP32."""
    byte, e8, e16, code, sign = _encode(x)
    shift = (e8.repeat_interleave(2, -1) + e16).repeat_interleave(4, -1)
    v = code.float() * torch.exp2(shift.float() - 2.0) * _scales(byte).unsqueeze(-1) * (1.0 - 2.0 * sign.float())
    return v.view(x.shape)


def _decode(units):
    """FP32 values of packed units [rows, n, 36]."""
    u = units.int()
    at = torch.arange(8, device=u.device, dtype=torch.int32)
    e8 = (u[..., 1:2] >> at) & 1
    e16 = torch.cat([(u[..., 2:3] >> at) & 1, (u[..., 3:4] >> at) & 1], -1)
    shift = (e8.repeat_interleave(2, -1) + e16).repeat_interleave(4, -1)
    code = torch.stack([u[..., 4:] & 15, u[..., 4:] >> 4], -1).view(*u.shape[:2], 64)
    v = (code & 7).float() * torch.exp2(shift.float() - 2.0) * (1.0 - 2.0 * (code >> 3).float())
    return (v * _scales(u[..., 0:1])).view(u.shape[0], -1)


def _act(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "relu":
        return (z > 0.0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    return torch.ones_like(z)


def _standard(v, kind):
    """v normalised without weight, and the factor it was scaled with."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * rstd, rstd


def _standard_grad(d, n, rstd, kind):
    d = d - n * (d * n).mean(-1, keepdim=True) - (d.mean(-1, keepdim=True) if kind == "layer" else 0.0)
    return d * rstd


def _gate_rows(s):
    return s["gate"].float().repeat_interleave(s["case"]["gate"], 0)[: s["case"]["M"]] if s["gate"] is not None else 1.0


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    p = s["x"].float()
    if c["post"] != "none":
        p = _standard(p, c["post"])[0] * s["wp"].float()
    h = c["scale"] * s["r"].float() + _gate_rows(s) * p
    y = _standard(h, c["pre"])[0] * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    return {"h": h.to(dt), "y": y.to(dt)}


def _plain_norm_grad(s):
    c, dt = s["case"], s["x"].dtype
    x, dy, w, gate = s["x"].float(), s["dy"].float(), s["w"].float(), _gate_rows(s)
    n, rstd = _standard(s["h"].float(), c["pre"])
    dh = s["dh"].float() + _standard_grad(dy * w, n, rstd, c["pre"])
    out = {"dresidual": (c["scale"] * dh).to(dt), "dweight": (dy * n).sum(0)}
    if s["b"] is not None:
        out["dbias"] = dy.sum(0)
    dp, p = dh * gate, x
    if c["post"] != "none":
        wp = s["wp"].float()
        xn, rx = _standard(x, c["post"])
        p = xn * wp
        out["dpost_weight"] = (dp * xn).sum(0)
        dx = _standard_grad(dp * wp, xn, rx, c["post"])
    else:
        dx = dp
    if s["gate"] is not None:
        row = torch.arange(c["M"], device=x.device) // c["gate"]
        out["dgate"] = torch.zeros(s["gate"].shape, device=x.device).index_add_(0, row, dh * p).to(dt)
    out["dx"] = dx.to(dt)
    return out


def _product(xq, units, bias):
    z = xq @ _decode(units).t()
    return z if bias is None else z + bias.float()


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        return _plain_norm(s)
    if op == "norm_grad":
        return _plain_norm_grad(s)
    dt = s["x"].dtype
    if op == "block":
        h = s["r"].float() + s["x"].float()
        y = _standard(h, "rms")[0] * s["w"].float()
        xq = _through_units(y.to(dt))
        f = _act(_product(xq, s["wg"], s["bg"]), c["act"]) * _product(xq, s["wu"], s["bu"])
        return {"y": (_product(_through_units(f.to(dt)), s["wd"], None) + h.to(dt).float()).to(dt)}
    xq = _through_units(s["x"])
    z = _product(xq, s["wg"], s["bg"])
    if op == "linear":
        y = _act(z, c["act"])
        return {"y": (y if s["r"] is None else y + s["r"].float()).to(dt)}
    if op == "gated":
        return {"y": (_act(z, c["act"]) * _product(xq, s["wu"], s["bu"])).to(dt)}
    dy = s["dy"].float()
    if op == "linear_grad":
        dz = dy * _act_slope(z, c["act"])
        return {"dx": (dz @ _decode(s["wg"])).to(dt), "dbias": dz.sum(0)}
    u = _product(xq, s["wu"], s["bu"])
    dg, du = dy * u * _act_slope(z, c["act"]), dy * _act(z, c["act"])
    return {"dx": (dg @ _decode(s["wg"]) + du @ _decode(s["wu"])).to(dt), "dbias_gate": dg.sum(0), "dbias_up": du.sum(0)}


# ------------------------------------------------------------------------------------------------ this package's calls
def _calls(s):
    import paper_2602_11287_b200 as hif4
    c, op = s["case"], s["case"]["op"]
    norm = {"none": hif4.HIF4_NORM_NONE, "rms": hif4.HIF4_NORM_RMS, "layer": hif4.HIF4_NORM_LAYER}
    act = {"none": hif4.HIF4_ACT_NONE, "relu": hif4.HIF4_ACT_RELU, "silu": hif4.HIF4_ACT_SILU, "gelu": hif4.HIF4_ACT_GELU,
           "gelu_tanh": hif4.HIF4_ACT_GELU_TANH}
    if op == "norm":
        h, y = hif4.hif4_block_norm(s["x"], s["w"], s["b"], residual=s["r"], res_scale=c["scale"], gate=s["gate"],
                                    rows_per_gate=c["gate"], post_weight=s["wp"], pre=norm[c["pre"]], post=norm[c["post"]], eps=EPS)
        return {"h": h, "y": y}
    if op == "norm_grad":
        d = hif4.hif4_block_norm_backward(s["dy"], s["h"], s["w"], dh=s["dh"], x=s["x"], bias=s["b"] is not None,
                                          res_scale=c["scale"], gate=s["gate"], rows_per_gate=c["gate"],
                                          post_weight=s["wp"], pre=norm[c["pre"]], post=norm[c["post"]], eps=EPS)
        return {k: v for k, v in d.items() if v is not None}
    if op == "block":
        h, y = hif4.hif4_block_norm(s["x"], s["w"], residual=s["r"], units=True, eps=EPS)
        f = hif4.hif4_gated_linear(y, s["wg"], s["wu"], s["bg"], s["bu"], act=act[c["act"]], dtype=s["x"].dtype, units=True)
        return {"y": hif4.hif4_linear_act(f, s["wd"], residual=h, dtype=s["x"].dtype)}
    if op == "linear":
        return {"y": hif4.hif4_linear_act(s["x"], s["wg"], s["bg"], residual=s["r"], act=act[c["act"]])}
    if op == "gated":
        return {"y": hif4.hif4_gated_linear(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=act[c["act"]])}
    if op == "linear_grad":
        dx, db = hif4.hif4_linear_act_backward(s["dy"], s["x"], s["wg"], s["bg"], act=act[c["act"]], want_dbias=True)
        return {"dx": dx, "dbias": db}
    dx, dbg, dbu = hif4.hif4_gated_linear_backward(s["dy"], s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=act[c["act"]], want_dbias=True)
    return {"dx": dx, "dbias_gate": dbg, "dbias_up": dbu}


def run(state):
    return _calls(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ definition, 64 bits
def _nearest(v, digits):
    """v rounded to `digits` binary digits of significand, ties to even."""
    m, e = torch.frexp(v)
    return torch.ldexp(torch.round(torch.ldexp(m, torch.full_like(e, digits))), e - digits)


def _to_type(v, dt):
    return v.to(dt).double()


def _hif4_64(v, digits):
    """Conversion of values v (64 bits) to HiF4 and back; products carry `digits` binary digits (8: BF16, 24: FP32)."""
    u = v.reshape(v.shape[0], -1, 16, 4)
    seventh = _nearest(torch.full((), 1.0 / 7.0, dtype=torch.float64, device=v.device), digits)
    peak = _nearest(u.abs().amax((-1, -2)) * seventh, digits).clamp(2.0 ** -48, 2.0 ** 15 * 1.5)
    scale = _nearest(peak, 3)
    one_m = torch.frexp(scale)[0] * 2.0
    inverse = _nearest(1.0 / one_m, digits) * (one_m / scale)
    t = _nearest(u.abs() * inverse[..., None, None], digits)
    p3 = t.amax(-1)
    p2 = p3.view(*p3.shape[:2], 8, 2).amax(-1, keepdim=True)
    two = torch.where(p2 >= 4.0, 2.0, 1.0).double().expand(*p3.shape[:2], 8, 2).reshape(p3.shape)
    step = two * torch.where(p3 >= 2.0 * two, 2.0, 1.0).double()
    q = torch.clamp(torch.round(4.0 * t / step[..., None]), max=7.0) / 4.0
    return (torch.where(torch.signbit(u), -q, q) * step[..., None] * scale[..., None, None]).reshape(v.shape)


def _weights_64(units):
    """[rows, cols] values of packed units, straight from the layout of a unit."""
    rows = units.shape[0]
    u = units.reshape(rows, -1, 36).long()
    meta = u[..., 0] | (u[..., 1] << 8) | (u[..., 2] << 16) | (u[..., 3] << 24)
    i = torch.arange(64, device=u.device)
    nib = (u[..., 4 + i // 2] >> (4 * (i % 2))) & 15
    two = torch.tensor(2.0, dtype=torch.float64, device=u.device)
    s1 = two ** ((meta & 255) // 4 - 48) * (1.0 + ((meta & 3).double()) / 4.0)
    micro = ((meta[..., None] >> (8 + i // 8)) & 1) + ((meta[..., None] >> (16 + i // 4)) & 1)
    sign = 1.0 - 2.0 * (nib // 8).double()
    return (sign * (nib % 8).double() / 4.0 * two ** micro * s1[..., None]).reshape(rows, -1)


def _act_64(z, act):
    """Activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if act == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * phi, phi + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    a = 2.0 * math.sqrt(2.0 / math.pi)
    s = torch.sigmoid(a * (z + 0.044715 * z ** 3))
    return z * s, s + z * s * (1.0 - s) * a * (1.0 + 0.134145 * z ** 2)


def _norm_64(v, kind):
    """Normalised rows and 1 / deviation."""
    centre = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    inv = ((v - centre).pow(2).sum(1, keepdim=True) / v.shape[1] + EPS).pow(-0.5)
    return (v - centre) * inv, inv


def _pull_64(d, n, inv, kind):
    """Gradient of the norm's input from that of its normalised rows."""
    width = d.shape[1]
    g = d - n * ((d * n).sum(1, keepdim=True) / width)
    if kind == "layer":
        g = g - d.sum(1, keepdim=True) / width
    return g * inv


def exact(case, seed):
    s = prepare(case, seed)
    op, dt, M = case["op"], DTYPES[case["dtype"]], case["M"]
    f = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if op in ("norm", "norm_grad"):
        x = f["x"]
        owner = torch.arange(M, device="cuda") // case["gate"] if case["gate"] else None
        gate = f["gate"][owner] if case["gate"] else torch.ones_like(x)
        xn, xi = _norm_64(x, case["post"]) if case["post"] != "none" else (x, None)
        wp = f["wp"] if f["wp"] is not None else 1.0
        if op == "norm":
            h = case["scale"] * f["r"] + gate * xn * wp
            y = _norm_64(h, case["pre"])[0] * f["w"]
            return {"h": h, "y": y + f["b"] if f["b"] is not None else y}
        n, inv = _norm_64(f["h"], case["pre"])
        dh = f["dh"] + _pull_64(f["dy"] * f["w"], n, inv, case["pre"])
        out = {"dresidual": case["scale"] * dh, "dweight": torch.einsum("mk,mk->k", f["dy"], n)}
        if f["b"] is not None:
            out["dbias"] = torch.einsum("mk->k", f["dy"])
        if case["post"] != "none":
            out["dpost_weight"] = torch.einsum("mk,mk,mk->k", dh, gate, xn)
            out["dx"] = _pull_64(dh * gate * wp, xn, xi, case["post"])
        else:
            out["dx"] = dh * gate
        if case["gate"]:
            pick = torch.nn.functional.one_hot(owner, f["gate"].shape[0]).double()
            out["dgate"] = pick.t() @ (dh * xn * wp)
        return out
    digits = 8 if dt == torch.bfloat16 else 24
    if op == "block":
        h = f["x"] + f["r"]
        xq = _hif4_64(_to_type(_norm_64(h, "rms")[0] * f["w"], dt), digits)
    else:
        xq = _hif4_64(f["x"], digits)
    wg = _weights_64(s["wg"])
    z = xq @ wg.t() + (f["bg"] if f["bg"] is not None else 0.0)
    a, slope = _act_64(z, case["act"])
    if op == "linear":
        return {"y": a + f["r"] if f["r"] is not None else a}
    if op == "linear_grad":
        dz = f["dy"] * slope
        return {"dx": dz @ wg, "dbias": dz.sum(0)}
    wu = _weights_64(s["wu"])
    u = xq @ wu.t() + (f["bu"] if f["bu"] is not None else 0.0)
    if op == "gated":
        return {"y": a * u}
    if op == "block":
        return {"y": _hif4_64(_to_type(a * u, dt), digits) @ _weights_64(s["wd"]).t() + _to_type(h, dt)}
    dg, du = f["dy"] * u * slope, f["dy"] * a
    return {"dx": dg @ wg + du @ wu, "dbias_gate": dg.sum(0), "dbias_up": du.sum(0)}
