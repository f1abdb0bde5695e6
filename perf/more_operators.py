"""The operators around the experts' products of a mixture-of-experts layer, and the products in microscaled 4-bit formats.

  route / route_grad      scores, balance bias, groups, top-k, weights
  rows                    order of the experts' rows and the rows themselves (as they are, as HiF4 units, MXFP4 or NVFP4)
  combine / combine_grad  weighted sum of the experts' outputs per token
  roundtrip               conversion to MXFP4 or NVFP4 (along the rows, or down the columns) and back
  product                 product of two operands in these formats
  layer                   routing, rows, grouped product and combination, as a served layer runs them

`run` computes a case with elementary torch operations in 32 bits (`own` false) or with this package's calls (`own`
true); `exact` computes it in 64 bits from the definitions.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BLOCK = {"mxfp4": 32, "nvfp4": 16}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # routing of one decoded token: latency only
        dict(name="route one token", op="route", T=1, E=256, k=8, score="sigmoid", bias=True, groups=8, kept=4, best=2, renorm=True,
             scale=2.5, dtype="fp32"),
        # of a prompt, with groups and a bias that balances the load
        dict(name="route prompt", op="route", T=16384, E=256, k=8, score="sigmoid", bias=True, groups=8, kept=4, best=2, renorm=True,
             scale=2.5, dtype="fp32"),
        # training step of a router over softmax scores
        dict(name="route gradient", op="route_grad", T=8190, E=100, k=6, score="softmax", bias=False, groups=1, kept=1, best=1, renorm=False,
             scale=1.0, dtype="bf16"),
        # rows of a small decoding batch as HiF4 units
        dict(name="rows of 8 tokens", op="rows", T=8, k=8, E=256, K=7168, fmt="hif4", dtype="bf16", drop=0.0),
        # of a prompt, moved as they are
        dict(name="rows of a prompt", op="rows", T=4096, k=8, E=256, K=7168, fmt="rows", dtype="bf16", drop=0.0),
        # the experts' FP32 outputs of a prompt back to tokens, with the residual
        dict(name="combine prompt", op="combine", T=4096, k=8, E=256, K=7168, rows="fp32", dtype="bf16", residual=True, drop=0.0),
        # training step behind the experts; every sixteenth token is padding, the width fills no tile
        dict(name="combine gradient", op="combine_grad", T=2047, k=6, E=64, K=2056, rows="bf16", dtype="bf16", residual=False, drop=0.0625),
        # activations of a prompt through NVFP4 with a gain for the tensor
        dict(name="roundtrip prompt", op="roundtrip", rows=8192, cols=5120, fmt="nvfp4", down=False, gain=True, dtype="bf16"),
        # a gradient's conversion down the columns, as the weight gradient's product takes it
        dict(name="roundtrip columns", op="roundtrip", rows=4096, cols=1000, fmt="mxfp4", down=True, gain=False, dtype="fp16"),
        # one token through a projection
        dict(name="product one token", op="product", M=1, N=14336, K=4096, fmt="nvfp4", alpha=True, dtype="bf16"),
        # a prompt through it
        dict(name="product prompt", op="product", M=4096, N=14336, K=4096, fmt="nvfp4", alpha=True, dtype="bf16"),
        # a layer of experts, from logits to the summed outputs
        dict(name="layer of experts", op="layer", T=1024, E=32, k=4, K=2048, N=7168, fmt="mxfp4", dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "route", "route_grad", "rows", "rows", "combine", "combine_grad", "roundtrip", "roundtrip", "product",
                     "product", "layer"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("route", "route_grad"):
        groups = rng.choice([1, 1, 4, 8])
        E = groups * _log_int(rng, 2, 512 // groups)
        kept = rng.randint(1, groups)
        best = rng.choice([1, 2])
        k = min(_log_int(rng, 1, 16), kept * (E // groups))
        return dict(op=op, T=_log_int(rng, 1, 8192), E=E, k=k, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups,
                    kept=kept, best=best, renorm=rng.random() < 0.5, scale=rng.choice([1.0, 2.5]), dtype=dtype)
    k, E = _log_int(rng, 1, 8), _log_int(rng, 8, 256)
    if op in ("rows", "combine", "combine_grad"):
        T, K = _log_int(rng, 1, 4096), 64 * _log_int(rng, 1, 112)
        if op != "rows" and rng.random() < 0.25:
            K = _log_int(rng, 16, 7168)
        while T * k * K > (4096 * 8 * 7168 if op == "rows" else 2047 * 6 * 7168):
            T = max(1, T // 2)
        case = dict(op=op, T=T, k=k, E=E, K=K, dtype=dtype, drop=rng.choice([0.0, 0.0, 0.1]))
        if op == "rows":
            case.update(fmt=rng.choice(["rows", "hif4", "mxfp4", "nvfp4"]))
            return case
        case.update(rows=rng.choice(["fp32", dtype]), residual=op == "combine" and rng.random() < 0.5)
        return case
    fmt = rng.choice(["mxfp4", "nvfp4"])
    if op == "roundtrip":
        down = rng.random() < 0.4
        rows, cols = _log_int(rng, 1, 8192), 64 * _log_int(rng, 1, 112)
        if down:
            rows, cols = cols, 8 * _log_int(rng, 1, 640)
        while rows * cols > 8192 * 5120:
            rows, cols = (rows, max(8, cols // 16 * 8)) if down else (max(1, rows // 2), cols)
        return dict(op=op, rows=rows, cols=cols, fmt=fmt, down=down, gain=rng.random() < 0.5, dtype=dtype)
    K = 256 * _log_int(rng, 1, 28) if rng.random() < 0.7 else 64 * _log_int(rng, 1, 112)
    N = 64 * _log_int(rng, 1, 224) if rng.random() < 0.7 else _log_int(rng, 8, 14336)
    if op == "product":
        M = _log_int(rng, 1, 4096)
        while M * N * K > 4096 * 14336 * 4096:
            M = max(1, M // 2)
        return dict(op=op, M=M, N=N, K=K, fmt=fmt, alpha=rng.random() < 0.5, dtype=dtype)
    E, k, T = _log_int(rng, 8, 32), _log_int(rng, 1, 4), _log_int(rng, 1, 1024)
    while E * N * K > 32 * 7168 * 2048:
        N = max(8, N // 2)
    return dict(op=op, T=T, E=E, k=k, K=K, N=N, fmt=fmt, dtype=rng.choice(["bf16", "fp16"]))


def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op == "route":                                 # logits in; ids and weights out
        return {"bytes": case["T"] * (case["E"] * e + case["k"] * 8), "flops": case["T"] * case["E"] * 10}
    if op == "route_grad":                            # logits, ids, weights' gradients in; logits' gradients out
        return {"bytes": case["T"] * (2 * case["E"] * e + case["k"] * 8), "flops": case["T"] * case["E"] * 10}
    if op in ("rows", "combine", "combine_grad"):
        T, K, R = case["T"], case["K"], case["T"] * case["k"]
        if op == "rows":                              # tokens and ids in; rows out
            return {"bytes": e * T * K + e * R * K + 8 * R, "flops": R * K}
        er = SIZE[case["rows"]]
        if op == "combine":
            return {"bytes": er * R * K + e * T * K * (2 if case["residual"] else 1) + 8 * R, "flops": 2 * R * K}
        return {"bytes": 2 * er * R * K + e * T * K + 12 * R, "flops": 3 * R * K}
    if op == "roundtrip":
        return {"bytes": 2 * e * case["rows"] * case["cols"], "flops": 8 * case["rows"] * case["cols"]}
    N, K, b = case["N"], case["K"], BLOCK[case["fmt"]]
    if op == "product":
        M = case["M"]
        return {"bytes": (M + N) * (K // 2 + K // b) + e * M * N, "flops": 2 * M * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    reached = min(E, T * k)
    return {"bytes": reached * N * (K // 2 + K // b) + e * T * (K + N) + 4 * T * E, "flops": 2 * T * k * N * K}


# ------------------------------------------------------------------------------------------------------------- inputs
def _activations(rows, cols, g, dtype):
    """Heavy-tailed activations with a few outlier channels, as hidden states have them."""
    z = torch.randn(rows, cols, generator=g, device="cuda")
    z *= torch.rsqrt(torch.rand(rows, cols, generator=g, device="cuda") + 0.05)
    z[:, torch.randperm(cols, generator=g, device="cuda")[: max(1, cols // 200)]] *= 20.0
    return z.to(dtype)


def _logits(T, E, g, dtype):
    """Router logits over experts of uneven popularity."""
    popular = -0.6 * torch.log(1.0 + torch.randperm(E, generator=g, device="cuda").float())
    return (1.5 * torch.randn(T, E, generator=g, device="cuda") + popular).to(dtype)


def _assignment(T, k, E, drop, g):
    """Distinct experts per token by popularity; tokens of padding have none (-1)."""
    k = min(k, E)
    ids = torch.sort(_logits(T, E, g, torch.float32), dim=1, descending=True, stable=True)[1][:, :k].int()
    if drop:
        ids[torch.rand(T, generator=g, device="cuda") < drop] = -1
    return ids.contiguous()


def _row_of(ids, E):
    """Row of each assignment (sorted by expert, then by token and place; -1: none) and the experts' first rows."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    order = torch.sort(key, stable=True)[1]
    row = torch.empty_like(order).scatter_(0, order, torch.arange(flat.numel(), device=flat.device))
    offsets = (key.unsqueeze(0) < torch.arange(E + 1, device=flat.device).unsqueeze(1)).sum(1)
    return torch.where(key < E, row, -1).view(ids.shape).int(), offsets


def _operand(rows, cols, fmt, g):
    """Codes [rows, cols / 2] and scales [words, rows, 16] of a Gaussian matrix, in slabs (what a program loads)."""
    codes = torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(rows, -(-(cols // BLOCK[fmt]) // 16) * 16, dtype=torch.uint8, device="cuda")
    slab = max(1, (1 << 24) // cols)
    for r in range(0, rows, slab):
        n = min(slab, rows - r)
        code, scale = _quantize(torch.randn(n, cols, generator=g, device="cuda") / 4.0, fmt)
        codes[r:r + n] = code[:, 0::2] | (code[:, 1::2] << 4)
        scales[r:r + n, : cols // BLOCK[fmt]] = scale
    return codes, scales.view(rows, -1, 16).transpose(0, 1).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, dt = case["op"], DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if op in ("route", "route_grad"):
        s["logits"] = _logits(case["T"], case["E"], g, dt)
        s["bias"] = 0.05 * torch.randn(case["E"], generator=g, device="cuda") if case["bias"] else None
        if op == "route_grad":
            s["ids"] = _choose(s["logits"], s["bias"], case)
            s["dw"] = torch.randn(case["T"], case["k"], generator=g, device="cuda")
        return s
    if op in ("rows", "combine", "combine_grad"):
        T, K = case["T"], case["K"]
        s["ids"] = _assignment(T, case["k"], case["E"], case["drop"], g)
        R = s["ids"].numel()
        if op == "rows":
            s["x"] = _activations(T, K, g, dt)
            # rows that no token has stay as they are, so the program holds the memory (zeros here)
            if case["fmt"] == "rows":
                s["out"] = torch.zeros(R, K, dtype=dt, device="cuda")
            elif case["fmt"] == "hif4":
                s["out"] = torch.zeros(R, K // 64, 36, dtype=torch.uint8, device="cuda")
            else:
                s["out"] = (torch.zeros(R, K // 2, dtype=torch.uint8, device="cuda"),
                            torch.zeros(-(-(K // BLOCK[case["fmt"]]) // 16), R, 16, dtype=torch.uint8, device="cuda"))
            return s
        s["row_of"], s["offsets"] = _row_of(s["ids"], case["E"])
        s["w"] = torch.rand(s["ids"].shape, generator=g, device="cuda") / s["ids"].shape[1]
        s["rows"] = torch.randn(R, K, generator=g, device="cuda").to(DTYPES[case["rows"]])
        s["r"] = _activations(T, K, g, dt) if case["residual"] else None
        if op == "combine_grad":
            s["dy"] = (torch.randn(T, K, generator=g, device="cuda") * 0.1).to(dt)
            s["out"] = torch.zeros(R, K, dtype=DTYPES[case["rows"]], device="cuda")
        return s
    if op == "roundtrip":
        s["x"] = _activations(case["rows"], case["cols"], g, dt)
        s["gain"] = (2688.0 / s["x"].float().abs().amax()).reshape(1) if case["gain"] else None
        return s
    if op == "product":
        s["a"] = _operand(case["M"], case["K"], case["fmt"], g)
        s["b"] = _operand(case["N"], case["K"], case["fmt"], g)
        s["alpha"] = 0.5 + torch.rand(1, generator=g, device="cuda") if case["alpha"] else None
        return s
    s["x"] = _activations(case["T"], case["K"], g, dt)
    s["logits"] = _logits(case["T"], case["E"], g, torch.float32)
    codes, scales = _operand(case["E"] * case["N"], case["K"], case["fmt"], g)
    s["w"] = codes.view(case["E"], case["N"], -1), scales.view(-1, case["E"], case["N"], 16).transpose(0, 1).contiguous()
    s["r"] = _activations(case["T"], case["N"], g, dt)
    return s


# --------------------------------------------------------------------------------------------------------- plain form
def _to_e2m1(q):
    """Nearest code 0..7 of E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6) of q >= 0, ties to even codes, saturating."""
    code = (q > 0.25).int()
    for border, closed in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += ((q >= border) if closed else (q > border)).int()
    return code


def _to_e4m3(v):
    """Nearest byte of E4M3 of v >= 0 (32 bits), ties to even, saturating at 448."""
    e = torch.floor(torch.log2(v.clamp(min=2.0 ** -20).double())).clamp(min=-6.0).float()
    m = torch.round(v * torch.exp2(3.0 - e))                    # 8..16, below 8 for subnormal numbers
    byte = ((e + 6.0) * 8.0 + m).int()
    return byte.clamp(max=0x7E)


def _from_e4m3(byte):
    e, m = (byte >> 3).float(), (byte & 7).float()
    return torch.where(e > 0, torch.exp2(e - 7.0) * (1.0 + m / 8.0), m * 2.0 ** -9)


def _quantize(x, fmt, gain=None):
    """Codes (one byte each, sign in bit 3) and scale bytes of x [rows, cols], in 32 bits."""
    v = x.float() if gain is None else x.float() * gain
    a = v.abs().view(v.shape[0], -1, BLOCK[fmt])
    peak = a.amax(-1)
    if fmt == "mxfp4":
        e = (((peak.view(torch.int32) >> 23) & 255) - 127 - 2).clamp(-127, 127)
        byte = torch.where(peak > 0.0, e + 127, 0)
        q = a * torch.exp2(-(byte - 127).double()).unsqueeze(-1)
        zero = peak == 0.0
    else:
        byte = _to_e4m3(peak / 6.0)
        zero = byte == 0
        q = a / torch.where(zero, 1.0, _from_e4m3(byte)).unsqueeze(-1)
    code = torch.where(zero.unsqueeze(-1), 0, _to_e2m1(q)).view(v.shape)
    return (code | (torch.signbit(v).int() << 3)).to(torch.uint8), byte.to(torch.uint8)


def _values(code, byte, fmt):
    """FP32 values of codes [rows, cols] and scale bytes [rows, blocks]."""
    c = code.int()
    m = (c & 7).float()
    a = torch.where(m < 2.0, 0.5 * m, torch.exp2(torch.floor(m / 2.0) - 1.0) * (1.0 + 0.5 * (m - 2.0 * torch.floor(m / 2.0))))
    scale = _from_e4m3(byte.int()) if fmt == "nvfp4" else torch.exp2(byte.double() - 127.0).float()
    v = a.view(a.shape[0], -1, BLOCK[fmt]) * scale.unsqueeze(-1)
    return v.view(a.shape) * (1.0 - 2.0 * (c >> 3).float())


def _operand_values(codes, scales, fmt):
    """FP32 values [.., rows, cols] of codes [.., rows, cols / 2] and scales [.., words, rows, 16]."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    byte = scales.transpose(-3, -2).flatten(-2)[..., : code.shape[-1] // BLOCK[fmt]]
    return _values(code.flatten(0, -2), byte.flatten(0, -2), fmt).view(code.shape)


def _hif4(x):
    """x converted to HiF4 units and back, FP32, by Algorithm 1 in the arithmetic of x (BF16, or FP32 for FP16 and FP32)."""
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
    code = torch.round(t.float() * torch.exp2(2.0 - shift.float())).clamp(max=7.0)
    scale = torch.exp2((byte >> 2).float() - 48.0) * (1.0 + (byte & 3).float() * 0.25)
    q = code * torch.exp2(shift.float() - 2.0) * scale.unsqueeze(-1) * (1.0 - 2.0 * torch.signbit(v).float())
    return q.view(x.shape)


def _scores(logits, score):
    """Scores in the type of the logits given (32 or 64 bits)."""
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-logits))
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    return p / p.sum(1, keepdim=True)


def _choose(logits, bias, c):
    """Ids by score and bias, in 64 bits: neighbours in the order differ by less than 32 hold."""
    l64 = logits.double()
    if bias is None and c["best"] == 1:
        choice = l64                                            # the order of the scores is that of the logits
    else:
        choice = _scores(l64, c["score"])
        if bias is not None:
            choice = choice + bias.double()
    if c["groups"] > 1:
        per = choice.view(choice.shape[0], c["groups"], -1)
        value = torch.sort(per, dim=2, descending=True)[0][:, :, : min(c["best"], per.shape[2])].sum(2)
        rank = torch.sort(value, dim=1, descending=True, stable=True)[1][:, : c["kept"]]
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, rank, True)
        choice = torch.where(keep.unsqueeze(2), per, -math.inf).view(choice.shape)
    return torch.sort(choice, dim=1, descending=True, stable=True)[1][:, : c["k"]].int()


def _route(logits, bias, c):
    ids = _choose(logits, bias, c)
    w = torch.gather(_scores(logits.float(), c["score"]), 1, ids.long())
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return ids, c["scale"] * w


def _route_grad(s):
    c, at = s["case"], s["ids"].long()
    p = _scores(s["logits"].float(), c["score"])
    w, g = torch.gather(p, 1, at), c["scale"] * s["dw"]
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        g = (g - (g * w).sum(1, keepdim=True) / total) / total
    ds = torch.zeros_like(p).scatter_add_(1, at, g)
    d = ds * p * (1.0 - p) if c["score"] == "sigmoid" else p * (ds - (ds * p).sum(1, keepdim=True))
    return {"dlogits": d.to(s["logits"].dtype)}


def _spread(values, row_of, count):
    """[count, cols] rows: that of each assignment, zeros where there is none."""
    at = row_of.reshape(-1).long()
    each = values.repeat_interleave(row_of.shape[1], 0)
    out = torch.zeros(count + 1, values.shape[1], dtype=values.dtype, device=values.device)
    out[torch.where(at >= 0, at, count)] = each
    return out[:count]


def _picked(rows, row_of):
    """[T, k, cols] rows of the assignments in 32 bits, zeros where there is none."""
    p = rows[row_of.long().clamp(min=0)].float()
    return torch.where((row_of >= 0).unsqueeze(-1), p, 0.0)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    dt = DTYPES[c["dtype"]]
    if op == "route":
        ids, w = _route(s["logits"], s["bias"], c)
        return {"ids": ids, "weights": w}
    if op == "route_grad":
        return _route_grad(s)
    if op == "rows":
        row_of, offsets = _row_of(s["ids"], c["E"])
        x = s["x"]
        if c["fmt"] == "hif4":
            x = _hif4(x)
        elif c["fmt"] != "rows":
            x = _values(*_quantize(x, c["fmt"]), c["fmt"])
        x = x.to(dt) if c["fmt"] == "rows" else x.to(torch.bfloat16)
        return {"rows": _spread(x, row_of, row_of.numel()), "row_of": row_of, "offsets": offsets}
    if op == "combine":
        y = (_picked(s["rows"], s["row_of"]) * s["w"].unsqueeze(-1)).sum(1)
        return {"y": (y if s["r"] is None else y + s["r"].float()).to(dt)}
    if op == "combine_grad":
        dy, picked = s["dy"].float(), _picked(s["rows"], s["row_of"])
        each = (dy.unsqueeze(1) * s["w"].unsqueeze(-1)).to(s["rows"].dtype)
        at = s["row_of"].reshape(-1).long()
        drows = torch.zeros(at.numel() + 1, c["K"], dtype=each.dtype, device=each.device)
        drows[torch.where(at >= 0, at, at.numel())] = each.view(at.numel(), -1)
        return {"drows": drows[: at.numel()], "dweights": (dy.unsqueeze(1) * picked).sum(-1)}
    if op == "roundtrip":
        x = s["x"].t() if c["down"] else s["x"]
        v = _values(*_quantize(x.contiguous(), c["fmt"], s["gain"]), c["fmt"])
        return {"values": (v if s["gain"] is None else v / s["gain"]).to(torch.bfloat16)}
    if op == "product":
        y = _operand_values(*s["a"], c["fmt"]) @ _operand_values(*s["b"], c["fmt"]).t()
        return {"y": (y if s["alpha"] is None else y * s["alpha"]).to(dt)}
    T, E = c["T"], c["E"]
    ids, w = _route(s["logits"], None, _router(c))
    # a token has an expert once at most, so T places per expert hold its rows
    x = _values(*_quantize(s["x"], c["fmt"]), c["fmt"])
    here = torch.zeros(E, T, dtype=torch.bool, device=x.device)
    here[ids.long(), torch.arange(T, device=x.device).unsqueeze(1)] = True
    b = _operand_values(*s["w"], c["fmt"])
    y = torch.bmm(torch.where(here.unsqueeze(-1), x, 0.0), b.transpose(1, 2))
    out = (y[ids.long(), torch.arange(T, device=x.device).unsqueeze(1)] * w.unsqueeze(-1)).sum(1)
    return {"y": (out + s["r"].float()).to(dt)}


def _router(c):
    return dict(k=c["k"], score="softmax", groups=1, kept=1, best=1, renorm=True, scale=1.0)


# ------------------------------------------------------------------------------------------------ this package's calls
def _calls(s):
    import paper_2602_11287_b200 as hif4
    c, op = s["case"], s["case"]["op"]
    dt = DTYPES[c["dtype"]]
    score = {"softmax": hif4.HIF4_SCORE_SOFTMAX, "sigmoid": hif4.HIF4_SCORE_SIGMOID}
    fmt = {"rows": None, "hif4": hif4.HIF4_FMT_HIF4, "mxfp4": hif4.HIF4_FMT_MXFP4, "nvfp4": hif4.HIF4_FMT_NVFP4}
    if op == "route":
        ids, w = hif4.hif4_route(s["logits"], c["k"], s["bias"], score=score[c["score"]], groups=c["groups"], top_groups=c["kept"],
                                 group_best=min(c["best"], c["E"] // c["groups"]), renormalize=c["renorm"], scale=c["scale"])
        return {"ids": ids, "weights": w}
    if op == "route_grad":
        return {"dlogits": hif4.hif4_route_backward(s["dw"], s["logits"], s["ids"], score=score[c["score"]], renormalize=c["renorm"],
                                                    scale=c["scale"])}
    if op == "rows":
        offsets, row_of = hif4.hif4_expert_plan(s["ids"], c["E"])
        rows = hif4.hif4_dispatch(s["x"], row_of, fmt=fmt[c["fmt"]], out=s["out"])
        if c["fmt"] == "hif4":
            rows = hif4.hif4_dequantize(rows)
        elif c["fmt"] != "rows":
            rows = hif4.hif4_bfp4_dequantize(rows, fmt[c["fmt"]])
        return {"rows": rows, "row_of": row_of, "offsets": offsets}
    if op == "combine":
        return {"y": hif4.hif4_combine(s["rows"], s["row_of"], s["w"], residual=s["r"], dtype=dt)}
    if op == "combine_grad":
        drows, dw = hif4.hif4_combine_backward(s["dy"], s["row_of"], s["w"], rows=s["rows"], out=s["out"])
        return {"drows": drows, "dweights": dw}
    if op == "roundtrip":
        q = (hif4.hif4_bfp4_quantize_transposed if c["down"] else hif4.hif4_bfp4_quantize)(s["x"], fmt[c["fmt"]], gain=s["gain"])
        return {"values": hif4.hif4_bfp4_dequantize(q, fmt[c["fmt"]], gain=s["gain"])}
    if op == "product":
        return {"y": hif4.hif4_bfp4_gemm(s["a"], s["b"], fmt[c["fmt"]], alpha=s["alpha"], dtype=dt)}
    ids, w = hif4.hif4_route(s["logits"], c["k"])
    offsets, row_of = hif4.hif4_expert_plan(ids, c["E"])
    rows = hif4.hif4_dispatch(s["x"], row_of, fmt=fmt[c["fmt"]])
    y = hif4.hif4_bfp4_grouped_gemm(rows, s["w"], offsets, fmt[c["fmt"]], dtype=torch.float32)
    return {"y": hif4.hif4_combine(y, row_of, w, residual=s["r"], dtype=dt)}


def run(state):
    return _calls(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ definition, 64 bits
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _nearest(v, digits):
    """v rounded to `digits` binary digits of significand, ties to even."""
    m, e = torch.frexp(v)
    return torch.ldexp(torch.round(torch.ldexp(m, torch.full_like(e, digits))), e - digits)


def _fp4_64(x, fmt, gain):
    """Conversion of x [rows, cols] to a microscaled format and back (not divided by the gain); x * gain carries 24 digits."""
    v = x.double() if gain is None else _nearest(x.double() * gain.double(), 24)
    u = v.reshape(v.shape[0], -1, BLOCK[fmt])
    peak = u.abs().amax(-1, keepdim=True)
    if fmt == "mxfp4":
        scale = torch.ldexp(torch.ones_like(peak), (torch.frexp(peak)[1] - 3).clamp(-127, 127))
    else:
        sixth = peak / 6.0
        step = torch.ldexp(torch.ones_like(sixth), (torch.frexp(sixth)[1] - 4).clamp(min=-9))
        scale = (torch.round(sixth / step) * step).clamp(max=448.0)
    q = torch.where(scale > 0, u.abs() / torch.where(scale > 0, scale, 1.0), 0.0).clamp(max=6.0)
    step = torch.where(q < 2.0, 0.5, torch.where(q < 4.0, 1.0, 2.0))
    q = torch.round(q / step) * step
    return (torch.where(torch.signbit(u), -q, q) * scale).reshape(v.shape)


def _packed_64(codes, scales, fmt):
    """Values of packed codes and scales, by the formats' tables."""
    grid = torch.tensor(_E2M1 + tuple(-m for m in _E2M1), dtype=torch.float64, device=codes.device)
    i = torch.arange(2 * codes.shape[1], device=codes.device)
    v = grid[((codes[:, i // 2] >> (4 * (i % 2))) & 15).long()]
    word = i // BLOCK[fmt] // 16
    b = scales[word, :, i // BLOCK[fmt] % 16].t().long()
    if fmt == "mxfp4":
        return torch.ldexp(v, b - 127)
    return v * torch.where(b < 8, b.double() / 512.0, torch.ldexp(1.0 + (b % 8).double() / 8.0, b // 8 - 7))


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


def _route_64(logits, bias, c):
    """(ids, weights) of the definition."""
    x = logits.double()
    s = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, 1)
    choice = x if bias is None and c["best"] == 1 else s if bias is None else s + bias.double()
    T, E = x.shape
    group = torch.arange(E, device=x.device) // (E // c["groups"])
    open_ = torch.zeros(T, c["groups"], dtype=torch.bool, device=x.device)
    value = torch.stack([choice[:, group == n].topk(min(c["best"], E // c["groups"]), 1)[0].sum(1) for n in range(c["groups"])], 1)
    for _ in range(c["kept"]):
        open_[torch.arange(T), torch.where(open_, -math.inf, value).argmax(1)] = True
    left = torch.where(open_[:, group], choice, -math.inf)
    ids = []
    for _ in range(c["k"]):
        best = left.amax(1, keepdim=True)
        at = torch.where(left == best, torch.arange(E, device=x.device), E).amin(1)
        ids.append(at)
        left[torch.arange(T), at] = -math.inf
    ids = torch.stack(ids, 1)
    w = s[torch.arange(T, device=x.device).unsqueeze(1), ids]
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return ids.int(), c["scale"] * w


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    digits = 8 if case["dtype"] == "bf16" else 24
    if op == "route":
        ids, w = _route_64(s["logits"], s["bias"], case)
        return {"ids": ids, "weights": w}
    if op == "route_grad":
        x = s["logits"].double().requires_grad_()
        p = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, 1)
        w = p.gather(1, s["ids"].long())
        w = case["scale"] * (w / w.sum(1, keepdim=True) if case["renorm"] else w)
        d, = torch.autograd.grad(w, x, s["dw"].double())
        return {"dlogits": d}
    if op in ("rows", "combine", "combine_grad"):
        T, E = case["T"], case["E"]
        flat = s["ids"].reshape(-1).long()
        fine = flat >= 0
        count = torch.bincount(flat[fine], minlength=E)
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), count.cumsum(0)])
        token = torch.argsort(torch.where(fine, flat, E), stable=True)[: int(offsets[-1])]
        if op == "rows":
            x = s["x"].double()
            if case["fmt"] == "hif4":
                x = _hif4_64(x, digits)
            elif case["fmt"] != "rows":
                x = _fp4_64(x, case["fmt"], None)
            rows = torch.zeros(flat.numel(), x.shape[1], dtype=torch.float64, device="cuda")
            rows[: token.numel()] = x[token // s["ids"].shape[1]]
            row_of = torch.full_like(flat, -1)
            row_of[token] = torch.arange(token.numel(), device="cuda")
            return {"rows": rows, "row_of": row_of.view(T, -1).int(), "offsets": offsets}
        w = s["w"].double().reshape(-1)
        if op == "combine":
            y = torch.zeros(T, case["K"], dtype=torch.float64, device="cuda") if s["r"] is None else s["r"].double()
            y.index_add_(0, token // s["ids"].shape[1], s["rows"][: token.numel()].double() * w[token].unsqueeze(1))
            return {"y": y}
        dy = s["dy"].double()[token // s["ids"].shape[1]]
        drows = torch.zeros(flat.numel(), case["K"], dtype=torch.float64, device="cuda")
        drows[: token.numel()] = dy * w[token].unsqueeze(1)
        dw = torch.zeros_like(w)
        dw[token] = torch.linalg.vecdot(dy, s["rows"][: token.numel()].double())
        return {"drows": drows, "dweights": dw.view(T, -1)}
    if op == "roundtrip":
        v = _fp4_64(s["x"].t() if case["down"] else s["x"], case["fmt"], s["gain"])
        return {"values": v if s["gain"] is None else v / s["gain"].double()}
    if op == "product":
        y = _packed_64(*s["a"], case["fmt"]) @ _packed_64(*s["b"], case["fmt"]).t()
        return {"y": y if s["alpha"] is None else y * s["alpha"].double()}
    ids, w = _route_64(s["logits"], None, _router(case))
    x, y = _fp4_64(s["x"], case["fmt"], None), s["r"].double()
    for e in range(case["E"]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        y.index_add_(0, t, (x[t] @ _packed_64(s["w"][0][e], s["w"][1][e], case["fmt"]).t()) * w[t, j].unsqueeze(1))
    return {"y": y}
