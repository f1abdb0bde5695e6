"""MXFP4 and NVFP4 from their definitions in 64 bits (conversion: FP32 steps, each rounded once), for the tests."""
import torch

BLOCK = {1: 32, 2: 16}                                   # by HIF4_FMT_*
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def scale_values(byte, fmt):
    b = byte.long()
    if fmt == 1:
        v = torch.ldexp(torch.ones_like(b, dtype=torch.float64), b - 127)
        return torch.where(b == 255, torch.nan, v)
    v = torch.where(b < 8, b.double() / 512.0, torch.ldexp(1.0 + (b % 8).double() / 8.0, b // 8 - 7))
    return torch.where(b == 127, torch.nan, v)


def values(codes, scales, fmt):
    """[.., rows, cols] of codes [.., rows, cols / 2] and scales [.., words, rows, 16]."""
    grid = torch.tensor(GRID + tuple(-m for m in GRID), dtype=torch.float64, device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    s = scales.transpose(-3, -2).flatten(-2)[..., : c.shape[-1] // BLOCK[fmt]]
    return grid[c.long()] * scale_values(s, fmt).repeat_interleave(BLOCK[fmt], -1)


def convert(x, fmt, gain=None):
    """(codes [rows, cols] one a byte, scale bytes [rows, blocks]) of x."""
    v = x.float() if gain is None else x.float() * gain.float()
    u = v.reshape(v.shape[0], -1, BLOCK[fmt])
    peak = u.abs().amax(-1)
    bad = u.isnan().any(-1)
    peak = torch.where(bad, 1.0, peak)
    if fmt == 1:
        e = (torch.frexp(torch.where(peak.isinf(), 1.5, peak))[1] - 3)
        e = torch.where(peak.isinf(), 126, torch.where(peak == 0, -127, e)).clamp(-127, 127)
        byte = e + 127
    else:
        sixth = (peak / 6.0).double().clamp(max=448.0)
        step = torch.ldexp(torch.ones_like(sixth), (torch.frexp(sixth)[1] - 4).clamp(min=-9))
        r = torch.round(sixth / step) * step
        table = scale_values(torch.arange(127, device=x.device), 2)
        byte = torch.searchsorted(table, r)
    scale = scale_values(byte, fmt).unsqueeze(-1)
    q = (u.abs().double() / torch.where(scale > 0, scale, 1.0)).float().double()
    q = torch.where((scale > 0) & (peak > 0).unsqueeze(-1), q, 0.0)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    code = torch.zeros(q.shape, dtype=torch.int64, device=x.device)
    for n in range(7):                                   # border between codes n and n + 1; a tie goes to the even one
        border = (grid[n] + grid[n + 1]) / 2
        code += ((q > border) if n % 2 == 0 else (q >= border)).long()
    code = code | (torch.signbit(u).long() << 3)
    code = torch.where(bad.unsqueeze(-1), 0, code)
    byte = torch.where(bad, 255 if fmt == 1 else 127, byte)
    return code.reshape(v.shape).to(torch.uint8), byte.to(torch.uint8)


def pack(code, byte):
    """codes [rows, cols / 2] and scales [words, rows, 16] as the library lays them out."""
    rows, blocks = byte.shape
    words = -(-blocks // 16)
    s = torch.zeros(rows, words * 16, dtype=torch.uint8, device=byte.device)
    s[:, :blocks] = byte
    return code[:, 0::2] | (code[:, 1::2] << 4), s.view(rows, words, 16).transpose(0, 1).contiguous()


def random_operand(rows, cols, fmt, g, groups=None):
    """Random codes and moderate scales."""
    lead = () if groups is None else (groups,)
    words = -(-(cols // BLOCK[fmt]) // 16)
    codes = torch.randint(0, 256, (*lead, rows, cols // 2), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    low, high = (120, 131) if fmt == 1 else (40, 72)
    scales = torch.randint(low, high, (*lead, words, rows, 16), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    return codes, scales
