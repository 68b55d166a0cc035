"""FP8 with a scale for each block of 128, from its definition, in 64 bits on the CPU."""
import torch

BLOCK = 128


def _codes(ratio):
    """E4M3 bytes of float64 values of at most 448 in magnitude, rounded to nearest even: from the type's table of values."""
    # (0 to 0x7E: zero, subnormals of 2^-9, then a fraction of three bits)
    table = torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127], dtype=torch.float64)
    a = ratio.abs()
    upper = torch.searchsorted(table, a.contiguous()).clamp(max=126)            # the first entry that is at least a
    lower = (upper - 1).clamp(min=0)
    to_upper, to_lower = table[upper] - a, a - table[lower]
    index = torch.where((to_upper < to_lower) | ((to_upper == to_lower) & (upper % 2 == 0)), upper, lower)
    return index.to(torch.uint8) | ((torch.signbit(ratio).to(torch.uint8)) << 7)


def quantize(x):
    """x [rows, cols] -> codes [rows, 64 * ceil(cols / 64)], scales [rows, 4 * ceil(cols / 512)] uint8, values [rows, cols] float64."""
    x = x.cpu().double()
    rows, cols = x.shape
    kb = -(-cols // BLOCK)
    v = torch.zeros((rows, kb * BLOCK), dtype=torch.float64)
    v[:, :cols] = x
    v = v.view(rows, kb, BLOCK)
    top = v.abs().amax(dim=2)
    finite = torch.isfinite(v).all(dim=2)
    safe = torch.where(finite & (top > 0), top, 1.0)
    f, e = torch.frexp(safe)                                                   # safe = f * 2^e, f in [1/2, 1); 448 = 7/8 * 2^9
    s = (e - 9 + (f > 0.875).int()).clamp(min=-127)
    s = torch.where(top > 0, s, -127)
    unit = torch.pow(torch.tensor(2.0, dtype=torch.float64), s.double())
    ok = finite.unsqueeze(2)
    codes = torch.where(ok, _codes(torch.where(ok, v, 0.0) / unit.unsqueeze(2)), 0)
    byte = torch.where(finite, s + 127, 255).to(torch.uint8)
    value = values(codes, byte).view(rows, -1)[:, :cols]
    pitch = -(-cols // 64) * 64
    out = torch.zeros((rows, kb * BLOCK), dtype=torch.uint8)
    out[:] = codes.view(rows, -1)
    scales = torch.zeros((rows, -(-kb // 4) * 4), dtype=torch.uint8)
    scales[:, :kb] = byte
    return out[:, :pitch].contiguous(), scales, value


def values(codes, byte):
    """codes [rows, kb, 128], byte [rows, kb] -> float64"""
    m, e = (codes & 7).double(), ((codes >> 3) & 15).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.pow(torch.tensor(2.0, dtype=torch.float64), e - 10))
    v = torch.where(codes >= 128, -v, v) * torch.pow(torch.tensor(2.0, dtype=torch.float64), byte.double() - 127).unsqueeze(2)
    return torch.where((byte == 255).unsqueeze(2), float("nan"), v)


def act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)) if not z.isnan().any() else torch.where(z.isnan(), z, z.clamp(min=0))
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    return z
