"""Plain 64-bit definitions of MXFP4, of the pointwise layer on it and of the norms around a block, and the error bounds of their fp32 kernels."""
import numpy as np
import torch

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U32 = 2.0 ** -24
ROUND = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: U32}      # unit roundoff of an output
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}    # half of the least subnormal


def quantize(x):
    """float64 [rows, cols] -> (codes [rows, 16*KB] uint8, scales [rows, 4*ceil(KB/4)] uint8), from the format's definition."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    kb = -(-cols // 32)
    v = np.zeros((rows, kb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, kb, 32)
    finite = np.isfinite(v).all(axis=-1)
    clean = np.where(np.isfinite(v), v, 0.0)
    top = np.abs(clean).max(axis=-1)
    exponent = np.frexp(np.where(top > 0, top, 1.0))[1] - 1
    byte = np.where(top > 0, np.maximum(exponent - 2, -127) + 127, 0)
    ratio = np.abs(clean) / np.ldexp(1.0, byte - 127)[..., None]
    distance = np.abs(ratio[..., None] - VALUES)
    nearest = distance.min(axis=-1, keepdims=True)
    tie = distance == nearest                                # of two nearest, the one whose code is even
    even = tie & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=-1), even.argmax(axis=-1), tie.argmax(axis=-1)).astype(np.uint8)
    code |= np.where(np.signbit(clean), 8, 0).astype(np.uint8)
    code = np.where(finite[..., None], code, 0).reshape(rows, kb * 32)
    scales = np.zeros((rows, -(-kb // 4) * 4), dtype=np.uint8)
    scales[:, :kb] = np.where(finite, byte, 255)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), scales


def dequantize(codes, scales, cols):
    """float64 [rows, cols]."""
    rows = codes.shape[0]
    code = np.stack([codes & 15, codes >> 4], axis=-1).reshape(rows, -1)
    value = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (value.reshape(rows, -1, 32) * scale[:, :value.shape[1] // 32, None]).reshape(rows, -1)[:, :cols]


def through_mx4(x):
    return dequantize(*quantize(x), np.asarray(x).shape[1])


def gelu(z):
    from scipy.special import ndtr
    return z * ndtr(z)


def pointwise(xq, wq, bias, residual, act):
    """(y, bound): act(wq xq + bias + residual) in 64 bits, and how far fp32 sums in any order may be from it before the last rounding.  `act`: 0 none,
    1 ReLU, 2 GELU, whose slope is at most 1.13 and whose normal distribution is within 1e-7."""
    z = xq @ wq.T
    size = np.abs(xq) @ np.abs(wq).T
    for extra in (bias, residual):
        if extra is not None:
            z = z + extra
            size = size + np.abs(extra)
    bound = (xq.shape[1] + 3) * U32 * size
    if act == 1:
        return np.maximum(z, 0.0), bound
    if act == 2:
        return gelu(z), 1.13 * bound + 2e-7 * np.abs(z)
    return z, bound


# ----------------------------------------------------------------------------------------------------------------------------
# norms; kind: 0 none, 1 LayerNorm, 2 RMS
# ----------------------------------------------------------------------------------------------------------------------------
def statistics(v, kind, eps):
    mean = v.mean(axis=1, keepdims=True) if kind == 1 else np.zeros((v.shape[0], 1))
    return v - mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(axis=1, keepdims=True) + eps)


def norm(v, kind, w, b, eps):
    if kind == 0:
        return v
    d, r = statistics(v, kind, eps)
    y = d * r * (1.0 if w is None else w)
    return y if b is None else y + b


def norm_grad(v, kind, dy, w, eps):
    """(dv, sum dy xh, sum dy)."""
    d, r = statistics(v, kind, eps)
    xh = d * r
    g = dy * (1.0 if w is None else w)
    inner = g - xh * (g * xh).mean(axis=1, keepdims=True)
    if kind == 1:
        inner = inner - g.mean(axis=1, keepdims=True)
    return r * inner, (dy * xh).sum(axis=0), dy.sum(axis=0)


def spread(gate, rows):
    return 1.0 if gate is None else np.repeat(gate, rows // gate.shape[0], axis=0)


def block_forward(p, kinds, eps=(1e-6, 1e-6)):
    """p: x, h, w, b, scale, gate, post_w, post_b (float64 or None) -> (x_out, y)."""
    x = p["x"]
    if p["h"] is not None:
        u = norm(p["h"], kinds[1], p["post_w"], p["post_b"], eps[1])
        x = x + u * (1.0 if p["scale"] is None else p["scale"]) * spread(p["gate"], len(x))
    return x, norm(x, kinds[0], p["w"], p["b"], eps[0]) if kinds[0] else None


def block_backward(p, kinds, dy, dx_out, eps=(1e-6, 1e-6)):
    """Gradients at p (whose x is x_out), by name."""
    x, rows = p["x"], len(p["x"] if p["x"] is not None else dx_out)
    out = {}
    t = 0.0 if dx_out is None else dx_out
    if kinds[0]:
        dv, out["dw"], out["db"] = norm_grad(x, kinds[0], dy, p["w"], eps[0])
        t = t + dv
    out["dx"] = t
    if p["h"] is None:
        return out
    u = norm(p["h"], kinds[1], p["post_w"], p["post_b"], eps[1])
    scale, gate = 1.0 if p["scale"] is None else p["scale"], spread(p["gate"], rows)
    out["dscale"] = (t * gate * u).sum(axis=0)
    if p["gate"] is not None:
        dg = (t * scale * u).reshape(p["gate"].shape[0], -1, t.shape[1]).sum(axis=1)
        out["dgate"] = dg if p["gate"].shape[1] == t.shape[1] else dg.sum(axis=1, keepdims=True)
    du = t * scale * gate
    out["dh"] = du
    if kinds[1]:
        out["dh"], out["dpost_w"], out["dpost_b"] = norm_grad(p["h"], kinds[1], du, p["post_w"], eps[1])
    return out


def close(got, want, bound, dtype, what):
    """got (device tensor, `dtype`) against want +- bound and one rounding."""
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    allowed = bound * (1 + ROUND[dtype]) + ROUND[dtype] * np.abs(want) + TINY[dtype]
    slack = np.abs(got - want) - allowed
    assert np.isfinite(got).all(), f"{what}: not finite"
    assert (slack <= 0).all(), f"{what}: off by {np.abs(got - want).flat[slack.argmax()]:.3e}, allowed {np.broadcast_to(allowed, slack.shape).flat[slack.argmax()]:.3e}"
