"""The 8-bit point of the pointwise layers with a scale for each block of 128 values, and the group norm of channels-last images with its
activation, as measurable cases: quantisation to FP8 E4M3 whose blocks of 128 channels share a power of two, the layer on such operands, the
gradient of a pointwise layer's weights and bias (from 16-bit operands, as they are), and the group norm in both directions.

A case is a dict of plain values; ``prepare`` draws its inputs on the GPU, ``run`` is one pass, either in elementary tensor
operations or through the library's entry points (``own``), and ``exact`` is the definition in 64 bits.  Sizes are those of the
library's own configurations (ResNet-50 and ConvNeXt-T at 224 x 224, batches of 1 to 128) and generic ones between them.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ITEM = {"f16": 2, "bf16": 2, "f32": 4}
BLOCK = 128
EPS = 1e-5
MAX_ELEMENTS = 401408 * 384
MAX_FLOPS = 2 * 8192 ** 3
ACTS = ("none", "relu", "gelu", "silu")


def _named(name, c):
    return dict(c, name=name) if name else c


def _quantize(name, rows, cols, dtype):
    return _named(name, {"kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype})


def _pw(name, rows, cin, cout, dtype="bf16", act="none", bias=True, residual=False, mask=True, quantized=False, transposed=False):
    """transposed: the weights lie as [cin, cout], as they do for the gradient of a layer's input."""
    return _named(name, {"kind": "pw", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype, "act": act, "bias": bias, "residual": residual,
                         "mask": mask, "quantized": quantized, "transposed": transposed})


def _wgrad(name, rows, cin, cout, dtype="bf16"):
    return _named(name, {"kind": "wgrad", "rows": rows, "cin": cin, "cout": cout, "dtype": dtype})


def _gn(name, images, h, w, channels, groups, dtype="bf16", act="silu", affine=True, grad=False):
    return _named(name, {"kind": "gn_bwd" if grad else "gn", "images": images, "h": h, "w": w, "channels": channels, "groups": groups,
                         "dtype": dtype, "act": act, "affine": affine})


def listed():
    return [
        # the smallest call: 49 pixels of a network's last stage (7x7, 768 channels, one image) to 8 bits and back
        _quantize("quantize_49x768", 49, 768, "f16"),
        # the widest activation of ConvNeXt-T stage 1 at batch 128: bound by memory
        _quantize("quantize_401408x384", 401408, 384, "bf16"),
        # ResNet-50's classifier on one image: a single row, latency counts
        _pw("pw_1x2048_1000", 1, 2048, 1000, mask=False),
        # the expansion that closes ResNet-50's first bottlenecks at batch 64: few channels, many rows, bound by memory
        _pw("pw_200704x64_256_relu_res", 200704, 64, 256, act="relu", residual=True),
        # ragged sizes of a pruned or hand-made network, on an activation that is already quantised
        _pw("pw_ragged_q_gelu", 1531, 1000, 777, "f16", act="gelu", quantized=True),
        # a large matrix product on operands that are already quantised
        _pw("pw_8192_q", 8192, 8192, 8192, bias=False, mask=False, quantized=True),
        # a training step of config 2's layer at batch 64: the gradient of 256 x 1024 weights over 12544 rows
        _wgrad("wgrad_12544x1024_256", 12544, 1024, 256),
        # the same over the most rows: ConvNeXt-T's stage-1 expansion at batch 128, a small matrix of very long sums
        _wgrad("wgrad_401408x96_384", 401408, 96, 384),
        # the smallest norm: one image's last stage, latency counts
        _gn("gn_1x7x7x768_silu", 1, 7, 7, 768, 32, "f16"),
        # ResNet-50's widest activation at batch 64 with its ReLU: bound by memory
        _gn("gn_64x56x56x256_relu", 64, 56, 56, 256, 32, act="relu"),
        # the gradient at ResNet-50's second stage, batch 64
        _gn("gn_bwd_64x28x28x512_relu", 64, 28, 28, 512, 32, act="relu", grad=True),
        # an odd image, groups that are no multiple of a vector, 32-bit data
        _gn("gn_bwd_ragged_silu_f32", 3, 17, 13, 330, 22, "f32", grad=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _up(n, unit, rng):
    """Half of the sizes are multiples of a vector, the others are what they are."""
    return max(unit, n // unit * unit) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["quantize", "pw", "pw", "pw", "wgrad", "wgrad", "gn", "gn", "gn_bwd", "gn_bwd"])
    if kind == "quantize":
        dtype = rng.choice(["f16", "bf16", "f32"])
        cols = _up(_log(rng, 8, 8192), 32, rng)
        return _quantize(None, _log(rng, 1, min(401408, MAX_ELEMENTS * 2 // ITEM[dtype] // cols)), cols, dtype)
    if kind in ("pw", "wgrad"):
        cin, cout = _up(_log(rng, 32, 8192), 32, rng), _up(_log(rng, 8, 8192), 32, rng)
        rows = _log(rng, 1, min(401408, MAX_ELEMENTS // max(cin, cout), MAX_FLOPS // (2 * cin * cout)))
        dtype = rng.choice(["f16", "bf16"])
        if kind == "wgrad":
            return _wgrad(None, rows, cin, cout, dtype)
        mask = cin % 4 == 0 and rng.random() < 0.5
        return _pw(None, rows, cin, cout, dtype, rng.choice(["none", "relu", "gelu"]), rng.random() < 0.75, rng.random() < 0.4, mask,
                   rng.random() < 0.4, rng.random() < 0.25)
    per = _log(rng, 1, 64)
    groups = _log(rng, 1, min(64, 2048 // per))
    if rng.random() < 0.5:
        groups, per = 32, max(1, per // 2 * 2)
    images, h, w = _log(rng, 1, 128), _log(rng, 1, 112), _log(rng, 1, 112)
    per = max(per, -(-16 // (h * w)))               # (statistics of a handful of values are none)
    images = max(1, min(images, MAX_ELEMENTS // 4 // (h * w * groups * per)))
    return _gn(None, images, h, w, groups * per, groups, rng.choice(["f16", "bf16", "bf16", "f32"]), rng.choice(ACTS), rng.random() < 0.8,
               kind == "gn_bwd")


# ----------------------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------------------
def _activation(g, rows, cols, dtype):
    """N(0, 1) with channels of different sizes, as the activations behind a norm are."""
    channel = torch.exp(0.7 * torch.randn(cols, generator=g, device="cuda"))
    if dtype == torch.float32:
        return torch.randn((rows, cols), generator=g, device="cuda").mul_(channel)
    return torch.randn((rows, cols), generator=g, device="cuda", dtype=dtype).mul_(channel.to(dtype))


def _vector(g, n, around, spread):
    return around + spread * torch.randn(n, generator=g, device="cuda")


def _inputs(case, seed):
    """Everything drawn, from the seed alone, in one order."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    d = {}
    if case["kind"] == "quantize":
        d["x"] = _activation(g, case["rows"], case["cols"], dtype)
    elif case["kind"] == "pw":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        d["x"] = _activation(g, rows, cin, dtype)
        d["W"] = (torch.randn((cout, cin), generator=g, device="cuda") * math.sqrt(2.0 / cin)).to(dtype)
        d["bias"] = _vector(g, cout, 0.0, 0.1) if case["bias"] else None
        d["residual"] = torch.randn((rows, cout), generator=g, device="cuda").to(dtype) if case["residual"] else None
        d["M"] = None
        if case["mask"]:
            # the two largest of every four are kept
            kept = d["W"].float().abs().view(cout, cin // 4, 4).topk(2, dim=-1).indices
            d["M"] = torch.zeros((cout, cin // 4, 4), dtype=torch.uint8, device="cuda").scatter_(2, kept, 1).view(cout, cin)
    elif case["kind"] == "wgrad":
        d["x"] = _activation(g, case["rows"], case["cin"], dtype)
        # gradients of a mean over the rows of a step: small, and of different sizes from channel to channel
        d["dy"] = _activation(g, case["rows"], case["cout"], dtype).mul_(2.0 ** -8)
    else:
        shape = (case["images"], case["h"], case["w"], case["channels"])
        d["x"] = _activation(g, shape[0] * shape[1] * shape[2], shape[3], dtype)
        # channels off zero, as they are behind a layer with a bias
        d["x"] = d["x"].add_(_vector(g, shape[3], 0.0, 0.5).to(dtype)).view(shape)
        d["gamma"] = _vector(g, shape[3], 1.0, 0.1) if case["affine"] else None
        d["beta"] = _vector(g, shape[3], 0.0, 0.1) if case["affine"] else None
        if case["kind"] == "gn_bwd":
            d["dy"] = torch.randn(shape, generator=g, device="cuda").to(dtype)
            # what the forward pass left: mean and reciprocal deviation of each image's groups
            v = d["x"].view(shape[0], -1, case["groups"], shape[3] // case["groups"])
            stats = torch.empty((shape[0], case["groups"], 2), device="cuda")
            for n in range(shape[0]):
                one = v[n].double()
                mean = one.mean(dim=(0, 2), keepdim=True)
                stats[n, :, 0] = mean.flatten()
                stats[n, :, 1] = torch.rsqrt((one - mean).square_().mean(dim=(0, 2)) + EPS)
            d["stats"] = stats
    return d


def prepare(case, seed):
    """What a program has in hand: activations, and weights that it laid out when it loaded them."""
    d = _inputs(case, seed)
    d["case"] = case
    if case["kind"] == "pw":
        W, M = d.pop("W"), d.pop("M")
        if own:
            import paper_2411_00288_amd as ss
            d["desc"] = ss.make_desc(case["cout"], case["cin"], 1, 1, _code(ss, case["dtype"]))
            if case["transposed"]:
                d["packed"] = ss.ss_f8_pack(d["desc"], W.t().contiguous(), None if M is None else M.t().contiguous(), transposed=True)
            else:
                d["packed"] = ss.ss_f8_pack(d["desc"], W, M)
            if case["quantized"]:
                d["codes"], d["scales"] = ss.ss_f8_quantize(d.pop("x"))
        else:
            d["Wq"] = _plain_blocks((W if M is None else W * M).float()).to(W.dtype)
            if case["quantized"]:
                d["x"] = _plain_blocks(d["x"].float()).to(d["x"].dtype)
    elif own and case["kind"] == "wgrad":
        import paper_2411_00288_amd as ss
        d["desc"] = ss.make_desc(case["cout"], case["cin"], 1, 1, _code(ss, case["dtype"]))
    elif own and case["kind"] in ("gn", "gn_bwd"):
        import paper_2411_00288_amd as ss
        act = {"none": ss.SS_ACT_NONE, "relu": ss.SS_ACT_RELU, "gelu": ss.SS_ACT_GELU, "silu": ss.SS_ACT_SILU}[case["act"]]
        d["desc"] = ss.make_groupnorm_desc(case["channels"], case["groups"], _code(ss, case["dtype"]), act, EPS)
    return d


def _code(ss, dtype):
    return {"f16": ss.SS_F16, "bf16": ss.SS_BF16, "f32": ss.SS_F32}[dtype]


# ----------------------------------------------------------------------------------------------------------------------------
# the plain form: elementary operations in 32 bits, rounded once
# ----------------------------------------------------------------------------------------------------------------------------
def _plain_blocks(x):
    """float32 [rows, cols] -> the values that its 8-bit form stands for."""
    rows, cols = x.shape
    padded = -cols % BLOCK
    v = torch.nn.functional.pad(x, (0, padded)) if padded else x
    v = v.reshape(rows, -1, BLOCK)
    largest = v.abs().amax(dim=-1, keepdim=True)
    # the scale's byte: the least power of two, 2^(byte - 127), that leaves nothing above 448
    byte = ((largest.view(torch.int32) + 0x1FFFFF) >> 23).sub_(8).clamp_(min=0)
    up = ((254 - byte) << 23).view(torch.float32)
    a = v * up
    exponent = (a.abs().view(torch.int32) >> 23).clamp_(min=121)                 # (-6, the least of a normal element)
    step = ((exponent - 3) << 23).view(torch.float32)                           # three bits of fraction
    a = torch.round(a / step).mul_(step)
    return (a / up).reshape(rows, cols + padded)[:, :cols]


def _plain_act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _plain_act_slope(z, act):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain_wgrad(s):
    case = s["case"]
    # sums over very many rows: parts in 32 bits, joined in 64
    dw = torch.zeros((case["cout"], case["cin"]), dtype=torch.float64, device="cuda")
    for at in range(0, case["rows"], 16384):
        dw += (s["dy"][at:at + 16384].float().t().contiguous() @ s["x"][at:at + 16384].float()).double()
    return {"dw": dw.float(), "db": s["dy"].float().sum(dim=0, dtype=torch.float64).float()}


def _plain_gn(s):
    case = s["case"]
    dtype, n, g = DTYPES[case["dtype"]], case["images"], case["groups"]
    c = case["channels"] // g
    v = s["x"].float().view(n, -1, g, c)
    mean = v.mean(dim=(1, 3), keepdim=True)
    z = v - mean
    r = torch.rsqrt((z * z).mean(dim=(1, 3), keepdim=True) + EPS)
    z = z * r
    if s["gamma"] is not None:
        z = z * s["gamma"].view(g, c) + s["beta"].view(g, c)
    stats = torch.stack([mean.view(n, g), r.view(n, g)], dim=2)
    return {"y": _plain_act(z, case["act"]).to(dtype).view(s["x"].shape), "stats": stats}


def _plain_gn_bwd(s):
    case = s["case"]
    dtype, n, g = DTYPES[case["dtype"]], case["images"], case["groups"]
    c = case["channels"] // g
    mean, r = s["stats"][:, :, 0].view(n, 1, g, 1), s["stats"][:, :, 1].view(n, 1, g, 1)
    v, t = s["x"].view(n, -1, g, c), s["dy"].float().view(n, -1, g, c)
    gamma = None if s["gamma"] is None else s["gamma"].view(g, c)
    if case["act"] == "relu":
        # which side of the corner: in 64 bits
        z = (v.double() - mean.double()) * r.double()
        if gamma is not None:
            z = z * gamma.double() + s["beta"].double().view(g, c)
        t = t * (z > 0)
        del z
    xh = (v.float() - mean) * r
    if case["act"] in ("gelu", "silu"):
        t = t * _plain_act_slope(xh if gamma is None else xh * gamma + s["beta"].view(g, c), case["act"])
    out = {}
    if gamma is not None:
        out["dgamma"] = (t * xh).sum(dim=1).sum(dim=0).flatten()
        out["dbeta"] = t.sum(dim=1).sum(dim=0).flatten()
        t = t * gamma
    dx = (t - t.mean(dim=(1, 3), keepdim=True) - xh * (t * xh).mean(dim=(1, 3), keepdim=True)) * r
    out["dx"] = dx.to(dtype).view(s["x"].shape)
    return out


def _plain(s):
    case = s["case"]
    dtype = DTYPES[case["dtype"]]
    if case["kind"] == "quantize":
        return _plain_blocks(s["x"].float()).to(dtype)
    if case["kind"] == "wgrad":
        return _plain_wgrad(s)
    if case["kind"] == "gn":
        return _plain_gn(s)
    if case["kind"] == "gn_bwd":
        return _plain_gn_bwd(s)
    x = s["x"].float()
    z = (x if case["quantized"] else _plain_blocks(x)) @ s["Wq"].float().t()
    if s["bias"] is not None:
        z += s["bias"]
    if s["residual"] is not None:
        z += s["residual"].float()
    return _plain_act(z, case["act"]).to(dtype)


# ----------------------------------------------------------------------------------------------------------------------------
# the library's calls
# ----------------------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2411_00288_amd as ss
    case = s["case"]
    if case["kind"] == "quantize":
        # to 8 bits, and what they stand for
        codes, scales = ss.ss_f8_quantize(s["x"])
        return ss.ss_f8_dequantize(codes, scales, case["cols"], s["x"].dtype)
    if case["kind"] == "pw":
        act = {"none": ss.SS_ACT_NONE, "relu": ss.SS_ACT_RELU, "gelu": ss.SS_ACT_GELU}[case["act"]]
        if case["quantized"]:
            return ss.ss_pw_f8_q_fwd(s["desc"], s["codes"], s["scales"], s["packed"], s["bias"], s["residual"], act)
        return ss.ss_pw_f8_fwd(s["desc"], s["x"], s["packed"], s["bias"], s["residual"], act)
    if case["kind"] == "wgrad":
        dw, db = ss.ss_pw_wgrad(s["desc"], s["dy"], s["x"])
        return {"dw": dw, "db": db}
    if case["kind"] == "gn":
        y, stats = ss.ss_groupnorm_fwd(s["desc"], s["x"], s["gamma"], s["beta"])
        return {"y": y, "stats": stats}
    grads = ss.ss_groupnorm_bwd(s["desc"], s["dy"], s["x"], s["stats"], s["gamma"], s["beta"])
    out = {} if s["gamma"] is None else {"dgamma": grads.dw, "dbeta": grads.db}
    out["dx"] = grads.dx
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ----------------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------------------------------------
def _code_bytes(rows, cols):
    """Codes and scales of rows."""
    return rows * (cols + -(-cols // BLOCK))


def work(case):
    w = ITEM[case["dtype"]]
    if case["kind"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": 2 * rows * cols * w + _code_bytes(rows, cols), "flops": 4 * rows * cols}   # x read, codes written, values written
    if case["kind"] == "pw":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        x = _code_bytes(rows, cin) if case["quantized"] else rows * cin * w
        return {"bytes": x + _code_bytes(cout, cin) + rows * cout * w * (2 if case["residual"] else 1) + 4 * cout * case["bias"],
                "flops": 2 * rows * cin * cout}
    if case["kind"] == "wgrad":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        return {"bytes": rows * (cin + cout) * w + 4 * cout * (cin + 1), "flops": 2 * rows * cin * cout}
    n = case["images"] * case["h"] * case["w"] * case["channels"]
    stats, vectors = 8 * case["images"] * case["groups"], 8 * case["channels"] * case["affine"]
    if case["kind"] == "gn":
        return {"bytes": 2 * n * w + stats + vectors, "flops": 10 * n}
    return {"bytes": 3 * n * w + stats + 2 * vectors, "flops": 20 * n}          # x, dy -> dx


# ----------------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, written apart from the plain form
# ----------------------------------------------------------------------------------------------------------------------------
def _exact_f8(x):
    """float64 or narrower [rows, cols] -> float64: what the blocks of 128 along the columns stand for."""
    rows, cols = x.shape
    out = torch.empty((rows, cols), dtype=torch.float64, device=x.device)
    part = max(1, (1 << 26) // cols)
    for at in range(0, rows, part):
        v = x[at:at + part].double()
        whole = torch.zeros((v.shape[0], -(-cols // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
        whole[:, :cols] = v
        whole = whole.unflatten(1, (-1, BLOCK))
        top = whole.abs().max(dim=2, keepdim=True).values
        # top = f * 2^e with f in [1/2, 1): at most 448 = 7/8 * 2^9 over the scale
        f, e = torch.frexp(torch.where(top > 0, top, 1.0))
        s = (e.long() - 9 + (f > 0.875)).clamp(min=-127)
        unit = torch.where(top > 0, (s + 1023 << 52).view(torch.float64), 1.0)
        # the type's own conversion rounds to nearest even; the quotient of a power of two has no more bits than x
        q = (whole / unit).float().to(torch.float8_e4m3fn).double() * unit
        out[at:at + part] = q.flatten(1)[:, :cols]
    return out


def _exact_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_gn(d, case):
    n, g = case["images"], case["groups"]
    ys, stats = [], []
    for i in range(n):
        v = d["x"][i].double().reshape(-1, g, case["channels"] // g).transpose(0, 1).reshape(g, -1)
        var, mean = torch.var_mean(v, dim=1, unbiased=False)
        r = 1 / torch.sqrt(var + EPS)
        z = ((v - mean[:, None]) * r[:, None]).view(g, -1, case["channels"] // g).transpose(0, 1).reshape(d["x"][i].shape)
        if d["gamma"] is not None:
            z = z * d["gamma"].double() + d["beta"].double()
        ys.append(_exact_act(z, case["act"]))
        stats.append(torch.stack([mean, r], dim=1))
    return {"y": torch.stack(ys), "stats": torch.stack(stats)}


def _exact_gn_bwd(d, case):
    """The statistics are inputs of the backward pass; dx contains their own dependence on x."""
    n, g, channels = case["images"], case["groups"], case["channels"]
    per = case["h"] * case["w"] * (channels // g)
    affine = d["gamma"] is not None
    gamma = d["gamma"].double() if affine else torch.ones(channels, dtype=torch.float64, device="cuda")
    beta = d["beta"].double() if affine else torch.zeros(channels, dtype=torch.float64, device="cuda")
    dgamma, dbeta, dx = torch.zeros_like(gamma), torch.zeros_like(gamma), torch.empty(d["x"].shape, dtype=torch.float64, device="cuda")

    def spread(group_values):
        return group_values.repeat_interleave(channels // g)

    def total(channel_values):
        return channel_values.view(g, -1).sum(dim=1)

    for i in range(n):
        mean, r = (spread(d["stats"][i, :, k].double()) for k in (0, 1))
        xh = (d["x"][i].double().view(-1, channels) - mean) * r
        z = (xh * gamma + beta).requires_grad_(True)
        _exact_act(z, case["act"]).backward(d["dy"][i].double().view(-1, channels))
        t = z.grad
        s0, s1 = t.sum(dim=0), (t * xh).sum(dim=0)
        dbeta += s0
        dgamma += s1
        dx[i] = (r * (gamma * t - spread(total(gamma * s0) / per) - xh * spread(total(gamma * s1) / per))).view(dx[i].shape)
    return {"dgamma": dgamma, "dbeta": dbeta, "dx": dx} if affine else {"dx": dx}


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "quantize":
        return _exact_f8(d["x"])
    if case["kind"] == "wgrad":
        dy = d["dy"].double()
        return {"dw": torch.matmul(dy.T, d["x"].double()), "db": dy.sum(dim=0)}
    if case["kind"] == "gn":
        return _exact_gn(d, case)
    if case["kind"] == "gn_bwd":
        return _exact_gn_bwd(d, case)
    W = d["W"].double()
    if d["M"] is not None:
        W = torch.where(d["M"] != 0, W, 0.0)
    Wq = _exact_f8(W)
    del W
    y = torch.matmul(_exact_f8(d["x"]), Wq.T)
    if d["bias"] is not None:
        y += d["bias"].double()
    if d["residual"] is not None:
        y += d["residual"].double()
    return _exact_act(y, case["act"])
