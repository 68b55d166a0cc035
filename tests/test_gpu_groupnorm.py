"""The group norm of channels-last images with its activation, and its gradient, against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
CODES = {"f16": 0, "bf16": 1, "f32": 4}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
EPS = 1e-5

# images, height, width, channels, groups
SHAPES = [(1, 1, 1, 32, 2), (2, 1, 1, 1, 1), (1, 1, 7, 3, 1), (3, 5, 1, 8, 8), (2, 7, 7, 24, 3), (2, 7, 7, 768, 32), (3, 17, 13, 330, 22), (1, 33, 31, 96, 32), (4, 14, 14, 40, 5),
          (1, 3, 3, 2056, 8), (2, 4, 4, 4097, 17), (1, 64, 64, 16, 1), (1, 2, 2, 5000, 1), (5, 28, 28, 64, 64), (1, 100, 90, 7, 7), (2, 57, 56, 256, 32), (1, 200, 120, 20, 2), (130, 3, 2, 72, 9)]


def data(seed, shape, dtype, off=0.5):
    g = torch.Generator().manual_seed(seed)
    c = shape[-1]
    x = torch.randn(shape, generator=g) * torch.exp(0.5 * torch.randn(c, generator=g)) + off * torch.randn(c, generator=g)
    return x.to(TYPES[dtype]), torch.randn(shape, generator=g).to(TYPES[dtype]), 1 + 0.2 * torch.randn(c, generator=g), 0.2 * torch.randn(c, generator=g)


def spread(v, c):
    return v.repeat_interleave(c // v.shape[-1], dim=-1)


def act(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return z * torch.special.ndtr(z)
    if kind == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def statistics(x, groups):
    n, c = x.shape[0], x.shape[-1]
    v = x.double().reshape(n, -1, groups, c // groups)
    mean = v.mean(dim=(1, 3))
    var = (v - mean[:, None, :, None]).square().mean(dim=(1, 3))
    return mean, var, 1 / torch.sqrt(var + EPS)


def check_forward(x, w, b, groups, kind, y, stats):
    n, c = x.shape[0], x.shape[-1]
    mean, var, r = statistics(x, groups)
    v = x.double().view(n, -1, c)
    m = v.shape[1] * (c // groups)
    size = v.view(n, -1, groups, c // groups).abs().amax(dim=(1, 3))
    # A sum of m values in the kernels' order: at most 64 + log2(m) additions to a value, each 2^-24 of the largest of the group; the mean takes part in every xh, the sum of squares
    # halves its relative error on the way to r.
    u = (80 + math.log2(m)) * 2.0 ** -24
    assert ((stats[..., 0].cpu().double() - mean).abs() <= u * size).all()
    dev = torch.sqrt(var + EPS)
    # (differences from the mean are off by u of the largest value; their squares' sum by twice that against the deviation, and by u of itself)
    rel = 2 * u + 2 * u * size / dev
    assert ((stats[..., 1].cpu().double() - r).abs() <= rel * r).all()
    xh = (v - spread(mean, c)[:, None]) * spread(r, c)[:, None]
    w, b = (torch.ones(c) if w is None else w).double(), (torch.zeros(c) if b is None else b).double()
    z = xh * w + b
    want = act(z, kind)
    dz = spread(u * size / dev, c)[:, None] * w.abs() + (spread(rel, c)[:, None] + 2.0 ** -22) * (xh * w).abs() + 2.0 ** -24 * z.abs()
    # an activation's slope is below 1.13; its own error: GELU in 16 bits 1e-7 of z and 4e-2 of values below 1e-2 (its lower tail), else a few roundings
    own = 2e-7 * z.abs() + 2.0 ** -21 * want.abs() + (4e-2 * want.abs() * (want.abs() < 1e-2) if kind == "gelu" else 0)
    tol = 1.13 * dz + own + want.abs() * torch.finfo(y.dtype).eps / 2 + 2.0 ** -25
    assert ((y.cpu().double().view(n, -1, c) - want).abs() <= tol).all()


@pytest.fixture(params=[None, 96], ids=["chosen", "passes"])
def kernel(request, force_tile):
    """The library's choice (the kernels that hold an image's groups, for most of these), or the passes over images of any size."""
    force_tile(request.param)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(ss, kernel, shape, dtype):
    kind = list(ACTS)[sum(shape) % 4]
    n, h, wd, c, groups = shape
    x, _, w, b = data(sum(shape), (n, h, wd, c), dtype)
    desc = ss.make_groupnorm_desc(c, groups, CODES[dtype], ACTS[kind], EPS)
    y, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
    assert y.shape == x.shape and y.dtype == x.dtype and stats.shape == (n, groups, 2)
    check_forward(x, w, b, groups, kind, y, stats)
    again = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
    assert torch.equal(y, again[0]) and torch.equal(stats, again[1])


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward_activations(ss, kernel, kind, dtype):
    x, _, w, b = data(3, (2, 9, 11, 48), dtype)
    w = w * 4
    desc = ss.make_groupnorm_desc(48, 6, CODES[dtype], ACTS[kind], EPS)
    check_forward(x, w, b, 6, kind, *ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda()))
    check_forward(x, None, None, 6, kind, *ss.ss_groupnorm_fwd(desc, x.cuda()))
    check_forward(x, w, None, 6, kind, *ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda()))


@pytest.mark.parametrize("pixels", [40, 5000])
def test_far_from_zero(ss, kernel, pixels):
    """Values whose mean is a thousand times their deviation: the sum of squares is no difference of large sums."""
    g = torch.Generator().manual_seed(9)
    x = 1000 + torch.randn((2, pixels, 32), generator=g)
    x[0, 0] = 0                                              # (a padded corner)
    desc = ss.make_groupnorm_desc(32, 4, ss.SS_F32, ss.SS_ACT_NONE, EPS)
    y, stats = ss.ss_groupnorm_fwd(desc, x.cuda())
    check_forward(x, None, None, 4, "none", y, stats)
    _, _, r = statistics(x, 4)
    assert ((stats[..., 1].cpu().double() / r - 1).abs() < 1e-3).all()


def check_backward(x, dy, w, b, groups, kind, stats, grads):
    """From the statistics that the call was given."""
    n, c = x.shape[0], x.shape[-1]
    v, d = x.double().view(n, -1, c), dy.double().view(n, -1, c)
    m = v.shape[1] * (c // groups)
    mean, r = (spread(stats[..., k].cpu().double(), c)[:, None] for k in (0, 1))
    wd, bd = (torch.ones(c) if w is None else w).double(), (torch.zeros(c) if b is None else b).double()
    xh = (v - mean) * r
    z = xh * wd + bd
    t = d * slope(z, kind)
    # t: an error of z of 2^-22 of its two parts, times the slope's own slope (below 1) and dy; and the slope's own error (GELU in 16 bits: 1e-6; a few roundings else)
    dt = d.abs() * ((0 if kind in ("none", "relu") else 2.0 ** -22 * ((xh * wd).abs() + bd.abs())) + (0 if kind in ("none", "relu") else 1e-6)) + 2.0 ** -23 * t.abs()
    s0, s1 = t.sum(dim=1), (t * xh).sum(dim=1)
    u = (80 + math.log2(max(m, 2))) * 2.0 ** -24
    e0, e1 = dt.sum(dim=1) + u * t.abs().sum(dim=1), (dt * xh.abs()).sum(dim=1) + (u + 2.0 ** -22) * (t * xh).abs().sum(dim=1)
    many = (n / 16 + 20) * 2.0 ** -24
    if w is not None:
        assert ((grads.dw.cpu().double() - s1.sum(dim=0)).abs() <= e1.sum(dim=0) + many * (t * xh).abs().sum(dim=(0, 1)) + 1e-30).all()
    else:
        assert grads.dw is None
    if b is not None:
        assert ((grads.db.cpu().double() - s0.sum(dim=0)).abs() <= e0.sum(dim=0) + many * t.abs().sum(dim=(0, 1)) + 1e-30).all()
    else:
        assert grads.db is None

    def over_group(s):
        return spread(s.view(n, groups, -1).sum(dim=2), c)[:, None] / m
    A, B = over_group(s0 * wd), over_group(s1 * wd)
    eA, eB = over_group(e0 * wd.abs() + u * (s0 * wd).abs()), over_group(e1 * wd.abs() + u * (s1 * wd).abs())
    want = r * (wd * t - A - xh * B)
    error = r * (wd.abs() * dt + eA + xh.abs() * eB + 2.0 ** -22 * ((wd * t).abs() + A.abs() + (xh * B).abs()))
    tol = error + want.abs() * torch.finfo(x.dtype).eps / 2 + 2.0 ** -25
    assert ((grads.dx.cpu().double().view(n, -1, c) - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(ss, kernel, shape, dtype):
    kind = list(ACTS)[(sum(shape) + 1) % 4]
    n, h, wd, c, groups = shape
    x, dy, w, b = data(sum(shape) + 1, (n, h, wd, c), dtype)
    desc = ss.make_groupnorm_desc(c, groups, CODES[dtype], ACTS[kind], EPS)
    _, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
    grads = ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda())
    assert grads.dx.shape == x.shape and grads.dx.dtype == x.dtype and grads.dw.shape == (c,) and grads.db.shape == (c,)
    check_backward(x, dy, w, b, groups, kind, stats, grads)
    for a, again in zip(grads, ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda())):
        assert torch.equal(a, again)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_activations(ss, kernel, kind, dtype):
    x, dy, w, b = data(4, (2, 9, 11, 48), dtype)
    w = w * 3
    desc = ss.make_groupnorm_desc(48, 6, CODES[dtype], ACTS[kind], EPS)
    _, stats = ss.ss_groupnorm_fwd(desc, x.cuda())
    for vectors in ((w, b), (None, None), (w, None), (None, b)):
        grads = ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, *(None if v is None else v.cuda() for v in vectors))
        check_backward(x, dy, *vectors, 6, kind, stats, grads)


def test_corner(ss, kernel):
    """The values that a ReLU's corner falls on: those whose sum in 32 bits rounds to the other side."""
    x = torch.randn((1, 64, 64, 8), generator=torch.Generator().manual_seed(8))
    desc = ss.make_groupnorm_desc(8, 2, ss.SS_F32, ss.SS_ACT_RELU, EPS)
    w = torch.full((8,), 1.7).cuda()
    _, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w)
    mean, r = (spread(stats[..., k].cpu().double(), 8) for k in (0, 1))
    for row in (5, 1000, 4095):
        # b such that this pixel's z is within a rounding of zero
        b = -((x.view(-1, 8)[row].double() - mean[0]) * r[0] * 1.7).float()
        dy = torch.ones((1, 64, 64, 8))
        grads = ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w, b.cuda())
        check_backward(x, dy, w.cpu(), b, 2, "relu", stats, grads)


def test_differences(ss):
    """Against differences of the loss sum(dy y) of a 64-bit forward pass."""
    x, dy, w, b = data(21, (2, 3, 3, 12), "f32")
    for kind in ("none", "gelu", "silu"):
        desc = ss.make_groupnorm_desc(12, 3, ss.SS_F32, ACTS[kind], EPS)
        _, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
        grads = ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda())

        def loss(x, w, b):
            mean, _, r = statistics(x, 3)
            z = (x.view(2, -1, 12) - spread(mean, 12)[:, None]) * spread(r, 12)[:, None] * w + b
            return (act(z, kind) * dy.double().view(2, -1, 12)).sum()
        args = [t.double() for t in (x, w, b)]
        for which, grad in enumerate((grads.dx, grads.dw, grads.db)):
            for i in range(0, args[which].numel(), 5):
                step = torch.zeros_like(args[which])
                step.view(-1)[i] = 1e-4
                up, down = ([a + step if k == which else a for k, a in enumerate(args)], [a - step if k == which else a for k, a in enumerate(args)])
                slope_ = (loss(*up) - loss(*down)) / 2e-4
                # (the difference's own error: 1e-8 of third derivatives of order 10; the gradient's: some hundred roundings)
                assert abs(slope_.item() - grad.view(-1)[i].item()) <= 2e-6 + 1e-4 * abs(slope_.item())


@pytest.mark.parametrize("dtype", TYPES)
def test_views(ss, kernel, dtype):
    """Channels of a wider tensor, from any element on; outputs that are the input; what lies beside them stays."""
    wide, dwide, w, b = data(31, (3, 6, 5, 50), dtype)
    wide, dwide, w, b = wide.cuda(), dwide.cuda(), w[:33].cuda(), b[:33].cuda()
    x, dy = wide[..., 5:38], dwide[..., 7:40]
    before = wide.clone()
    desc = ss.make_groupnorm_desc(33, 11, CODES[dtype], ss.SS_ACT_SILU, EPS)
    y, stats = ss.ss_groupnorm_fwd(desc, x.contiguous(), w, b)
    g = ss.ss_groupnorm_bwd(desc, dy.contiguous(), x.contiguous(), stats, w, b)
    for one, other in zip(g, ss.ss_groupnorm_bwd(desc, dy, x, stats, w, b)):
        assert torch.equal(one, other)
    given = torch.empty_like(stats)
    out, s = ss.ss_groupnorm_fwd(desc, x, w, b, y=x, stats=given)
    assert out is x and s is given and torch.equal(x, y) and torch.equal(given, stats)
    assert torch.equal(wide[..., :5], before[..., :5]) and torch.equal(wide[..., 38:], before[..., 38:])


def test_streams_and_graphs(ss, kernel):
    """Another stream; a captured pass, both ways, replayed with other data between eager calls."""
    x, dy, w, b = (t.cuda() for t in data(41, (2, 20, 20, 64), "bf16"))
    desc = ss.make_groupnorm_desc(64, 8, ss.SS_BF16, ss.SS_ACT_GELU, EPS)
    want, stats = ss.ss_groupnorm_fwd(desc, x, w, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, s2 = ss.ss_groupnorm_fwd(desc, x, w, b, stream=side)
    g2 = ss.ss_groupnorm_bwd(desc, dy, x, s2, w, b, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(want, y2) and torch.equal(stats, s2)
    for one, other in zip(g2, ss.ss_groupnorm_bwd(desc, dy, x, stats, w, b)):
        assert torch.equal(one, other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, s3 = ss.ss_groupnorm_fwd(desc, x, w, b)
        g3 = ss.ss_groupnorm_bwd(desc, dy, x, s3, w, b)
    for k in range(3):
        a, d, _, _ = data(50 + k, (2, 20, 20, 64), "bf16")
        x.copy_(a)
        dy.copy_(d)
        want, stats = ss.ss_groupnorm_fwd(desc, x, w, b)
        grads = ss.ss_groupnorm_bwd(desc, dy, x, stats, w, b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, y3) and torch.equal(stats, s3)
        for one, other in zip(grads, g3):
            assert torch.equal(one, other)


def test_nan_stays_in_its_group(ss, kernel):
    x, dy, w, b = data(61, (3, 10, 9, 40), "f32")
    x[1, 4, 4, 13] = float("nan")
    x[2, 0, 0, 39] = float("inf")
    desc = ss.make_groupnorm_desc(40, 5, ss.SS_F32, ss.SS_ACT_RELU, EPS)
    y, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
    bad = torch.zeros((3, 10, 9, 40), dtype=torch.bool)
    bad[1, ..., 8:16], bad[2, ..., 32:] = True, True
    assert torch.equal(y.cpu().isnan(), bad)
    grads = ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda())
    assert torch.equal(grads.dx.cpu().isnan(), bad)


def test_nothing(ss):
    desc = ss.make_groupnorm_desc(24, 3, ss.SS_F16, ss.SS_ACT_SILU, EPS)
    w = torch.ones(24, device="cuda")
    for shape in ((0, 5, 5, 24), (4, 0, 5, 24)):
        x = torch.empty(shape, dtype=torch.float16, device="cuda")
        y, stats = ss.ss_groupnorm_fwd(desc, x, w, w)
        assert y.shape == shape and stats.shape == (shape[0], 3, 2)
        g = ss.ss_groupnorm_bwd(desc, x, x, stats, w, w)
        assert g.dx.shape == shape and not g.dw.any() and not g.db.any()


def test_refusals(ss):
    x = torch.ones((2, 3, 3, 24), dtype=torch.float16, device="cuda")
    desc = ss.make_groupnorm_desc(24, 3, ss.SS_F16, ss.SS_ACT_SILU, EPS)
    w = torch.ones(24, device="cuda")
    _, stats = ss.ss_groupnorm_fwd(desc, x)
    make = ss.make_groupnorm_desc
    reserved = make(24, 3, ss.SS_F16)
    reserved.reserved = 1
    for call in (lambda: ss.ss_groupnorm_fwd(make(24, 5, ss.SS_F16), x), lambda: ss.ss_groupnorm_fwd(make(24, 0, ss.SS_F16), x), lambda: ss.ss_groupnorm_fwd(make(24, 3, ss.SS_F8), x),
                 lambda: ss.ss_groupnorm_fwd(make(24, 3, ss.SS_F16, 4), x), lambda: ss.ss_groupnorm_fwd(make(24, 3, ss.SS_F16, 0, -1.0), x),
                 lambda: ss.ss_groupnorm_fwd(make(24, 3, ss.SS_F16, 0, float("nan")), x), lambda: ss.ss_groupnorm_fwd(reserved, x), lambda: ss.ss_groupnorm_fwd(desc, x.float()),
                 lambda: ss.ss_groupnorm_fwd(desc, x.cpu()), lambda: ss.ss_groupnorm_fwd(desc, x[..., :16]), lambda: ss.ss_groupnorm_fwd(desc, x.transpose(1, 3)),
                 lambda: ss.ss_groupnorm_fwd(desc, x[0, 0, 0]), lambda: ss.ss_groupnorm_fwd(desc, x, w[:23]), lambda: ss.ss_groupnorm_fwd(desc, x, w.half()),
                 lambda: ss.ss_groupnorm_fwd(desc, x, stats=stats[:1]), lambda: ss.ss_groupnorm_fwd(desc, x, y=x[:1]), lambda: ss.ss_groupnorm_fwd(desc, x[:, :, ::2]),
                 lambda: ss.ss_groupnorm_bwd(desc, x, x, None), lambda: ss.ss_groupnorm_bwd(desc, x[:1], x, stats), lambda: ss.ss_groupnorm_bwd(desc, x, x, stats[:1]),
                 lambda: ss.ss_groupnorm_bwd(desc, x.view(3, 2, 3, 24), x, stats),
                 lambda: ss.ss_groupnorm_bwd(desc, x, x, stats, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
                 lambda: ss.ss_groupnorm_workspace_bytes(make(16392, 1, ss.SS_F16), 1, 1), lambda: ss.ss_groupnorm_workspace_bytes(desc, 1, (1 << 24) + 1),
                 lambda: ss.ss_groupnorm_workspace_bytes(desc, 1 << 20, 1 << 20), lambda: ss.ss_groupnorm_workspace_bytes(desc, -1, 5)):
        with pytest.raises(ss.SSError):
            call()
