"""The group norm and the weight gradient where offsets pass 32 bits, and of more images than one launch has threads for."""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5
HALF = torch.finfo(torch.bfloat16).eps / 2                       # a rounding to bfloat16: 2^-8 of the value


def need(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GB of free device memory")


def reference(x, dy, w, b, groups):
    """images [n, pixels, c] -> y, dx, dw, db in 64 bits (no activation)."""
    n, px, c = x.shape
    v = x.double().view(n, px, groups, c // groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    r = 1 / torch.sqrt((v - mean).square().mean(dim=(1, 3), keepdim=True) + EPS)
    xh = (v - mean) * r
    t = dy.double().view(v.shape)
    wd = w.double().view(groups, -1)
    g = t * wd
    dx = r * (g - g.mean(dim=(1, 3), keepdim=True) - xh * (g * xh).mean(dim=(1, 3), keepdim=True))
    return (xh * wd + b.double().view(groups, -1)).view(x.shape), dx.view(x.shape), (t * xh).sum(dim=(0, 1)).flatten(), t.sum(dim=(0, 1)).flatten()


@pytest.mark.parametrize("kernel", [None, 96])
def test_many_images(ss, force_tile, kernel):
    """2^25 images of two pixels and eight channels: 2^33 threads, in pieces of images; every one compared."""
    need(24)
    n, c, groups = (1 << 25) + 5, 8, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn((n, 2, c), generator=g, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w, b = 1 + 0.1 * torch.randn(c, generator=g, device="cuda"), 0.1 * torch.randn(c, generator=g, device="cuda")
    desc = ss.make_groupnorm_desc(c, groups, ss.SS_BF16, ss.SS_ACT_NONE, EPS)
    force_tile(kernel)
    y, stats = ss.ss_groupnorm_fwd(desc, x, w, b)
    grads = ss.ss_groupnorm_bwd(desc, dy, x, stats, w, b)
    dw, db = torch.zeros(c, dtype=torch.float64, device="cuda"), torch.zeros(c, dtype=torch.float64, device="cuda")
    size = torch.zeros(c, dtype=torch.float64, device="cuda")
    step = 1 << 22
    for at in range(0, n, step):
        wy, wdx, part_w, part_b = reference(x[at:at + step], dy[at:at + step], w, b, groups)
        # (eight values to the statistics: their errors are some 2^-20 of the result, which is rounded to half a step; where a group's deviation is small dx is large, and so is its error)
        assert bool(((y[at:at + step].double() - wy).abs() <= wy.abs() * HALF + 1e-5).all()), at
        largest = wdx.abs().view(-1, 2, groups, c // groups).amax(dim=(1, 3), keepdim=True).expand(-1, 2, -1, c // groups).reshape(wdx.shape)
        r = stats[at:at + step, :, 1].double().repeat_interleave(c // groups, dim=1).unsqueeze(1)
        assert bool(((grads.dx[at:at + step].double() - wdx).abs() <= wdx.abs() * HALF + 1e-5 * (largest + r)).all()), at
        dw += part_w
        db += part_b
        size += dy[at:at + step].double().abs().sum(dim=(0, 1))
    # n values to a sum, in 16 slices of n / 16: n / 16 additions, whose roundings are of either sign; six of their standard deviations
    tol = 6 * (n / 16) ** 0.5 * 2.0 ** -24 * size
    assert bool(((grads.db.double() - db).abs() <= tol).all()) and bool(((grads.dw.double() - dw).abs() <= 3 * tol).all())


@pytest.mark.parametrize("pixels,c,groups", [(1 << 24, 136, 2)])
def test_long_image(ss, pixels, c, groups):
    """An image of more than 2^31 values: its statistics, and pixels from its beginning, middle and end."""
    need(40)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((1, pixels, c), dtype=torch.bfloat16, device="cuda")
    dy = torch.empty_like(x)
    step = 1 << 20
    for at in range(0, pixels, step):
        x[0, at:at + step] = torch.randn((step, c), generator=g, device="cuda").bfloat16() + at / pixels
        dy[0, at:at + step] = torch.randn((step, c), generator=g, device="cuda").bfloat16()
    w = 1 + 0.1 * torch.randn(c, generator=g, device="cuda")
    desc = ss.make_groupnorm_desc(c, groups, ss.SS_BF16, ss.SS_ACT_NONE, EPS)
    y, stats = ss.ss_groupnorm_fwd(desc, x, w)
    grads = ss.ss_groupnorm_bwd(desc, dy, x, stats, w)
    m = pixels * (c // groups)

    def parts():
        for at in range(0, pixels, step):
            yield at, x[0, at:at + step].double().view(step, groups, -1), dy[0, at:at + step].double().view(step, groups, -1)
    mean = sum(v.sum(dim=(0, 2)) for _, v, _ in parts()) / m
    var = sum((v - mean.view(1, -1, 1)).square().sum(dim=(0, 2)) for _, v, _ in parts()) / m
    r = 1 / torch.sqrt(var + EPS)
    # a thread adds thousands of values, which are at most seven in magnitude
    assert bool(((stats[0, :, 0].double() - mean).abs() <= 1e-5).all()) and bool(((stats[0, :, 1].double() - r).abs() <= 1e-5).all())
    wd = w.double().view(groups, -1)
    s0, s1 = sum(t.sum(dim=0) for _, _, t in parts()), sum((t * ((v - mean.view(1, -1, 1)) * r.view(1, -1, 1))).sum(dim=0) for _, v, t in parts())
    assert bool(((grads.dw.double() - s1.flatten()).abs() <= 1e-5 * pixels ** 0.5 * 64).all())
    A, B = (wd * s0).sum(dim=1) / m, (wd * s1).sum(dim=1) / m
    for at in (0, pixels // 2 - 3, pixels - 1000):
        v, t = x[0, at:at + 1000].double().view(1000, groups, -1), dy[0, at:at + 1000].double().view(1000, groups, -1)
        xh = (v - mean.view(1, -1, 1)) * r.view(1, -1, 1)
        want_y, want_dx = xh * wd, r.view(1, -1, 1) * (wd * t - A.view(1, -1, 1) - xh * B.view(1, -1, 1))
        for got, want in ((y, want_y), (grads.dx, want_dx)):
            assert bool(((got[0, at:at + 1000].double().view(want.shape) - want).abs() <= want.abs() * HALF + 1e-4).all()), at


def test_weight_gradient_of_long_sums(ss):
    """x of more than 2^31 values; integers, whose sums fp32 holds."""
    need(16)
    rows, cin, cout = 2_200_003, 1000, 24
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randint(-1, 2, (rows, cin), generator=g, dtype=torch.int8, device="cuda").half()
    dy = torch.randint(-1, 2, (rows, cout), generator=g, dtype=torch.int8, device="cuda").half()
    dw, db = ss.ss_pw_wgrad(ss.make_desc(cout, cin, 1, 1, ss.SS_F16), dy, x)
    want = torch.zeros((cout, cin), dtype=torch.float64, device="cuda")
    for at in range(0, rows, 1 << 18):
        want += (dy[at:at + (1 << 18)].float().t().contiguous() @ x[at:at + (1 << 18)].float()).double()
    assert torch.equal(dw.double(), want) and torch.equal(db.double(), dy.double().sum(dim=0))
