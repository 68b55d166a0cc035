"""A training step of a block of a channels-last network, as the calls are used together: group norm with SiLU, an FP8 pointwise layer with a residual, and back."""
import pytest
import torch

import f8_reference as ref

pytestmark = pytest.mark.gpu
EPS = 1e-5
HALF = torch.finfo(torch.bfloat16).eps / 2                       # a rounding to bfloat16: 2^-8 of the value


def normalise(x, groups):
    n, c = x.shape[0], x.shape[-1]
    v = x.view(n, -1, groups, c // groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    return ((v - mean) / torch.sqrt((v - mean).square().mean(dim=(1, 3), keepdim=True) + EPS)).reshape(x.shape)


@pytest.mark.parametrize("shape,cout,groups", [((2, 7, 7, 96), 160, 32), ((1, 13, 9, 70), 33, 5)])
def test_block(ss, shape, cout, groups):
    g = torch.Generator().manual_seed(7)
    n, h, wd, c = shape
    x, res, dy = (torch.randn((n, h, wd, k), generator=g).bfloat16() for k in (c, cout, cout))
    W, gamma, beta = (torch.randn((cout, c), generator=g) / c ** 0.5).bfloat16(), 1 + 0.1 * torch.randn(c, generator=g), 0.1 * torch.randn(c, generator=g)
    bias = torch.randn(cout, generator=g)
    norm = ss.make_groupnorm_desc(c, groups, ss.SS_BF16, ss.SS_ACT_SILU, EPS)
    layer, back = ss.make_desc(cout, c, 1, 1, ss.SS_BF16), ss.make_desc(c, cout, 1, 1, ss.SS_BF16)
    dev = [t.cuda() for t in (x, res, dy, W, gamma, beta, bias)]
    X, RES, DY, WT, GAMMA, BETA, BIAS = dev
    forward, backward = ss.ss_f8_pack(layer, WT), ss.ss_f8_pack(back, WT, transposed=True)
    u, stats = ss.ss_groupnorm_fwd(norm, X, GAMMA, BETA)
    y = ss.ss_pw_f8_fwd(layer, u, forward, BIAS, RES)
    du = ss.ss_pw_f8_fwd(back, DY, backward)
    dw, db = ss.ss_pw_wgrad(layer, DY, u)
    grads = ss.ss_groupnorm_bwd(norm, du, X, stats, GAMMA, BETA)

    # each call against its definition at what the call before it gave
    z = normalise(x.double(), groups) * gamma.double() + beta.double()
    assert ((u.cpu().double() - z * torch.sigmoid(z)).abs() <= HALF * z.abs() + 1e-5).all()
    uq, Wq = ref.quantize(u.cpu().view(-1, c))[2], ref.quantize(W)[2]
    want = uq @ Wq.t() + bias.double() + res.double().view(-1, cout)
    # (half a step; what the FP8 instruction drops: 2^-13 of the largest of eight products, of each)
    slack = 2.0 ** -13 * c * uq.abs().amax() * Wq.abs().amax()
    assert ((y.cpu().double().view(-1, cout) - want).abs() <= HALF * want.abs() + slack).all()
    gq, Wt = ref.quantize(dy.view(-1, cout))[2], ref.quantize(W.t().contiguous())[2]
    want = gq @ Wt.t()
    slack = 2.0 ** -13 * cout * gq.abs().amax() * Wt.abs().amax()
    assert ((du.cpu().double().view(-1, c) - want).abs() <= HALF * want.abs() + slack).all()
    flat_dy, flat_u = dy.double().view(-1, cout), u.cpu().double().view(-1, c)
    assert ((dw.cpu().double() - flat_dy.t() @ flat_u).abs() <= 2.0 ** -18 * (flat_dy.abs().t() @ flat_u.abs())).all()
    assert ((db.cpu().double() - flat_dy.sum(dim=0)).abs() <= 2.0 ** -18 * flat_dy.abs().sum(dim=0)).all()
    xs, ws, bs = (t.double().requires_grad_(True) for t in (x, gamma, beta))
    z = normalise(xs, groups) * ws + bs
    (z * torch.sigmoid(z) * du.cpu().double()).sum().backward()
    assert ((grads.dx.cpu().double() - xs.grad).abs() <= HALF * xs.grad.abs() + 1e-5 * xs.grad.abs().amax()).all()
    for got, want in ((grads.dw, ws.grad), (grads.db, bs.grad)):
        assert ((got.cpu().double() - want).abs() <= 1e-5 * want.abs().amax() + 1e-5 * want.abs()).all()

    # the same step captured, replayed with other data between eager calls
    torch.cuda.synchronize()

    def step():
        u, stats = ss.ss_groupnorm_fwd(norm, X, GAMMA, BETA)
        y = ss.ss_pw_f8_fwd(layer, u, forward, BIAS, RES)
        du = ss.ss_pw_f8_fwd(back, DY, backward)
        return (u, stats, y, du, *ss.ss_pw_wgrad(layer, DY, u), *ss.ss_groupnorm_bwd(norm, du, X, stats, GAMMA, BETA))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for k in range(3):
        X.copy_(torch.randn(shape, generator=g).bfloat16())
        DY.copy_(torch.randn(dy.shape, generator=g).bfloat16())
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        for one, other in zip(captured, eager):
            assert torch.equal(one, other)
