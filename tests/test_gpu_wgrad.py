"""The gradient of a pointwise layer's weights and bias, against 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
KERNELS = {"tile_64": 90, "tile_128": 91, "tile_256": 92}


def operands(seed, rows, cin, cout, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cin), generator=g) * torch.exp(torch.randn(cin, generator=g))
    return (torch.randn((rows, cout), generator=g) * 2.0 ** -6 * torch.exp(torch.randn((rows, 1), generator=g))).to(TYPES[dtype]), x.to(TYPES[dtype])


def check(dy, x, dw, db):
    dy, x = dy.double(), x.double()
    rows = x.shape[0]
    # each product, exact in fp32, meets at most rows / 8 + 70 additions (the instruction's own, the steps' and the parts'), each 2^-23 of the sum of magnitudes; 2^-126 where the sums are
    # smaller than fp32 goes
    tol = (rows / 8 + 70) * 2.0 ** -23 * (dy.abs().t() @ x.abs()) + 2.0 ** -126
    assert ((dw.cpu().double() - dy.t() @ x).abs() <= tol).all()
    if db is not None:
        assert ((db.cpu().double() - dy.sum(dim=0)).abs() <= (rows / 8 + 70) * 2.0 ** -24 * dy.abs().sum(dim=0)).all()


@pytest.mark.parametrize("kernel", [None, *KERNELS])
@pytest.mark.parametrize("rows,cin,cout,dtype", [(1, 1, 1, "f16"), (1, 96, 40, "bf16"), (2, 7, 3, "bf16"), (15, 8, 8, "f16"), (64, 33, 70, "f16"), (127, 130, 65, "bf16"), (128, 64, 32, "f16"),
                                                 (129, 100, 100, "bf16"), (500, 300, 77, "f16"), (1100, 260, 300, "bf16"), (2100, 48, 515, "bf16"), (9000, 96, 50, "f16"), (3001, 5, 300, "f16")])
def test_weight_gradient(ss, force_tile, kernel, rows, cin, cout, dtype):
    dy, x = operands(rows + cin + cout, rows, cin, cout, dtype)
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == "f16" else ss.SS_BF16)
    force_tile(None if kernel is None else KERNELS[kernel])
    dw, db = ss.ss_pw_wgrad(desc, dy.cuda(), x.cuda())
    again = ss.ss_pw_wgrad(desc, dy.cuda(), x.cuda())
    assert torch.equal(dw, again[0]) and torch.equal(db, again[1])
    check(dy, x, dw, db)


def test_difference(ss):
    """Against differences of the layer's own output: sum dy (W + e) x - sum dy (W - e) x over 2 e is the gradient, as the layer is linear."""
    dy, x = operands(3, 40, 12, 10, "bf16")
    W, e = torch.randn((10, 12), generator=torch.Generator().manual_seed(4)).double(), 0.5
    dw, db = ss.ss_pw_wgrad(ss.make_desc(10, 12, 1, 1, ss.SS_BF16), dy.cuda(), x.cuda())

    def loss(W, b):
        return (dy.double() * (x.double() @ W.t() + b)).sum()
    for o, c in ((0, 0), (3, 11), (9, 5)):
        step = torch.zeros_like(W)
        step[o, c] = e
        slope = (loss(W + step, 0.0) - loss(W - step, 0.0)) / (2 * e)
        assert abs(slope.item() - dw[o, c].item()) <= 80 * 2.0 ** -23 * (dy.double().abs()[:, o] @ x.double().abs()[:, c]).item()
        b = torch.zeros(10, dtype=torch.float64)
        b[o] = e
        slope = (loss(W, b) - loss(W, -b)) / (2 * e)
        assert abs(slope.item() - db[o].item()) <= 80 * 2.0 ** -23 * dy.double().abs()[:, o].sum().item()


def test_forms(ss):
    """Views of wider tensors, given outputs, several leading dimensions, no bias, no rows, another stream."""
    dy, x = (t.cuda() for t in operands(5, 200, 150, 90, "f16"))
    x, dy = x[:, 11:111], dy[:, 1:61]
    desc = ss.make_desc(60, 100, 1, 1, ss.SS_F16)
    want = ss.ss_pw_wgrad(desc, dy.contiguous(), x.contiguous())
    check(dy.cpu(), x.cpu(), *want)
    buffer = torch.full((60 * 100 + 1,), 5.0, device="cuda")
    dw, none = ss.ss_pw_wgrad(desc, dy, x, dw=buffer[1:].view(60, 100), with_bias=False)
    assert none is None and torch.equal(dw, want[0]) and buffer[0] == 5
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dw, db = ss.ss_pw_wgrad(desc, dy.contiguous().view(2, 10, 10, 60), x.contiguous().view(2, 10, 10, 100), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(dw, want[0]) and torch.equal(db, want[1])
    dw, db = ss.ss_pw_wgrad(desc, dy[:0], x[:0])
    assert not dw.any() and not db.any() and dw.shape == (60, 100)


def test_not_a_number(ss):
    """A NaN in x spoils its channel's column, one in dy its row; the rows behind the last are not read for it."""
    dy, x = operands(6, 300, 70, 80, "bf16")
    x[299, 7], dy[150, 33] = float("nan"), float("inf")
    wide_x, wide_dy = torch.full((512, 70), float("nan"), dtype=torch.bfloat16), torch.full((512, 80), float("nan"), dtype=torch.bfloat16)
    wide_x[:300], wide_dy[:300] = x, dy
    for kernel in KERNELS.values():
        ss.ss_debug_force_tile(kernel)
        dw, db = ss.ss_pw_wgrad(ss.make_desc(80, 70, 1, 1, ss.SS_BF16), wide_dy.cuda()[:300], wide_x.cuda()[:300])
        ss.ss_debug_force_tile(-1)
        bad = torch.zeros((80, 70), dtype=torch.bool)
        bad[:, 7], bad[33] = True, True
        assert torch.equal(~dw.isfinite().cpu(), bad)
        assert torch.equal(~db.isfinite().cpu(), torch.arange(80) == 33)


def test_replayed(ss):
    """A captured call, replayed with other data between eager calls, gives the eager result."""
    desc = ss.make_desc(96, 130, 1, 1, ss.SS_F16)
    dy, x = (t.cuda() for t in operands(7, 3000, 130, 96, "f16"))
    ws = torch.empty(ss.ss_pw_wgrad_workspace_bytes(desc, 3000), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty((96, 130), device="cuda"), torch.empty(96, device="cuda")
    ss.ss_pw_wgrad(desc, dy, x, dw, db, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ss.ss_pw_wgrad(desc, dy, x, dw, db, workspace=ws)
    for k in range(3):
        a, b = operands(20 + k, 3000, 130, 96, "f16")
        dy.copy_(a)
        x.copy_(b)
        want = ss.ss_pw_wgrad(desc, dy, x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, want[0]) and torch.equal(db, want[1])


def test_refusals(ss):
    desc = ss.make_desc(60, 100, 1, 1, ss.SS_F16)
    x, dy = torch.ones((5, 100), dtype=torch.float16, device="cuda"), torch.ones((5, 60), dtype=torch.float16, device="cuda")
    for call in (lambda: ss.ss_pw_wgrad(desc, dy[:4], x), lambda: ss.ss_pw_wgrad(desc, dy, x.bfloat16()), lambda: ss.ss_pw_wgrad(desc, dy.cpu(), x), lambda: ss.ss_pw_wgrad(desc, None, x),
                 lambda: ss.ss_pw_wgrad(desc, dy, x.t().contiguous().t()), lambda: ss.ss_pw_wgrad(desc, dy, x, dw=torch.empty((60, 99), device="cuda")),
                 lambda: ss.ss_pw_wgrad(desc, dy, x, db=torch.empty(59, device="cuda")), lambda: ss.ss_pw_wgrad(desc, dy, x, db=torch.empty(60, device="cuda"), with_bias=False),
                 lambda: ss.ss_pw_wgrad(desc, dy, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                 lambda: ss.ss_pw_wgrad(ss.make_desc(60, 100, 1, 1, ss.SS_F8), dy, x), lambda: ss.ss_pw_wgrad_workspace_bytes(ss.make_desc(60, 100, 3, 3, ss.SS_F16), 5),
                 lambda: ss.ss_pw_wgrad_workspace_bytes(desc, 1 << 31), lambda: ss.ss_pw_wgrad_workspace_bytes(desc, -1)):
        with pytest.raises(ss.SSError):
            call()
