"""Norms before and after a block with gate, residual scale and residual sum, and their gradient, against 64-bit definitions.

Bounds: a row's sum adds at most 16 values in a lane, then 6 + 16 partial sums, so that a mean is off by at most 40 u times the mean magnitude and a
factor by as much of itself; a normalised value d r is then within 128 u of the row's largest |v| times r.  Sums over `rows` rows add up one
rounding each on top."""
import itertools

import numpy as np
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = {torch.float16: "SS_F16", torch.bfloat16: "SS_BF16", torch.float32: "SS_F32"}
C = 128 * ref.U32


def _draw(rows, cols, dtype, gate, seed, offset=0.0):
    rng = np.random.default_rng(seed)
    t = lambda *shape: torch.from_numpy(rng.standard_normal(shape)).cuda()
    p = {"x": (t(rows, cols) + offset).to(dtype), "h": (t(rows, cols) * 1.5).to(dtype), "w": (1 + 0.2 * t(cols)).float(), "b": t(cols).float(),
         "scale": (0.3 * t(cols)).float(), "gate": None if gate is None else t(*gate).to(dtype), "post_w": (1 + 0.2 * t(cols)).float(), "post_b": (0.2 * t(cols)).float()}
    return p, t(rows, cols).to(dtype), t(rows, cols).to(dtype)


def _wide(p):
    return {k: None if v is None else v.double().cpu().numpy() for k, v in p.items()}


def _slack(v, kind, w, b, eps):
    """How far a norm of v may be off, for inputs that are exact."""
    if kind == 0:
        return 0.0
    _, r = ref.statistics(v, kind, eps)
    w = 1.0 if w is None else np.abs(w)
    return C * (np.abs(v).max(axis=1, keepdims=True) * r * w * 2 + (0.0 if b is None else np.abs(b)))


def _gain(v, kind, w, eps):
    """Largest change of a norm's output for a change of one of its inputs' magnitude."""
    if kind == 0:
        return 0.0
    d, r = ref.statistics(v, kind, eps)
    return 3 * r * (1.0 if w is None else np.abs(w)) * (1 + np.abs(d * r))


def _check_forward(ss, p, kinds, dtype, out, eps):
    q = _wide(p)
    x_out, y = ref.block_forward(q, kinds, eps)
    bound = np.zeros_like(x_out)
    if q["h"] is not None:
        factor = np.abs((1.0 if q["scale"] is None else q["scale"]) * ref.spread(q["gate"], len(x_out)))
        u = ref.norm(q["h"], kinds[1], q["post_w"], q["post_b"], eps[1])
        bound = bound + factor * _slack(q["h"], kinds[1], q["post_w"], q["post_b"], eps[1]) + 4 * ref.U32 * (np.abs(q["x"]) + 2 * factor * np.abs(u))
        ref.close(out[0] if isinstance(out, tuple) else out, x_out, bound, dtype, "x_out")
    if kinds[0]:
        change = _gain(x_out, kinds[0], q["w"], eps[0]) * bound.max(axis=1, keepdims=True)
        ref.close(out[-1] if isinstance(out, tuple) else out, y, change + _slack(x_out, kinds[0], q["w"], q["b"], eps[0]), dtype, "y")


def _check_backward(p, kinds, dy, dx_out, dtype, grads, eps):
    q = _wide(p)
    dy, dx_out = (None if v is None else v.double().cpu().numpy() for v in (dy, dx_out))
    want = ref.block_backward(q, kinds, dy, dx_out, eps)
    rows = len(want["dx"])

    def norm_bounds(v, kind, g_out, w, g_error, ep):
        """(of dv, of sum dy xh, of sum dy) for an incoming gradient that is off by g_error."""
        d, r = ref.statistics(v, kind, ep)
        top = (np.abs(v).max(axis=1, keepdims=True) * r + 1) * (1 + np.abs(d * r).max(axis=1, keepdims=True))
        w = 1.0 if w is None else np.abs(w)
        g = (np.abs(g_out) * w).max(axis=1, keepdims=True)
        dv = r * top * (4 * C * g + 3 * (g_error * w).max(axis=1, keepdims=True)) if kind else g_error
        mag = np.abs(g_out)
        return dv, (mag * top * 2 * C + g_error * top + rows * ref.U32 * mag * np.abs(d * r)).sum(axis=0), (g_error + rows * ref.U32 * mag).sum(axis=0)

    bounds = {}
    zero = np.zeros_like(want["dx"])
    bounds["dx"] = zero
    if kinds[0]:
        bounds["dx"], bounds["dw"], bounds["db"] = norm_bounds(q["x"], kinds[0], dy, q["w"], zero, eps[0])
    t, dt = want["dx"], bounds["dx"] + 4 * ref.U32 * np.abs(want["dx"])
    bounds["dx"] = dt
    if q["h"] is not None:
        u = ref.norm(q["h"], kinds[1], q["post_w"], q["post_b"], eps[1])
        du = _slack(q["h"], kinds[1], q["post_w"], q["post_b"], eps[1]) + 4 * ref.U32 * np.abs(u)
        scale, gate = np.abs(1.0 if q["scale"] is None else q["scale"]), np.abs(ref.spread(q["gate"], rows))
        product = dt * np.abs(u) + np.abs(t) * du + 4 * ref.U32 * np.abs(t * u)
        bounds["dscale"] = ((product + rows * ref.U32 * np.abs(t * u)) * gate * np.ones_like(t)).sum(axis=0)
        if q["gate"] is not None:
            groups = q["gate"].shape[0]
            each = ((product + (rows // groups + 64) * ref.U32 * np.abs(t * u)) * scale).reshape(groups, -1, t.shape[1]).sum(axis=1)
            bounds["dgate"] = each if q["gate"].shape[1] == t.shape[1] else each.sum(axis=1, keepdims=True)
        g, ge = t * scale * gate, dt * scale * gate + 4 * ref.U32 * np.abs(t) * scale * gate
        bounds["dh"] = ge
        if kinds[1]:
            bounds["dh"], bounds["dpost_w"], bounds["dpost_b"] = norm_bounds(q["h"], kinds[1], g, q["post_w"], ge, eps[1])
    present = {"dx": True, "dh": q["h"] is not None, "dgate": q["gate"] is not None, "dw": q["w"] is not None, "db": q["b"] is not None,
               "dscale": q["scale"] is not None, "dpost_w": q["post_w"] is not None, "dpost_b": q["post_b"] is not None}
    for name, value in grads._asdict().items():
        assert (value is not None) == present[name], name
        if value is not None:
            ref.close(value, want[name], bounds[name], dtype if name in ("dx", "dh", "dgate") else torch.float32, name)


def _run(ss, rows, cols, dtype, kinds, gate, parts, seed, eps=(1e-6, 1e-5), offset=0.0):
    p, dy, dx_out = _draw(rows, cols, dtype, gate, seed, offset)
    for name in ("w", "b", "scale", "post_w", "post_b", "h"):
        if name not in parts:
            p[name] = None
    if not kinds[0]:
        p["w"] = p["b"] = None
    if not kinds[1]:
        p["post_w"] = p["post_b"] = None
    desc = ss.make_norm_desc(cols, getattr(ss, DTYPES[dtype]), kinds[0], eps[0], kinds[1], eps[1])
    names = ("w", "b", "h", "scale", "gate", "post_w", "post_b")
    out = ss.ss_norm_fwd(desc, p["x"], *(p[n] for n in names))
    _check_forward(ss, p, kinds, dtype, out, eps)
    if not kinds[0]:
        dy = None
    at = dict(p, x=p["x"])                                       # any stream will do as x_out
    grads = ss.ss_norm_bwd(desc, dy, at["x"] if kinds[0] else None, *(p[n] for n in names), dx_out=dx_out)
    _check_backward(at, kinds, dy, dx_out, dtype, grads, eps)
    if kinds[0]:
        grads = ss.ss_norm_bwd(desc, dy, at["x"], *(p[n] for n in names))
        _check_backward(at, kinds, dy, None, dtype, grads, eps)


ALL = ("w", "b", "scale", "post_w", "post_b", "h")


# one row and channel to rows of every width class (16 to 1024 lanes, one and two runs), whole vectors and odd ones
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (5, 7), (70, 96), (33, 128), (17, 129), (9, 255), (40, 256), (21, 500), (12, 768), (6, 1000), (7, 1024), (5, 1027),
                                       (4, 2048), (3, 4096), (3, 4099), (2, 8192), (2, 8200), (2, 16384), (1, 12345)])
def test_widths(ss, dtype, rows, cols):
    _run(ss, rows, cols, dtype, (1, 0) if cols > 1 else (2, 0), None, ALL, rows + cols)
    _run(ss, rows, cols, dtype, (2, 2), (rows, cols), ALL, rows + cols + 1)


@pytest.mark.parametrize("kinds", [k for k in itertools.product((0, 1, 2), (0, 1, 2))])
@pytest.mark.parametrize("gate", [None, (60, 1), (60, 72), (12, 1), (12, 72), (1, 1), (1, 72), (30, 1), (30, 72)])
def test_kinds_and_gates(ss, kinds, gate):
    _run(ss, 60, 72, torch.bfloat16 if gate is None or gate[1] == 1 else torch.float32, kinds, gate, ALL, 10 * kinds[0] + kinds[1])


@pytest.mark.parametrize("parts", [("w", "b"), ("w",), (), ("h",), ("h", "scale"), ("h", "w", "post_w"), ("h", "b", "post_b", "scale")])
@pytest.mark.parametrize("kinds", [(1, 0), (2, 0), (1, 2), (2, 1)])
def test_missing_operands(ss, parts, kinds):
    if "h" not in parts:
        kinds = (kinds[0], 0)
    _run(ss, 37, 100, torch.float16, kinds, None, parts, len(parts))


# many workgroups, groups cut into strips, groups shared by a workgroup, groups of fewer rows than a workgroup takes at once
@pytest.mark.parametrize("rows,cols,gate", [(5000, 96, None), (6272, 96, (2, 1)), (6272, 40, (2, 40)), (9000, 64, (4500, 1)), (3000, 64, (1000, 64)), (4096, 200, (1, 200)),
                                            (2500, 520, (5, 1)), (1200, 1500, (3, 1500))])
def test_many_rows(ss, rows, cols, gate):
    _run(ss, rows, cols, torch.float32, (1, 2), gate, ALL, rows)


def test_a_mean_that_dwarfs_the_variance(ss):
    """Rows around 100 with unit variance: the variance is a mean of squared differences, not a difference of large sums."""
    _run(ss, 64, 384, torch.float32, (1, 0), None, ALL, 5, offset=100.0)


def test_empty_and_constant_rows(ss):
    desc = ss.make_norm_desc(96, ss.SS_F16, ss.SS_NORM_LAYER, 1e-6, ss.SS_NORM_RMS, 1e-6)
    x = torch.zeros((4, 96), dtype=torch.float16, device="cuda")
    x[1] = 2.0
    h = torch.zeros_like(x)
    w, b = torch.full((96,), 3.0, device="cuda"), torch.linspace(0, 1, 96, device="cuda")
    gate = torch.zeros((4, 1), dtype=torch.float16, device="cuda")
    x_out, y = ss.ss_norm_fwd(desc, x, w, b, h, None, gate, w, None)
    assert torch.equal(x_out, x) and torch.equal(y, b.half().expand(4, 96))
    g = ss.ss_norm_bwd(desc, torch.zeros_like(x), x_out, w, b, h, None, gate, w, None)
    assert all((v == 0).all() for v in g if v is not None)
    none = ss.ss_norm_fwd(desc, x[:0], w, b, h[:0])
    assert none[0].shape == none[1].shape == (0, 96)
    g = ss.ss_norm_bwd(desc, x[:0], x[:0], w, b, h[:0], w, None, w, None)
    assert g.dx.shape == (0, 96) and all((v == 0).all() and v.shape == (96,) for v in (g.dw, g.db, g.dscale, g.dpost_w))


def test_a_nan_stays_in_its_row(ss):
    for cols in (64, 500, 3000):
        p, dy, dx_out = _draw(20, cols, torch.float32, (20, 1), cols)
        desc = ss.make_norm_desc(cols, ss.SS_F32, ss.SS_NORM_LAYER, 1e-6, ss.SS_NORM_RMS, 1e-6)
        names = ("w", "b", "h", "scale", "gate", "post_w", "post_b")
        clean = ss.ss_norm_fwd(desc, p["x"], *(p[n] for n in names))
        p["x"][3, 5] = float("nan")
        p["h"][11, 0] = float("inf")
        bad = ss.ss_norm_fwd(desc, p["x"], *(p[n] for n in names))
        keep = [i for i in range(20) if i not in (3, 11)]
        for a, c in zip(bad, clean):
            assert torch.equal(a[keep], c[keep])
        assert torch.isnan(bad[1][[3, 11]]).all()
        grads = ss.ss_norm_bwd(desc, dy, clean[0], *(p[n] for n in names), dx_out=dx_out)      # h's infinity: its own row of dh, and the sums
        assert torch.isfinite(grads.dx).all() and torch.isfinite(grads.dh[keep]).all() and torch.isfinite(grads.dw).all()


def test_views_in_place_streams_and_graph(ss):
    p, dy, dx_out = _draw(50, 100, torch.bfloat16, (50, 1), 8)
    desc = ss.make_norm_desc(100, ss.SS_BF16, ss.SS_NORM_RMS, 1e-6)
    want = ss.ss_norm_fwd(desc, p["x"], p["w"], None, p["h"], p["scale"], p["gate"])
    wide = torch.zeros((50, 111), dtype=torch.bfloat16, device="cuda")
    wide[:, 5:105] = p["x"]
    y = torch.full((50, 120), 9.0, dtype=torch.bfloat16, device="cuda")
    h = torch.zeros((50, 203), dtype=torch.bfloat16, device="cuda")
    h[:, 101:201] = p["h"]
    got = ss.ss_norm_fwd(desc, wide[:, 5:105], p["w"], None, h[:, 101:201], p["scale"], p["gate"], x_out=wide[:, 5:105], y=y[:, 7:107])   # the stream in place
    assert torch.equal(wide[:, 5:105], want[0]) and torch.equal(got[1], want[1])
    assert (wide[:, :5] == 0).all() and (wide[:, 105:] == 0).all() and (y[:, :7] == 9).all() and (y[:, 107:] == 9).all()
    images = p["x"].view(5, 5, 2, 100)
    out = ss.ss_norm_fwd(desc, images, p["w"], None, p["h"].view(5, 5, 2, 100), p["scale"], p["gate"].view(5, 5, 2, 1))
    assert out[0].shape == images.shape and torch.equal(out[1].view(50, 100), want[1])
    grads = ss.ss_norm_bwd(desc, dy, want[0], p["w"], None, p["h"], p["scale"], p["gate"], dx_out=dx_out)
    again = ss.ss_norm_bwd(desc, torch.nn.functional.pad(dy, (1, 2))[:, 1:101], wide[:, 5:105], p["w"], None, h[:, 101:201], p["scale"], p["gate"], dx_out=dx_out)
    assert all(torch.equal(a, b) for a, b in zip(grads, again) if a is not None)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = ss.ss_norm_fwd(desc, p["x"], p["w"], None, p["h"], p["scale"], p["gate"], stream=stream)
    back = ss.ss_norm_bwd(desc, dy, other[0], p["w"], None, p["h"], p["scale"], p["gate"], dx_out=dx_out, stream=stream)
    stream.synchronize()
    assert torch.equal(other[1], want[1]) and all(torch.equal(a, b) for a, b in zip(grads, back) if a is not None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x_out, y = ss.ss_norm_fwd(desc, p["x"], p["w"], None, p["h"], p["scale"], p["gate"])
        grads = ss.ss_norm_bwd(desc, dy, x_out, p["w"], None, p["h"], p["scale"], p["gate"], dx_out=dx_out)
    for _ in range(4):
        p["x"].mul_(0.7)
        eager = ss.ss_norm_fwd(desc, p["x"], p["w"], None, p["h"], p["scale"], p["gate"])
        eager = (*eager, *ss.ss_norm_bwd(desc, dy, eager[0], p["w"], None, p["h"], p["scale"], p["gate"], dx_out=dx_out))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((x_out, y, *grads), eager) if a is not None)


def test_rows_beyond_32_bit_offsets(ss):
    pitch = (1 << 30) + 8
    buffer = torch.zeros(2 * pitch + 64, dtype=torch.float16, device="cuda")
    far = buffer.as_strided((3, 64), (pitch, 1))
    p, dy, _ = _draw(3, 64, torch.float16, None, 4)
    desc = ss.make_norm_desc(64, ss.SS_F16)
    far.copy_(p["x"])
    want = ss.ss_norm_fwd(desc, p["x"], p["w"], p["b"])
    assert torch.equal(ss.ss_norm_fwd(desc, far, p["w"], p["b"]), want)
    grads, near = (ss.ss_norm_bwd(desc, dy, x, p["w"], p["b"]) for x in (far, p["x"]))
    assert torch.equal(grads.dx, near.dx) and torch.equal(grads.dw, near.dw)
    ss.ss_norm_fwd(desc, p["x"], p["w"], p["b"], y=far)
    assert torch.equal(far.contiguous(), want)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", [(1, 32), (50, 96), (7, 100), (3, 768), (2, 1111), (3, 4096), (1, 16384)])
def test_quantised_output(ss, dtype, rows, cols):
    """y in MXFP4, quantised from fp32: an element may differ from the definition's only where that lies on a halfway point within the norm's bound, and a
    scale only where the largest is at a power of two."""
    p, _, _ = _draw(rows, cols, dtype, None, cols)
    desc = ss.make_norm_desc(cols, getattr(ss, DTYPES[dtype]), ss.SS_NORM_LAYER, 1e-6)
    x_out, codes, scales = ss.ss_norm_mx4_fwd(desc, p["x"], p["w"], p["b"], p["h"], p["scale"])
    assert torch.equal(x_out, ss.ss_norm_fwd(desc, p["x"], p["w"], p["b"], p["h"], p["scale"])[0])
    q = _wide(p)
    xo, y = ref.block_forward(q, (1, 0))
    bound = _slack(xo, 1, q["w"], q["b"], 1e-6) + _gain(xo, 1, q["w"], 1e-6) * 16 * ref.U32 * (np.abs(q["x"]) + np.abs(q["h"])).max(axis=1, keepdims=True)
    low, high = ref.through_mx4(y - bound), ref.through_mx4(y + bound)
    got = ref.dequantize(codes.cpu().numpy(), scales.cpu().numpy(), cols)
    assert codes.shape == (rows, -(-cols // 32) * 16) and scales.shape == (rows, -(-cols // 128) * 4)
    kb = -(-cols // 32)
    assert (scales.cpu().numpy()[:, kb:] == 0).all()
    settled = (low == high)
    tops = np.zeros((rows, kb * 32))
    tops[:, :cols] = np.abs(y)
    btop = np.zeros((rows, kb * 32))
    btop[:, :cols] = bound
    tops, btop = tops.reshape(rows, kb, 32).max(axis=-1), btop.reshape(rows, kb, 32).max(axis=-1)
    same_scale = np.frexp(tops - btop)[1] == np.frexp(tops + btop)[1]
    settled &= np.repeat(same_scale, 32, axis=1)[:, :cols]
    assert settled.mean() > 0.98
    want = ref.through_mx4(y)
    assert np.array_equal(got[settled], want[settled])
    alone = ss.ss_norm_mx4_fwd(desc, p["x"], p["w"], p["b"])
    assert len(alone) == 2 and alone[0].shape == codes.shape


def test_refusals(ss):
    p, dy, dx_out = _draw(8, 64, torch.float16, (8, 1), 1)
    desc = ss.make_norm_desc(64, ss.SS_F16, ss.SS_NORM_LAYER, 1e-6, ss.SS_NORM_RMS, 1e-6)
    bare = ss.make_norm_desc(64, ss.SS_F16, ss.SS_NORM_LAYER, 1e-6)
    none = ss.make_norm_desc(64, ss.SS_F16, ss.SS_NORM_NONE)
    x, h, w = p["x"], p["h"], p["w"]

    def refused(call, *a, status=ss.SS_ERR_INVALID_ARG, **k):
        with pytest.raises(ss.SSError) as e:
            call(*a, **k)
        assert e.value.status == status

    refused(ss.ss_norm_fwd, desc, x.bfloat16(), w, None, h)
    refused(ss.ss_norm_fwd, desc, x.cpu(), w, None, h)
    refused(ss.ss_norm_fwd, desc, x[:, :63], w, None, h)
    refused(ss.ss_norm_fwd, desc, x, w[:63], None, h)
    refused(ss.ss_norm_fwd, desc, x, w.half(), None, h)
    refused(ss.ss_norm_fwd, desc, x, w, None, h[:4])
    refused(ss.ss_norm_fwd, desc, x, w, None, h, None, p["gate"][:3])                 # 3 does not divide 8
    refused(ss.ss_norm_fwd, desc, x, w, None, h, None, p["gate"].float())
    refused(ss.ss_norm_fwd, desc, x, w)                                             # a norm of a block that is not there
    refused(ss.ss_norm_fwd, bare, x, w, None, None, w)
    refused(ss.ss_norm_fwd, bare, x, w, None, None, None, p["gate"])
    refused(ss.ss_norm_fwd, none, x)
    refused(ss.ss_norm_fwd, ss.make_norm_desc(64, ss.SS_F16, 7), x, w)
    refused(ss.ss_norm_fwd, ss.make_norm_desc(64, ss.SS_F16, eps=-1e-6), x, w)
    refused(ss.ss_norm_fwd, bare, x.t())
    refused(ss.ss_norm_fwd, bare, x, y=torch.empty((8, 64), device="cuda"))
    refused(ss.ss_norm_mx4_fwd, bare, x, w, None, codes=torch.empty((8, 16), dtype=torch.uint8, device="cuda"))
    refused(ss.ss_norm_mx4_fwd, none, x, None, None, h)
    wide = torch.empty((2, 16400), dtype=torch.float16, device="cuda")
    refused(ss.ss_norm_fwd, ss.make_norm_desc(16400, ss.SS_F16), wide, status=ss.SS_ERR_UNSUPPORTED)
    refused(ss.ss_norm_bwd, bare, None, x, w)
    refused(ss.ss_norm_bwd, bare, dy, None, w)
    refused(ss.ss_norm_bwd, bare, dy[:4], x, w)
    refused(ss.ss_norm_bwd, bare, dy, x, w, None, None, w)
    refused(ss.ss_norm_bwd, desc, dy, x, w, None, h, None, p["gate"][:3])
    refused(ss.ss_norm_bwd, none, None, None, None, None, h)
    refused(ss.ss_norm_bwd, none, dy, x, None, None, h, dx_out=dx_out)
    refused(ss.ss_norm_bwd, desc, dy, x, w, None, h, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), status=ss.SS_ERR_WORKSPACE)
