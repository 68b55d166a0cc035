"""Norms around a block, and their gradient, on tensors beyond the last-level cache (more than 256 MB read and written), whose lines the kernels do not keep: every row, column
sum and gate against the definition in fp64 on the GPU.  Every width class of the kernels, without a block output too; bounds as in test_gpu_norm.py."""
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = {torch.float16: "SS_F16", torch.bfloat16: "SS_BF16", torch.float32: "SS_F32"}
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U, C = ref.U32, 128 * ref.U32
EPS = (1e-6, 1e-5)
LARGE = 256 << 20


def _top(v):
    return v.abs().amax(dim=1, keepdim=True)


def _statistics(v, kind, eps):
    d = v - v.mean(dim=1, keepdim=True) if kind == 1 else v
    return d, 1.0 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + eps)


def _norm(v, kind, w, b, eps):
    if kind == 0:
        return v
    d, r = _statistics(v, kind, eps)
    return d * r * w + b


def _slack(v, kind, w, b, eps):
    if kind == 0:
        return 0.0
    _, r = _statistics(v, kind, eps)
    return C * (_top(v) * r * w.abs() * 2 + b.abs())


def _close(got, want, bound, dtype, what):
    unit, tiny = ref.ROUND[dtype], ref.TINY[dtype]
    over = (got.double() - want).abs() - (bound * (1 + unit) + unit * want.abs() + tiny)
    assert bool((over <= 0).all()), (what, float(over.max()), torch.nonzero(~(over <= 0))[:3].tolist())


class Case:
    def __init__(self, ss, rows, cols, dtype, kinds, gate, block=True, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.rows, self.cols, self.dtype, self.kinds = rows, cols, dtype, kinds
        self.x = t(rows, cols).to(dtype)
        self.w, self.b = (1 + 0.2 * t(cols), t(cols)) if kinds[0] else (None, None)
        self.h = self.scale = self.gate = self.post_w = self.post_b = None
        if block:
            self.h, self.scale = (1.5 * t(rows, cols)).to(dtype), 0.3 * t(cols)
            self.gate = None if gate is None else t(*gate).to(dtype)
            if kinds[1]:
                self.post_w, self.post_b = 1 + 0.2 * t(cols), 0.2 * t(cols)
        self.dy, self.dx_out = t(rows, cols).to(dtype) if kinds[0] else None, t(rows, cols).to(dtype)
        self.desc = ss.make_norm_desc(cols, getattr(ss, DTYPES[dtype]), kinds[0], EPS[0], kinds[1], EPS[1])

    def operands(self):
        return self.w, self.b, self.h, self.scale, self.gate, self.post_w, self.post_b

    def wide(self, name, first, last):
        v = getattr(self, name)
        if v is None:
            return None
        if name == "gate":
            per = self.rows // v.shape[0]
            return v.double()[torch.arange(first, last, device="cuda") // per]
        return v.double() if v.dim() == 1 else v[first:last].double()

    def pieces(self):
        """Rows in whole groups of the gate, at most about 32 million values of each tensor in fp64 at once."""
        per = 1 if self.gate is None else self.rows // self.gate.shape[0]
        step = max(1, (32 << 20) // self.cols // per) * per
        return [(at, min(at + step, self.rows)) for at in range(0, self.rows, step)]


def _check_forward(case, out):
    x_out, y = out if isinstance(out, tuple) else (out, None) if case.kinds[0] == 0 else (None, out)
    for a, z in case.pieces():
        p = {n: case.wide(n, a, z) for n in ("x", "h", "w", "b", "scale", "gate", "post_w", "post_b")}
        want, bound = p["x"], torch.zeros((), dtype=torch.float64, device="cuda")
        if p["h"] is not None:
            factor = p["scale"] * (1.0 if p["gate"] is None else p["gate"])
            u = _norm(p["h"], case.kinds[1], p["post_w"], p["post_b"], EPS[1])
            bound = factor.abs() * _slack(p["h"], case.kinds[1], p["post_w"], p["post_b"], EPS[1]) + 4 * U * (p["x"].abs() + 2 * (factor * u).abs())
            want = p["x"] + factor * u
            _close(x_out[a:z], want, bound, case.dtype, "x_out")
            bound = _top(bound)
        if case.kinds[0]:
            d, r = _statistics(want, case.kinds[0], EPS[0])
            gain = 3 * r * p["w"].abs() * (1 + (d * r).abs())
            _close(y[a:z], d * r * p["w"] + p["b"], gain * bound + _slack(want, case.kinds[0], p["w"], p["b"], EPS[0]), case.dtype, "y")


def _check_backward(case, grads):
    kinds, rows = case.kinds, case.rows
    sums = {}

    def add(name, want, bound):
        old = sums.get(name, (0.0, 0.0))
        sums[name] = (old[0] + want.sum(dim=0), old[1] + bound.sum(dim=0))

    def through(v, kind, g_out, w, error, eps, names):
        """(dv, its bound) of a norm for an incoming gradient that is off by `error`; adds its vectors' gradients."""
        d, r = _statistics(v, kind, eps)
        xh, g = d * r, g_out * w
        dv = r * (g - xh * (g * xh).mean(dim=1, keepdim=True) - (g.mean(dim=1, keepdim=True) if kind == 1 else 0.0))
        top = (_top(v) * r + 1) * (1 + _top(xh))
        mag = g_out.abs()
        add(names[0], g_out * xh, mag * top * 2 * C + error * top + rows * U * mag * xh.abs())
        add(names[1], g_out, error + rows * U * mag)
        return dv, r * top * (4 * C * _top(g) + 3 * _top(error * w.abs()))

    gates = []
    for a, z in case.pieces():
        p = {n: case.wide(n, a, z) for n in ("x", "h", "w", "scale", "gate", "post_w", "post_b", "dy", "dx_out")}
        t, dt = p["dx_out"], torch.zeros_like(p["dx_out"])
        if kinds[0]:
            dv, dt = through(p["x"], kinds[0], p["dy"], p["w"], dt, EPS[0], ("dw", "db"))
            t = t + dv
        dt = dt + 4 * U * t.abs()
        _close(grads.dx[a:z], t, dt, case.dtype, "dx")
        if p["h"] is None:
            continue
        u = _norm(p["h"], kinds[1], p["post_w"], p["post_b"], EPS[1])
        du = _slack(p["h"], kinds[1], p["post_w"], p["post_b"], EPS[1]) + 4 * U * u.abs()
        gate = torch.ones((), dtype=torch.float64, device="cuda") if p["gate"] is None else p["gate"]
        product = dt * u.abs() + t.abs() * du + 4 * U * (t * u).abs()
        add("dscale", t * gate * u, (product + rows * U * (t * u).abs()) * gate.abs())
        if p["gate"] is not None:
            per = rows // case.gate.shape[0]
            fold = lambda v: v.reshape((z - a) // per, per, case.cols).sum(dim=1)
            want, bound = fold(t * p["scale"] * u), fold((product + (per + 64) * U * (t * u).abs()) * p["scale"].abs())
            one = case.gate.shape[1] == 1
            gates.append((want.sum(dim=1, keepdim=True), bound.sum(dim=1, keepdim=True)) if one else (want, bound))
        factor = p["scale"] * gate
        g, ge = t * factor, dt * factor.abs() + 4 * U * (t * factor).abs()
        if kinds[1]:
            g, ge = through(p["h"], kinds[1], g, p["post_w"], ge, EPS[1], ("dpost_w", "dpost_b"))
        _close(grads.dh[a:z], g, ge, case.dtype, "dh")
    for name, (want, bound) in sums.items():
        _close(getattr(grads, name), want, bound, F32, name)
    if gates:
        _close(grads.dgate, torch.cat([w for w, _ in gates]), torch.cat([b for _, b in gates]), case.dtype, "dgate")


def _run(ss, case, forward=True):
    item = 4 if case.dtype == F32 else 2
    n = case.rows * case.cols * item
    if forward:
        assert n * (4 if case.h is not None else 2) > LARGE and case.cols % 8 == 0
        _check_forward(case, ss.ss_norm_fwd(case.desc, case.x, *case.operands()))
    assert n * (6 if case.h is not None else 4) > LARGE
    x_out = case.x if case.kinds[0] else None
    grads = ss.ss_norm_bwd(case.desc, case.dy, x_out, *case.operands(), dx_out=case.dx_out)
    _check_backward(case, grads)
    again = ss.ss_norm_bwd(case.desc, case.dy, x_out, *case.operands(), dx_out=case.dx_out)
    assert all(torch.equal(u, v) for u, v in zip(grads, again) if u is not None)


# rows of 16 to 1024 lanes, one and two runs to the lane
WIDTHS = [(401408, 96), (200704, 192), (140000, 256), (90000, 384), (70000, 512), (36000, 1000), (20000, 2048), (9000, 4096), (4400, 8192), (2200, 16384), (2800, 12344)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", WIDTHS)
def test_widths(ss, dtype, rows, cols):
    _run(ss, Case(ss, rows, cols, dtype, (1, 0), None))
    _run(ss, Case(ss, rows, cols, dtype, (2, 1), (rows // 8, cols)))


@pytest.mark.parametrize("kinds", [(a, b) for a in (0, 1, 2) for b in (0, 1, 2)])
@pytest.mark.parametrize("gate", [(128, 1), (128, 96), (401408, 1), (401408, 96)])
def test_kinds_and_gates(ss, kinds, gate):
    _run(ss, Case(ss, 401408, 96, BF16, kinds, gate, seed=sum(kinds) + gate[0]))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rows,cols", [(800000, 96), (100000, 768), (17000, 4096)])
def test_without_a_block_output(ss, dtype, kind, rows, cols):
    _run(ss, Case(ss, rows, cols, dtype, (kind, 0), None, block=False))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", [(401408, 96), (100000, 768), (20000, 4096)])
def test_quantised_output(ss, dtype, rows, cols):
    """The MXFP4 form is that of a part of the rows, which is small enough for the other kernels: the rows do not know of each other."""
    case = Case(ss, rows, cols, dtype, (1, 0), None)
    x_out, codes, scales = ss.ss_norm_mx4_fwd(case.desc, case.x, *case.operands())
    for a in (0, rows // 2 - 100, rows - 700):
        part = ss.ss_norm_mx4_fwd(case.desc, case.x[a:a + 700], case.w, case.b, case.h[a:a + 700], case.scale)
        assert all(torch.equal(v[a:a + 700], p) for v, p in zip((x_out, codes, scales), part))


def test_in_place_and_inside_wider_tensors(ss):
    """The stream in place, and operands at odd places of wider tensors."""
    case = Case(ss, 401408, 96, BF16, (1, 0), (128, 1))
    want = ss.ss_norm_fwd(case.desc, case.x, *case.operands())
    wide = torch.full((401408, 111), 9.0, dtype=BF16, device="cuda")
    wide[:, 5:101] = case.x
    got = ss.ss_norm_fwd(case.desc, wide[:, 5:101], *case.operands(), x_out=wide[:, 5:101], y=case.h)
    assert torch.equal(wide[:, 5:101], want[0]) and torch.equal(got[1], want[1]) and got[1].data_ptr() == case.h.data_ptr()
    assert bool((wide[:, :5] == 9).all()) and bool((wide[:, 101:] == 9).all())
