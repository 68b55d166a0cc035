"""Norms around a block at the edges of their arguments: no rows, vectors that have no meaning in the call."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {torch.float16: "SS_F16", torch.bfloat16: "SS_BF16", torch.float32: "SS_F32"}


def _poison(shape, dtype):
    """Leaves NaN in the memory that the next allocation of this shape is likely to get."""
    torch.full(shape, float("nan"), dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", [(1, 1), (4, 1), (4, 96), (700, 96)])
@pytest.mark.parametrize("stream", [False, True])
def test_gradient_of_a_gate_that_saw_no_rows(ss, dtype, shape, stream):
    """x [0, 96] with a gate that has rows: its gradient is a sum over nothing."""
    desc = ss.make_norm_desc(96, getattr(ss, DTYPES[dtype]))
    none = torch.empty((0, 96), dtype=dtype, device="cuda")
    w, gate = torch.ones(96, device="cuda"), torch.ones(shape, dtype=dtype, device="cuda")
    _poison(shape, dtype)
    g = ss.ss_norm_bwd(desc, none, none, w, None, none, w, gate, dx_out=none, stream=torch.cuda.current_stream() if stream else None)
    assert g.dgate.shape == shape and g.dgate.dtype == dtype and (g.dgate == 0).all()
    assert (g.dw == 0).all() and (g.dscale == 0).all() and g.dx.shape == g.dh.shape == (0, 96)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("gate_cols", [1, 96])
@pytest.mark.parametrize("vectors", [False, True])
def test_no_rows_at_the_c_interface(ss, dtype, gate_cols, vectors):
    """The call itself writes the gate's zeros, with and without the channel vectors' next to them."""
    from paper_2411_00288_amd import binding
    desc = ss.make_norm_desc(96, getattr(ss, DTYPES[dtype]))
    row = torch.zeros(96, dtype=dtype, device="cuda")
    gate, dgate = (torch.ones((1500, gate_cols), dtype=dtype, device="cuda") for _ in range(2))
    dw = torch.ones(96, device="cuda")
    io = binding.ss_norm_grad_io(rows=0, groups=1499, gate_cols=gate_cols)
    for name in ("dy", "x_out", "h", "dx", "dh"):
        setattr(io, name, row.data_ptr())
        setattr(io, f"ld{name}", 96)
    io.gate, io.dgate = gate.data_ptr(), dgate.data_ptr()
    if vectors:
        io.dw = dw.data_ptr()
    call = lambda: binding._lib.ss_norm_bwd(ctypes.byref(desc), ctypes.byref(io), None, 0, binding._stream_ptr())
    assert call() == ss.SS_OK
    torch.cuda.synchronize()
    assert (dgate[:1499] == 0).all() and (dgate[1499] == 1).all() and (dw == (0 if vectors else 1)).all()      # (and nothing behind the gate)
    io.groups = -1
    assert call() == ss.SS_ERR_INVALID_ARG
    io.groups = 2 ** 31
    assert call() == ss.SS_ERR_UNSUPPORTED
