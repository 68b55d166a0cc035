"""Tensors of rows in which some leading dimension is zero: no rows, whichever dimension it is, in every call that takes rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(0,), (0, 5), (3, 0), (3, 0, 7), (0, 0), (2, 3, 0), (0, 1), (1, 0)]


@pytest.mark.parametrize("lead", SHAPES)
@pytest.mark.parametrize("dtype,code", [(torch.float16, "SS_F16"), (torch.bfloat16, "SS_BF16"), (torch.float32, "SS_F32")])
def test_norms_and_quantisation(ss, lead, dtype, code):
    x = torch.empty((*lead, 64), dtype=dtype, device="cuda")
    codes, scales = ss.ss_mx4_quantize(x)
    assert codes.shape == (*lead, 32) and scales.shape == (*lead, 4)
    assert ss.ss_mx4_dequantize(codes, scales, 64, dtype).shape == x.shape
    w = torch.ones(64, device="cuda")
    desc = ss.make_norm_desc(64, getattr(ss, code))
    assert ss.ss_norm_fwd(desc, x, w).shape == x.shape
    out = ss.ss_norm_fwd(desc, x, w, w, x, w)
    assert out[0].shape == out[1].shape == x.shape
    assert ss.ss_norm_mx4_fwd(desc, x, w)[0].shape == codes.shape
    grads = ss.ss_norm_bwd(desc, x, x, w, w, x, w, dx_out=x)
    assert grads.dx.shape == grads.dh.shape == x.shape and all((v == 0).all() for v in (grads.dw, grads.db, grads.dscale))


@pytest.mark.parametrize("lead", SHAPES)
def test_pointwise(ss, lead):
    x = torch.empty((*lead, 64), dtype=torch.bfloat16, device="cuda")
    desc = ss.make_desc(40, 64, 1, 1, ss.SS_BF16)
    packed = ss.ss_mx4_pack(desc, torch.randn((40, 64), device="cuda").bfloat16())
    residual = torch.empty((*lead, 40), dtype=torch.bfloat16, device="cuda")
    assert ss.ss_pw_mx4_fwd(desc, x, packed, None, residual).shape == residual.shape
    assert ss.ss_pw_mx4_q_fwd(desc, *ss.ss_mx4_quantize(x), packed, None, residual, ss.SS_ACT_GELU).shape == residual.shape


def test_views_without_rows(ss):
    """Empty parts of wider tensors, with any strides; rows that are not there need no even spacing, those that are do."""
    wide = torch.zeros((4, 6, 100), dtype=torch.float16, device="cuda")
    for view in (wide[:, :0, 3:67], wide[:0, :, 3:67], wide.transpose(0, 1)[:, 2:2, :64]):
        assert ss.ss_mx4_quantize(view)[0].shape == (*view.shape[:-1], 32)
    with pytest.raises(ss.SSError):
        ss.ss_mx4_quantize(wide[:, :5, 3:67])
    with pytest.raises(ss.SSError):
        ss.ss_mx4_quantize(wide[:, :5, 3:67], stream=torch.cuda.current_stream())
