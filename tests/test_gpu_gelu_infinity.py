"""GELU of infinities: z Phi(z) has the limits +infinity at +infinity and 0 at -infinity.  In every kernel that has the activation; the other channels do not
notice."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [(torch.float16, "SS_F16"), (torch.bfloat16, "SS_BF16")]
INF = float("inf")


def _bias(cout):
    """A bias whose first channels are an infinity of either sign, a NaN, and the largest finite value; and GELU of it."""
    b = torch.linspace(-3, 3, cout, device="cuda")
    b[:4] = torch.tensor([INF, -INF, float("nan"), 3.4e38])
    want = b.double()
    want = want * torch.special.ndtr(want)
    want[0], want[1] = INF, 0.0
    return b, want


def _check(y, want, dtype):
    """Every row of y is GELU of the bias, up to the output's rounding and the 1e-7 of Phi."""
    y, want = y.reshape(-1, y.shape[-1]), want.to(dtype)
    assert torch.equal(torch.isnan(y), torch.isnan(want).expand_as(y))
    assert torch.equal(torch.isinf(y), torch.isinf(want).expand_as(y)) and (y[:, 0] == INF).all()
    at = torch.isfinite(want)
    got, ref = y[:, at].double(), want[at].double()
    assert ((got - ref).abs() <= torch.finfo(dtype).eps * ref.abs() + 1e-6).all()


@pytest.mark.parametrize("dtype,code", TYPES)
@pytest.mark.parametrize("kernel", range(70, 79))
@pytest.mark.parametrize("rows,cin,cout", [(32, 64, 128), (300, 96, 72)])
def test_pointwise_4bit(ss, force_tile, dtype, code, kernel, rows, cin, cout):
    desc = ss.make_desc(cout, cin, 1, 1, getattr(ss, code))
    packed = ss.ss_mx4_pack(desc, torch.zeros((cout, cin), dtype=dtype, device="cuda"))
    x = torch.randn((rows, cin), device="cuda").to(dtype)
    bias, want = _bias(cout)
    codes, scales = ss.ss_mx4_quantize(x)
    force_tile(kernel)
    y = ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, bias, None, ss.SS_ACT_GELU) if kernel < 75 else ss.ss_pw_mx4_fwd(desc, x, packed, bias, None, ss.SS_ACT_GELU)
    _check(y, want, dtype)
    residual = torch.zeros((rows, cout), dtype=dtype, device="cuda")
    residual[-1, 5], residual[0, 6] = INF, -INF
    zero = torch.zeros(cout, device="cuda")
    y = (ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, zero, residual, ss.SS_ACT_GELU) if kernel < 75
         else ss.ss_pw_mx4_fwd(desc, x, packed, zero, residual, ss.SS_ACT_GELU))
    assert y[-1, 5] == INF and y[0, 6] == 0 and int((y == 0).sum()) == rows * cout - 1


@pytest.mark.parametrize("dtype,code", TYPES)
@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("N,H,W,cin,cout,k", [(1, 1, 1, 32, 64, 1), (1, 4, 4, 256, 64, 1), (1, 9, 9, 32, 40, 3), (2, 56, 56, 64, 256, 1), (8, 28, 28, 64, 64, 3)])
def test_convolution(ss, dtype, code, sparse, N, H, W, cin, cout, k):
    desc = ss.make_desc(cout, cin, k, k, getattr(ss, code))
    W0 = torch.zeros((cout, cin * k * k), dtype=dtype, device="cuda")
    M = torch.tensor([1, 0, 1, 0], dtype=torch.uint8, device="cuda").repeat(cout, cin * k * k // 4)
    x = torch.randn((N, H, W, cin), device="cuda").to(dtype)
    bias, want = _bias(cout)
    pad = (k // 2, k // 2)
    y = (ss.ss_conv2d_fwd(desc, x, ss.ss_mask_compress(desc, W0, M), bias, (1, 1), pad, ss.SS_ACT_GELU) if sparse
         else ss.ss_conv2d_dense_fwd(desc, x, ss.ss_dense_pack(desc, W0, M), bias, (1, 1), pad, ss.SS_ACT_GELU))
    _check(y, want, dtype)


@pytest.mark.parametrize("C,N,H", [(96, 1, 7), (96, 1, 56), (96, 8, 112), (64, 2, 30), (128, 4, 56)])
def test_between_two_layers(ss, C, N, H):
    """An infinity in the intermediate of the inverted bottleneck: it reaches every output through the second layer's positive weights."""
    dtype = torch.bfloat16
    one, two = ss.make_desc(4 * C, C, 1, 1, ss.SS_BF16), ss.make_desc(C, 4 * C, 1, 1, ss.SS_BF16)
    first = ss.ss_dense_pack(one, torch.zeros((4 * C, C), dtype=dtype, device="cuda"), None)
    second = ss.ss_dense_pack(two, torch.ones((C, 4 * C), dtype=dtype, device="cuda"), None)
    bias = torch.zeros(4 * C, device="cuda")
    x = torch.randn((N, H, H, C), device="cuda").to(dtype)
    call = lambda: ss.ss_conv2d_pw_fused_dense_fwd(one, x, first, bias, (1, 1), (0, 0), ss.SS_ACT_GELU, two, second, torch.zeros(C, device="cuda"))
    assert (call() == 0).all()
    bias[17] = INF
    assert (call() == INF).all()
