"""The pointwise layer on FP8 blocks over odd numbers of reduction steps (of 64): half a block behind one, two or three whole ones, and behind a loop of four."""
import pytest
import torch

import f8_reference as ref
from test_gpu_f8_blocks import KERNELS, bound, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel", [None, *KERNELS])
@pytest.mark.parametrize("rows,cin,cout,dtype", [(130, 192, 130, torch.bfloat16), (300, 320, 260, torch.float16), (64, 448, 96, torch.bfloat16), (257, 576, 257, torch.float16),
                                                 (515, 704, 300, torch.bfloat16), (100, 810, 65, torch.float16), (290, 960, 513, torch.bfloat16), (200, 1045, 70, torch.float16)])
def test_odd_steps(ss, force_tile, kernel, rows, cin, cout, dtype):
    assert -(-cin // 64) % 2 == 1
    g = gen(rows + cin + cout)
    # every block of a size of its own, so that another's codes or scales in its place are no small error
    size = torch.exp2(torch.arange(-(-cin // 128)) * 5 % 9 - 4.0).repeat_interleave(128)[:cin]
    x, W = (torch.randn((rows, cin), generator=g) * size).to(dtype), (torch.randn((cout, cin), generator=g) / size).to(dtype)
    bias = torch.randn(cout, generator=g)
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == torch.float16 else ss.SS_BF16)
    packed = ss.ss_f8_pack(desc, W.cuda())
    Wq, xq = ref.quantize(W)[2], ref.quantize(x)[2]
    want = xq @ Wq.t() + bias.double()
    tol = bound(Wq, xq, want, dtype, cin)
    force_tile(None if kernel is None else KERNELS[kernel])
    codes, scales = ss.ss_f8_quantize(x.cuda())
    for y in (ss.ss_pw_f8_q_fwd(desc, codes, scales, packed, bias.cuda()), ss.ss_pw_f8_fwd(desc, x.cuda(), packed, bias.cuda())):
        assert ((y.cpu().double() - want).abs() <= tol).all()
