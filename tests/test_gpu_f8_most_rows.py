"""Quantisation and the pointwise layer on FP8 blocks on more rows than one launch has threads for (2^32): small integers, which the type holds, so that every row is
compared for equality."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS = (1 << 30) + (1 << 26) + 77
STEP = 1 << 26


def test_every_row(ss, force_tile):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 180 << 30:
        pytest.skip("needs 180 GB of free device memory")
    cin, cout = 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((ROWS, cin), dtype=torch.float16, device="cuda")
    for at in range(0, ROWS, STEP):
        part = x[at:at + STEP]
        part.copy_(torch.randint(-4, 5, part.shape, generator=g, dtype=torch.int8, device="cuda"))
    codes, scales = ss.ss_f8_quantize(x)
    y = torch.empty((ROWS, cout), dtype=torch.float16, device="cuda")
    ss.ss_f8_dequantize(codes, scales, cin, torch.float16, out=y)
    for at in range(0, ROWS, STEP):
        assert bool((y[at:at + STEP] == x[at:at + STEP]).all()), at
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16)
    W = torch.randint(-1, 2, (cout, cin), generator=g, device="cuda").half()
    packed, bias, wide = ss.ss_f8_pack(desc, W), torch.arange(cout, device="cuda").float(), W.float().t().contiguous()
    for kernel, call in ((80, lambda: ss.ss_pw_f8_q_fwd(desc, codes, scales, packed, bias, None, 0, y)), (None, lambda: ss.ss_pw_f8_fwd(desc, x, packed, bias, None, 0, y)),
                         (86, lambda: ss.ss_pw_f8_fwd(desc, x, packed, bias, None, 0, y))):
        force_tile(kernel)
        y.fill_(float("nan"))
        call()
        for at in range(0, ROWS, STEP):
            assert bool((y[at:at + STEP] == (x[at:at + STEP].float() @ wide + bias).half()).all()), (kernel, at)
    del x, y, codes, scales
    torch.cuda.empty_cache()
