"""Quantisation and the pointwise MXFP4 layer on more rows than one launch has threads for (2^32), which the calls take up to 2^31 - 1 rows of.

Values are small integers and halves that MXFP4 holds, so that quantisation loses nothing and the sums are exact: every row is compared for equality."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS = (1 << 30) + (1 << 26) + 77
STEP = 1 << 26


@pytest.fixture
def memory():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def test_every_row(ss, memory, force_tile):
    cin, cout = 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((ROWS, cin), dtype=torch.float16, device="cuda")
    for at in range(0, ROWS, STEP):
        part = x[at:at + STEP]
        part.copy_(torch.randint(-4, 5, part.shape, generator=g, dtype=torch.int8, device="cuda"))
    codes = torch.full((ROWS, 16), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((ROWS, 4), 0xAA, dtype=torch.uint8, device="cuda")
    ss.ss_mx4_quantize(x, codes, scales)
    back = ss.ss_mx4_dequantize(codes, scales, cin, torch.float16)
    for at in range(0, ROWS, STEP):
        assert bool((back[at:at + STEP] == x[at:at + STEP]).all()), at
        assert not bool((scales[at:at + STEP, 1:] != 0).any()) and not bool((codes[at:at + STEP, 4:] != 0).any()), at
    del back
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16)
    W = torch.randint(-1, 2, (cout, cin), generator=g, device="cuda").half()
    packed = ss.ss_mx4_pack(desc, W)
    bias = torch.arange(cout, device="cuda").float()
    wide = W.float().t().contiguous()
    y = torch.empty((ROWS, cout), dtype=torch.float16, device="cuda")

    def check(what):
        for at in range(0, ROWS, STEP):
            want = (x[at:at + STEP].float() @ wide + bias).half()
            assert bool((y[at:at + STEP] == want).all()), (what, at)

    for kernel in (None, 70, 71, 72):
        force_tile(kernel)
        y.fill_(float("nan"))
        ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, bias, None, 0, y)
        check(kernel)
    for kernel in (None, 76, 77):
        force_tile(kernel)
        y.fill_(float("nan"))
        ss.ss_pw_mx4_fwd(desc, x, packed, bias, None, 0, y)
        check(kernel)
    force_tile(None)
    y.copy_(x)                                                    # a residual that is the output, in every piece
    ss.ss_pw_mx4_fwd(desc, x, packed, bias, y, 0, y)
    for at in range(0, ROWS, STEP):
        part = x[at:at + STEP].float()
        assert bool((y[at:at + STEP] == (part @ wide + bias + part).half()).all()), at
