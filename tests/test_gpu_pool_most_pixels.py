"""Max pooling of more outputs than one launch has threads for (2^32, eight channels each): every one is written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_every_output(ss):
    side = 46341                                                 # (two images of side^2 pixels are just over 2^32)
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 170 << 30:
        pytest.skip("needs 170 GB of free device memory")
    x = torch.empty((2, side, side, 8), dtype=torch.float16, device="cuda")
    y = torch.full_like(x, float("nan"))
    for n in range(2):
        for at in range(0, side, 4096):
            x[n, at:at + 4096].view(torch.int16).copy_(torch.randint(0, 20000, x[n, at:at + 4096].shape, dtype=torch.int16, device="cuda"))
    ss.ss_maxpool2d(x, 1, 1, 0, y=y)                              # a window of one pixel: the input itself
    for n in range(2):
        for at in range(0, side, 4096):
            assert torch.equal(y[n, at:at + 4096].view(torch.int16), x[n, at:at + 4096].view(torch.int16)), (n, at)
    del x, y
    torch.cuda.empty_cache()
