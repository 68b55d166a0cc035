"""The group norm in passes over few images of many channels: what many chunks leave is joined without the error of as many additions in 32 bits.

Values of one sign and of nearly one size, whose sums are rounded the same way at every addition, to the bounds of the other tests (64 + log2(m) additions to a value)."""
import pytest
import torch

from test_gpu_groupnorm import CODES, EPS, TYPES, check_backward, check_forward

pytestmark = pytest.mark.gpu

# images, height, width, channels, groups
SHAPES = [(1, 64, 64, 1280, 1), (1, 112, 112, 1032, 8), (1, 72, 64, 2048, 32), (1, 40, 40, 1100, 1100), (2, 24, 24, 16384, 2), (1, 150, 150, 264, 1)]


def values(seed, shape, dtype, around, spread):
    g = torch.Generator().manual_seed(seed)
    return (around + spread * torch.randn(shape, generator=g)).to(TYPES[dtype])


@pytest.mark.parametrize("spread", [0.0, 0.02])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward(ss, force_tile, shape, dtype, spread):
    n, h, wd, c, groups = shape
    x, dy = values(1, (n, h, wd, c), dtype, 0.7, spread), values(2, (n, h, wd, c), dtype, 0.1, spread)
    desc = ss.make_groupnorm_desc(c, groups, CODES[dtype], ss.SS_ACT_NONE, EPS)
    force_tile(96)
    w, b = torch.full((c,), 1.1), torch.full((c,), 0.3)
    y, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
    check_forward(x, w, b, groups, "none", y, stats)
    check_backward(x, dy, w, b, groups, "none", stats, ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda()))


def test_chunks_leave_little(ss):
    """What the chunks leave is an eighth of 16-bit data at most, and a group's no more than a workgroup joins at 128 values to the thread."""
    for images, pixels, c, groups in ((1, 112 * 112, 2048, 32), (1, 64 * 64, 1280, 1), (2, 96 * 96, 1000, 8), (1, 32 * 32, 16384, 32), (1, 512 * 512, 128, 32), (4, 64 * 64, 640, 2)):
        ws = ss.ss_groupnorm_workspace_bytes(ss.make_groupnorm_desc(c, groups, ss.SS_F32), images, pixels)
        if ws == 0:                                          # (held)
            continue
        assert ws <= images * (pixels * c * 2 // 8 + groups * 8) + 256
        assert ws / 8 <= images * groups * (128 * 1024 + 1) + 32
