"""The group norm where a workgroup holds its share, with up to 16 rows to the thread: enough images that the plan takes workgroups of 256 threads, in whole runs of channels and cut ones."""
import pytest
import torch

from test_gpu_groupnorm import ACTS, CODES, EPS, TYPES, check_backward, check_forward, data

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("channels,groups", [(64, 8), (60, 12), (48, 24), (33, 3)])
@pytest.mark.parametrize("pixels", [150, 330, 430, 800])
def test_many_rows(ss, pixels, channels, groups, dtype):
    images = 260
    kind = list(ACTS)[(pixels + channels) % 4]
    x, dy, w, b = data(pixels + channels, (images, pixels, channels), dtype)
    desc = ss.make_groupnorm_desc(channels, groups, CODES[dtype], ACTS[kind], EPS)
    if dtype != "f32" or pixels <= 330:
        # nothing but the images' sums: it is held
        assert ss.ss_groupnorm_workspace_bytes(desc, images, pixels) == 0 and ss.ss_groupnorm_workspace_bytes(desc, images, pixels, True) == images * channels * 8
    y, stats = ss.ss_groupnorm_fwd(desc, x.cuda(), w.cuda(), b.cuda())
    check_forward(x, w, b, groups, kind, y, stats)
    check_backward(x, dy, w, b, groups, kind, stats, ss.ss_groupnorm_bwd(desc, dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda()))
