"""The group norm's gradient through the C interface with dx in dy's place, and in neither's: the bits of the binding's call, and what lies beside the channels stays."""
import ctypes

import pytest
import torch

from test_gpu_groupnorm import ACTS, CODES, EPS, TYPES, data

pytestmark = pytest.mark.gpu


def ptr(t):
    return ctypes.c_void_p(t.data_ptr())


@pytest.mark.parametrize("tile", [None, 96], ids=["chosen", "passes"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("images,pixels,c,groups,kind", [(2, 49, 24, 3, "relu"), (3, 1000, 64, 8, "silu"), (1, 5000, 33, 11, "gelu"), (2, 300, 1030, 5, "none"), (260, 330, 60, 12, "relu"),
                                                         (1, 70, 7, 7, "silu")])
def test_dx_is_dy(ss, force_tile, tile, dtype, images, pixels, c, groups, kind):
    x, dy, w, b = (t.cuda() for t in data(pixels + c, (images, pixels, c), dtype))
    desc = ss.make_groupnorm_desc(c, groups, CODES[dtype], ACTS[kind], EPS)
    force_tile(tile)
    _, stats = ss.ss_groupnorm_fwd(desc, x, w, b)
    want = ss.ss_groupnorm_bwd(desc, dy, x, stats, w, b)
    ws = torch.empty(max(16, ss.ss_groupnorm_workspace_bytes(desc, images, pixels, True)), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty_like(w), torch.empty_like(b)
    wide = torch.full((images, pixels, c + 9), 3.0, dtype=TYPES[dtype], device="cuda")
    inner = wide[..., 5:5 + c]
    for src, dst in ((inner, inner), (dy, inner)):
        wide.fill_(3.0)
        inner.copy_(dy)
        torch.cuda.synchronize()
        status = ss.binding._lib.ss_groupnorm_bwd(ctypes.byref(desc), ptr(src), src.stride(1), ptr(x), c, images, pixels, ptr(stats), ptr(w), ptr(b), ptr(dst), dst.stride(1), ptr(dw), ptr(db),
                                                  ptr(ws), ws.numel(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert status == ss.SS_OK
        assert torch.equal(inner, want.dx) and torch.equal(dw, want.dw) and torch.equal(db, want.db)
        assert bool((wide[..., :5] == 3).all()) and bool((wide[..., 5 + c:] == 3).all())
