"""The group norm's activations and their slopes at infinities, which a bias may be: their limits, in every type."""
import pytest
import torch

from test_gpu_groupnorm import ACTS, CODES, EPS, TYPES, data

pytestmark = pytest.mark.gpu
C, GROUPS, UP, DOWN = 16, 4, [1, 6, 15], [0, 7, 9]


@pytest.mark.parametrize("tile", [None, 96], ids=["chosen", "passes"])
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_limits(ss, force_tile, tile, kind, dtype):
    x, dy, w, b = (t.cuda() for t in data(5, (2, 6, 5, C), dtype))
    desc = ss.make_groupnorm_desc(C, GROUPS, CODES[dtype], ACTS[kind], EPS)
    force_tile(tile)
    infinite, far = b.clone(), b.clone()
    infinite[UP], infinite[DOWN] = float("inf"), float("-inf")
    far[UP], far[DOWN] = 3e4, -3e4                            # (where slopes are 1 and 0 to the last bit)
    usual, _ = ss.ss_groupnorm_fwd(desc, x, w, b)
    y, stats = ss.ss_groupnorm_fwd(desc, x, w, infinite)
    rest = [c for c in range(C) if c not in UP + DOWN]
    assert torch.equal(y[..., rest], usual[..., rest])
    assert bool((y[..., UP] == float("inf")).all())
    assert bool((y[..., DOWN] == (float("-inf") if kind == "none" else 0)).all())
    for got, want in zip(ss.ss_groupnorm_bwd(desc, dy, x, stats, w, infinite), ss.ss_groupnorm_bwd(desc, dy, x, stats, w, far)):
        assert bool(want.isfinite().all()) and torch.equal(got, want)
