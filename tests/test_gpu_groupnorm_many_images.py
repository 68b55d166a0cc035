"""The group norm's gradients of its vectors over very many images, of values of one sign and one size: sums whose additions all round the same way."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tile", [None, 96], ids=["chosen", "passes"])
@pytest.mark.parametrize("images", [300, 511, 512, 4099, (1 << 20) + 3])
def test_vectors(ss, force_tile, tile, images):
    c, groups, pixels = 24, 3, 2
    # statistics as given: xh is x
    stats = torch.tensor([0.0, 1.0], device="cuda").expand(images, groups, 2).contiguous()
    x = torch.full((images, pixels, c), 0.7, device="cuda") + 0.01 * torch.arange(c, device="cuda")
    dy = torch.full((images, pixels, c), 0.1, device="cuda") + 0.003 * torch.arange(c, device="cuda")
    desc = ss.make_groupnorm_desc(c, groups, ss.SS_F32, ss.SS_ACT_NONE)
    force_tile(tile)
    grads = ss.ss_groupnorm_bwd(desc, dy, x, stats, torch.ones(c, device="cuda"), torch.zeros(c, device="cuda"))
    n = images * pixels
    for got, want in ((grads.db, dy[0, 0].double() * n), (grads.dw, dy[0, 0].double() * x[0, 0].double() * n)):
        # (an image's: a product, one addition of two pixels, a factor and a rounding; the images', in 64 bits: a rounding)
        assert bool((got.double() - want).abs().le(6 * 2.0 ** -24 * want).all())
