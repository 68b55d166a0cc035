"""The tests' own definition of FP8 blocks against torch's conversion and by hand."""
import torch

from f8_reference import quantize


def test_codes_are_the_types():
    """With the scale divided out a value's code is torch's conversion to the type (nearest even), whose bytes are the format's."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((40, 300), generator=g) * torch.exp(4 * torch.randn((40, 1), generator=g))
    codes, scales, value = quantize(x)
    unit = torch.pow(2.0, scales[:, :3].double() - 127).repeat_interleave(128, dim=1)[:, :300]
    want = (x.double() / unit).float().to(torch.float8_e4m3fn)
    assert torch.equal(codes[:, :300], want.view(torch.uint8))
    assert torch.equal(value, want.double() * unit)
    assert not codes[:, 300:].any()


def test_scales_by_hand():
    x = torch.zeros((6, 130))
    x[0, 5], x[1, 5], x[2, 5], x[3, 5] = 448.0, 449.0, 1.0, 1.75
    x[4, 129] = float("inf")
    codes, scales, value = quantize(x)
    assert scales[:, 0].tolist() == [127, 128, 119, 119, 0, 0] and scales[:, 1].tolist() == [0, 0, 0, 0, 255, 0] and not scales[:, 2:].any()
    assert codes[0, 5] == 0x7E and codes[2, 5] == 0x78 and codes[3, 5] == 0x7E
    assert value[1, 5] == 448.0 and value[4, 128:].isnan().all() and not value[4, :128].any()


def test_nothing_saturates():
    """Every value keeps a relative error of half a step, or half the least step of its block."""
    g = torch.Generator().manual_seed(4)
    x = torch.rand((500, 128), generator=g).double() * torch.pow(2.0, 30 * torch.rand((500, 1), generator=g).double() - 15)
    _, scales, value = quantize(x)
    least = 2.0 ** -10 * torch.pow(2.0, scales[:, :1].double() - 127)
    assert ((value - x).abs() <= torch.maximum(x * 2.0 ** -4, least)).all()
