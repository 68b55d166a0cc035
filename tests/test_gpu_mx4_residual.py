"""The pointwise MXFP4 layer on 16-bit rows with a residual, whose output leaves past the caches at any size: small integers, which the types hold, so that every value is compared for
equality, on whole tiles and ragged ones, in place, inside wider tensors."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kernel", [None, 76, 77])
@pytest.mark.parametrize("rows,cin,cout", [(64, 64, 64), (128, 64, 256), (33000, 64, 64), (40000, 96, 128), (300, 256, 192), (1000, 200, 96), (257, 64, 320), (96, 300, 128), (32768, 31, 64)])
def test_equal(ss, force_tile, dtype, kernel, rows, cin, cout):
    g = torch.Generator(device="cuda").manual_seed(rows + cin)
    t = TYPES[dtype]
    ints = lambda low, high, *s: torch.randint(low, high, s, generator=g, device="cuda").float()
    # (blocks whose largest is 4 hold the integers to 4; sums stay below 256 in magnitude, which bfloat16 holds)
    x, W, residual, bias = ints(-1, 2, rows, cin), (ints(0, 8, cout, cin) == 0).float() - (ints(0, 8, cout, cin) == 0).float(), ints(-8, 9, rows, cout), ints(-3, 4, cout)
    want = x @ W.t() + bias + residual
    assert float(want.abs().max()) <= 256
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == "f16" else ss.SS_BF16)
    packed = ss.ss_mx4_pack(desc, W.to(t))
    force_tile(kernel)
    wide = torch.full((rows, cout + 11), 7.0, dtype=t, device="cuda")
    for act in (0, 1):
        expected = (want.clamp(min=0) if act else want).to(t)
        assert torch.equal(ss.ss_pw_mx4_fwd(desc, x.to(t), packed, bias, residual.to(t), act), expected)
        inner = wide.fill_(7.0)[:, 3:3 + cout]
        inner.copy_(residual)
        assert torch.equal(ss.ss_pw_mx4_fwd(desc, x.to(t), packed, bias, inner, act, inner), expected)
        assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 3 + cout:] == 7).all())
