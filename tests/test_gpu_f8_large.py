"""Pointwise layers on FP8 blocks that move more than most of the last-level cache: every kernel that stores past it, forced in turn, every element against 64 bits.

The definition is evaluated on the GPU in fp64, from the values that the codes stand for (compared bit by bit elsewhere)."""
import pytest
import torch

import f8_reference as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
TILE64, TILE128, TILE256, ROWS, ROWS128, CODES = 80, 81, 82, 86, 87, 88
LARGE = 192 << 20


def tops(v):
    """The largest magnitude of each eight neighbouring columns."""
    return torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 8)).view(len(v), -1, 8).amax(dim=2)


class Layer:
    def __init__(self, ss, rows, cin, cout, dtype, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.ss, self.dtype = ss, dtype
        self.desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == F16 else ss.SS_BF16)
        self.x = (randn(rows, cin) * torch.exp(0.7 * randn(cin))).to(dtype)
        W = (randn(cout, cin) * (2.0 / cin) ** 0.5).to(dtype)
        self.packed, self.bias, self.residual = ss.ss_f8_pack(self.desc, W), randn(cout), randn(rows, cout).to(dtype)
        self.codes, self.scales = ss.ss_f8_quantize(self.x)
        self.xq = ss.ss_f8_dequantize(self.codes, self.scales, cin, torch.float32)
        self.wq = ref.quantize(W)[2].cuda()

    def run(self, kernel, *a):
        if kernel <= TILE256:
            return self.ss.ss_pw_f8_q_fwd(self.desc, self.codes, self.scales, self.packed, *a)
        return self.ss.ss_pw_f8_fwd(self.desc, self.x, self.packed, *a)

    def off(self, y, bias, residual, act):
        """How far y is outside of its bound, at the most (not above 0 where it is right).

        Additions in fp32, at most K / 64 + 70 that a product meets, each 2^-23 of the sum of magnitudes; eight neighbouring products lose at most 2^-13 of the largest
        each, which is at most the product of the largest of either side; GELU's slope is below 1.13 and its own error 2e-7 of its argument; half a step of the output."""
        unit, tiny, K = torch.finfo(self.dtype).eps / 2, 2.0 ** -25, self.xq.shape[1]
        worst = float("-inf")
        for at in range(0, len(y), 65536):
            xq = self.xq[at:at + 65536].double()
            z, size, dropped = xq @ self.wq.t(), xq.abs() @ self.wq.abs().t(), tops(xq) @ tops(self.wq).t()
            for extra in (self.bias.double() if bias else None, residual[at:at + 65536].double() if residual is not None else None):
                if extra is not None:
                    z, size = z + extra, size + extra.abs()
            bound = (K / 64 + 70) * 2.0 ** -23 * size + 8 * 2.0 ** -13 * dropped
            if act == 2:
                z, bound = z * torch.special.ndtr(z), 1.13 * bound + 2e-7 * z.abs()
            got = y[at:at + 65536].double()
            over = (got - z).abs() - (bound * (1 + unit) + unit * z.abs() + tiny)
            worst = max(worst, float(torch.where(over.isnan(), float("inf"), over).max()))
        return worst


# whole tiles of every size, and rows and channels that end inside one; the second moves enough only with its residual
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,cin,cout", [(401408, 96, 384), (200704, 64, 256), (401421, 64, 352), (350021, 200, 448)])
def test_outputs_that_pass_the_caches(ss, force_tile, dtype, rows, cin, cout):
    assert rows * (2 * cout + cin) * 2 > LARGE                       # (16-bit rows with a residual)
    layer = Layer(ss, rows, cin, cout, dtype, rows + cin)
    y = torch.empty((rows, cout), dtype=dtype, device="cuda")
    for kernel in (TILE64, TILE128, TILE256, ROWS, ROWS128, CODES):
        force_tile(kernel)
        for act in (0, 2):
            y.fill_(float("nan"))
            layer.run(kernel, layer.bias, None, act, y)
            assert layer.off(y, True, None, act) <= 0, (kernel, act, "bias")
            assert layer.off(y, False, None, act) > 0, (kernel, act, "the definition without the bias is another")
            y.copy_(layer.residual)                                  # the output is the residual
            layer.run(kernel, None, y, act, y)
            assert layer.off(y, False, layer.residual, act) <= 0, (kernel, act, "residual")


def test_a_wider_tensor_past_the_caches(ss, force_tile):
    """Rows inside a wider tensor, at an odd place: nothing outside of them is written."""
    rows, cin, cout = 360000, 96, 384
    layer = Layer(ss, rows, cin, cout, BF16, 5)
    out = torch.empty((rows, cout + 7), dtype=BF16, device="cuda")
    inner = out[:, 3:3 + cout]
    for kernel in (TILE64, TILE128, TILE256, ROWS, ROWS128, CODES):
        force_tile(kernel)
        out.fill_(7.0)
        layer.run(kernel, layer.bias, None, 0, inner)
        assert layer.off(inner, True, None, 0) <= 0, kernel
        assert bool((out[:, :3] == 7).all()) and bool((out[:, 3 + cout:] == 7).all()), kernel
