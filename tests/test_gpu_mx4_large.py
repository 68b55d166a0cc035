"""Pointwise MXFP4 layers whose output passes the caches by (more than 256 MB of it): every kernel that stores such an output, forced in turn, whole rows against 64 bits.

The definition is evaluated on the GPU in fp64, from the values that the codes stand for (compared bit by bit elsewhere).  Bounds are those of ``rows_reference.pointwise``."""
import numpy as np
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
TILE64, TILE128, TILE256, ROWS, ROWS128, CODES = 70, 71, 72, 76, 77, 78
LARGE = 256 << 20


class Layer:
    def __init__(self, ss, rows, cin, cout, dtype, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == F16 else ss.SS_BF16)
        self.x = (randn(rows, cin) * torch.exp(0.7 * randn(cin))).to(dtype)
        W = (randn(cout, cin) * np.sqrt(2.0 / cin)).to(dtype)
        self.packed, self.bias = ss.ss_mx4_pack(self.desc, W), 0.1 * randn(cout)
        self.residual = randn(rows, cout).to(dtype)
        self.codes, self.scales = ss.ss_mx4_quantize(self.x)
        self.xq = ss.ss_mx4_dequantize(self.codes, self.scales, cin, torch.float32)
        self.wq = torch.from_numpy(ref.through_mx4(W.double().cpu().numpy())).cuda()
        self.dtype = dtype

    def check(self, y, bias, residual, act, what):
        """y against act(wq xq + bias + residual): at most the fp32 sums' bound and one rounding off, in every element."""
        unit, tiny = ref.ROUND[self.dtype], ref.TINY[self.dtype]
        for at in range(0, len(y), 65536):
            xq = self.xq[at:at + 65536].double()
            z, size = xq @ self.wq.t(), xq.abs() @ self.wq.abs().t()
            for extra in (self.bias.double() if bias else None, residual[at:at + 65536].double() if residual is not None else None):
                if extra is not None:
                    z, size = z + extra, size + extra.abs()
            bound = (xq.shape[1] + 3) * ref.U32 * size
            if act == 2:
                z, bound = z * torch.special.ndtr(z), 1.13 * bound + 2e-7 * z.abs()
            got = y[at:at + 65536].double()
            over = (got - z).abs() - (bound * (1 + unit) + unit * z.abs() + tiny)
            assert bool((over <= 0).all()), (what, at, torch.nonzero(~(over <= 0))[:4].tolist(), float(over.max()))


# a whole number of tiles of every size, and rows and channels that end inside one
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,cin,cout", [(401408, 96, 384), (350021, 200, 448), (401421, 64, 352), (401408, 300, 384)])
def test_outputs_that_pass_the_caches(ss, force_tile, dtype, rows, cin, cout):
    assert rows * cout * 2 > LARGE
    layer = Layer(ss, rows, cin, cout, dtype, rows + cin)
    y = torch.empty((rows, cout), dtype=dtype, device="cuda")
    for kernel in (TILE64, TILE128, TILE256, ROWS, ROWS128, CODES):
        if kernel == ROWS128 and cin > 256:
            continue
        force_tile(kernel)
        for act in (0, 2):
            call = ((lambda *a: ss.ss_pw_mx4_q_fwd(layer.desc, layer.codes, layer.scales, layer.packed, *a)) if kernel <= TILE256
                    else (lambda *a: ss.ss_pw_mx4_fwd(layer.desc, layer.x, layer.packed, *a)))
            y.fill_(float("nan"))
            call(layer.bias, None, act, y)
            layer.check(y, True, None, act, (kernel, act, "bias"))
            with pytest.raises(AssertionError):                      # (the definition without the bias is another)
                layer.check(y, False, None, act, (kernel, act, "no bias"))
            y.copy_(layer.residual)                                  # the output is the residual
            call(None, y, act, y)
            layer.check(y, False, layer.residual, act, (kernel, act, "residual"))


def test_eight_waves_past_the_caches(ss, force_tile):
    """Fewer rows of many channels: the kernel with rows in LDS with eight waves, one chunk of the reduction and several."""
    for cin in (96, 700):
        layer = Layer(ss, 20013, cin, 8192, BF16, cin)
        force_tile(ROWS)
        for act in (0, 2):
            y = torch.full((20013, 8192), float("nan"), dtype=BF16, device="cuda")
            ss.ss_pw_mx4_fwd(layer.desc, layer.x, layer.packed, layer.bias, layer.residual, act, y)
            layer.check(y, True, layer.residual, act, (cin, act))


def test_a_wider_tensor_past_the_caches(ss, force_tile):
    """Rows inside a wider tensor, at an odd place: nothing outside of them is written."""
    rows, cin, cout = 360000, 96, 384
    layer = Layer(ss, rows, cin, cout, BF16, 5)
    out = torch.empty((rows, cout + 7), dtype=BF16, device="cuda")
    inner = out[:, 3:3 + cout]
    for kernel in (TILE64, TILE128, TILE256, ROWS, ROWS128):
        force_tile(kernel)
        out.fill_(7.0)
        if kernel <= TILE256:
            ss.ss_pw_mx4_q_fwd(layer.desc, layer.codes, layer.scales, layer.packed, layer.bias, None, 0, inner)
        else:
            ss.ss_pw_mx4_fwd(layer.desc, layer.x, layer.packed, layer.bias, None, 0, inner)
        layer.check(inner, True, None, 0, kernel)
        assert bool((out[:, :3] == 7).all()) and bool((out[:, 3 + cout:] == 7).all()), kernel


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,cin,cout", [(33000, 544, 128), (40000, 300, 64), (32768, 1000, 192), (33000, 2100, 64)])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_whole_tiles_of_longer_reductions(ss, force_tile, dtype, rows, cin, cout, act):
    """Many rows with channels in whole pairs of tiles, output kept in the caches: the walk without bounds checks, with four waves and with eight."""
    layer = Layer(ss, rows, cin, cout, dtype, rows)
    force_tile(ROWS)
    y = ss.ss_pw_mx4_fwd(layer.desc, layer.x, layer.packed, layer.bias, layer.residual, act)
    if act == 1:
        # (ReLU of both: the bound of the sums holds behind it)
        assert bool((y >= 0).all())
        plain = ss.ss_pw_mx4_fwd(layer.desc, layer.x, layer.packed, layer.bias, layer.residual, 0)
        assert torch.equal(y, plain.clamp(min=0))
    else:
        layer.check(y, True, layer.residual, act, act)


def test_the_librarys_own_choice_on_many_rows(ss):
    """What the choice takes for layers of many rows and long reductions, with and without LDS for two workgroups."""
    for rows, cin, cout in ((20000, 4096, 1024), (32768, 2048, 512), (20000, 8192, 256), (40000, 1024, 1024)):
        layer = Layer(ss, rows, cin, cout, BF16, cin)
        layer.check(ss.ss_pw_mx4_fwd(layer.desc, layer.x, layer.packed, layer.bias, layer.residual, 2), True, layer.residual, 2, (rows, cin, cout))
