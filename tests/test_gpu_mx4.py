"""MXFP4 on the GPU: quantisation bit for bit against the format's definition, the way back, packed weights, and the pointwise layer on them."""
import numpy as np
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def _values(rows, cols, dtype, seed, spread=4.0):
    """Rows of very different magnitudes, with zeros of both signs and halfway points among them."""
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, -(-cols // 32)))).repeat(32, axis=1)[:, :cols]
    v = np.where(rng.random(v.shape) < 0.1, rng.choice([0.0, -0.0, 0.25, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.75], v.shape), v)
    return torch.from_numpy(v).cuda().to(dtype)


def _same(x, codes, scales):
    want = ref.quantize(x.double().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy().reshape(want[1].shape), want[1])
    assert np.array_equal(codes.cpu().numpy().reshape(want[0].shape), want[0])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 96), (49, 768), (7, 129), (130, 1111), (1, 8192), (513, 40)])
def test_quantize_and_back(ss, dtype, rows, cols):
    x = _values(rows, cols, dtype, rows * 10000 + cols)
    codes, scales = ss.ss_mx4_quantize(x)
    _same(x, codes, scales)
    values = ref.dequantize(codes.cpu().numpy(), scales.cpu().numpy(), cols)
    for out in (F16, BF16, F32):
        y = ss.ss_mx4_dequantize(codes, scales, cols, out)
        # (a block with an infinity, which the spread gives in float16, stands for NaN; a value beyond float16's range for its infinity)
        assert np.array_equal(y.double().cpu().numpy(), torch.from_numpy(values).to(out).double().numpy(), equal_nan=True)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_special_blocks(ss, dtype):
    """Blocks with a NaN, an infinity, nothing, the type's smallest and largest values; their neighbours do not notice."""
    info = torch.finfo(dtype)
    x = torch.full((12, 96), 1.5, dtype=dtype, device="cuda")
    smallest = torch.tensor(info.smallest_normal * info.eps, dtype=torch.float64).to(dtype)
    for i, v in enumerate([float("nan"), float("inf"), -float("inf"), info.max, info.min, info.smallest_normal, float(smallest), 0.0, -0.0]):
        x[i, 32:64] = v if i != 1 else 0.0
        x[i, 40] = v
    x[9, 32:64] = torch.linspace(-3, 3, 32).to(dtype) * float(smallest)
    x[10] = 0.0
    codes, scales = ss.ss_mx4_quantize(x)
    _same(x, codes, scales)
    back = ss.ss_mx4_dequantize(codes, scales, 96, F32)
    assert torch.isnan(back[:3, 32:64]).all() and (back[:9, :32] == 1.5).all() and (back[:9, 64:] == 1.5).all() and (back[10] == 0).all()
    assert torch.isfinite(back[3:]).all()


def test_every_16bit_pattern(ss):
    """All finite binary16 and bfloat16 values as the only value of a block, and as a small one next to a larger."""
    for dtype in (F16, BF16):
        bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
        bits = bits[torch.isfinite(bits)]
        x = torch.zeros((bits.numel(), 64), dtype=dtype)
        x[:, 0] = bits
        x[:, 33] = bits
        x[:, 40] = (bits.float() * 3.0).clamp(torch.finfo(dtype).min, torch.finfo(dtype).max).to(dtype)
        x = x.cuda()
        _same(x, *ss.ss_mx4_quantize(x))


def test_quantize_strides_streams_and_given_outputs(ss):
    wide = _values(40, 300, BF16, 5)
    for view in (wide[:, 3:203], wide[::2, :128], wide[5:6, 1:], wide.view(5, 8, 300)[:, :, 100:], wide[:0], wide[:, :1]):
        codes, scales = ss.ss_mx4_quantize(view)
        assert codes.shape[:-1] == view.shape[:-1]
        _same(view.reshape(-1, view.shape[-1]), codes, scales)
    given = torch.full((40, 160), 7, dtype=torch.uint8, device="cuda"), torch.full((40, 12), 7, dtype=torch.uint8, device="cuda")
    codes, scales = ss.ss_mx4_quantize(wide, *given)
    assert codes is given[0] and scales is given[1]
    _same(wide, codes, scales)
    out = torch.zeros((40, 400), dtype=BF16, device="cuda")
    back = ss.ss_mx4_dequantize(codes, scales, 300, BF16, out[:, 50:350])
    assert back.data_ptr() == out[:, 50:].data_ptr() and (out[:, :50] == 0).all() and (out[:, 350:] == 0).all()
    assert torch.equal(back, ss.ss_mx4_dequantize(codes, scales, 300, BF16))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    on_stream = ss.ss_mx4_quantize(wide, stream=stream)
    again = ss.ss_mx4_dequantize(*on_stream, 300, BF16, stream=stream)
    stream.synchronize()
    assert torch.equal(on_stream[0], codes) and torch.equal(again, back)


def test_rows_beyond_32_bit_offsets(ss):
    """Rows far enough apart that the third begins beyond 2^31 elements."""
    pitch = (1 << 30) + 8
    buffer = torch.empty(2 * pitch + 96, dtype=F16, device="cuda")
    x = buffer.as_strided((3, 96), (pitch, 1))
    x.copy_(_values(3, 96, F16, 9))
    codes, scales = ss.ss_mx4_quantize(x)
    _same(x, codes, scales)
    x.zero_()
    ss.ss_mx4_dequantize(codes, scales, 96, F16, x)
    assert torch.equal(x.contiguous(), ss.ss_mx4_dequantize(codes, scales, 96, F16))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("cout,cin,masked", [(1, 1, False), (33, 100, True), (96, 384, True), (64, 31, False), (5, 520, True)])
def test_packed_weights(ss, dtype, cout, cin, masked):
    W = _values(cout, cin, dtype, cout + cin, spread=1.0)
    rng = np.random.default_rng(cin)
    M = torch.from_numpy((rng.random((cout, cin)) < 0.5).astype(np.uint8)).cuda() if masked else None
    if masked:
        M[0] = 0                                                  # a row whose mask leaves nothing
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == F16 else ss.SS_BF16)
    before = W.clone()
    packed = ss.ss_mx4_pack(desc, W, M)
    want = ref.through_mx4((W if M is None else torch.where(M != 0, W, torch.zeros_like(W))).double().cpu().numpy())
    assert torch.equal(ss.ss_mx4_unpack(desc, packed).cpu(), torch.from_numpy(want).to(dtype))
    assert torch.equal(W, before)
    # the layout that the header documents
    kb, mt, ks = -(-cin // 32), -(-cout // 32), -(-(-(-cin // 32)) // 2)
    raw = packed.cpu().numpy()
    masked_w = (W if M is None else torch.where(M != 0, W, torch.zeros_like(W))).double().cpu().numpy()
    codes, scales = ref.quantize(masked_w)
    tiles = raw[256:256 + mt * ks * 1024].reshape(mt, ks, 2, 32, 16)
    whole = np.zeros((mt * 32, ks * 2, 16), dtype=np.uint8)
    whole[:cout, :kb] = codes.reshape(cout, kb, 16)
    assert np.array_equal(tiles, whole.reshape(mt, 32, ks, 2, 16).transpose(0, 2, 3, 1, 4))
    kq = -(-ks // 4)
    stiles = raw[256 + mt * ks * 1024:256 + mt * ks * 1024 + mt * kq * 256].reshape(mt, kq, 2, 32, 4)
    swhole = np.zeros((mt * 32, kq * 8), dtype=np.uint8)
    swhole[:cout, :kb] = scales[:, :kb]
    assert np.array_equal(stiles, swhole.reshape(mt, 32, kq, 4, 2).transpose(0, 2, 4, 1, 3))


def _layer(ss, rows, cin, cout, dtype, seed, masked=True, spread=0.7):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((rows, cin)) * np.exp(spread * rng.standard_normal(cin))).cuda().to(dtype)
    W = torch.from_numpy(rng.standard_normal((cout, cin)) * np.sqrt(2.0 / cin)).cuda().to(dtype)
    M = torch.from_numpy((rng.random((cout, cin)) < 0.5).astype(np.uint8)).cuda() if masked else None
    bias = torch.from_numpy(0.1 * rng.standard_normal(cout)).cuda().float()
    residual = torch.from_numpy(rng.standard_normal((rows, cout))).cuda().to(dtype)
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == F16 else ss.SS_BF16)
    Wm = W if M is None else torch.where(M != 0, W, torch.zeros_like(W))
    return desc, x, ss.ss_mx4_pack(desc, W, M), bias, residual, ref.through_mx4(x.double().cpu().numpy()), ref.through_mx4(Wm.double().cpu().numpy())


# one row to several tiles of pixels; reductions of less than a block to several chunks; output channels of less than a vector to several tiles
SHAPES = [(1, 1, 1), (1, 32, 8), (1, 2048, 1000), (2, 96, 33), (5, 100, 64), (16, 512, 40), (17, 1024, 136), (31, 64, 96), (32, 8192, 32), (33, 288, 300), (49, 768, 264),
          (64, 256, 256), (65, 320, 31), (100, 1000, 777), (129, 96, 384), (200, 384, 96), (257, 544, 288), (300, 2048, 64), (515, 160, 520), (1000, 33, 7), (1, 8192, 1024),
          (3, 4000, 2000), (2049, 128, 128), (1531, 1000, 777), (70, 5000, 100), (33, 8192, 40), (600, 4800, 700)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_pointwise(ss, dtype, rows, cin, cout):
    desc, x, packed, bias, residual, xq, wq = _layer(ss, rows, cin, cout, dtype, rows + cin + cout)
    b, r = bias.double().cpu().numpy(), residual.double().cpu().numpy()
    codes, scales = ss.ss_mx4_quantize(x)
    for act, use_b, use_r in [(ss.SS_ACT_NONE, False, False), (ss.SS_ACT_RELU, True, True), (ss.SS_ACT_GELU, True, False), (ss.SS_ACT_NONE, False, True)]:
        want, bound = ref.pointwise(xq, wq, b if use_b else None, r if use_r else None, act)
        args = (bias if use_b else None, residual if use_r else None, act)
        y = ss.ss_pw_mx4_fwd(desc, x, packed, *args)
        ref.close(y, want, bound, dtype, f"from 16 bits, act {act}")
        ref.close(ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, *args), want, bound, dtype, f"quantised, act {act}")


@pytest.mark.parametrize("rows,cin,cout", [(1, 200, 40), (20, 96, 100), (70, 1000, 37), (300, 130, 264)])
def test_pointwise_views(ss, rows, cin, cout):
    """Operands at odd places and pitches, an output that is the residual, and one inside a wider tensor whose other columns stay."""
    desc, x, packed, bias, residual, xq, wq = _layer(ss, rows, cin, cout, BF16, 77 + rows)
    plain = ss.ss_pw_mx4_fwd(desc, x, packed, bias, residual, ss.SS_ACT_RELU)
    wide = torch.zeros((rows, cin + 9), dtype=BF16, device="cuda")
    wide[:, 3:3 + cin] = x
    out = torch.full((rows, cout + 5), 3.0, dtype=BF16, device="cuda")
    out[:, 1:1 + cout] = residual
    y = ss.ss_pw_mx4_fwd(desc, wide[:, 3:3 + cin], packed, bias, out[:, 1:1 + cout], ss.SS_ACT_RELU, y=out[:, 1:1 + cout])
    assert y.data_ptr() == out[:, 1:].data_ptr() and torch.equal(y, plain)
    assert (out[:, 0] == 3).all() and (out[:, 1 + cout:] == 3).all()
    codes, scales = ss.ss_mx4_quantize(x)
    out[:, 1:1 + cout] = residual
    assert torch.equal(ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, bias, out[:, 1:1 + cout], ss.SS_ACT_RELU, y=out[:, 1:1 + cout]),
                       ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, bias, residual, ss.SS_ACT_RELU))
    assert (out[:, 0] == 3).all() and (out[:, 1 + cout:] == 3).all()
    image = x.new_empty((2, rows, 1, cin)).copy_(x.view(1, rows, 1, cin))
    both = ss.ss_pw_mx4_fwd(desc, image, packed, bias)
    assert both.shape == (2, rows, 1, cout) and torch.equal(both[0], both[1])


@pytest.mark.parametrize("rows", [1, 40, 600])
def test_a_nan_stays_in_its_row(ss, rows):
    desc, x, packed, bias, _, xq, wq = _layer(ss, rows + 2, 160, 72, F16, rows)
    clean = ss.ss_pw_mx4_fwd(desc, x, packed, bias)
    x[1, 70] = float("nan")
    x[rows, 0] = float("inf")
    codes, scales = ss.ss_mx4_quantize(x)
    keep = [i for i in range(rows + 2) if i not in (1, rows)]
    for y in (ss.ss_pw_mx4_fwd(desc, x, packed, bias), ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, bias)):
        assert torch.isnan(y[1]).all() and torch.isnan(y[rows]).all()
        ref.close(y[keep], *ref.pointwise(xq[keep], wq, bias.double().cpu().numpy(), None, 0), F16, "other rows")
    W = torch.ones((72, 160), dtype=F16, device="cuda")
    W[7, 159] = float("nan")
    y = ss.ss_pw_mx4_fwd(desc, torch.ones((rows, 160), dtype=F16, device="cuda"), ss.ss_mx4_pack(desc, W))
    assert torch.isnan(y[:, 7]).all() and (y[:, [i for i in range(72) if i != 7]] == 160).all()


def test_pointwise_empty_stream_and_graph(ss):
    desc, x, packed, bias, residual, _, _ = _layer(ss, 300, 256, 200, BF16, 3)
    assert ss.ss_pw_mx4_fwd(desc, x[:0], packed).shape == (0, 200)
    assert ss.ss_pw_mx4_q_fwd(desc, *ss.ss_mx4_quantize(x[:0]), packed).shape == (0, 200)
    want = ss.ss_pw_mx4_fwd(desc, x, packed, bias, residual, ss.SS_ACT_GELU)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    y = ss.ss_pw_mx4_fwd(desc, x, packed, bias, residual, ss.SS_ACT_GELU, stream=stream)
    stream.synchronize()
    assert torch.equal(y, want)
    for rows in (1, 16, 300):
        xs, rs = x[:rows].clone(), residual[:rows].clone()
        y = torch.empty((rows, 200), dtype=BF16, device="cuda")
        graph = torch.cuda.CUDAGraph()
        ss.ss_pw_mx4_fwd(desc, xs, packed, bias, rs, ss.SS_ACT_GELU, y)
        with torch.cuda.graph(graph):
            ss.ss_pw_mx4_fwd(desc, xs, packed, bias, rs, ss.SS_ACT_GELU, y)
        for turn in range(4):
            xs.mul_(-0.5)
            eager = ss.ss_pw_mx4_fwd(desc, xs, packed, bias, rs, ss.SS_ACT_GELU)
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, eager), (rows, turn)


def test_refusals(ss):
    desc, x, packed, bias, residual, _, _ = _layer(ss, 8, 64, 48, F16, 4)
    codes, scales = ss.ss_mx4_quantize(x)

    def refused(call, *a, status=ss.SS_ERR_INVALID_ARG, **k):
        with pytest.raises(ss.SSError) as e:
            call(*a, **k)
        assert e.value.status == status

    refused(ss.ss_mx4_quantize, x.cpu())
    refused(ss.ss_mx4_quantize, x.int())
    refused(ss.ss_mx4_quantize, x.t())
    refused(ss.ss_mx4_quantize, x.view(2, 4, 64).transpose(0, 1))
    refused(ss.ss_mx4_quantize, x[:, :0])
    refused(ss.ss_mx4_quantize, x, codes[:4])
    refused(ss.ss_mx4_quantize, x, codes, scales[:, :2])
    refused(ss.ss_mx4_quantize, x, codes.int())
    refused(ss.ss_mx4_dequantize, codes, scales, 96)
    refused(ss.ss_mx4_dequantize, codes, scales[:4], 64)
    refused(ss.ss_mx4_dequantize, codes, scales, 64, torch.float64)
    refused(ss.ss_mx4_dequantize, codes, scales, 64, F16, torch.empty((8, 63), dtype=F16, device="cuda"))
    refused(ss.ss_mx4_pack, desc, x)
    refused(ss.ss_mx4_pack, desc, torch.empty((48, 64), dtype=BF16, device="cuda"))
    refused(ss.ss_mx4_pack, desc, torch.empty((48, 64), dtype=F16, device="cuda"), packed=packed[:-1])
    refused(ss.ss_mx4_pack, ss.make_desc(48, 64, 3, 3), x, status=ss.SS_ERR_UNSUPPORTED)
    refused(ss.ss_pw_mx4_fwd, desc, x.bfloat16(), packed)
    refused(ss.ss_pw_mx4_fwd, desc, x[:, :63], packed)
    refused(ss.ss_pw_mx4_fwd, desc, x, packed[:-256])
    refused(ss.ss_pw_mx4_fwd, desc, x, packed, bias[:-1])
    refused(ss.ss_pw_mx4_fwd, desc, x, packed, bias.half())
    refused(ss.ss_pw_mx4_fwd, desc, x, packed, None, residual[:4])
    refused(ss.ss_pw_mx4_fwd, desc, x, packed, None, None, 3)
    refused(ss.ss_pw_mx4_fwd, desc, x, packed, y=torch.empty((8, 48), dtype=BF16, device="cuda"))
    long, xl, pl, _, _, _, _ = _layer(ss, 64, 8192, 8, F16, 4)                     # (its codes are made in the workspace)
    assert ss.ss_pw_mx4_workspace_bytes(long, 64) >= 64 * 4352
    refused(ss.ss_pw_mx4_fwd, long, xl, pl, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"), status=ss.SS_ERR_WORKSPACE)
    refused(ss.ss_pw_mx4_q_fwd, desc, codes[:, :16], scales, packed)
    refused(ss.ss_pw_mx4_q_fwd, desc, codes, scales[:4], packed)
    refused(ss.ss_pw_mx4_q_fwd, desc, x, scales, packed)


# every kernel in turn (ids of include/ss_debug.h): whole tiles and cut ones, less than a scale word of the reduction and several
@pytest.mark.parametrize("kernel", range(70, 79))
@pytest.mark.parametrize("rows,cin,cout", [(1, 8, 1), (32, 300, 96), (64, 96, 64), (70, 1000, 100), (128, 64, 256), (300, 544, 320), (517, 256, 70)])
def test_every_kernel(ss, force_tile, kernel, rows, cin, cout):
    desc, x, packed, bias, residual, xq, wq = _layer(ss, rows, cin, cout, BF16, 3 * rows + cin)
    want, bound = ref.pointwise(xq, wq, bias.double().cpu().numpy(), residual.double().cpu().numpy(), ss.SS_ACT_RELU)
    codes, scales = ss.ss_mx4_quantize(x)
    force_tile(kernel)
    if kernel < 75:
        ref.close(ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed, bias, residual, ss.SS_ACT_RELU), want, bound, BF16, f"kernel {kernel}")
    else:
        ref.close(ss.ss_pw_mx4_fwd(desc, x, packed, bias, residual, ss.SS_ACT_RELU), want, bound, BF16, f"kernel {kernel}")


def test_small_integers_are_exact(ss, force_tile):
    """Integers up to 6 with a power of two as each block's scale: every kernel gives the same, exact sums."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.choice([-6.0, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], (200, 320))).cuda().to(F16)
    W = torch.from_numpy(rng.choice([-1.0, 0, 0.5, 1], (96, 320))).cuda().to(F16)
    x[:, ::32] = 4.0                                              # (each block's largest is 4 or 6: scale 1)
    W[:, ::32] = 1.0                                              # (scale 1/4: all of these values are there)
    desc = ss.make_desc(96, 320, 1, 1, ss.SS_F16)
    packed, want = ss.ss_mx4_pack(desc, W), (x.double() @ W.double().t()).cpu()
    codes, scales = ss.ss_mx4_quantize(x)
    for kernel in range(70, 75):
        force_tile(kernel)
        assert torch.equal(ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed).double().cpu(), want.half().double()), kernel
    for kernel in range(76, 79):
        force_tile(kernel)
        assert torch.equal(ss.ss_pw_mx4_fwd(desc, x, packed).double().cpu(), want.half().double()), kernel


def test_outputs_beyond_the_caches(ss):
    """More than 128 MB of output (whose lines are not kept) and more than 2^31 bytes of it: rows at both ends, and those around the 2^31st byte."""
    rows, cin, cout = 4200000, 32, 256
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((rows, cin), generator=g, device="cuda").half()
    W = torch.randn((cout, cin), generator=g, device="cuda").half()
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16)
    packed = ss.ss_mx4_pack(desc, W)
    wq = ref.through_mx4(W.double().cpu().numpy())
    codes, scales = ss.ss_mx4_quantize(x)
    around = torch.cat([torch.arange(0, 70), torch.arange(2 ** 22 - 70, 2 ** 22 + 70), torch.arange(rows - 70, rows)])
    want, bound = ref.pointwise(ref.through_mx4(x[around].double().cpu().numpy()), wq, None, None, 0)
    for y in (ss.ss_pw_mx4_fwd(desc, x, packed), ss.ss_pw_mx4_q_fwd(desc, codes, scales, packed)):
        ref.close(y[around], want, bound, F16, "rows")
        del y


@pytest.mark.parametrize("rows,cin,cout", [(33000, 544, 70), (32801, 300, 96), (70000, 264, 33)])
def test_many_rows_of_longer_reductions(ss, rows, cin, cout):
    desc, x, packed, bias, residual, xq, wq = _layer(ss, rows, cin, cout, BF16, rows)
    want, bound = ref.pointwise(xq, wq, bias.double().cpu().numpy(), residual.double().cpu().numpy(), ss.SS_ACT_GELU)
    ref.close(ss.ss_pw_mx4_fwd(desc, x, packed, bias, residual, ss.SS_ACT_GELU), want, bound, BF16, "rows")
