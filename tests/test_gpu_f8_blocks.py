"""FP8 with a scale for each block of 128: quantisation, packing and the pointwise layer, against the definition in 64 bits."""
import pytest
import torch

import f8_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows_of(g, rows, cols, dtype):
    """Blocks of different sizes, among them zeros."""
    x = torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, -(-cols // 64)), generator=g)).repeat_interleave(64, dim=1)[:, :cols]
    x[torch.rand((rows, cols), generator=g) < 0.1] = 0
    if rows > 2:
        x[rows // 2] = 0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 8), (5, 64), (4, 65), (7, 127), (3, 128), (9, 129), (5, 300), (3, 512), (2, 513), (6, 1000), (300, 96), (2, 5000)])
def test_quantize_bits(ss, dtype, rows, cols):
    x = rows_of(gen(rows * 1000 + cols), rows, cols, TYPES[dtype])
    codes, scales, value = ref.quantize(x)
    got_codes, got_scales = ss.ss_f8_quantize(x.cuda())
    assert torch.equal(got_scales.cpu(), scales)
    # (a zero's sign is kept)
    assert torch.equal(got_codes.cpu(), codes)
    back = ss.ss_f8_dequantize(got_codes, got_scales, cols, torch.float32).cpu()
    assert torch.equal(back.double(), value)
    assert torch.equal(ss.ss_f8_dequantize(got_codes, got_scales, cols, TYPES[dtype]).cpu(), value.to(TYPES[dtype]))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_every_exponent_and_nan(ss, dtype):
    """Blocks of every size that the type has, down to its subnormals; infinities and NaN."""
    t = TYPES[dtype]
    lo, hi = (-24, 15) if dtype == "f16" else (-149, 127)
    g = gen(5)
    x = (torch.rand((hi - lo + 1, 128), generator=g, dtype=torch.float64) * 2 - 1) * torch.pow(2.0, torch.arange(lo, hi + 1).double()).unsqueeze(1) * 1.99
    x = x.clamp(-torch.finfo(t).max, torch.finfo(t).max).to(t)
    x = torch.cat([x, torch.full((1, 128), torch.finfo(t).max, dtype=t), torch.ones((3, 128), dtype=t)])
    x[-1, 3], x[-2, 127], x[-3, 0] = float("nan"), float("inf"), float("-inf")
    codes, scales, value = ref.quantize(x)
    got_codes, got_scales = ss.ss_f8_quantize(x.cuda())
    assert torch.equal(got_scales.cpu(), scales) and torch.equal(got_codes.cpu(), codes)
    back = ss.ss_f8_dequantize(got_codes, got_scales, 128, torch.float32).cpu()
    # (rounded to the type: a block's largest may be rounded up to 2^128, which fp32 gives as infinity)
    value = value.float()
    assert torch.equal(back.isnan(), value.isnan()) and torch.equal(torch.where(back.isnan(), 0, back), torch.where(value.isnan(), 0, value))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_views(ss, dtype):
    """Rows of a wider tensor, from any element on; outputs given; another stream."""
    whole = rows_of(gen(6), 40, 333, TYPES[dtype]).cuda()
    x = whole[3:, 5:205]
    codes, scales, value = ref.quantize(x)
    out_c, out_s = torch.empty((37, 256), dtype=torch.uint8, device="cuda"), torch.empty((37, 4), dtype=torch.uint8, device="cuda")
    got = ss.ss_f8_quantize(x, out_c, out_s)
    assert got[0] is out_c and got[1] is out_s
    assert torch.equal(out_c.cpu(), codes) and torch.equal(out_s.cpu(), scales)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c2, s2 = ss.ss_f8_quantize(x, stream=side)
    wide = torch.full((37, 400), 3.0, dtype=TYPES[dtype], device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    ss.ss_f8_dequantize(c2, s2, 200, TYPES[dtype], out=wide[:, 100:300], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(c2.cpu(), codes) and torch.equal(wide[:, 100:300].cpu(), value.to(TYPES[dtype]))
    assert (wide[:, :100] == 3).all() and (wide[:, 300:] == 3).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("cout,cin", [(1, 1), (5, 7), (32, 64), (33, 65), (70, 200), (96, 512), (40, 777), (31, 1500)])
@pytest.mark.parametrize("mask", [False, True])
def test_pack(ss, dtype, cout, cin, mask):
    g = gen(cout * 7 + cin)
    t = TYPES[dtype]
    W = rows_of(g, cout, cin, t)
    M = (torch.rand((cout, cin), generator=g) < 0.5).to(torch.uint8) if mask else None
    masked = W if M is None else W * M
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == "f16" else ss.SS_BF16)
    packed = ss.ss_f8_pack(desc, W.cuda(), None if M is None else M.cuda())
    ss.ss_weights_check(desc, packed, ss.SS_WEIGHTS_F8)
    assert torch.equal(ss.ss_f8_unpack(desc, packed).cpu(), ref.quantize(masked)[2].to(t))
    turned = ss.ss_f8_pack(desc, W.t().contiguous().cuda(), None if M is None else M.t().contiguous().cuda(), transposed=True)
    ss.ss_weights_check(desc, turned, ss.SS_WEIGHTS_F8)
    differ = (packed != turned).cpu().view(-1)
    # a masked weight is +0 either way
    assert not differ.any()
    with pytest.raises(ss.SSError):
        ss.ss_weights_check(desc, packed, False)
    with pytest.raises(ss.SSError):
        ss.ss_weights_check(ss.make_desc(cout + 1 if cout % 32 else cout, cin + 64, 1, 1, desc.dtype), torch.cat([packed, packed, packed]), ss.SS_WEIGHTS_F8)


def bound(W, x, out, dtype, K):
    """How far a product may be off: half a step of the output (2^-25 where it is subnormal); the additions in fp32, of which a product, exact in fp32, meets at most K / 64 + 70
    (the instruction's own, the steps', the waves' and the bias's), each 2^-23 of the sum of magnitudes; and what the FP8 instruction drops: it adds the
    products of eight neighbouring channels first and keeps of each what is not below 2^-13 of the largest, so each loses at most 2^-13 of that."""
    size = x.abs() @ W.abs().t()
    W8, x8 = (torch.nn.functional.pad(t.abs(), (0, -K % 8)).view(t.shape[0], -1, 8) for t in (W, x))
    dropped = torch.zeros_like(size)
    for k in range(W8.shape[1]):
        dropped += 8 * 2.0 ** -13 * (x8[:, k].unsqueeze(1) * W8[:, k].unsqueeze(0)).amax(dim=2)
    return out.abs() * torch.finfo(dtype).eps / 2 + (K / 64 + 70) * 2.0 ** -23 * size + dropped + 2.0 ** -25


KERNELS = {"tile_64": 80, "tile_128": 81, "tile_256": 82, "few_32": 83, "few_64": 84, "few16": 85, "rows": 86, "rows_128": 87, "codes": 88}


@pytest.mark.parametrize("kernel", [None, *KERNELS])
@pytest.mark.parametrize("rows,cin,cout,dtype,act", [(1, 1, 1, "f16", "none"), (1, 2048, 1000, "bf16", "none"), (5, 64, 96, "f16", "relu"), (33, 128, 32, "bf16", "gelu"),
                                                     (100, 200, 130, "f16", "gelu"), (257, 321, 260, "bf16", "relu"), (64, 450, 257, "bf16", "none"), (70, 1000, 300, "f16", "gelu"),
                                                     (300, 577, 513, "f16", "none"), (31, 1664, 40, "bf16", "relu")])
def test_product(ss, force_tile, kernel, rows, cin, cout, dtype, act):
    g = gen(rows + cin * 3 + cout * 5)
    t = TYPES[dtype]
    x, W = rows_of(g, rows, cin, t), (torch.randn((cout, cin), generator=g) / cin ** 0.5).to(t)
    bias, res = torch.randn(cout, generator=g), torch.randn((rows, cout), generator=g).to(t)
    M = (torch.rand((cout, cin), generator=g) < 0.5).to(torch.uint8) if cin % 4 == 0 else None
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == "f16" else ss.SS_BF16)
    packed = ss.ss_f8_pack(desc, W.cuda(), None if M is None else M.cuda())
    Wq, xq = ref.quantize(W if M is None else W * M)[2], ref.quantize(x)[2]
    kinds = {"none": ss.SS_ACT_NONE, "relu": ss.SS_ACT_RELU, "gelu": ss.SS_ACT_GELU}
    force_tile(None if kernel is None else KERNELS[kernel])
    codes, scales = ss.ss_f8_quantize(x.cuda())
    got_q = ss.ss_pw_f8_q_fwd(desc, codes, scales, packed, bias.cuda(), res.cuda(), kinds[act])
    got = ss.ss_pw_f8_fwd(desc, x.cuda(), packed, bias.cuda(), res.cuda(), kinds[act])
    plain = ss.ss_pw_f8_q_fwd(desc, codes, scales, packed)
    z = xq @ Wq.t()
    full = z + bias.double() + res.double()
    want = ref.act(full, act)
    # (an activation's slope is below 1.13; its own error, 1e-6 of the value and 1e-7)
    tol = 1.13 * bound(Wq, xq, full, t, cin) + want.abs() * (torch.finfo(t).eps / 2 + 4e-2 * (act == "gelu") * (want.abs() < 1e-2)) + 2e-7
    assert ((got_q.cpu().double() - want).abs() <= tol).all()
    assert ((got.cpu().double() - want).abs() <= tol).all()
    assert ((plain.cpu().double() - z).abs() <= bound(Wq, xq, z, t, cin)).all()


def test_product_nan_stays_in_its_row(ss, force_tile):
    """A row with a NaN or an infinity gives NaN in that row alone, a weight row with one in that channel alone."""
    g = gen(11)
    x, W = torch.randn((300, 200), generator=g).bfloat16(), torch.randn((300, 200), generator=g).bfloat16()
    x[17, 150], x[200, 3], W[44, 199] = float("nan"), float("inf"), float("-inf")
    desc = ss.make_desc(300, 200, 1, 1, ss.SS_BF16)
    packed = ss.ss_f8_pack(desc, W.cuda())
    for kernel in (None, *KERNELS.values()):
        force_tile(kernel)
        y = ss.ss_pw_f8_fwd(desc, x.cuda(), packed).cpu()
        bad = torch.zeros((300, 300), dtype=torch.bool)
        bad[17], bad[200], bad[:, 44] = True, True, True
        assert torch.equal(y.isnan(), bad)


def test_product_views(ss):
    """Rows of wider tensors, outputs that keep what is beside them, a residual that is the output."""
    g = gen(12)
    wide_x, wide_y = torch.randn((90, 300), generator=g).half().cuda(), torch.randn((90, 200), generator=g).half().cuda()
    x, y = wide_x[:, 7:207], wide_y[:, 9:109]
    before, old = wide_y.clone(), y.clone()
    W = (torch.randn((100, 200), generator=g) / 14).half()
    desc = ss.make_desc(100, 200, 1, 1, ss.SS_F16)
    packed = ss.ss_f8_pack(desc, W.cuda())
    assert ss.ss_pw_f8_fwd(desc, x, packed, residual=y, y=y) is y
    assert torch.equal(y, ss.ss_pw_f8_fwd(desc, x.contiguous(), packed, residual=old))
    assert torch.equal(wide_y[:, :9], before[:, :9]) and torch.equal(wide_y[:, 109:], before[:, 109:])


def test_input_gradient(ss):
    """The forward weights, packed transposed, give the gradient of the input: dx = q(dy) q(W^T)^T."""
    g = gen(13)
    W, dy = (torch.randn((70, 150), generator=g) / 8).bfloat16(), torch.randn((45, 70), generator=g).bfloat16()
    desc_t = ss.make_desc(150, 70, 1, 1, ss.SS_BF16)
    got = ss.ss_pw_f8_fwd(desc_t, dy.cuda(), ss.ss_f8_pack(desc_t, W.cuda(), transposed=True)).cpu().double()
    Wq, gq = ref.quantize(W.t().contiguous())[2], ref.quantize(dy)[2]
    want = gq @ Wq.t()
    assert ((got - want).abs() <= bound(Wq, gq, want, torch.bfloat16, 70)).all()


def test_no_rows(ss):
    desc = ss.make_desc(60, 100, 1, 1, ss.SS_F16)
    packed = ss.ss_f8_pack(desc, torch.ones((60, 100), dtype=torch.float16, device="cuda"))
    x = torch.empty((0, 100), dtype=torch.float16, device="cuda")
    codes, scales = ss.ss_f8_quantize(x)
    assert codes.shape == (0, 128) and scales.shape == (0, 4)
    assert ss.ss_pw_f8_fwd(desc, x, packed).shape == (0, 60) and ss.ss_pw_f8_q_fwd(desc, codes, scales, packed).shape == (0, 60)
    assert ss.ss_f8_dequantize(codes, scales, 100, torch.float16).shape == (0, 100)


def test_refusals(ss):
    desc = ss.make_desc(60, 100, 1, 1, ss.SS_F16)
    W = torch.ones((60, 100), dtype=torch.float16, device="cuda")
    packed = ss.ss_f8_pack(desc, W)
    x = torch.ones((5, 100), dtype=torch.float16, device="cuda")
    codes, scales = ss.ss_f8_quantize(x)
    dy = torch.ones((5, 60), dtype=torch.float16, device="cuda")
    for call in (lambda: ss.ss_f8_quantize(x.cpu()), lambda: ss.ss_f8_quantize(x.t()), lambda: ss.ss_f8_quantize(x.double()), lambda: ss.ss_f8_quantize(x, codes[:, :64]),
                 lambda: ss.ss_f8_dequantize(codes, scales, 129), lambda: ss.ss_f8_dequantize(codes, scales[:4], 100),
                 lambda: ss.ss_f8_pack(desc, W.t().contiguous()), lambda: ss.ss_f8_pack(desc, W, transposed=True), lambda: ss.ss_f8_pack(desc, W.bfloat16()),
                 lambda: ss.ss_pw_f8_fwd(desc, x.bfloat16(), packed), lambda: ss.ss_pw_f8_fwd(desc, x[:, :99], packed), lambda: ss.ss_pw_f8_fwd(desc, x, packed[:-1]),
                 lambda: ss.ss_pw_f8_fwd(desc, x, packed, act=3), lambda: ss.ss_pw_f8_fwd(desc, x, packed, bias=torch.ones(59, device="cuda")),
                 lambda: ss.ss_pw_f8_fwd(desc, x, packed, residual=dy[:4]), lambda: ss.ss_pw_f8_q_fwd(desc, codes[:4], scales, packed),
                 lambda: ss.ss_f8_packed_bytes(ss.make_desc(8, 8, 3, 3, ss.SS_F16)), lambda: ss.ss_f8_packed_bytes(ss.make_desc(8, 8, 1, 1, ss.SS_F8)),
                 lambda: ss.ss_f8_packed_bytes(ss.make_desc(8, (1 << 22) + 1, 1, 1, ss.SS_F16))):
        with pytest.raises(ss.SSError):
            call()
