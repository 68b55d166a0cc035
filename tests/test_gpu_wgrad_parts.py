"""The weight gradient's join of the sums' parts: few and many, of matrices whose size is no multiple of a vector, into outputs on any element; and subnormal operands."""
import pytest
import torch

from test_gpu_wgrad import KERNELS, check, operands

pytestmark = pytest.mark.gpu


def gradient(ss, dy, x, dtype):
    rows, cout, cin = len(x), dy.shape[1], x.shape[1]
    out = torch.full((cout * cin + 2,), 5.0, device="cuda")
    bias = torch.full((cout + 2,), 5.0, device="cuda")
    dw, db = ss.ss_pw_wgrad(ss.make_desc(cout, cin, 1, 1, ss.SS_F16 if dtype == "f16" else ss.SS_BF16), dy.cuda(), x.cuda(), dw=out[1:-1].view(cout, cin), db=bias[1:-1])
    assert out[0] == 5 and out[-1] == 5 and bias[0] == 5 and bias[-1] == 5
    return dw, db


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,cin,cout", [(700, 33, 65), (9001, 33, 65), (5000, 1, 3), (6001, 131, 129), (520, 7, 9)])
def test_sizes(ss, rows, cin, cout, dtype):
    assert cin * cout % 4
    dy, x = operands(rows + cin, rows, cin, cout, dtype)
    check(dy, x, *gradient(ss, dy, x, dtype))


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("parts", [1, 2, 3, 15, 16, 17, 40])
@pytest.mark.parametrize("rows,cin,cout", [(5003, 33, 65), (5003, 100, 36), (None, 33, 65)])
def test_parts(ss, force_tile, force_split, kernel, parts, rows, cin, cout):
    chunk = {"tile_64": 128, "tile_128": 64, "tile_256": 32}[kernel]
    rows = parts * 384 - 5 if rows is None else rows         # (as many as asked for; otherwise whole chunks of rows may leave fewer)
    per = -(-(-(-rows // parts)) // chunk) * chunk
    made = -(-rows // per)
    dy, x = operands(parts, rows, cin, cout, "bf16")
    force_tile(KERNELS[kernel])
    force_split(parts)
    desc = ss.make_desc(cout, cin, 1, 1, ss.SS_BF16)
    assert ss.ss_pw_wgrad_workspace_bytes(desc, rows) == (-(-made * cout * cin * 4 // 256) * 256 if made > 1 else 0) + made * cout * 4
    dw, db = gradient(ss, dy, x, "bf16")
    check(dy, x, dw, db)
    again = gradient(ss, dy, x, "bf16")
    assert torch.equal(dw, again[0]) and torch.equal(db, again[1])


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_subnormal_operands(ss, force_tile, kernel, dtype):
    """Gradients below the types' least normal value count as what they are."""
    g = torch.Generator().manual_seed(3)
    t, least = (torch.float16, 2.0 ** -24) if dtype == "f16" else (torch.bfloat16, 2.0 ** -133)
    steps = torch.randint(1, 1024 if dtype == "f16" else 128, (600, 70), generator=g).double()
    dy, x = (steps * least).to(t), (torch.randn((600, 50), generator=g) * 256).to(t)
    assert torch.equal(dy.double(), steps * least)
    force_tile(KERNELS[kernel])
    dw, db = gradient(ss, dy, x, dtype)
    if dtype == "f16":
        check(dy, x, dw, db)
    else:
        # (the bias's sums are subnormal in fp32, too, or little more)
        check(dy, x, dw, None)
        assert bool(((db.cpu().double() - dy.double().sum(dim=0)).abs() <= 2.0 ** -126).all())
