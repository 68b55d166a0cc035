"""The 64-bit definitions that the GPU tests compare with: the MXFP4 format's closed forms, and gradients against differences."""
import numpy as np
import pytest

import rows_reference as ref


def test_format_closed_forms():
    one = np.zeros((1, 32))
    one[0, :13] = [6, -6, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.0, 0.5]
    codes, scales = ref.quantize(one)
    got = ref.dequantize(codes, scales, 32)[0, :13]
    assert scales[0].tolist() == [127, 0, 0, 0]
    assert got.tolist() == [6, -6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, 0, 0.5] and np.signbit(got[11])
    # the scale is two below the exponent of the largest: 7.9 saturates at 6, 8 does not
    assert ref.through_mx4(np.full((1, 1), 7.9))[0, 0] == 6 and ref.through_mx4(np.full((1, 1), 8.0))[0, 0] == 8
    assert ref.quantize(np.zeros((2, 33)))[1].tolist() == [[0, 0, 0, 0]] * 2
    assert ref.quantize(np.full((1, 1), 2.0 ** -149))[1][0, 0] == 0
    assert ref.quantize(np.array([[np.nan] + [0] * 31 + [np.inf]]))[1][0].tolist() == [255, 255, 0, 0]


def test_every_value_survives():
    for e in (-120, -1, 0, 7, 100):
        v = np.concatenate([ref.VALUES, -ref.VALUES])[None] * 2.0 ** e
        assert np.array_equal(ref.through_mx4(v), v)


@pytest.mark.parametrize("kinds", [(1, 0), (2, 0), (1, 1), (2, 2), (1, 2), (0, 1), (2, 1), (0, 0)])
@pytest.mark.parametrize("gate", [None, (6, 1), (2, 1), (6, 7), (3, 7)])
def test_gradients_against_differences(kinds, gate):
    rng = np.random.default_rng(kinds[0] * 10 + kinds[1])
    p = {"x": rng.standard_normal((6, 7)), "h": rng.standard_normal((6, 7)), "w": 1 + 0.3 * rng.standard_normal(7), "b": rng.standard_normal(7),
         "scale": rng.standard_normal(7), "gate": None if gate is None else rng.standard_normal(gate), "post_w": 1 + 0.3 * rng.standard_normal(7),
         "post_b": rng.standard_normal(7)}
    dy, dx_out = rng.standard_normal((6, 7)), rng.standard_normal((6, 7))

    def loss(q):
        x_out, y = ref.block_forward(q, kinds)
        return (x_out * dx_out).sum() + (0.0 if y is None else (y * dy).sum())

    at = dict(p, x=ref.block_forward(p, kinds)[0])
    grads = ref.block_backward(at, kinds, dy, dx_out)
    names = {"x": "dx", "h": "dh", "scale": "dscale"}
    names.update({"w": "dw", "b": "db"} if kinds[0] else {})
    names.update({"post_w": "dpost_w", "post_b": "dpost_b"} if kinds[1] else {})
    names.update({"gate": "dgate"} if gate else {})
    for name, g in names.items():
        for i in np.ndindex(p[name].shape):
            up, down = ({**p, name: p[name].copy()} for _ in range(2))
            up[name][i] += 1e-5
            down[name][i] -= 1e-5
            assert abs((loss(up) - loss(down)) / 2e-5 - grads[g][i]) < 1e-6 * (1 + abs(grads[g][i])), (name, i)


def test_host_side_sizes_and_refusals():
    import paper_2411_00288_amd as ss
    assert ss.ss_mx4_packed_bytes(ss.make_desc(40, 100, 1, 1)) == 256 + 2 * 2 * 1024 + 2 * 256       # 4 blocks: 2 steps, 1 scale word
    assert ss.ss_mx4_packed_bytes(ss.make_desc(1, 1, 1, 1, ss.SS_BF16)) == 256 + 1024 + 256
    for bad, code in [(ss.make_desc(8, 8, 3, 3), ss.SS_ERR_UNSUPPORTED), (ss.make_desc(8, 8, 1, 1, ss.SS_I8), ss.SS_ERR_UNSUPPORTED),
                      (ss.make_desc(8, 0, 1, 1), ss.SS_ERR_INVALID_ARG), (ss.make_desc(8, 8, 1, 1, ss.SS_F32), ss.SS_ERR_INVALID_ARG)]:
        for query in (ss.ss_mx4_packed_bytes, lambda d: ss.ss_pw_mx4_workspace_bytes(d, 4)):
            with pytest.raises(ss.SSError) as e:
                query(bad)
            assert e.value.status == code
    with pytest.raises(ss.SSError):
        ss.ss_pw_mx4_workspace_bytes(ss.make_desc(8, 8, 1, 1), -1)
    norm = ss.make_norm_desc(96)
    assert ss.ss_norm_bwd_workspace_bytes(norm, 0) == 0 and ss.ss_norm_bwd_workspace_bytes(norm, 64, 8, 1) > 0
    for bad in [(ss.make_norm_desc(0), 4, 0, 0), (ss.make_norm_desc(8, ss.SS_I8), 4, 0, 0), (ss.make_norm_desc(8, norm=3), 4, 0, 0), (ss.make_norm_desc(8, post=-1), 4, 0, 0),
                (ss.make_norm_desc(8, eps=-1.0), 4, 0, 0), (ss.make_norm_desc(8, eps=float("nan")), 4, 0, 0), (ss.make_norm_desc(8, post_eps=float("inf")), 4, 0, 0),
                (norm, -1, 0, 0), (norm, 4, 3, 1), (norm, 4, 0, 1), (norm, 4, 2, 7)]:
        with pytest.raises(ss.SSError) as e:
            ss.ss_norm_bwd_workspace_bytes(*bad)
        assert e.value.status == ss.SS_ERR_INVALID_ARG
    with pytest.raises(ss.SSError) as e:
        ss.ss_norm_bwd_workspace_bytes(ss.make_norm_desc(16385), 4)
    assert e.value.status == ss.SS_ERR_UNSUPPORTED
