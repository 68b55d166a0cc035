"""What the calls on FP8 blocks, the weight gradient and the group norm refuse, through the C interface: none of these reaches a device."""
import ctypes

import pytest

import paper_2411_00288_amd as ss

lib = ss.binding._lib
P = ctypes.c_void_p(4096)                                       # an aligned address that nothing reads
ODD = ctypes.c_void_p(4097)
INVALID, UNSUPPORTED, WORKSPACE = ss.SS_ERR_INVALID_ARG, ss.SS_ERR_UNSUPPORTED, ss.SS_ERR_WORKSPACE


@pytest.mark.parametrize("args,status", [
    ((None, 5, 64, 64, 0, P, P), INVALID), ((P, -1, 64, 64, 0, P, P), INVALID), ((P, 5, 0, 64, 0, P, P), INVALID), ((P, 5, 64, 63, 0, P, P), INVALID),
    ((P, 5, 64, 64, 2, P, P), INVALID), ((P, 5, 64, 64, 0, ODD, P), INVALID), ((P, 5, 64, 64, 0, P, ODD), INVALID), ((ODD, 5, 64, 64, 0, P, P), INVALID),
    ((P, 1 << 31, 64, 64, 0, P, P), UNSUPPORTED), ((P, 5, (1 << 22) + 1, 1 << 23, 0, P, P), UNSUPPORTED), ((P, 5, 64, 1 << 31, 0, P, P), UNSUPPORTED),
    ((None, 0, 64, 64, 0, None, None), ss.SS_OK)])
def test_quantize(args, status):
    assert lib.ss_f8_quantize(*args, None) == status
    x, rows, cols, ld, dtype, codes, scales = args
    assert lib.ss_f8_dequantize(codes, scales, rows, cols, dtype, x, ld, None) == status


def test_weights():
    size = ctypes.c_size_t()
    for desc, status in ((ss.make_desc(64, 64, 1, 1, ss.SS_F16), ss.SS_OK), (ss.make_desc(64, 64, 3, 3, ss.SS_F16), UNSUPPORTED), (ss.make_desc(64, 64, 1, 1, ss.SS_F8), UNSUPPORTED),
                         (ss.make_desc(0, 64, 1, 1, ss.SS_F16), INVALID), (ss.make_desc(1, (1 << 22) + 1, 1, 1, ss.SS_F16), UNSUPPORTED), (ss.make_desc(1 << 26, 1, 1, 1, ss.SS_F16), UNSUPPORTED)):
        assert lib.ss_f8_packed_bytes(ctypes.byref(desc), ctypes.byref(size)) == status
        assert lib.ss_f8_unpack(ctypes.byref(desc), None, P, None) == (status or INVALID)
        assert lib.ss_f8_pack(ctypes.byref(desc), None, None, 0, P, None) == (status or INVALID)
    desc = ss.make_desc(100, 200, 1, 1, ss.SS_BF16)
    assert ss.ss_f8_packed_bytes(desc) == 256 + 4 * 4 * 2048 + 4 * 1 * 128
    assert lib.ss_f8_pack(ctypes.byref(desc), P, None, 2, P, None) == INVALID
    assert lib.ss_f8_pack(ctypes.byref(desc), P, None, 0, ODD, None) == INVALID
    assert lib.ss_weights_check(ctypes.byref(ss.make_desc(8, 8, 3, 3, ss.SS_F16)), P, ss.SS_WEIGHTS_F8, None) == UNSUPPORTED


def test_layer():
    d = ctypes.byref(ss.make_desc(100, 200, 1, 1, ss.SS_BF16))

    def fwd(x=P, rows=5, ldx=200, packed=P, bias=None, residual=None, ldr=0, act=0, y=P, ldy=100, ws=None, ws_bytes=0):
        return lib.ss_pw_f8_fwd(d, x, rows, ldx, packed, bias, residual, ldr, act, y, ldy, ws, ws_bytes, None)
    for call, status in ((dict(x=None), INVALID), (dict(x=ODD), INVALID), (dict(ldx=199), INVALID), (dict(rows=-1), INVALID), (dict(packed=None), INVALID), (dict(packed=ODD), INVALID),
                         (dict(y=None), INVALID), (dict(ldy=99), INVALID), (dict(act=3), INVALID), (dict(act=-1), INVALID), (dict(residual=P, ldr=99), INVALID),
                         (dict(bias=ctypes.c_void_p(4098)), INVALID), (dict(rows=1 << 31), UNSUPPORTED), (dict(ldx=1 << 31), UNSUPPORTED), (dict(ldy=1 << 31), UNSUPPORTED),
                         (dict(rows=0, x=None, packed=None, y=None), ss.SS_OK)):
        assert fwd(**call) == status, call
    big = ss.make_desc(8192, 8192, 1, 1, ss.SS_BF16)
    need = ss.ss_pw_f8_workspace_bytes(big, 4096)
    assert need >= 4096 * 8192 + 4096 * 64
    args = (ctypes.byref(big), P, 4096, 8192, P, None, None, 0, 0, P, 8192)
    assert lib.ss_pw_f8_fwd(*args, P, need - 1, None) == WORKSPACE and lib.ss_pw_f8_fwd(*args, None, need, None) == WORKSPACE and lib.ss_pw_f8_fwd(*args, ODD, need, None) == WORKSPACE
    assert lib.ss_pw_f8_q_fwd(d, None, P, 5, P, None, None, 0, 0, P, 100, None) == INVALID
    assert lib.ss_pw_f8_q_fwd(d, P, ODD, 5, P, None, None, 0, 0, P, 100, None) == INVALID


def test_weight_gradient():
    desc = ss.make_desc(100, 200, 1, 1, ss.SS_BF16)
    d, need = ctypes.byref(desc), ss.ss_pw_wgrad_workspace_bytes(desc, 50)

    def call(dy=P, lddy=100, x=P, ldx=200, rows=50, dw=P, db=None, ws=P, ws_bytes=need):
        return lib.ss_pw_wgrad(d, dy, lddy, x, ldx, rows, dw, db, ws, ws_bytes, None)
    for args, status in ((dict(dy=None), INVALID), (dict(x=ODD), INVALID), (dict(lddy=99), INVALID), (dict(ldx=199), INVALID), (dict(rows=-1), INVALID), (dict(dw=None), INVALID),
                         (dict(dw=ctypes.c_void_p(4098)), INVALID), (dict(db=ctypes.c_void_p(4098)), INVALID), (dict(ldx=(1 << 23) + 1), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
                         (dict(ws=None), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE), (dict(ws=ctypes.c_void_p(4104)), WORKSPACE)):
        assert call(**args) == status, args
    assert ss.ss_pw_wgrad_workspace_bytes(desc, 0) == 0


def test_group_norm():
    desc = ss.make_groupnorm_desc(24, 3, ss.SS_F16, ss.SS_ACT_SILU)

    def fwd(desc=desc, x=P, ldx=24, images=2, pixels=9, y=P, ldy=24, stats=P, ws=None, ws_bytes=0):
        return lib.ss_groupnorm_fwd(ctypes.byref(desc), x, ldx, images, pixels, None, None, y, ldy, stats, ws, ws_bytes, None)

    def bwd(desc=desc, dy=P, lddy=24, x=P, ldx=24, images=2, pixels=9, stats=P, dx=P, lddx=24, ws=P, ws_bytes=1 << 20):
        return lib.ss_groupnorm_bwd(ctypes.byref(desc), dy, lddy, x, ldx, images, pixels, stats, None, None, dx, lddx, None, None, ws, ws_bytes, None)
    make = ss.make_groupnorm_desc
    for bad, status in ((make(24, 5, 0), INVALID), (make(24, 0, 0), INVALID), (make(0, 1, 0), INVALID), (make(24, 3, 2), INVALID), (make(24, 3, 0, 4), INVALID), (make(24, 3, 0, -1), INVALID),
                        (make(24, 3, 0, 0, -1e-9), INVALID), (make(24, 3, 0, 0, float("inf")), INVALID), (make(24, 3, 0, 0, float("nan")), INVALID), (make(16400, 1, 0), UNSUPPORTED)):
        assert fwd(bad) == status and bwd(bad) == status
    for args, status in ((dict(x=None), INVALID), (dict(x=ODD), INVALID), (dict(ldx=23), INVALID), (dict(images=-1), INVALID), (dict(pixels=-1), INVALID), (dict(images=1 << 31), UNSUPPORTED),
                         (dict(pixels=(1 << 24) + 1), UNSUPPORTED), (dict(images=1 << 16, pixels=1 << 16), UNSUPPORTED), (dict(ldx=(1 << 19) + 1), UNSUPPORTED), (dict(stats=ctypes.c_void_p(4100)), INVALID)):
        assert fwd(**args) == status and bwd(**args) == status, args
    assert fwd(y=None) == INVALID and fwd(ldy=23) == INVALID
    assert bwd(dy=None) == INVALID and bwd(lddy=23) == INVALID and bwd(dx=None) == INVALID and bwd(stats=None) == INVALID and bwd(ws=None) == WORKSPACE
    assert fwd(images=0, x=None, y=None) == ss.SS_OK and fwd(pixels=0, x=None, y=None) == ss.SS_OK
    large = make(2048, 1, ss.SS_F32)
    assert fwd(large, ldx=2048, ldy=2048, pixels=100000) == WORKSPACE
