"""Binding over the C ABI declared in include/ss.h.

Argument marshalling only: every step of the path (compression, convolution, epilogue) runs in
the HIP library.  PyTorch provides device memory and the stream.  There is no fallback: if the
library has not been built, importing fails with an instruction to build it.

A plain good call goes through the extension module ``_native`` (csrc/ss_python.cpp): it checks, allocates
and enqueues in compiled code.  Where that declines (returns None: something is wrong with the arguments, or an option it
does not handle, such as an explicit stream), the checks below find the reason and report it, or make the call through
ctypes.
"""
from __future__ import annotations

import ctypes
from pathlib import Path
from typing import NamedTuple

import torch

_HERE = Path(__file__).resolve().parent
LIB_PATH = _HERE / "libss.so"

SS_OK = 0
SS_ERR_INVALID_ARG, SS_ERR_BAD_MASK, SS_ERR_UNSUPPORTED, SS_ERR_WORKSPACE, SS_ERR_HIP = -1, -2, -3, -4, -5
SS_F16, SS_BF16, SS_I8, SS_F8, SS_F32 = 0, 1, 2, 3, 4
SS_K_CRS, SS_K_RSC = 0, 1
SS_ACT_NONE, SS_ACT_RELU, SS_ACT_GELU, SS_ACT_SILU = 0, 1, 2, 3
SS_WEIGHTS_DENSE, SS_WEIGHTS_SPARSE, SS_WEIGHTS_MX4, SS_WEIGHTS_F8 = 0, 1, 2, 3
SS_NORM_NONE, SS_NORM_LAYER, SS_NORM_RMS = 0, 1, 2

EXPORTS = ["ss_status_string", "ss_packed_bytes", "ss_dense_bytes", "ss_mask_compress", "ss_mask_decompress",
           "ss_dense_pack", "ss_conv2d_workspace_bytes", "ss_conv2d_fwd", "ss_conv2d_dense_fwd",
           "ss_conv2d_res_fwd", "ss_conv2d_dense_res_fwd", "ss_mask_update_compress", "ss_maxpool2d", "ss_dwconv2d_fwd",
           "ss_conv2d_q8_fwd", "ss_conv2d_q8_dense_fwd", "ss_conv2d_pw_fused_fwd", "ss_conv2d_pw_fused_dense_fwd",
           "ss_weights_check", "ss_conv2d_fwd_static_ws", "ss_conv2d_pw_fused_query", "ss_conv2d_pw2_fused_fwd", "ss_conv2d_pw2_fused_dense_fwd",
           "ss_conv2d_pw2_fused_query", "ss_conv2d_maxpool_dense_fwd", "ss_conv2d_maxpool_dense_query",
           "ss_mx4_quantize", "ss_mx4_dequantize", "ss_mx4_packed_bytes", "ss_mx4_pack", "ss_mx4_unpack", "ss_pw_mx4_workspace_bytes",
           "ss_pw_mx4_fwd", "ss_pw_mx4_q_fwd", "ss_f8_quantize", "ss_f8_dequantize", "ss_f8_packed_bytes", "ss_f8_pack", "ss_f8_unpack",
           "ss_pw_f8_workspace_bytes", "ss_pw_f8_fwd", "ss_pw_f8_q_fwd", "ss_pw_wgrad_workspace_bytes", "ss_pw_wgrad", "ss_norm_fwd", "ss_norm_bwd_workspace_bytes", "ss_norm_bwd",
           "ss_groupnorm_workspace_bytes", "ss_groupnorm_fwd", "ss_groupnorm_bwd"]
DEBUG_EXPORTS = ["ss_debug_force_tile", "ss_debug_limit_blocks", "ss_debug_force_split", "ss_debug_issue_peak", "ss_debug_lds_bandwidth"]          # include/ss_debug.h: test hooks


class ss_weight_desc(ctypes.Structure):
    _fields_ = [("cout", ctypes.c_int32), ("cin", ctypes.c_int32), ("kh", ctypes.c_int32), ("kw", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("korder", ctypes.c_int32)]


class ss_norm_desc(ctypes.Structure):
    _fields_ = [("cols", ctypes.c_int32), ("dtype", ctypes.c_int32), ("norm", ctypes.c_int32), ("post", ctypes.c_int32),
                ("eps", ctypes.c_float), ("post_eps", ctypes.c_float)]


class ss_groupnorm_desc(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int32), ("groups", ctypes.c_int32), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("eps", ctypes.c_float),
                ("reserved", ctypes.c_int32)]


def _fields(text):
    """Fields of a struct of ss.h: a name with "#" is an int32, with "=" an int64, any other a pointer."""
    return [(n.rstrip("#="), ctypes.c_int32 if n.endswith("#") else ctypes.c_int64 if n.endswith("=") else ctypes.c_void_p) for n in text.split()]


class ss_norm_io(ctypes.Structure):
    _fields_ = _fields("rows= groups= gate_cols# x ldx= h ldh= gate scale post_w post_b x_out ldx_out= w b y ldy= codes scales")


class ss_norm_grad_io(ctypes.Structure):
    _fields_ = _fields("rows= groups= gate_cols# dy lddy= x_out ldx_out= dx_out lddx_out= h ldh= gate w scale post_w post_b dx lddx= dh lddh= "
                       "dgate dw db dscale dpost_w dpost_b")


class SSError(RuntimeError):
    def __init__(self, status: int, what: str, detail=None):
        self.status = status
        self.detail = detail
        super().__init__(f"{what}: {status_string(status)}" + (f" {detail}" if detail is not None else ""))


def _load() -> ctypes.CDLL:
    if not LIB_PATH.exists():
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()' "
            "or python paper_2411_00288_amd/build.py). There is no CPU fallback.")
    lib = ctypes.CDLL(str(LIB_PATH))
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dp = ctypes.POINTER(ss_weight_desc)
    lib.ss_status_string.restype = ctypes.c_char_p
    lib.ss_status_string.argtypes = [ctypes.c_int]
    lib.ss_packed_bytes.argtypes = [dp, ctypes.POINTER(sz)]
    lib.ss_dense_bytes.argtypes = [dp, ctypes.POINTER(sz)]
    lib.ss_mask_compress.argtypes = [dp, vp, vp, vp, ctypes.POINTER(i32), vp]
    lib.ss_mask_update_compress.argtypes = [dp, vp, vp, vp, vp, ctypes.POINTER(i32), vp]
    lib.ss_maxpool2d.argtypes = [vp, i32, i32, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.ss_dwconv2d_fwd.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, i32, i32, i32, i32, i32, vp, vp]
    lib.ss_mask_decompress.argtypes = [dp, vp, vp, vp]
    lib.ss_dense_pack.argtypes = [dp, vp, vp, vp, vp]
    lib.ss_conv2d_workspace_bytes.argtypes = [dp, i32, i32, i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
    conv_args = [dp, vp, i32, i32, i32, vp, vp, i32, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.ss_conv2d_fwd.argtypes = conv_args
    lib.ss_conv2d_dense_fwd.argtypes = conv_args
    res_args = conv_args[:7] + [vp] + conv_args[7:]          # residual after bias
    lib.ss_conv2d_res_fwd.argtypes = res_args
    lib.ss_conv2d_dense_res_fwd.argtypes = res_args
    q8_args = [dp, vp, i32, i32, i32, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.ss_conv2d_q8_fwd.argtypes = q8_args
    lib.ss_conv2d_q8_dense_fwd.argtypes = q8_args
    fused_args = [dp, vp, i32, i32, i32, vp, vp, i32, i32, i32, i32, i32, dp, vp, vp, vp, i32, vp, vp]
    lib.ss_conv2d_pw_fused_fwd.argtypes = fused_args
    lib.ss_conv2d_pw_fused_dense_fwd.argtypes = fused_args
    lib.ss_weights_check.argtypes = [dp, vp, i32, vp]
    lib.ss_conv2d_pw_fused_query.argtypes = [dp, i32, i32, i32, i32, dp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    third_args = fused_args[:-1] + [dp, vp, vp, i32, vp, vp]
    lib.ss_conv2d_pw2_fused_fwd.argtypes = third_args
    lib.ss_conv2d_pw2_fused_dense_fwd.argtypes = third_args
    lib.ss_conv2d_pw2_fused_query.argtypes = [dp, i32, i32, i32, i32, i32, i32, i32, dp, dp, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.ss_conv2d_maxpool_dense_fwd.argtypes = conv_args[:13] + [vp, vp]    # y, pooled, stream
    lib.ss_conv2d_maxpool_dense_query.argtypes = [dp] + [i32] * 8 + [ctypes.POINTER(i32)]
    lib.ss_conv2d_fwd_static_ws.argtypes = conv_args[:13] + [vp]            # no workspace pair
    i64, nd = ctypes.c_int64, ctypes.POINTER(ss_norm_desc)
    lib.ss_mx4_quantize.argtypes = [vp, i64, i32, i64, i32, vp, vp, vp]
    lib.ss_mx4_dequantize.argtypes = [vp, vp, i64, i32, i32, vp, i64, vp]
    lib.ss_mx4_packed_bytes.argtypes = [dp, ctypes.POINTER(sz)]
    lib.ss_mx4_pack.argtypes = [dp, vp, vp, vp, vp]
    lib.ss_mx4_unpack.argtypes = [dp, vp, vp, vp]
    lib.ss_pw_mx4_workspace_bytes.argtypes = [dp, i64, ctypes.POINTER(sz)]
    lib.ss_pw_mx4_fwd.argtypes = [dp, vp, i64, i64, vp, vp, vp, i64, i32, vp, i64, vp, sz, vp]
    lib.ss_pw_mx4_q_fwd.argtypes = [dp, vp, vp, i64, vp, vp, vp, i64, i32, vp, i64, vp]
    lib.ss_f8_quantize.argtypes = lib.ss_mx4_quantize.argtypes
    lib.ss_f8_dequantize.argtypes = lib.ss_mx4_dequantize.argtypes
    lib.ss_f8_packed_bytes.argtypes = lib.ss_mx4_packed_bytes.argtypes
    lib.ss_f8_pack.argtypes = [dp, vp, vp, i32, vp, vp]
    lib.ss_f8_unpack.argtypes = lib.ss_mx4_unpack.argtypes
    lib.ss_pw_f8_workspace_bytes.argtypes = lib.ss_pw_mx4_workspace_bytes.argtypes
    lib.ss_pw_f8_fwd.argtypes = lib.ss_pw_mx4_fwd.argtypes
    lib.ss_pw_f8_q_fwd.argtypes = lib.ss_pw_mx4_q_fwd.argtypes
    lib.ss_pw_wgrad_workspace_bytes.argtypes = lib.ss_pw_mx4_workspace_bytes.argtypes
    lib.ss_pw_wgrad.argtypes = [dp, vp, i64, vp, i64, i64, vp, vp, vp, sz, vp]
    lib.ss_norm_fwd.argtypes = [nd, ctypes.POINTER(ss_norm_io), vp]
    lib.ss_norm_bwd_workspace_bytes.argtypes = [nd, i64, i64, i32, ctypes.POINTER(sz)]
    lib.ss_norm_bwd.argtypes = [nd, ctypes.POINTER(ss_norm_grad_io), vp, sz, vp]
    gd = ctypes.POINTER(ss_groupnorm_desc)
    lib.ss_groupnorm_workspace_bytes.argtypes = [gd, i64, i64, i32, ctypes.POINTER(sz)]
    lib.ss_groupnorm_fwd.argtypes = [gd, vp, i64, i64, i64, vp, vp, vp, i64, vp, vp, sz, vp]
    lib.ss_groupnorm_bwd.argtypes = [gd, vp, i64, vp, i64, i64, i64, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
    lib.ss_debug_force_tile.argtypes = [i32]
    lib.ss_debug_limit_blocks.argtypes = [i32]
    lib.ss_debug_force_split.argtypes = [i32]
    lib.ss_debug_issue_peak.argtypes = [i32, i32, vp, sz, ctypes.POINTER(ctypes.c_float), vp]
    lib.ss_debug_lds_bandwidth.argtypes = [i32, i32, i32, vp, sz, ctypes.POINTER(ctypes.c_float), vp]
    for name in EXPORTS[1:] + DEBUG_EXPORTS:
        getattr(lib, name).restype = ctypes.c_int
    return lib


_lib = _load()
from . import _native  # noqa: E402  (links against the library loaded above)


def status_string(status: int) -> str:
    return _lib.ss_status_string(int(status)).decode()


def make_desc(cout, cin, kh, kw, dtype=SS_F16, korder=SS_K_CRS) -> ss_weight_desc:
    return ss_weight_desc(int(cout), int(cin), int(kh), int(kw), int(dtype), int(korder))


def _stream_ptr(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dev_ptr(t, name, dtypes=None, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise SSError(SS_ERR_INVALID_ARG, f"{name} is None")
    if not t.is_cuda:
        raise SSError(SS_ERR_INVALID_ARG, f"{name} must live in device memory")
    if not t.is_contiguous():
        raise SSError(SS_ERR_INVALID_ARG, f"{name} must be contiguous")
    if dtypes is not None and t.dtype not in dtypes:
        raise SSError(SS_ERR_INVALID_ARG, f"{name} has dtype {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


_T16 = (torch.float16, torch.bfloat16, torch.int16, torch.uint16)
_T8 = (torch.int8, torch.uint8, torch.float8_e4m3fn)


def _wtypes(desc):
    """Tensor dtypes accepted for weights of a descriptor."""
    return _T8 if desc.dtype in (SS_I8, SS_F8) else _T16


def torch_dtype(dtype: int):
    return {SS_F16: torch.float16, SS_BF16: torch.bfloat16, SS_I8: torch.int8, SS_F8: torch.uint8}[dtype]


def ss_packed_bytes(desc: ss_weight_desc) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_packed_bytes(ctypes.byref(desc), ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_packed_bytes")
    return int(out.value)


def ss_dense_bytes(desc: ss_weight_desc) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_dense_bytes(ctypes.byref(desc), ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_dense_bytes")
    return int(out.value)


def _failed(r, what):
    """Raises the SSError for the (status, row, block) of a call that the compiled path made and that failed: it is not made again."""
    raise SSError(r[0], what, detail=(r[1], r[2]) if r[0] == SS_ERR_BAD_MASK else None)


def ss_mask_compress(desc: ss_weight_desc, W: torch.Tensor, M: torch.Tensor, packed: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """W [cout, K] 16-bit, M [cout, K] uint8 (device) -> packed uint8 buffer (device)."""
    if stream is None:
        r = _native.pack(0, desc, W, None, M, packed)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_mask_compress")
    K = desc.cin * desc.kh * desc.kw
    if W is not None and W.numel() != desc.cout * K or M is not None and M.numel() != desc.cout * K:
        raise SSError(SS_ERR_INVALID_ARG, "ss_mask_compress: W/M size does not match the descriptor")
    if packed is None:
        packed = torch.empty(ss_packed_bytes(desc), dtype=torch.uint8, device=W.device)
    elif packed.numel() * packed.element_size() < ss_packed_bytes(desc):
        raise SSError(SS_ERR_INVALID_ARG, "ss_mask_compress: packed buffer too small")
    bad = (ctypes.c_int32 * 2)(-1, -1)
    st = _lib.ss_mask_compress(ctypes.byref(desc), _dev_ptr(W, "W", _wtypes(desc)), _dev_ptr(M, "M", (torch.uint8, torch.bool)),
                               _dev_ptr(packed, "packed"), bad, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_mask_compress", detail=(bad[0], bad[1]) if st == SS_ERR_BAD_MASK else None)
    return packed


def ss_mask_update_compress(desc: ss_weight_desc, W: torch.Tensor, U: torch.Tensor, M: torch.Tensor,
                            packed: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """W <- round16(W + U) in place, and packed <- compress(W, M): re-packing after a weight update."""
    if stream is None:
        r = _native.pack(1, desc, W, U, M, packed)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_mask_update_compress")
    K = desc.cin * desc.kh * desc.kw
    if W is None or U is None or M is None or W.numel() != desc.cout * K or U.numel() != desc.cout * K or \
            M.numel() != desc.cout * K or U.dtype != W.dtype:
        raise SSError(SS_ERR_INVALID_ARG, "ss_mask_update_compress: W/U/M do not match the descriptor")
    if packed is None:
        packed = torch.empty(ss_packed_bytes(desc), dtype=torch.uint8, device=W.device)
    elif packed.numel() * packed.element_size() < ss_packed_bytes(desc):
        raise SSError(SS_ERR_INVALID_ARG, "ss_mask_update_compress: packed buffer too small")
    bad = (ctypes.c_int32 * 2)(-1, -1)
    st = _lib.ss_mask_update_compress(ctypes.byref(desc), _dev_ptr(W, "W", _T16), _dev_ptr(U, "U", _T16),
                                      _dev_ptr(M, "M", (torch.uint8, torch.bool)), _dev_ptr(packed, "packed"), bad,
                                      _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_mask_update_compress", detail=(bad[0], bad[1]) if st == SS_ERR_BAD_MASK else None)
    return packed


def ss_mask_decompress(desc: ss_weight_desc, packed: torch.Tensor, out: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    K = desc.cin * desc.kh * desc.kw
    if out is None:
        out = torch.empty((desc.cout, K), dtype=torch_dtype(desc.dtype), device=packed.device)
    st = _lib.ss_mask_decompress(ctypes.byref(desc), _dev_ptr(packed, "packed"), _dev_ptr(out, "out", _wtypes(desc)),
                                 _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_mask_decompress")
    return out


def ss_dense_pack(desc: ss_weight_desc, W: torch.Tensor, M: torch.Tensor | None, dense: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
    if stream is None:
        r = _native.pack(2, desc, W, None, M, dense)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_dense_pack")
    K = desc.cin * desc.kh * desc.kw
    if W.numel() != desc.cout * K or (M is not None and M.numel() != desc.cout * K):
        raise SSError(SS_ERR_INVALID_ARG, "ss_dense_pack: W/M size does not match the descriptor")
    if dense is None:
        dense = torch.empty(ss_dense_bytes(desc), dtype=torch.uint8, device=W.device)
    elif dense.numel() * dense.element_size() < ss_dense_bytes(desc):
        raise SSError(SS_ERR_INVALID_ARG, "ss_dense_pack: dense buffer too small")
    st = _lib.ss_dense_pack(ctypes.byref(desc), _dev_ptr(W, "W", _wtypes(desc)),
                            _dev_ptr(M, "M", (torch.uint8, torch.bool), allow_none=True),
                            _dev_ptr(dense, "dense"), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_dense_pack")
    return dense


def ss_weights_check(desc: ss_weight_desc, weights: torch.Tensor, sparse: bool | int = True, stream=None) -> None:
    """Raises unless `weights` was written for `desc` by the matching packing call (and, for the sparse form, with a
    valid mask); sparse: True, False, or SS_WEIGHTS_MX4 / SS_WEIGHTS_F8 for weights of ss_mx4_pack / ss_f8_pack.  One stream
    synchronisation; call once per buffer at set-up."""
    kind = sparse if sparse in (SS_WEIGHTS_MX4, SS_WEIGHTS_F8) else SS_WEIGHTS_SPARSE if sparse else SS_WEIGHTS_DENSE
    need = (ss_dense_bytes, ss_packed_bytes, ss_mx4_packed_bytes, ss_f8_packed_bytes)[kind](desc)
    if weights is None or weights.numel() * weights.element_size() < need:
        raise SSError(SS_ERR_INVALID_ARG, "ss_weights_check: buffer smaller than the descriptor's size query")
    st = _lib.ss_weights_check(ctypes.byref(desc), _dev_ptr(weights, "weights"), kind, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_weights_check")


def ss_debug_force_tile(tile_id: int) -> None:
    """Test hook (include/ss_debug.h): force the convolution kernels' tile variant; negative = library's choice."""
    _lib.ss_debug_force_tile(int(tile_id))


def ss_debug_limit_blocks(n: int) -> None:
    """Test hook (include/ss_debug.h): cap the workgroups of the resident-grid kernels; 0 = no cap."""
    _lib.ss_debug_limit_blocks(int(n))


def ss_debug_force_split(n: int) -> None:
    """Test hook (include/ss_debug.h): force the number of workgroups per output tile; 0 = the library decides."""
    _lib.ss_debug_force_split(int(n))


def ss_debug_issue_peak(dtype: int = SS_F16, sparse: bool = True, stream=None) -> float:
    """Calibration probe (include/ss_debug.h): register-only issue rate of the matrix instruction, dense-equivalent
    TFLOP/s."""
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    out = ctypes.c_float(0.0)
    st = _lib.ss_debug_issue_peak(int(dtype), 1 if sparse else 0, _dev_ptr(scratch, "scratch"), scratch.numel(),
                                  ctypes.byref(out), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_debug_issue_peak")
    return float(out.value)


def ss_debug_lds_bandwidth(write: int, waves_per_simd: int, row_bytes: int = 592, stream=None) -> float:
    """Calibration probe (include/ss_debug.h): LDS bandwidth of one compute unit, GB/s."""
    scratch = torch.empty(2 << 20, dtype=torch.uint8, device="cuda")
    out = ctypes.c_float(0.0)
    st = _lib.ss_debug_lds_bandwidth(int(write), int(waves_per_simd), int(row_bytes), _dev_ptr(scratch, "scratch"),
                                     scratch.numel(), ctypes.byref(out), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_debug_lds_bandwidth")
    return float(out.value)


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _check_operands(what, desc, wbuf, bias, sparse):
    """Sizes the asynchronous calls rely on and cannot check themselves: a short buffer would be read past its end."""
    need = ss_packed_bytes(desc) if sparse else ss_dense_bytes(desc)
    if _nbytes(wbuf) < need:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: weight buffer holds {_nbytes(wbuf)} bytes, the descriptor needs {need}")
    if bias is not None and bias.numel() < desc.cout:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: bias holds {bias.numel()} values, cout is {desc.cout}")


def ss_conv2d_workspace_bytes(desc, N, H, W, stride=(1, 1), pad=(0, 0)) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_conv2d_workspace_bytes(ctypes.byref(desc), N, H, W, stride[0], stride[1], pad[0], pad[1],
                                        ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_conv2d_workspace_bytes")
    return int(out.value)


def out_shape(desc, N, H, W, stride=(1, 1), pad=(0, 0)):
    if stride[0] <= 0 or stride[1] <= 0 or pad[0] < 0 or pad[1] < 0:
        raise SSError(SS_ERR_INVALID_ARG, "stride must be positive and pad non-negative")
    Ho = (H + 2 * pad[0] - desc.kh) // stride[0] + 1
    Wo = (W + 2 * pad[1] - desc.kw) // stride[1] + 1
    return (N, Ho, Wo, desc.cout)


def _conv_args(what, desc, x, wbuf, bias, stride, pad, act, y, workspace, stream, residual=None, with_res=False):
    if x is None or x.dim() != 4 or x.shape[3] != desc.cin:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: x must be NHWC with cin channels")
    N, H, W, _ = x.shape
    _check_operands(what, desc, wbuf, bias, "dense" not in what)
    shp = out_shape(desc, N, H, W, stride, pad)
    if shp[1] <= 0 or shp[2] <= 0:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: empty output")
    if y is None:
        y = torch.empty(shp, dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: y must be {shp} {x.dtype}")
    need = ss_conv2d_workspace_bytes(desc, N, H, W, stride, pad)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > 0 and workspace is None:
        workspace = torch.zeros(need, dtype=torch.uint8, device=x.device)      # the ticket counters must start at zero
        ws_bytes = need
    if residual is not None and (tuple(residual.shape) != shp or residual.dtype != x.dtype or not residual.is_contiguous()):
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: residual must be contiguous {shp} {x.dtype}")
    head = (ctypes.byref(desc), _dev_ptr(x, "x", (torch_dtype(desc.dtype),)), N, H, W, _dev_ptr(wbuf, "weights"),
            _dev_ptr(bias, "bias", (torch.float32,), allow_none=True))
    tail = (stride[0], stride[1], pad[0], pad[1], act,
            _dev_ptr(y, "y"), _dev_ptr(workspace, "workspace", allow_none=True), ws_bytes)
    args = head + ((_dev_ptr(residual, "residual", allow_none=True),) if with_res else ()) + tail
    return args, y, workspace


def _conv(fn, what, desc, x, wbuf, bias, stride, pad, act, y, workspace, stream, residual=None, with_res=False):
    args, y, _ws = _conv_args(what, desc, x, wbuf, bias, stride, pad, act, y, workspace, stream, residual, with_res)
    st = fn(*args, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return y


def _launch(what, kind, desc1, desc2, x, w1, w2, scale, bias1, bias2, residual, y, workspace, nhw, stride, pad, act1, act2=0, pool=None, third=None):
    """The callable that enqueues a marshalled call on torch's current stream (arguments checked by the caller).  third: descriptor, weights,
    bias, activation and output of a third layer."""
    def failed(st):
        raise SSError(st, what)
    tensors = (x, w1, w2, scale, bias1, bias2, residual, y, workspace)
    ptr = lambda t: None if t is None else t.data_ptr()
    last = None if third is None else (third[0], ptr(third[1]), ptr(third[2]), int(third[3]), ptr(third[4]))
    return _native.launch(kind, desc1, desc2, tuple(map(ptr, tensors)), _nbytes(workspace),
                          tuple(nhw), (stride[0], stride[1], pad[0], pad[1]), int(act1), int(act2), pool, last, (tensors, third), failed)


def prepare_conv2d(desc, x, wbuf, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None, workspace=None,
                   sparse=True, residual=None):
    """Marshal the arguments of ss_conv2d_fwd / ss_conv2d_dense_fwd (ss_conv2d_res_fwd / ss_conv2d_dense_res_fwd
    when a residual is given) once and return (launch, y):
    ``launch()`` enqueues the call on the current torch stream.  For launch-bound loops and graph
    capture, where per-call Python argument checking would dominate.  The tensors passed here
    must stay alive and in place for as long as ``launch`` is used."""
    with_res = residual is not None
    what = ("ss_conv2d_res_fwd" if sparse else "ss_conv2d_dense_res_fwd") if with_res else \
           ("ss_conv2d_fwd" if sparse else "ss_conv2d_dense_fwd")
    _args, y, ws = _conv_args(what, desc, x, wbuf, bias, stride, pad, act, y, workspace, None, residual, with_res)
    return _launch(what, 0 if sparse else 1, desc, None, x, wbuf, None, None, bias, None, residual, y, ws, x.shape[:3], stride, pad, act), y


def prepare_conv2d_maxpool_dense(desc, x, dense, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_RELU, y=None, pooled=None):
    """Marshal the arguments of ss_conv2d_maxpool_dense_fwd once; returns (launch, y, pooled), as prepare_conv2d does."""
    what = "ss_conv2d_maxpool_dense_fwd"
    _args, y, _ws = _conv_args(what, desc, x, dense, bias, stride, pad, act, y, None, None)
    N, Ho, Wo, C = y.shape
    shp = (N, (Ho - 1) // 2 + 1, (Wo - 1) // 2 + 1, C)
    if pooled is None:
        pooled = torch.empty(shp, dtype=y.dtype, device=y.device)
    elif tuple(pooled.shape) != shp or pooled.dtype != y.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: pooled must be {shp} {y.dtype}")
    _dev_ptr(pooled, "pooled")
    return _launch(what, 9, desc, None, x, dense, None, None, bias, None, None, y, pooled, x.shape[:3], stride, pad, act), y, pooled


def ss_conv2d_maxpool_dense_query(desc, nhw, stride, pad, act=SS_ACT_RELU):
    """Would ss_conv2d_maxpool_dense_fwd take the layer on an input of nhw = (N, H, W)?"""
    sup = ctypes.c_int32(0)
    st = _lib.ss_conv2d_maxpool_dense_query(ctypes.byref(desc), nhw[0], nhw[1], nhw[2], stride[0], stride[1], pad[0], pad[1], act, ctypes.byref(sup))
    if st != SS_OK:
        raise SSError(st, "ss_conv2d_maxpool_dense_query")
    return bool(sup.value)


def ss_conv2d_maxpool_dense_fwd(desc, x, dense, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_RELU, y=None, pooled=None):
    """The dense first layer of an image network and the 3x3 max pooling behind it in one kernel; returns (y, pooled)."""
    launch, y, pooled = prepare_conv2d_maxpool_dense(desc, x, dense, bias, stride, pad, act, y, pooled)
    launch()
    return y, pooled


def ss_conv2d_fwd(desc, x, packed, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None, workspace=None,
                  stream=None) -> torch.Tensor:
    """2:4-sparse convolution: x NHWC [N,H,W,cin] -> y NHWC [N,Ho,Wo,cout] (same 16-bit dtype)."""
    if stream is None:
        r = _native.conv(0, desc, x, packed, None, bias, None, stride, pad, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_conv2d_fwd")
    return _conv(_lib.ss_conv2d_fwd, "ss_conv2d_fwd", desc, x, packed, bias, stride, pad, act, y, workspace, stream)


def ss_conv2d_fwd_static_ws(desc, x, packed, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None,
                            stream=None) -> torch.Tensor:
    """ss_conv2d_fwd without a workspace argument: a split reduction's scratch is the library's own device array.
    `y` should be passed by callers that must not allocate (it is allocated here otherwise)."""
    what = "ss_conv2d_fwd_static_ws"
    if x is None or x.dim() != 4 or x.shape[3] != desc.cin:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: x must be NHWC with cin channels")
    N, H, W, _ = x.shape
    _check_operands(what, desc, packed, bias, True)
    shp = out_shape(desc, N, H, W, stride, pad)
    if shp[1] <= 0 or shp[2] <= 0:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: empty output")
    if y is None:
        y = torch.empty(shp, dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: y must be {shp} {x.dtype}")
    st = _lib.ss_conv2d_fwd_static_ws(ctypes.byref(desc), _dev_ptr(x, "x", (torch_dtype(desc.dtype),)), N, H, W,
                                      _dev_ptr(packed, "weights"), _dev_ptr(bias, "bias", (torch.float32,), allow_none=True),
                                      stride[0], stride[1], pad[0], pad[1], act, _dev_ptr(y, "y"), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return y


def ss_conv2d_dense_fwd(desc, x, dense, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None,
                        workspace=None, stream=None) -> torch.Tensor:
    """The dense-MFMA twin on the operand built by ss_dense_pack."""
    if stream is None:
        r = _native.conv(1, desc, x, dense, None, bias, None, stride, pad, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_conv2d_dense_fwd")
    return _conv(_lib.ss_conv2d_dense_fwd, "ss_conv2d_dense_fwd", desc, x, dense, bias, stride, pad, act, y,
                 workspace, stream)


def ss_conv2d_res_fwd(desc, x, packed, bias=None, residual=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None,
                      workspace=None, stream=None) -> torch.Tensor:
    """2:4-sparse convolution closing a residual block: y = act(conv(x) + bias + residual), residual NHWC like y."""
    if stream is None:
        r = _native.conv(0, desc, x, packed, None, bias, residual, stride, pad, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_conv2d_res_fwd")
    return _conv(_lib.ss_conv2d_res_fwd, "ss_conv2d_res_fwd", desc, x, packed, bias, stride, pad, act, y, workspace,
                 stream, residual, True)


def ss_conv2d_dense_res_fwd(desc, x, dense, bias=None, residual=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE,
                            y=None, workspace=None, stream=None) -> torch.Tensor:
    """The dense-MFMA twin of ss_conv2d_res_fwd."""
    if stream is None:
        r = _native.conv(1, desc, x, dense, None, bias, residual, stride, pad, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_conv2d_dense_res_fwd")
    return _conv(_lib.ss_conv2d_dense_res_fwd, "ss_conv2d_dense_res_fwd", desc, x, dense, bias, stride, pad, act, y,
                 workspace, stream, residual, True)


def _q8_args(what, desc, x, wbuf, scale, bias, stride, pad, act, y, workspace):
    if x is None or x.dim() != 4 or x.shape[3] != desc.cin:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: x must be NHWC with cin channels")
    N, H, W, _ = x.shape
    _check_operands(what, desc, wbuf, bias, "dense" not in what)
    if scale is not None and scale.numel() < desc.cout:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: scale holds {scale.numel()} values, cout is {desc.cout}")
    shp = out_shape(desc, N, H, W, stride, pad)
    if shp[1] <= 0 or shp[2] <= 0:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: empty output")
    if y is None:
        y = torch.empty(shp, dtype=torch.float16, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != torch.float16:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: y must be {shp} float16")
    need = ss_conv2d_workspace_bytes(desc, N, H, W, stride, pad)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if need > 0 and workspace is None:
        workspace = torch.zeros(need, dtype=torch.uint8, device=x.device)
        ws_bytes = need
    xtypes = (torch.int8,) if desc.dtype == SS_I8 else (torch.uint8, torch.float8_e4m3fn)
    args = (ctypes.byref(desc), _dev_ptr(x, "x", xtypes), N, H, W, _dev_ptr(wbuf, "weights"),
            _dev_ptr(scale, "scale", (torch.float32,), allow_none=True),
            _dev_ptr(bias, "bias", (torch.float32,), allow_none=True), stride[0], stride[1], pad[0], pad[1], act,
            SS_F16, _dev_ptr(y, "y"), _dev_ptr(workspace, "workspace", allow_none=True), ws_bytes)
    return args, y, workspace


def prepare_conv2d_q8(desc, x, wbuf, scale=None, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None,
                      workspace=None, sparse=True):
    """prepare_conv2d for the 8-bit integer entry points: returns (launch, y)."""
    what = "ss_conv2d_q8_fwd" if sparse else "ss_conv2d_q8_dense_fwd"
    _args, y, ws = _q8_args(what, desc, x, wbuf, scale, bias, stride, pad, act, y, workspace)
    return _launch(what, 2 if sparse else 3, desc, None, x, wbuf, None, scale, bias, None, None, y, ws, x.shape[:3], stride, pad, act), y


def ss_conv2d_q8_fwd(desc, x, packed, scale=None, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None,
                     workspace=None, stream=None) -> torch.Tensor:
    """2:4-sparse convolution on 8-bit operands (int8, or FP8 E4M3 bytes): x NHWC -> y NHWC float16 =
    act(scale * sum + bias)."""
    if stream is None:
        r = _native.conv(2, desc, x, packed, scale, bias, None, stride, pad, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_conv2d_q8_fwd")
    args, y, _ws = _q8_args("ss_conv2d_q8_fwd", desc, x, packed, scale, bias, stride, pad, act, y, workspace)
    st = _lib.ss_conv2d_q8_fwd(*args, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_conv2d_q8_fwd")
    return y


def ss_conv2d_q8_dense_fwd(desc, x, dense, scale=None, bias=None, stride=(1, 1), pad=(0, 0), act=SS_ACT_NONE, y=None,
                           workspace=None, stream=None) -> torch.Tensor:
    """The dense integer-MFMA twin of ss_conv2d_q8_fwd."""
    if stream is None:
        r = _native.conv(3, desc, x, dense, scale, bias, None, stride, pad, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_conv2d_q8_dense_fwd")
    args, y, _ws = _q8_args("ss_conv2d_q8_dense_fwd", desc, x, dense, scale, bias, stride, pad, act, y, workspace)
    st = _lib.ss_conv2d_q8_dense_fwd(*args, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_conv2d_q8_dense_fwd")
    return y


def _prepare_fused(what, third, desc1, x, w1, bias1, stride, pad, act1, desc2, w2, bias2, residual, act2, y, sparse):
    """Checks and marshals a fused pair, with its third layer (descriptor, weights, bias, activation, output or None) if there is one."""
    if x is None or x.dim() != 4 or x.shape[3] != desc1.cin:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: x must be NHWC with cin channels")
    N, H, W, _ = x.shape
    _check_operands(what, desc1, w1, bias1, sparse)
    _check_operands(what, desc2, w2, bias2, sparse)
    shp1 = out_shape(desc1, N, H, W, stride, pad)
    if shp1[1] <= 0 or shp1[2] <= 0:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: empty output")
    shp = (N, shp1[1], shp1[2], desc2.cout)
    if y is None:
        y = torch.empty(shp, dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: y must be {shp} {x.dtype}")
    if residual is not None and (tuple(residual.shape) != shp or residual.dtype != x.dtype or not residual.is_contiguous()):
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: residual must be contiguous {shp} {x.dtype}")
    for t, name, dtypes in ((x, "x", (torch_dtype(desc1.dtype),)), (w1, "weights 1", None), (w2, "weights 2", None), (y, "y", None)):
        _dev_ptr(t, name, dtypes)
    for t, name in ((bias1, "bias1"), (bias2, "bias2")):
        _dev_ptr(t, name, (torch.float32,), allow_none=True)
    _dev_ptr(residual, "residual", allow_none=True)
    if third is None:
        return _launch(what, 4 if sparse else 5, desc1, desc2, x, w1, w2, None, bias1, bias2, residual, y, None, (N, H, W), stride, pad,
                       act1, act2), y
    desc3, w3, bias3, act3, y3 = third
    _check_operands(what, desc3, w3, bias3, sparse)
    shp3 = shp[:3] + (desc3.cout,)
    if y3 is None:
        y3 = torch.empty(shp3, dtype=x.dtype, device=x.device)
    elif tuple(y3.shape) != shp3 or y3.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: y3 must be {shp3} {x.dtype}")
    _dev_ptr(w3, "weights 3")
    _dev_ptr(y3, "y3")
    _dev_ptr(bias3, "bias3", (torch.float32,), allow_none=True)
    return _launch(what, 7 if sparse else 8, desc1, desc2, x, w1, w2, None, bias1, bias2, residual, y, None, (N, H, W), stride, pad,
                   act1, act2, third=(desc3, w3, bias3, act3, y3)), y, y3


def prepare_conv2d_pw_fused(desc1, x, w1, bias1, stride, pad, act1, desc2, w2, bias2=None, residual=None,
                            act2=SS_ACT_NONE, y=None, sparse=True):
    """Marshal the arguments of ss_conv2d_pw_fused_fwd / ss_conv2d_pw_fused_dense_fwd once; returns (launch, y)."""
    what = "ss_conv2d_pw_fused_fwd" if sparse else "ss_conv2d_pw_fused_dense_fwd"
    return _prepare_fused(what, None, desc1, x, w1, bias1, stride, pad, act1, desc2, w2, bias2, residual, act2, y, sparse)


def prepare_conv2d_pw2_fused(desc1, x, w1, bias1, stride, pad, act1, desc2, w2, bias2, residual, act2, desc3, w3, bias3=None,
                             act3=SS_ACT_NONE, y2=None, y3=None, sparse=True):
    """Marshal the arguments of ss_conv2d_pw2_fused_fwd / ss_conv2d_pw2_fused_dense_fwd once; returns (launch, y2, y3)."""
    what = "ss_conv2d_pw2_fused_fwd" if sparse else "ss_conv2d_pw2_fused_dense_fwd"
    return _prepare_fused(what, (desc3, w3, bias3, act3, y3), desc1, x, w1, bias1, stride, pad, act1, desc2, w2, bias2, residual, act2, y2, sparse)


def ss_conv2d_pw2_fused_query(desc1, nhw, stride, pad, desc2, desc3, sparse=True):
    """(supported, pays): would the three layers run in one kernel, and does the library expect that, on an input of nhw = (N, H, W), to beat the
    pair and the third call?"""
    sup, pays = ctypes.c_int32(0), ctypes.c_int32(0)
    st = _lib.ss_conv2d_pw2_fused_query(ctypes.byref(desc1), nhw[0], nhw[1], nhw[2], stride[0], stride[1], pad[0], pad[1], ctypes.byref(desc2), ctypes.byref(desc3),
                                        1 if sparse else 0, ctypes.byref(sup), ctypes.byref(pays))
    if st != SS_OK:
        raise SSError(st, "ss_conv2d_pw2_fused_query")
    return bool(sup.value), bool(pays.value)


def ss_conv2d_pw2_fused_fwd(desc1, x, packed1, bias1, stride, pad, act1, desc2, packed2, bias2, residual, act2, desc3, packed3, bias3=None,
                            act3=SS_ACT_NONE, y2=None, y3=None):
    """ss_conv2d_pw_fused_fwd and the 1x1 masked convolution that reads its output; returns (y2, y3)."""
    launch, y2, y3 = prepare_conv2d_pw2_fused(desc1, x, packed1, bias1, stride, pad, act1, desc2, packed2, bias2, residual, act2, desc3, packed3,
                                              bias3, act3, y2, y3, sparse=True)
    launch()
    return y2, y3


def ss_conv2d_pw2_fused_dense_fwd(desc1, x, dense1, bias1, stride, pad, act1, desc2, dense2, bias2, residual, act2, desc3, dense3, bias3=None,
                                  act3=SS_ACT_NONE, y2=None, y3=None):
    """The dense twin of ss_conv2d_pw2_fused_fwd."""
    launch, y2, y3 = prepare_conv2d_pw2_fused(desc1, x, dense1, bias1, stride, pad, act1, desc2, dense2, bias2, residual, act2, desc3, dense3,
                                              bias3, act3, y2, y3, sparse=False)
    launch()
    return y2, y3


def ss_conv2d_pw_fused_query(desc1, stride, pad, desc2, sparse=True):
    """(supported, pays): would the fused entry point take this pair, and does the library expect it to beat two calls?"""
    sup, pays = ctypes.c_int32(0), ctypes.c_int32(0)
    st = _lib.ss_conv2d_pw_fused_query(ctypes.byref(desc1), stride[0], stride[1], pad[0], pad[1], ctypes.byref(desc2),
                                       1 if sparse else 0, ctypes.byref(sup), ctypes.byref(pays))
    if st != SS_OK:
        raise SSError(st, "ss_conv2d_pw_fused_query")
    return bool(sup.value), bool(pays.value)


def ss_conv2d_pw_fused_fwd(desc1, x, packed1, bias1, stride, pad, act1, desc2, packed2, bias2=None, residual=None,
                           act2=SS_ACT_NONE, y=None) -> torch.Tensor:
    """k x k masked convolution followed by a 1x1 masked convolution (+ residual), the intermediate kept on chip."""
    r = _native.fused(1, desc1, x, packed1, bias1, stride, pad, act1, desc2, packed2, bias2, residual, act2, y)
    if r is not None:
        return r if type(r) is not tuple else _failed(r, "ss_conv2d_pw_fused_fwd")
    launch, y = prepare_conv2d_pw_fused(desc1, x, packed1, bias1, stride, pad, act1, desc2, packed2, bias2, residual,
                                        act2, y, sparse=True)
    launch()
    return y


def ss_conv2d_pw_fused_dense_fwd(desc1, x, dense1, bias1, stride, pad, act1, desc2, dense2, bias2=None, residual=None,
                                 act2=SS_ACT_NONE, y=None) -> torch.Tensor:
    """The dense twin of ss_conv2d_pw_fused_fwd."""
    r = _native.fused(0, desc1, x, dense1, bias1, stride, pad, act1, desc2, dense2, bias2, residual, act2, y)
    if r is not None:
        return r if type(r) is not tuple else _failed(r, "ss_conv2d_pw_fused_dense_fwd")
    launch, y = prepare_conv2d_pw_fused(desc1, x, dense1, bias1, stride, pad, act1, desc2, dense2, bias2, residual,
                                        act2, y, sparse=False)
    launch()
    return y


def ss_maxpool2d(x: torch.Tensor, k: int = 3, stride: int = 2, pad: int = 1, y: torch.Tensor | None = None,
                 stream=None) -> torch.Tensor:
    """NHWC max pooling of a 16-bit tensor (positions outside the image do not take part)."""
    if stream is None:
        r = _native.maxpool(x, k, stride, pad, y)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_maxpool2d")
    if x is None or x.dim() != 4 or x.dtype not in _T16 or stride <= 0:
        raise SSError(SS_ERR_INVALID_ARG, "ss_maxpool2d: x must be a 16-bit NHWC tensor")
    N, H, W, C = x.shape
    shp = (N, (H + 2 * pad - k) // stride + 1, (W + 2 * pad - k) // stride + 1, C)
    if y is None:
        y = torch.empty(shp, dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"ss_maxpool2d: y must be {shp} {x.dtype}")
    st = _lib.ss_maxpool2d(_dev_ptr(x, "x"), N, H, W, C, SS_F16 if x.dtype == torch.float16 else SS_BF16, k, stride, pad,
                           _dev_ptr(y, "y"), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_maxpool2d")
    return y


def prepare_maxpool2d(x, k=3, stride=2, pad=1, y=None):
    """Marshal the arguments of ss_maxpool2d once; returns (launch, y), as prepare_conv2d does."""
    if x is None or x.dim() != 4 or x.dtype not in _T16 or stride <= 0:
        raise SSError(SS_ERR_INVALID_ARG, "ss_maxpool2d: x must be a 16-bit NHWC tensor")
    N, H, W, C = x.shape
    shp = (N, (H + 2 * pad - k) // stride + 1, (W + 2 * pad - k) // stride + 1, C)
    if y is None:
        y = torch.empty(shp, dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"ss_maxpool2d: y must be {shp} {x.dtype}")
    _dev_ptr(x, "x")
    _dev_ptr(y, "y")
    return _launch("ss_maxpool2d", 6, None, None, x, None, None, None, None, None, None, y, None, (N, H, W), (stride, stride),
                   (pad, pad), 0, 0, (C, SS_F16 if x.dtype == torch.float16 else SS_BF16, k)), y


def ss_dwconv2d_fwd(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, pad=(0, 0), act=SS_ACT_NONE,
                    y: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Depthwise convolution, stride 1: x NHWC 16-bit, w [kh, kw, C] of the same dtype -> y NHWC."""
    if stream is None:
        r = _native.dwconv(x, w, bias, pad, act, y)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_dwconv2d_fwd")
    if x is None or w is None or x.dim() != 4 or w.dim() != 3 or w.shape[2] != x.shape[3] or w.dtype != x.dtype or \
            x.dtype not in (torch.float16, torch.bfloat16):
        raise SSError(SS_ERR_INVALID_ARG, "ss_dwconv2d_fwd: x must be NHWC 16-bit and w [kh, kw, C] of the same dtype")
    N, H, W, C = x.shape
    kh, kw = int(w.shape[0]), int(w.shape[1])
    shp = (N, H + 2 * pad[0] - kh + 1, W + 2 * pad[1] - kw + 1, C)
    if shp[1] <= 0 or shp[2] <= 0:
        raise SSError(SS_ERR_INVALID_ARG, "ss_dwconv2d_fwd: empty output")
    if y is None:
        y = torch.empty(shp, dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != shp or y.dtype != x.dtype:
        raise SSError(SS_ERR_INVALID_ARG, f"ss_dwconv2d_fwd: y must be {shp} {x.dtype}")
    st = _lib.ss_dwconv2d_fwd(_dev_ptr(x, "x"), N, H, W, C, SS_F16 if x.dtype == torch.float16 else SS_BF16,
                              _dev_ptr(w, "w"), _dev_ptr(bias, "bias", (torch.float32,), allow_none=True), kh, kw,
                              pad[0], pad[1], act, _dev_ptr(y, "y"), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, "ss_dwconv2d_fwd")
    return y


# --------------------------------------------------------------------------------------------
# Rows of channels (pixels, tokens): MXFP4 and the norms around a block
# --------------------------------------------------------------------------------------------
_ROW_TYPES = {torch.float16: SS_F16, torch.bfloat16: SS_BF16, torch.float32: SS_F32}
_ROW_DTYPES = {code: dtype for dtype, code in _ROW_TYPES.items()}


def _pitch(t, what, name):
    """(rows, pitch) of a tensor of rows: the last dimension is dense, and the others step through memory as one."""
    rows, ld = 1, 0
    if t.dim() == 0 or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: the channels of {name} must be contiguous")
    if t.numel() == 0:
        return 0, t.shape[-1]                                # (whichever dimension is the empty one: there are no rows to be spaced)
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if rows == 1:
            ld = stride
        elif stride != ld * rows:
            raise SSError(SS_ERR_INVALID_ARG, f"{what}: the rows of {name} must be evenly spaced")
        rows *= size
    return rows, ld if rows > 1 else t.shape[-1]


def _row_tensor(what, name, t, cols, dtype, rows=None):
    """Checks a tensor of rows; (address, rows, pitch)."""
    if t is None:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} is None")
    if not t.is_cuda:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} must live in device memory")
    if t.dim() == 0 or t.shape[-1] != cols or (dtype is not None and t.dtype != dtype) or t.dtype not in _ROW_TYPES:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} must be [..., {cols}] {dtype or 'float16, bfloat16 or float32'}")
    n, ld = _pitch(t, what, name)
    if rows is not None and n != rows:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} has {n} rows, not {rows}")
    return ctypes.c_void_p(t.data_ptr()), n, ld


def _channel_vector(what, name, t, cols):
    if t is not None and t.numel() != cols:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} holds {t.numel()} values, not {cols}")
    return _dev_ptr(t, f"{what}: {name}", (torch.float32,), allow_none=True)


def _byte_tensor(what, name, t, rows, cols):
    """Codes or scales of a quantised activation: whole, 8-bit, dense."""
    p = _dev_ptr(t, f"{what}: {name}", (torch.uint8,))
    if t.dim() == 0 or t.shape[-1] != cols or (rows is not None and t.numel() != rows * cols):
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} must be [..., {cols}] uint8" + ("" if rows is None else f" of {rows} rows"))
    return p


def _mx4_sizes(cols):
    """Bytes of a row's codes and scales."""
    blocks = (cols + 31) // 32
    return 16 * blocks, (blocks + 3) // 4 * 4


def _on(stream, device):
    """Allocations made inside belong to the stream that the call is enqueued on."""
    return torch.cuda.stream(torch.cuda.current_stream(device) if stream is None else stream)


def ss_mx4_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None, stream=None):
    """x [..., cols] float16, bfloat16 or float32 -> (codes [..., 16*ceil(cols/32)], scales [..., 4*ceil(cols/128)]) uint8 (include/ss.h, MXFP4)."""
    if stream is None:
        r = _native.mx4_quantize(x, codes, scales)
        if r is not None:
            return r if type(r[0]) is not int else _failed(r, "ss_mx4_quantize")
    return _quantize("ss_mx4_quantize", _mx4_sizes, x, codes, scales, stream)


def _quantize(what, sizes, x, codes, scales, stream):
    if x is None or x.dim() == 0 or x.shape[-1] == 0:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: x must be [..., cols]")
    cols = x.shape[-1]
    px, rows, ld = _row_tensor(what, "x", x, cols, None)
    nc, ns = sizes(cols)
    with _on(stream, x.device):
        codes = torch.empty((*x.shape[:-1], nc), dtype=torch.uint8, device=x.device) if codes is None else codes
        scales = torch.empty((*x.shape[:-1], ns), dtype=torch.uint8, device=x.device) if scales is None else scales
    st = getattr(_lib, what)(px, rows, cols, ld, _ROW_TYPES[x.dtype], _byte_tensor(what, "codes", codes, rows, nc),
                              _byte_tensor(what, "scales", scales, rows, ns), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return codes, scales


def ss_mx4_dequantize(codes: torch.Tensor, scales: torch.Tensor, cols: int, dtype=torch.bfloat16, out: torch.Tensor | None = None,
                      stream=None) -> torch.Tensor:
    """The values [..., cols] that codes and scales stand for."""
    if stream is None:
        r = _native.mx4_dequantize(codes, scales, cols, _ROW_TYPES.get(dtype, -1), out)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_mx4_dequantize")
    return _dequantize("ss_mx4_dequantize", _mx4_sizes, codes, scales, cols, dtype, out, stream)


def _dequantize(what, sizes, codes, scales, cols, dtype, out, stream):
    if dtype not in _ROW_TYPES or cols <= 0:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: dtype {dtype}, {cols} channels")
    nc, ns = sizes(cols)
    pc = _byte_tensor(what, "codes", codes, None, nc)
    rows = codes.numel() // nc
    ps = _byte_tensor(what, "scales", scales, rows, ns)
    with _on(stream, codes.device):
        out = torch.empty((*codes.shape[:-1], cols), dtype=dtype, device=codes.device) if out is None else out
    po, _, ld = _row_tensor(what, "out", out, cols, dtype, rows)
    st = getattr(_lib, what)(pc, ps, rows, cols, _ROW_TYPES[dtype], po, ld, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return out


def ss_mx4_packed_bytes(desc: ss_weight_desc) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_mx4_packed_bytes(ctypes.byref(desc), ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_mx4_packed_bytes")
    return int(out.value)


def ss_mx4_pack(desc: ss_weight_desc, W: torch.Tensor, M: torch.Tensor | None = None, packed: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """W [cout, cin] 16-bit, M [cout, cin] uint8 or None -> the masked weights in MXFP4, laid out for ss_pw_mx4_fwd."""
    return _pack("ss_mx4_pack", desc, ss_mx4_packed_bytes(desc), W, M, (), packed, stream)


def _pack(what, desc, need, W, M, more, packed, stream):
    """Checks and makes a packing call for block-scaled weights; `more`: its arguments behind the mask."""
    if W is None or W.numel() != desc.cout * desc.cin or (M is not None and M.numel() != desc.cout * desc.cin):
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: W/M size does not match the descriptor")
    pw, pm = _dev_ptr(W, "W", (torch_dtype(desc.dtype),)), _dev_ptr(M, "M", (torch.uint8, torch.bool), allow_none=True)
    if packed is None:
        with _on(stream, W.device):
            packed = torch.empty(need, dtype=torch.uint8, device=W.device)
    elif _nbytes(packed) < need:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: packed buffer too small")
    st = getattr(_lib, what)(ctypes.byref(desc), pw, pm, *more, _dev_ptr(packed, "packed"), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return packed


def ss_mx4_unpack(desc: ss_weight_desc, packed: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The values [cout, cin] that packed weights stand for."""
    return _unpack("ss_mx4_unpack", desc, ss_mx4_packed_bytes(desc), packed, out, stream)


def _unpack(what, desc, need, packed, out, stream):
    if _nbytes(packed) < need:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: packed buffer too small")
    if out is None:
        with _on(stream, packed.device):
            out = torch.empty((desc.cout, desc.cin), dtype=torch_dtype(desc.dtype), device=packed.device)
    elif out.numel() != desc.cout * desc.cin:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: out does not match the descriptor")
    st = getattr(_lib, what)(ctypes.byref(desc), _dev_ptr(packed, "packed"), _dev_ptr(out, "out", (torch_dtype(desc.dtype),)), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return out


def ss_pw_mx4_workspace_bytes(desc: ss_weight_desc, rows: int) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_pw_mx4_workspace_bytes(ctypes.byref(desc), rows, ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_pw_mx4_workspace_bytes")
    return int(out.value)


def _pw(what, desc, need, scratch, head, rows, lead, device, packed, bias, residual, act, y, workspace, stream):
    """Checks and makes a pointwise call on block-scaled operands; `need`: bytes of its weights, `scratch`: what tells the bytes of its workspace, or None,
    `head`: its activation's arguments, `lead`: the leading dimensions of y."""
    if _nbytes(packed) < need:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: weight buffer holds {_nbytes(packed)} bytes, the descriptor needs {need}")
    dtype = torch_dtype(desc.dtype)
    pb = _channel_vector(what, "bias", bias, desc.cout)
    pr, ldr = None, 0
    if residual is not None:
        pr, _, ldr = _row_tensor(what, "residual", residual, desc.cout, dtype, rows)
    with _on(stream, device):
        if y is None:
            y = torch.empty((*lead, desc.cout), dtype=dtype, device=device)
        py, _, ldy = _row_tensor(what, "y", y, desc.cout, dtype, rows)
        args = (ctypes.byref(desc), *head, _dev_ptr(packed, "packed"), pb, pr, ldr, act, py, ldy)
        if scratch is not None:
            need = scratch(desc, rows)
            if need > 0 and workspace is None:
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
            st = getattr(_lib, what)(*args, _dev_ptr(workspace, "workspace", allow_none=True), _nbytes(workspace), _stream_ptr(stream))
        else:
            st = getattr(_lib, what)(*args, _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return y


def ss_pw_mx4_fwd(desc: ss_weight_desc, x: torch.Tensor, packed: torch.Tensor, bias=None, residual=None, act=SS_ACT_NONE, y=None, workspace=None,
                  stream=None) -> torch.Tensor:
    """Pointwise layer on MXFP4 operands: x [..., cin] 16-bit, quantised on the way -> y [..., cout]."""
    if stream is None:
        r = _native.pw_mx4(desc, x, None, packed, bias, residual, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_pw_mx4_fwd")
    what = "ss_pw_mx4_fwd"
    px, rows, ld = _row_tensor(what, "x", x, desc.cin, torch_dtype(desc.dtype))
    return _pw(what, desc, ss_mx4_packed_bytes(desc), ss_pw_mx4_workspace_bytes, (px, rows, ld), rows, x.shape[:-1], x.device, packed, bias, residual, act, y, workspace, stream)


def ss_pw_mx4_q_fwd(desc: ss_weight_desc, codes: torch.Tensor, scales: torch.Tensor, packed: torch.Tensor, bias=None, residual=None, act=SS_ACT_NONE,
                    y=None, stream=None) -> torch.Tensor:
    """The same on an activation that ss_mx4_quantize (or ss_norm_mx4_fwd) has quantised: [..., cin] as codes and scales -> y [..., cout]."""
    if stream is None:
        r = _native.pw_mx4(desc, codes, scales, packed, bias, residual, act, y, None)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_pw_mx4_q_fwd")
    what = "ss_pw_mx4_q_fwd"
    nc, ns = _mx4_sizes(desc.cin)
    pc = _byte_tensor(what, "codes", codes, None, nc)
    rows = codes.numel() // nc
    return _pw(what, desc, ss_mx4_packed_bytes(desc), None, (pc, _byte_tensor(what, "scales", scales, rows, ns), rows), rows, codes.shape[:-1], codes.device, packed,
               bias, residual, act, y, None, stream)


def _f8_sizes(cols):
    """Bytes of a row's codes and scales."""
    return (cols + 63) // 64 * 64, (cols + 511) // 512 * 4


def ss_f8_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None, stream=None):
    """x [..., cols] float16, bfloat16 or float32 -> (codes [..., 64*ceil(cols/64)], scales [..., 4*ceil(cols/512)]) uint8 (include/ss.h, FP8 with a scale
    for each block of 128)."""
    if stream is None:
        r = _native.f8_quantize(x, codes, scales)
        if r is not None:
            return r if type(r[0]) is not int else _failed(r, "ss_f8_quantize")
    return _quantize("ss_f8_quantize", _f8_sizes, x, codes, scales, stream)


def ss_f8_dequantize(codes: torch.Tensor, scales: torch.Tensor, cols: int, dtype=torch.bfloat16, out: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """The values [..., cols] that codes and scales stand for."""
    if stream is None:
        r = _native.f8_dequantize(codes, scales, cols, _ROW_TYPES.get(dtype, -1), out)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_f8_dequantize")
    return _dequantize("ss_f8_dequantize", _f8_sizes, codes, scales, cols, dtype, out, stream)


def ss_f8_packed_bytes(desc: ss_weight_desc) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_f8_packed_bytes(ctypes.byref(desc), ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_f8_packed_bytes")
    return int(out.value)


def ss_f8_pack(desc: ss_weight_desc, W: torch.Tensor, M: torch.Tensor | None = None, transposed: bool = False, packed: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
    """W [cout, cin] 16-bit, M [cout, cin] uint8 or None -> the masked weights in FP8, laid out for ss_pw_f8_fwd.  transposed: W and M are [cin, cout] (the
    gradient of a layer's input takes the layer's own weights so, with a descriptor of cout and cin exchanged)."""
    shape = (desc.cin, desc.cout) if transposed else (desc.cout, desc.cin)
    for name, t in (("W", W), ("M", M)):
        if t is not None and t.dim() == 2 and tuple(t.shape) != shape:
            raise SSError(SS_ERR_INVALID_ARG, f"ss_f8_pack: {name} is {tuple(t.shape)}, not {shape}")
    return _pack("ss_f8_pack", desc, ss_f8_packed_bytes(desc), W, M, (int(bool(transposed)),), packed, stream)


def ss_f8_unpack(desc: ss_weight_desc, packed: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The values [cout, cin] that packed weights stand for."""
    return _unpack("ss_f8_unpack", desc, ss_f8_packed_bytes(desc), packed, out, stream)


def ss_pw_f8_workspace_bytes(desc: ss_weight_desc, rows: int) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_pw_f8_workspace_bytes(ctypes.byref(desc), rows, ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_pw_f8_workspace_bytes")
    return int(out.value)


def ss_pw_f8_fwd(desc: ss_weight_desc, x: torch.Tensor, packed: torch.Tensor, bias=None, residual=None, act=SS_ACT_NONE, y=None, workspace=None,
                 stream=None) -> torch.Tensor:
    """Pointwise or linear layer on FP8 operands: x [..., cin] 16-bit, quantised on the way -> y [..., cout]."""
    if stream is None:
        r = _native.pw_f8(desc, x, None, packed, bias, residual, act, y, workspace)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_pw_f8_fwd")
    what = "ss_pw_f8_fwd"
    px, rows, ld = _row_tensor(what, "x", x, desc.cin, torch_dtype(desc.dtype))
    return _pw(what, desc, ss_f8_packed_bytes(desc), ss_pw_f8_workspace_bytes, (px, rows, ld), rows, x.shape[:-1], x.device, packed, bias, residual, act, y, workspace,
               stream)


def ss_pw_f8_q_fwd(desc: ss_weight_desc, codes: torch.Tensor, scales: torch.Tensor, packed: torch.Tensor, bias=None, residual=None, act=SS_ACT_NONE,
                   y=None, stream=None) -> torch.Tensor:
    """The same on an activation that ss_f8_quantize has quantised: [..., cin] as codes and scales -> y [..., cout]."""
    if stream is None:
        r = _native.pw_f8(desc, codes, scales, packed, bias, residual, act, y, None)
        if r is not None:
            return r if type(r) is not tuple else _failed(r, "ss_pw_f8_q_fwd")
    what = "ss_pw_f8_q_fwd"
    nc, ns = _f8_sizes(desc.cin)
    pc = _byte_tensor(what, "codes", codes, None, nc)
    rows = codes.numel() // nc
    return _pw(what, desc, ss_f8_packed_bytes(desc), None, (pc, _byte_tensor(what, "scales", scales, rows, ns), rows), rows, codes.shape[:-1], codes.device, packed,
               bias, residual, act, y, None, stream)


def ss_pw_wgrad_workspace_bytes(desc: ss_weight_desc, rows: int) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_pw_wgrad_workspace_bytes(ctypes.byref(desc), rows, ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_pw_wgrad_workspace_bytes")
    return int(out.value)


def ss_pw_wgrad(desc: ss_weight_desc, dy: torch.Tensor, x: torch.Tensor, dw=None, db=None, with_bias: bool = True, workspace=None, stream=None):
    """Gradient of a pointwise or linear layer's weights and bias: dy [..., cout] (of what stands before the activation), x [..., cin] -> (dw [cout, cin], db [cout] or None) float32,
    from 16-bit operands as they are, whatever the type of the forward product."""
    if stream is None:
        r = _native.pw_wgrad(desc, dy, x, dw, db, int(with_bias), workspace)
        if r is not None:
            return r if type(r[0]) is not int else _failed(r, "ss_pw_wgrad")
    what = "ss_pw_wgrad"
    dtype = torch_dtype(desc.dtype)
    pd, rows, ldd = _row_tensor(what, "dy", dy, desc.cout, dtype)
    px, _, ldx = _row_tensor(what, "x", x, desc.cin, dtype, rows)
    if not with_bias and db is not None:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: db without a bias")
    need = ss_pw_wgrad_workspace_bytes(desc, rows)
    with _on(stream, x.device):
        dw = torch.empty((desc.cout, desc.cin), dtype=torch.float32, device=x.device) if dw is None else dw
        if with_bias and db is None:
            db = torch.empty(desc.cout, dtype=torch.float32, device=x.device)
        if need > 0 and workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    st = _lib.ss_pw_wgrad(ctypes.byref(desc), pd, ldd, px, ldx, rows, _channel_vector(what, "dw", dw, desc.cout * desc.cin), _channel_vector(what, "db", db, desc.cout),
                             _dev_ptr(workspace, "workspace", allow_none=True), _nbytes(workspace), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return dw, db


def make_norm_desc(cols, dtype=SS_BF16, norm=SS_NORM_LAYER, eps=1e-6, post=SS_NORM_NONE, post_eps=1e-6) -> ss_norm_desc:
    """The norm of a block's input, and the one of its output (`post`); dtype: of every activation."""
    return ss_norm_desc(int(cols), int(dtype), int(norm), int(post), float(eps), float(post_eps))


# An empty tensor has no address, by which the library tells an operand from none; it gets this one, which no call without rows reads or writes at.
_NOWHERE = ctypes.c_void_p(4096)


def _norm_io(what, io, desc, rows, gate, vectors, tensors):
    """Fills a struct of ss.h: the gate, the channel vectors and the tensors of rows, by their names."""
    dtype = _ROW_DTYPES.get(desc.dtype)
    io.rows = rows
    if gate is not None:
        if gate.dtype != dtype or gate.dim() == 0 or gate.shape[-1] not in (1, desc.cols):
            raise SSError(SS_ERR_INVALID_ARG, f"{what}: gate must be [..., 1] or [..., {desc.cols}] {dtype}")
        io.gate_cols = gate.shape[-1]
        io.groups = gate.numel() // io.gate_cols
        io.gate = _dev_ptr(gate, f"{what}: gate") if gate.numel() else _NOWHERE
    for name, t in vectors.items():
        setattr(io, name, _channel_vector(what, name, t, desc.cols))
    for name, t in tensors.items():
        if t is not None:
            p, _, ld = _row_tensor(what, name, t, desc.cols, dtype, rows)
            setattr(io, name, p if rows else _NOWHERE)
            setattr(io, f"ld{name}", ld)


def _norm_fwd(what, desc, x, w, b, h, scale, gate, post_w, post_b, x_out, y, codes, scales, stream):
    dtype = _ROW_DTYPES.get(desc.dtype)
    _, rows, _ = _row_tensor(what, "x", x, desc.cols, dtype)
    io = ss_norm_io()
    quantised = what == "ss_norm_mx4_fwd"
    with _on(stream, x.device):
        if h is not None and x_out is None:
            x_out = torch.empty(x.shape, dtype=dtype, device=x.device)
        if quantised:
            nc, ns = _mx4_sizes(desc.cols)
            codes = torch.empty((*x.shape[:-1], nc), dtype=torch.uint8, device=x.device) if codes is None else codes
            scales = torch.empty((*x.shape[:-1], ns), dtype=torch.uint8, device=x.device) if scales is None else scales
        elif y is None and desc.norm != SS_NORM_NONE:
            y = torch.empty(x.shape, dtype=dtype, device=x.device)
    _norm_io(what, io, desc, rows, gate, {"w": w, "b": b, "scale": scale, "post_w": post_w, "post_b": post_b},
             {"x": x, "h": h, "x_out": x_out, "y": y})
    if quantised:
        io.codes, io.scales = (p if rows else _NOWHERE for p in (_byte_tensor(what, "codes", codes, rows, nc), _byte_tensor(what, "scales", scales, rows, ns)))
    st = _lib.ss_norm_fwd(ctypes.byref(desc), ctypes.byref(io), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    out = (codes, scales) if quantised else () if y is None else (y,)
    out = out if h is None else (x_out, *out)
    return out if len(out) > 1 else out[0]


def ss_norm_fwd(desc: ss_norm_desc, x, w=None, b=None, h=None, scale=None, gate=None, post_w=None, post_b=None, x_out=None, y=None, stream=None):
    """x_out = x + scale * gate * post(h), y = norm(x_out) -> (x_out, y); without a block output h: y = norm(x) -> y; with SS_NORM_NONE -> x_out.

    x, h [..., cols]; w, b, scale, post_w, post_b [cols] float32; gate [groups, 1] or [groups, cols] of x's type, each of its rows for
    rows / groups consecutive rows of x."""
    if stream is None:
        r = _native.norm_fwd(desc, x, w, b, h, scale, gate, post_w, post_b, x_out, y)
        if r is not None:
            return r if type(r) is not tuple or type(r[0]) is not int else _failed(r, "ss_norm_fwd")
    return _norm_fwd("ss_norm_fwd", desc, x, w, b, h, scale, gate, post_w, post_b, x_out, y, None, None, stream)


def ss_norm_mx4_fwd(desc: ss_norm_desc, x, w=None, b=None, h=None, scale=None, gate=None, post_w=None, post_b=None, x_out=None, codes=None, scales=None,
                    stream=None):
    """ss_norm_fwd with y in MXFP4: -> (x_out, codes, scales), or (codes, scales) without h."""
    if stream is None:
        r = _native.norm_mx4_fwd(desc, x, w, b, h, scale, gate, post_w, post_b, x_out, codes, scales)
        if r is not None:
            return r if type(r[0]) is not int else _failed(r, "ss_norm_mx4_fwd")
    return _norm_fwd("ss_norm_mx4_fwd", desc, x, w, b, h, scale, gate, post_w, post_b, x_out, None, codes, scales, stream)


class NormGrads(NamedTuple):
    """Gradients of ss_norm_fwd; None where the call had no such operand."""
    dx: torch.Tensor
    dh: torch.Tensor | None
    dgate: torch.Tensor | None
    dw: torch.Tensor | None
    db: torch.Tensor | None
    dscale: torch.Tensor | None
    dpost_w: torch.Tensor | None
    dpost_b: torch.Tensor | None


def ss_norm_bwd_workspace_bytes(desc: ss_norm_desc, rows: int, groups: int = 0, gate_cols: int = 0) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_norm_bwd_workspace_bytes(ctypes.byref(desc), rows, groups, gate_cols, ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_norm_bwd_workspace_bytes")
    return int(out.value)


def ss_norm_bwd(desc: ss_norm_desc, dy, x_out, w=None, b=None, h=None, scale=None, gate=None, post_w=None, post_b=None, dx_out=None, workspace=None,
                stream=None) -> NormGrads:
    """Gradient of ss_norm_fwd.  dy: of y (None with SS_NORM_NONE); dx_out: of x_out, or None; x_out, h and the other operands as in the forward
    call (x_out = its x where there was no h).  The gradient of a vector that is None is not returned."""
    if stream is None:
        r = _native.norm_bwd(desc, dy, x_out, w, b, h, scale, gate, post_w, post_b, dx_out, workspace)
        if r is not None:
            return NormGrads(*r) if len(r) == 8 else _failed(r, "ss_norm_bwd")
    what = "ss_norm_bwd"
    dtype = _ROW_DTYPES.get(desc.dtype)
    like = x_out if desc.norm != SS_NORM_NONE else dx_out
    _, rows, _ = _row_tensor(what, "x_out" if like is x_out else "dx_out", like, desc.cols, dtype)
    io = ss_norm_grad_io()
    with _on(stream, like.device):
        dx = torch.empty(like.shape, dtype=dtype, device=like.device)
        dh = None if h is None else torch.empty(h.shape, dtype=dtype, device=like.device)
        dgate = None if gate is None else torch.empty(gate.shape, dtype=gate.dtype, device=like.device)
        dw, db, dscale, dpost_w, dpost_b = (None if v is None else torch.empty(v.shape, dtype=torch.float32, device=like.device)
                                            for v in (w, b, scale, post_w, post_b))
        _norm_io(what, io, desc, rows, gate,
                 {"w": w, "scale": scale, "post_w": post_w, "post_b": post_b, "dw": dw, "db": db, "dscale": dscale, "dpost_w": dpost_w, "dpost_b": dpost_b},
                 {"dy": dy, "x_out": x_out, "dx_out": dx_out, "h": h, "dx": dx, "dh": dh})
        _channel_vector(what, "b", b, desc.cols)
        if dgate is not None:
            io.dgate = _dev_ptr(dgate, "dgate") if dgate.numel() else _NOWHERE
        need = ss_norm_bwd_workspace_bytes(desc, rows, io.groups, io.gate_cols)
        if need > 0 and workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
        st = _lib.ss_norm_bwd(ctypes.byref(desc), ctypes.byref(io), _dev_ptr(workspace, "workspace", allow_none=True), _nbytes(workspace), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return NormGrads(dx, dh, dgate, dw, db, dscale, dpost_w, dpost_b)


# --------------------------------------------------------------------------------------------
# Group norm of channels-last images
# --------------------------------------------------------------------------------------------
def make_groupnorm_desc(channels, groups, dtype=SS_BF16, act=SS_ACT_NONE, eps=1e-5) -> ss_groupnorm_desc:
    """Group norm over `groups` groups of neighbouring channels, with the activation behind it; dtype: of every activation."""
    return ss_groupnorm_desc(int(channels), int(groups), int(dtype), int(act), float(eps), 0)


def ss_groupnorm_workspace_bytes(desc: ss_groupnorm_desc, images: int, pixels: int, backward: bool = False) -> int:
    out = ctypes.c_size_t(0)
    st = _lib.ss_groupnorm_workspace_bytes(ctypes.byref(desc), images, pixels, int(bool(backward)), ctypes.byref(out))
    if st != SS_OK:
        raise SSError(st, "ss_groupnorm_workspace_bytes")
    return int(out.value)


def _images(what, name, t, desc, like=None):
    """Checks a tensor of images [images, ..., channels]; (address, images, pixels, pitch)."""
    p, rows, ld = _row_tensor(what, name, t, desc.channels, _ROW_DTYPES.get(desc.dtype))
    if t.dim() < 2:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} must be [images, ..., {desc.channels}]")
    images = t.shape[0]
    pixels = 1
    for size in t.shape[1:-1]:
        pixels *= size
    if like is not None and (images, pixels) != like:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: {name} has {images} images of {pixels} pixels, not {like[0]} of {like[1]}")
    return p, images, pixels, ld


def _group_stats(what, stats, images, desc):
    if stats.numel() != images * desc.groups * 2:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: stats must be [{images}, {desc.groups}, 2] float32")
    return _dev_ptr(stats, f"{what}: stats", (torch.float32,))


def ss_groupnorm_fwd(desc: ss_groupnorm_desc, x: torch.Tensor, w=None, b=None, y=None, stats=None, workspace=None, stream=None):
    """y = act(groupnorm(x) * w + b) -> (y, stats): x [images, ..., channels], channels last; w, b [channels] float32 or None; stats [images, groups, 2] float32,
    mean and reciprocal deviation, which ss_groupnorm_bwd takes."""
    if stream is None:
        r = _native.groupnorm_fwd(desc, x, w, b, y, stats, workspace)
        if r is not None:
            return r if type(r[0]) is not int else _failed(r, "ss_groupnorm_fwd")
    what = "ss_groupnorm_fwd"
    px, images, pixels, ldx = _images(what, "x", x, desc)
    need = ss_groupnorm_workspace_bytes(desc, images, pixels)
    with _on(stream, x.device):
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if y is None else y
        stats = torch.empty((images, desc.groups, 2), dtype=torch.float32, device=x.device) if stats is None else stats
        if need > 0 and workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    py, _, ldy = _row_tensor(what, "y", y, desc.channels, x.dtype, images * pixels)
    st = _lib.ss_groupnorm_fwd(ctypes.byref(desc), px, ldx, images, pixels, _channel_vector(what, "w", w, desc.channels), _channel_vector(what, "b", b, desc.channels),
                               py, ldy, _group_stats(what, stats, images, desc), _dev_ptr(workspace, "workspace", allow_none=True), _nbytes(workspace), _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return y, stats


class GroupNormGrads(NamedTuple):
    """Gradients of ss_groupnorm_fwd; None where the call had no such operand."""
    dx: torch.Tensor
    dw: torch.Tensor | None
    db: torch.Tensor | None


def ss_groupnorm_bwd(desc: ss_groupnorm_desc, dy: torch.Tensor, x: torch.Tensor, stats: torch.Tensor, w=None, b=None, workspace=None, stream=None) -> GroupNormGrads:
    """Gradient of ss_groupnorm_fwd for a gradient dy of y; x, w and b as in the forward call, stats as it gave them."""
    if stream is None:
        r = _native.groupnorm_bwd(desc, dy, x, stats, w, b, workspace)
        if r is not None:
            return GroupNormGrads(*r) if type(r[0]) is not int else _failed(r, "ss_groupnorm_bwd")
    what = "ss_groupnorm_bwd"
    px, images, pixels, ldx = _images(what, "x", x, desc)
    pd, _, _, ldd = _images(what, "dy", dy, desc, (images, pixels))
    if stats is None:
        raise SSError(SS_ERR_INVALID_ARG, f"{what}: stats is None")
    ps, pw, pb = _group_stats(what, stats, images, desc), _channel_vector(what, "w", w, desc.channels), _channel_vector(what, "b", b, desc.channels)
    need = ss_groupnorm_workspace_bytes(desc, images, pixels, True)
    with _on(stream, x.device):
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dw, db = (None if v is None else torch.empty(v.shape, dtype=torch.float32, device=x.device) for v in (w, b))
        if need > 0 and workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    st = _lib.ss_groupnorm_bwd(ctypes.byref(desc), pd, ldd, px, ldx, images, pixels, ps, pw, pb, ctypes.c_void_p(dx.data_ptr()), desc.channels,
                               _dev_ptr(dw, "dw", allow_none=True), _dev_ptr(db, "db", allow_none=True), _dev_ptr(workspace, "workspace", allow_none=True), _nbytes(workspace),
                               _stream_ptr(stream))
    if st != SS_OK:
        raise SSError(st, what)
    return GroupNormGrads(dx, dw, db)
