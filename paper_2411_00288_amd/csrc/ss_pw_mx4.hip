// Pointwise layer on MXFP4 operands: y = act(Wq xq + bias + residual).
#include "ss_mx4.h"
#include <algorithm>

namespace ss {

struct PwArgs {
    const uint8_t *codes, *scales;         // quantised activation
    const uint8_t *w;                      // first weight tile
    const uint8_t *w_scales;               // first word of their scales
    const float *bias;
    const uint16_t *residual;
    uint16_t *y;
    long long ldr, ldy;
    int P, cout, K, act;
};

// One product of 32 output channels and 32 pixels over 64 reduction indices: lane l gives the 32 values of block l/32 of weight row l%32 and of
// pixel l%32, and the byte of their scales; it gets the channels 8*(v/4) + 4*(l/32) + v%4, v = 0..15, of pixel l%32.
template <int SEL>
__device__ __forceinline__ f32x16 mma_mx4(const u32x4 &a, const u32x4 &b, const f32x16 &c, uint32_t scale_a, uint32_t scale_b)
{
    const i32x8 wide_a = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, wide_b = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide_a, wide_b, c, 4, 4, SEL, (int)scale_a, SEL, (int)scale_b);
}

// A wave makes one 32 x 32 tile, straight from memory.
template <int DT>
__global__ __launch_bounds__(256) void pw_mx4_kernel(PwArgs p)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, KB = (p.K + 31) / 32, S = (KB + 3) / 4 * 4, Ks = (KB + 1) / 2, Kq = (Ks + 3) / 4;
    const int mt = blockIdx.y * 2 + wave / 2;
    const long long px = ((long long)blockIdx.x * 2 + wave % 2) * 32 + lane % 32;
    if (mt * 32 >= p.cout) return;
    const bool in = px < p.P;
    f32x16 acc = {};
    for (int ks = 0; ks < Ks; ks++) {
        const int b = 2 * ks + lane / 32;
        const u32x4 wa = *reinterpret_cast<const u32x4 *>(p.w + (((size_t)mt * Ks + ks) * 64 + lane) * 16);
        const uint32_t sa = p.w_scales[(((size_t)mt * Kq + ks / 4) * 64 + lane) * 4 + ks % 4];
        u32x4 xb = {};
        uint32_t sb = 0;
        if (in && b < KB) {
            xb = *reinterpret_cast<const u32x4 *>(p.codes + (px * KB + b) * 16);
            sb = p.scales[px * S + b];
        }
        acc = mma_mx4<0>(wa, xb, acc, sa, sb);
    }
    if (!in) return;
#pragma unroll
    for (int q = 0; q < 4; q++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int o = mt * 32 + 8 * q + 4 * (lane / 32) + e;
            if (o >= p.cout) continue;
            float v = acc[4 * q + e];
            if (p.bias != nullptr) v += p.bias[o];
            if (p.residual != nullptr) v += widen<DT>(p.residual[px * p.ldr + o]);
            if (p.act == SS_ACT_RELU) v = floor_at(v, 0.f);
            if (p.act == SS_ACT_GELU) v = gelu_cdf<DT>(v);
            store1<DT>(p.y + px * p.ldy + o, v);
        }
}

namespace {

int check_pw(const ss_weight_desc *d, int64_t rows, const void *packed, const float *bias, const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy)
{
    const int st = check_desc(d, false);
    if (st != SS_OK) return st;
    if (d->kh != 1 || d->kw != 1 || is_byte_type(d->dtype)) return SS_ERR_UNSUPPORTED;
    if (act != SS_ACT_NONE && act != SS_ACT_RELU && act != SS_ACT_GELU) return SS_ERR_INVALID_ARG;
    if (rows < 0 || ldy < d->cout || (residual && ldr < d->cout)) return SS_ERR_INVALID_ARG;
    if (rows > INT32_MAX || ldy > INT32_MAX || (residual && ldr > INT32_MAX)) return SS_ERR_UNSUPPORTED;
    if (rows == 0) return SS_OK;
    if (!packed || !y || !aligned(packed, 16) || !aligned(y, 2) || !aligned(bias, 4) || !aligned(residual, 2)) return SS_ERR_INVALID_ARG;
    return SS_OK;
}

size_t codes_bytes(const Mx4Dims &t, int64_t rows) { return ((size_t)rows * t.KB * 16 + 255) / 256 * 256; }

int product(const ss_weight_desc *d, const uint8_t *codes, const uint8_t *scales, int64_t rows, const void *packed, const float *bias, const void *residual, int64_t ldr,
            int32_t act, void *y, int64_t ldy, hipStream_t s)
{
    const Mx4Dims t = mx4_dims(d->cout, d->cin);
    PwArgs a{};
    a.codes = codes;
    a.scales = scales;
    a.w = static_cast<const uint8_t *>(packed) + kHeaderBytes;
    a.w_scales = a.w + (size_t)t.Mt * t.Ks * 1024;
    a.bias = bias;
    a.residual = static_cast<const uint16_t *>(residual);
    a.y = static_cast<uint16_t *>(y);
    a.ldr = ldr;
    a.ldy = ldy;
    a.P = (int)rows;
    a.cout = d->cout;
    a.K = d->cin;
    a.act = act;
    const dim3 grid((unsigned)((rows + 63) / 64), (unsigned)((t.Mt + 1) / 2));
    if (grid.y > 65535) return SS_ERR_UNSUPPORTED;
    d->dtype == SS_F16 ? pw_mx4_kernel<SS_F16><<<grid, dim3(256), 0, s>>>(a) : pw_mx4_kernel<SS_BF16><<<grid, dim3(256), 0, s>>>(a);
    return launched();
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_pw_mx4_q_fwd(const ss_weight_desc *desc, const void *codes, const void *scales, int64_t rows, const void *packed, const float *bias,
                               const void *residual, int64_t ldr, int32_t act, void *y, int64_t ldy, void *stream)
{
    const int st = check_pw(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!codes || !scales || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    return product(desc, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), rows, packed, bias, residual, ldr, act, y, ldy,
                   static_cast<hipStream_t>(stream));
}

extern "C" int ss_pw_mx4_workspace_bytes(const ss_weight_desc *desc, int64_t rows, size_t *bytes)
{
    const int st = check_desc(desc, false);
    if (st != SS_OK) return st;
    if (desc->kh != 1 || desc->kw != 1 || is_byte_type(desc->dtype)) return SS_ERR_UNSUPPORTED;
    if (!bytes || rows < 0) return SS_ERR_INVALID_ARG;
    if (rows > INT32_MAX) return SS_ERR_UNSUPPORTED;
    const Mx4Dims t = mx4_dims(desc->cout, desc->cin);
    *bytes = codes_bytes(t, rows) + (size_t)rows * t.S;
    return SS_OK;
}

extern "C" int ss_pw_mx4_fwd(const ss_weight_desc *desc, const void *x, int64_t rows, int64_t ldx, const void *packed, const float *bias, const void *residual,
                             int64_t ldr, int32_t act, void *y, int64_t ldy, void *workspace, size_t ws_bytes, void *stream)
{
    int st = check_pw(desc, rows, packed, bias, residual, ldr, act, y, ldy);
    if (st != SS_OK) return st;
    if (ldx < desc->cin) return SS_ERR_INVALID_ARG;
    if (ldx > INT32_MAX) return SS_ERR_UNSUPPORTED;
    if (rows == 0) return SS_OK;
    if (!x || !aligned(x, 2)) return SS_ERR_INVALID_ARG;
    size_t need = 0;
    st = ss_pw_mx4_workspace_bytes(desc, rows, &need);
    if (st != SS_OK) return st;
    if (need > 0 && (!workspace || !aligned(workspace, 16) || ws_bytes < need)) return SS_ERR_WORKSPACE;
    const Mx4Dims t = mx4_dims(desc->cout, desc->cin);
    uint8_t *codes = static_cast<uint8_t *>(workspace), *scales = codes + codes_bytes(t, rows);
    st = mx4_quantize(x, rows, desc->cin, ldx, desc->dtype, codes, scales, static_cast<hipStream_t>(stream));
    if (st != SS_OK) return st;
    return product(desc, codes, scales, rows, packed, bias, residual, ldr, act, y, ldy, static_cast<hipStream_t>(stream));
}
