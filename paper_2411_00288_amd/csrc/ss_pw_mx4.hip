// Pointwise layer on MXFP4 operands: y = act(Wq xq + bias + residual).
#include "ss_mx4.h"
#include <algorithm>
#include <type_traits>

namespace ss {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
struct __attribute__((packed, aligned(2))) Half16 { u32x2 v; };        // four 16-bit values

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

constexpr int kChunk = 8;                                  // blocks of a reduction chunk: 256 channels, four steps, one scale word

// A wave's MI x NI tiles of sums, finished and stored: bias, residual, activation, rounding, whole 16-byte runs where the channels allow it.
template <int DT, int MI, int NI>
__device__ __forceinline__ void pw_store(const PwArgs &p, const f32x16 (&acc)[MI][NI], int mt0, long long px0, int lane)
{
    const int half = lane / 32;
#pragma unroll
    for (int i = 0; i < MI; i++) {
        const int o0 = (mt0 + i) * 32;
        if (o0 >= p.cout) return;
        float bias[16];
#pragma unroll
        for (int v = 0; v < 16; v++) {
            const int o = o0 + 8 * (v / 4) + 4 * half + v % 4;
            bias[v] = p.bias != nullptr && o < p.cout ? p.bias[o] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < NI; j++) {
            __builtin_amdgcn_sched_barrier(0);
            const long long px = px0 + j * 32 + lane % 32;
            const bool in = px < p.P;
            float z[16];
#pragma unroll
            for (int v = 0; v < 16; v++) z[v] = acc[i][j][v] + bias[v];
            if (p.residual != nullptr && in) {
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int o = o0 + 8 * q + 4 * half;
                    const uint16_t *src = p.residual + px * p.ldr + o;
                    if (o + 4 <= p.cout) {
                        const u32x2 r = reinterpret_cast<const Half16 *>(src)->v;
                        z[4 * q] += widen<DT>((uint16_t)r[0]);
                        z[4 * q + 1] += widen<DT>((uint16_t)(r[0] >> 16));
                        z[4 * q + 2] += widen<DT>((uint16_t)r[1]);
                        z[4 * q + 3] += widen<DT>((uint16_t)(r[1] >> 16));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (o + e < p.cout) z[4 * q + e] += widen<DT>(src[e]);
                    }
                }
            }
            if (p.act == SS_ACT_RELU) {
#pragma unroll
                for (int v = 0; v < 16; v++) z[v] = floor_at(z[v], 0.f);
            } else if (p.act == SS_ACT_GELU) {
#pragma unroll
                for (int v = 0; v < 16; v++) z[v] = gelu_cdf<DT>(z[v]);
            }
            // the two lanes of a pixel trade runs of four channels, so that each holds 16 in a row
            uint32_t d[4][2];
#pragma unroll
            for (int q = 0; q < 4; q++) {
                d[q][0] = cvt_pack2<DT>(z[4 * q], z[4 * q + 1]);
                d[q][1] = cvt_pack2<DT>(z[4 * q + 2], z[4 * q + 3]);
            }
            u32x4 run[2];
#pragma unroll
            for (int q = 0; q < 2; q++)
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const auto s = __builtin_amdgcn_permlane32_swap(d[q][e], d[q + 2][e], false, false);
                    run[q][e] = s[0];
                    run[q][2 + e] = s[1];
                }
            if (!in) continue;
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const int o = o0 + 16 * half + 8 * q;
                uint16_t *dst = p.y + px * p.ldy + o;
                if (o + 8 <= p.cout) {
                    reinterpret_cast<Vec16 *>(dst)->v = run[q];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        if (o + e < p.cout) dst[e] = (uint16_t)(run[q][e / 2] >> (16 * (e % 2)));
                }
            }
        }
    }
}

// Large products: four waves, MI x NI tiles of 32 x 32 each, make 64 MI output channels and 64 NI pixels.
//   weights     straight from memory into registers, in the instruction's own order, three steps (of 64 reduction indices) ahead
//   activation  256 channels at a time through two LDS buffers, filled from registers that were loaded a chunk earlier; 16-byte pieces trade
//               places within their row so that neither the fill nor a wave's read of 32 rows meets a bank twice
// A reduction past the last block meets zero scales on both sides; rows past the last read zeros from the buffer's end.
template <int DT, int MI, int NI>
__global__ __launch_bounds__(256, MI * NI >= 16 ? 1 : 2) void pw_mx4_tile_kernel(PwArgs p, int tiles_m, int tiles_n)
{
    constexpr int BN = 64 * NI, PIECES = BN * kChunk / 256;
    __shared__ __attribute__((aligned(16))) uint8_t codes_s[2][BN * kChunk * 16];
    __shared__ uint32_t scales_s[2][2][BN];                // [buffer][half][pixel]: the four steps' bytes
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int KB = (p.K + 31) / 32, S = (KB + 3) / 4 * 4, Ks = (KB + 1) / 2, Kq = (Ks + 3) / 4, Mt = (p.cout + 31) / 32;
    // An XCD (workgroups b, b + 8, ...) works on neighbouring tiles, in bands of eight tiles of channels: 32 of them in flight read 8 + 4 panels.
    const int total = tiles_m * tiles_n, xcd = blockIdx.x % 8;
    const int id = xcd * (total / 8) + min(xcd, total % 8) + blockIdx.x / 8;
    const int band = id / (8 * tiles_n), band_m = min(8, tiles_m - band * 8), in_band = id - band * 8 * tiles_n;
    const int tm = band * 8 + in_band % band_m, tn = in_band / band_m;
    const int mt0 = tm * 2 * MI + __builtin_amdgcn_readfirstlane(wave / 2) * MI;
    const long long row0 = (long long)tn * BN;
    const unsigned pitch = (unsigned)KB * 16u;
    const int rows = (int)min((long long)BN, p.P - row0);
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.codes) + row0 * pitch, 0, (int)(rows * pitch), 0x00020000);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.scales) + row0 * S, 0, rows * S, 0x00020000);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w), 0, Mt * Ks * 1024, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p.w_scales), 0, Mt * Kq * 256, 0x00020000);
    u32x4 piece[PIECES];
    uint32_t ps[2];
    auto fetch = [&](int q) {                               // chunk q of the activation, to registers
#pragma unroll
        for (int i = 0; i < PIECES; i++) {
            const int at = tid + 256 * i, row = at / 8, b = q * kChunk + at % 8;
            piece[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, (int)(row * pitch + b * 16), 0, 0));
        }
#pragma unroll
        for (int d = 0; d < 2; d++) {
            const int b = q * kChunk + 4 * d;              // (past a row's scales: past the buffer's end, which reads zero)
            ps[d] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, b < S ? tid * S + b : -4, 0, 0);
        }
    };
    auto fill = [&](int buf) {
#pragma unroll
        for (int i = 0; i < PIECES; i++) {
            const int at = tid + 256 * i, row = at / 8, b = at % 8;
            *reinterpret_cast<u32x4 *>(codes_s[buf] + row * 128 + ((b ^ (row & 7) ^ ((row >> 3) & 1)) * 16)) = piece[i];
        }
        if (BN >= 256 || tid < BN) {
            scales_s[buf][0][tid] = __builtin_amdgcn_perm(ps[1], ps[0], 0x06040200u);
            scales_s[buf][1][tid] = __builtin_amdgcn_perm(ps[1], ps[0], 0x07050301u);
        }
    };
    u32x4 wa[4][MI];
    uint32_t sa[MI], na[MI];
    auto weights = [&](int ks, u32x4 (&to)[MI]) {
        const int k = min(ks, Ks - 1);                     // (a step past the last has zero scales, a tile past the last is not stored)
#pragma unroll
        for (int i = 0; i < MI; i++)
            to[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, lane * 16, (min(mt0 + i, Mt - 1) * Ks + k) * 1024, 0));
    };
    auto weight_scales = [&](int q, uint32_t (&to)[MI]) {
#pragma unroll
        for (int i = 0; i < MI; i++)
            to[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(ra, lane * 4, (min(mt0 + i, Mt - 1) * Kq + min(q, Kq - 1)) * 256, 0);
    };
    f32x16 acc[MI][NI] = {};
    fetch(0);
    weight_scales(0, sa);
#pragma unroll
    for (int s = 0; s < 3; s++) weights(s, wa[s]);
    fill(0);
    __syncthreads();
    const int px0 = (wave % 2) * NI * 32, half = lane / 32;
    // (no branches: the compiler moves matrix instructions behind one, away from their loads; what is fetched behind the last chunk is not used)
    for (int q = 0; q < Kq; q++) {
        const int buf = q & 1;
        fetch(q + 1);
        weight_scales(q + 1, na);
        uint32_t sb[NI];
#pragma unroll
        for (int j = 0; j < NI; j++) sb[j] = scales_s[buf][half][px0 + j * 32 + lane % 32];
#pragma unroll
        for (int s = 0; s < 4; s++) {
            __builtin_amdgcn_sched_barrier(0);              // (loads stay in their step: moved ahead they take more registers than there are)
            weights(q * 4 + s + 3, wa[(s + 3) % 4]);
            u32x4 xb[NI];
#pragma unroll
            for (int j = 0; j < NI; j++) {
                const int row = px0 + j * 32 + lane % 32, b = 2 * s + half;
                xb[j] = *reinterpret_cast<const u32x4 *>(codes_s[buf] + row * 128 + ((b ^ (row & 7) ^ ((row >> 3) & 1)) * 16));
            }
#pragma unroll
            for (int i = 0; i < MI; i++)
#pragma unroll
                for (int j = 0; j < NI; j++) {
                    if (s == 0) acc[i][j] = mma_mx4<0>(wa[s][i], xb[j], acc[i][j], sa[i], sb[j]);
                    if (s == 1) acc[i][j] = mma_mx4<1>(wa[s][i], xb[j], acc[i][j], sa[i], sb[j]);
                    if (s == 2) acc[i][j] = mma_mx4<2>(wa[s][i], xb[j], acc[i][j], sa[i], sb[j]);
                    if (s == 3) acc[i][j] = mma_mx4<3>(wa[s][i], xb[j], acc[i][j], sa[i], sb[j]);
                }
        }
        __builtin_amdgcn_sched_barrier(0);
        fill(buf ^ 1);
#pragma unroll
        for (int i = 0; i < MI; i++) sa[i] = na[i];
        lds_barrier();
    }
    pw_store<DT, MI, NI>(p, acc, mt0, row0 + px0, lane);
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
    const auto go = [&](auto mi, auto ni) -> int {
        constexpr int MI = decltype(mi)::value, NI = decltype(ni)::value;
        const long long tm = (t.Mt + 2 * MI - 1) / (2 * MI), tn = (rows + 64 * NI - 1) / (64 * NI);
        if (tm * tn > 0x7FFFFFFFll) return SS_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)(tm * tn)), block(256);
        d->dtype == SS_F16 ? pw_mx4_tile_kernel<SS_F16, MI, NI><<<grid, block, 0, s>>>(a, (int)tm, (int)tn)
                           : pw_mx4_tile_kernel<SS_BF16, MI, NI><<<grid, block, 0, s>>>(a, (int)tm, (int)tn);
        return launched();
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    const long long cus = std::max(compute_units(), 1);
    const auto tiles = [&](int mi, int ni) { return (long long)((t.Mt + 2 * mi - 1) / (2 * mi)) * ((rows + 64 * ni - 1) / (64 * ni)); };
    if (tiles(4, 4) >= cus) return go(Four{}, Four{});
    if (tiles(2, 2) >= cus) return go(Two{}, Two{});
    return go(One{}, One{});
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
