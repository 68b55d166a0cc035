// Quantisation to MXFP4 and back, and the packing of weights for the pointwise layer on such operands.
#include "ss_mx4.h"
#include "ss_conv_params.h"
#include <type_traits>

namespace ss {

// One thread per run of 8 values, four runs a thread; the quad of lanes that holds a block finds its scale among itself.  Bound by memory: 2 bytes
// read and 0.53 written for a 16-bit value.  `runs` = 16 * ceil(blocks / 4) to the row, so that a quad is never split between rows and the
// scales' surplus bytes are written too.
// WIDE: rows of at least 8.  LAST: a tensor too large for the caches, whose lines are not kept in them (401408 x 384 to codes and back 151 -> 129 us, 50176 x 768,
// which fit, 33 -> 36).
template <int DT, bool WIDE, bool LAST>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const char *__restrict__ x, long long ldx, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                           long long total, int cols, unsigned runs, unsigned mul, unsigned sh)
{
    const int KB = (cols + 31) / 32, S = (int)runs / 4;
    const long long first = (long long)blockIdx.x * 1024 + threadIdx.x;
    Run<DT> v[4];
    long long row[4];
    int run[4];
#pragma unroll
    for (int u = 0; u < 4; u++) {
        const long long i = first + u * 256;
        if (total < 1ll << 31)                           // uniform
            row[u] = (long long)(((unsigned long long)(unsigned)i * mul) >> sh);
        else
            row[u] = i / runs;
        run[u] = (int)(i - row[u] * runs);
        if constexpr (WIDE)                              // (past the last run: the first row)
            v[u] = load_wide<DT, LAST>(x + (i < total ? row[u] * ldx : 0ll) * item_bytes<DT>(), run[u] * 8, cols);
        else
            v[u] = load_run<DT>(x + (row[u] * ldx + run[u] * 8) * item_bytes<DT>(), i < total ? cols - run[u] * 8 : 0);
    }
#pragma unroll
    for (int u = 0; u < 4; u++) {
        if (first + u * 256 >= total) return;
        if constexpr (WIDE) place_wide<DT>(v[u], run[u] * 8, cols, true);
        const uint32_t byte = mx4_scale(quad_max(magnitude<DT>(v[u])));
        if (run[u] < 4 * KB) *reinterpret_cast<uint32_t *>(codes + (row[u] * KB * 4 + run[u]) * 4) = mx4_codes<DT>(v[u], byte);
        if (run[u] % 4 == 0) scales[row[u] * S + run[u] / 4] = (uint8_t)byte;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, char *__restrict__ y, long long ldy,
                                                             long long total, int cols, unsigned runs, unsigned mul, unsigned sh)
{
    const int KB = (cols + 31) / 32, S = (KB + 3) / 4 * 4;
    const long long first = (long long)blockIdx.x * 1024 + threadIdx.x;
    uint32_t c[4], b[4];
    long long row[4];
    int run[4];
#pragma unroll
    for (int u = 0; u < 4; u++) {
        const long long i = first + u * 256;
        if (total < 1ll << 31)                           // uniform
            row[u] = (long long)(((unsigned long long)(unsigned)i * mul) >> sh);
        else
            row[u] = i / runs;
        run[u] = (int)(i - row[u] * runs);
        if (i < total) {
            c[u] = *reinterpret_cast<const uint32_t *>(codes + (row[u] * KB * 4 + run[u]) * 4);
            b[u] = scales[row[u] * S + run[u] / 4];
        }
    }
#pragma unroll
    for (int u = 0; u < 4; u++) {
        if (first + u * 256 >= total) return;
        float v[8];
        mx4_values8(c[u], b[u], v);
        store8<DT>(y + (row[u] * ldy + run[u] * 8) * item_bytes<DT>(), cols - run[u] * 8, v);
    }
}

// Weights, once per update: a thread takes one block of one row, masks it, quantises it and puts it where the matrix instruction's lane expects it.
template <int DT>
__global__ __launch_bounds__(256) void mx4_pack_kernel(const uint16_t *__restrict__ W, const uint8_t *__restrict__ M, uint8_t *__restrict__ packed, int cout, int K,
                                                       int Mt, int Ks, int Kq, PackHeader hdr)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<uint32_t *>(packed)[threadIdx.x] = threadIdx.x < kHdrWords ? hdr.w[threadIdx.x] : 0u;
    const int slots = 8 * Kq;                              // blocks of a row, with those that pad the scale words
    const int row = (int)(i / slots), b = (int)(i - (long long)row * slots), mt = row >> 5;
    if (mt >= Mt) return;
    const int ks = b >> 1, lane = (row & 31) + 32 * (b & 1);
    float v[4][8];
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; q++) {
        const int k = b * 32 + q * 8, n = row < cout ? K - k : 0;
        load8<DT>(W + (size_t)row * K + k, n, v[q]);
        if (M != nullptr)
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (e < n && M[(size_t)row * K + k + e] == 0) v[q][e] = 0.f;
        m = max(m, magnitude8(v[q]));
    }
    const uint32_t byte = mx4_scale(m);
    if (ks < Ks) {
        u32x4 c;
#pragma unroll
        for (int q = 0; q < 4; q++) c[q] = mx4_codes8(v[q], byte);
        *reinterpret_cast<u32x4 *>(packed + kHeaderBytes + (((size_t)mt * Ks + ks) * 64 + lane) * 16) = c;
    }
    packed[kHeaderBytes + (size_t)Mt * Ks * 1024 + (((size_t)mt * Kq + ks / 4) * 64 + lane) * 4 + ks % 4] = (uint8_t)byte;
}

template <int DT>
__global__ __launch_bounds__(256) void mx4_unpack_kernel(const uint8_t *__restrict__ packed, uint16_t *__restrict__ W, int cout, int K, int Mt, int Ks, int Kq)
{
    const int KB = (K + 31) / 32;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / KB), b = (int)(i - (long long)row * KB), mt = row >> 5;
    if (row >= cout) return;
    const int ks = b >> 1, lane = (row & 31) + 32 * (b & 1);
    const u32x4 c = *reinterpret_cast<const u32x4 *>(packed + kHeaderBytes + (((size_t)mt * Ks + ks) * 64 + lane) * 16);
    const uint32_t byte = packed[kHeaderBytes + (size_t)Mt * Ks * 1024 + (((size_t)mt * Kq + ks / 4) * 64 + lane) * 4 + ks % 4];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        float v[8];
        mx4_values8(c[q], byte, v);
        store8<DT>(W + (size_t)row * K + b * 32 + q * 8, K - b * 32 - q * 8, v);
    }
}

int mx4_quantize(const void *x, int64_t rows, int cols, int64_t ldx, int dtype, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    const Mx4Dims t = mx4_dims(1, cols);
    const unsigned runs = (unsigned)t.S * 4;
    unsigned mul, sh;
    fast_div_setup(runs, &mul, &sh);
    const long long piece = piece_rows(runs / 4);
    const auto go = [&](auto kern) {
        for (long long at = 0; at < rows; at += piece) {
            const long long total = std::min(piece, (long long)rows - at) * runs;
            kern<<<dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, s>>>(static_cast<const char *>(x) + at * ldx * (dtype == SS_F32 ? 4 : 2), (long long)ldx,
                                                                              codes + at * t.KB * 16, scales + at * t.S, total, cols, runs, mul, sh);
        }
    };
    const auto pick = [&](auto wide, auto last) {
        constexpr bool WIDE = decltype(wide)::value, LAST = decltype(last)::value;
        dtype == SS_F16 ? go(mx4_quantize_kernel<SS_F16, WIDE, LAST>) : dtype == SS_BF16 ? go(mx4_quantize_kernel<SS_BF16, WIDE, LAST>) : go(mx4_quantize_kernel<SS_F32, WIDE, LAST>);
    };
    if (cols < 8)
        pick(std::false_type{}, std::false_type{});
    else
        rows * (int64_t)cols * (dtype == SS_F32 ? 4 : 2) > 192ll << 20 ? pick(std::true_type{}, std::true_type{}) : pick(std::true_type{}, std::false_type{});
    return launched();
}

namespace {

int check_mx4_desc(const ss_weight_desc *d)
{
    const int st = check_desc(d, false);
    if (st != SS_OK) return st;
    return d->kh == 1 && d->kw == 1 && !is_byte_type(d->dtype) ? SS_OK : SS_ERR_UNSUPPORTED;
}

// rows x cols of an activation: SS_OK, or why it is refused
int check_rows(int64_t rows, int32_t cols, int64_t ld, int32_t dtype)
{
    if (rows < 0 || cols <= 0 || ld < cols || (dtype != SS_F16 && dtype != SS_BF16 && dtype != SS_F32)) return SS_ERR_INVALID_ARG;
    return rows <= INT32_MAX && cols <= (1 << 24) && ld <= INT32_MAX ? SS_OK : SS_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_mx4_quantize(const void *x, int64_t rows, int32_t cols, int64_t ldx, int32_t dtype, void *codes, void *scales, void *stream)
{
    const int st = check_rows(rows, cols, ldx, dtype);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!x || !codes || !scales || !aligned(x, dtype == SS_F32 ? 4 : 2) || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    return mx4_quantize(x, rows, cols, ldx, dtype, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales), static_cast<hipStream_t>(stream));
}

extern "C" int ss_mx4_dequantize(const void *codes, const void *scales, int64_t rows, int32_t cols, int32_t dtype, void *y, int64_t ldy, void *stream)
{
    const int st = check_rows(rows, cols, ldy, dtype);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!y || !codes || !scales || !aligned(y, dtype == SS_F32 ? 4 : 2) || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    const Mx4Dims t = mx4_dims(1, cols);
    const unsigned runs = (unsigned)t.KB * 4;
    unsigned mul, sh;
    fast_div_setup(runs, &mul, &sh);
    const long long piece = piece_rows(runs / 4);
    const auto go = [&](auto kern) {
        for (long long at = 0; at < rows; at += piece) {
            const long long total = std::min(piece, (long long)rows - at) * runs;
            kern<<<dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(
                static_cast<const uint8_t *>(codes) + at * t.KB * 16, static_cast<const uint8_t *>(scales) + at * t.S,
                static_cast<char *>(y) + at * ldy * (dtype == SS_F32 ? 4 : 2), (long long)ldy, total, cols, runs, mul, sh);
        }
    };
    dtype == SS_F16 ? go(mx4_dequantize_kernel<SS_F16>) : dtype == SS_BF16 ? go(mx4_dequantize_kernel<SS_BF16>) : go(mx4_dequantize_kernel<SS_F32>);
    return launched();
}

extern "C" int ss_mx4_packed_bytes(const ss_weight_desc *desc, size_t *packed_bytes)
{
    const int st = check_mx4_desc(desc);
    if (st != SS_OK) return st;
    if (!packed_bytes) return SS_ERR_INVALID_ARG;
    *packed_bytes = mx4_packed_size(mx4_dims(desc->cout, desc->cin));
    return SS_OK;
}

extern "C" int ss_mx4_pack(const ss_weight_desc *desc, const void *W, const uint8_t *M, void *packed, void *stream)
{
    const int st = check_mx4_desc(desc);
    if (st != SS_OK) return st;
    if (!W || !packed || !aligned(W, 2) || !aligned(packed, 16)) return SS_ERR_INVALID_ARG;
    const Mx4Dims t = mx4_dims(desc->cout, desc->cin);
    TileDims td{};
    td.Mt = t.Mt;
    td.Ks = t.Ks;
    const PackHeader hdr = pack_header(kMagicMx4, desc, td);
    const long long blocks = ((long long)t.Mt * 32 * 8 * t.Kq + 255) / 256;
    if (blocks > 0x7FFFFFFFll) return SS_ERR_UNSUPPORTED;
    const auto go = [&](auto kern) {
        kern<<<dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(static_cast<const uint16_t *>(W), M, static_cast<uint8_t *>(packed), desc->cout,
                                                                                         desc->cin, t.Mt, t.Ks, t.Kq, hdr);
    };
    desc->dtype == SS_F16 ? go(mx4_pack_kernel<SS_F16>) : go(mx4_pack_kernel<SS_BF16>);
    return launched();
}

extern "C" int ss_mx4_unpack(const ss_weight_desc *desc, const void *packed, void *W, void *stream)
{
    const int st = check_mx4_desc(desc);
    if (st != SS_OK) return st;
    if (!W || !packed || !aligned(W, 2) || !aligned(packed, 16)) return SS_ERR_INVALID_ARG;
    const Mx4Dims t = mx4_dims(desc->cout, desc->cin);
    const long long blocks = ((long long)desc->cout * t.KB + 255) / 256;
    if (blocks > 0x7FFFFFFFll) return SS_ERR_UNSUPPORTED;
    const auto go = [&](auto kern) {
        kern<<<dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(static_cast<const uint8_t *>(packed), static_cast<uint16_t *>(W), desc->cout,
                                                                                         desc->cin, t.Mt, t.Ks, t.Kq);
    };
    desc->dtype == SS_F16 ? go(mx4_unpack_kernel<SS_F16>) : go(mx4_unpack_kernel<SS_BF16>);
    return launched();
}
