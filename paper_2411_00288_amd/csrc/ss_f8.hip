// Quantisation to FP8 with a scale for each block of 128 and back, and the packing of weights.
#include "ss_f8.h"
#include "ss_conv_params.h"
#include <type_traits>

namespace ss {

// One thread per run of 8 values, four runs a thread; the 16 lanes that hold a block find its scale among themselves.  Bound by memory: 2 bytes read and 1.01 written for
// a 16-bit value: 401408 x 384 in bfloat16 75 us (6.2 TB/s); of narrow rows lanes have no channels (401408 x 64 21 us, 3.6 TB/s).  `runs` = 16 * blocks to the row, so that a block is
// never split between rows.  WIDE: rows of at least 8.  LAST: a tensor too large for the caches, whose lines are not kept in them.
template <int DT, bool WIDE, bool LAST>
__global__ __launch_bounds__(256) void f8_quantize_kernel(const char *__restrict__ x, long long ldx, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales,
                                                          long long total, int cols, unsigned runs, unsigned mul, unsigned sh)
{
    const int KB = (int)runs / 16, S = (KB + 3) / 4 * 4, P = (cols + 63) / 64 * 64;
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
        if (first + u * 256 >= total) return;            // (a block's 16 lanes leave together)
        if constexpr (WIDE) place_wide<DT>(v[u], run[u] * 8, cols, true);
        const uint32_t byte = f8_scale(row16_max(magnitude<DT>(v[u])));
        const u32x2 c = f8_codes<DT>(v[u], byte);
        if (run[u] * 8 < P) {
            u32x2 *const to = reinterpret_cast<u32x2 *>(codes + row[u] * P + run[u] * 8);
            if constexpr (LAST)
                __builtin_nontemporal_store(c, to);
            else
                *to = c;
        }
        const int b = run[u] / 16, lane = run[u] % 16;
        if (lane == 0)
            scales[row[u] * S + b] = (uint8_t)byte;
        else if (b == KB - 1 && b + lane < S)
            scales[row[u] * S + b + lane] = 0;
    }
}

// Back: 401408 x 384 to bfloat16 75 to 87 us.
template <int DT>
__global__ __launch_bounds__(256) void f8_dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, char *__restrict__ y, long long ldy,
                                                            long long total, int cols, unsigned runs, unsigned mul, unsigned sh)
{
    const int KB = (cols + 127) / 128, S = (KB + 3) / 4 * 4, P = (cols + 63) / 64 * 64;
    const long long first = (long long)blockIdx.x * 1024 + threadIdx.x;
    u32x2 c[4];
    uint32_t b[4];
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
            c[u] = *reinterpret_cast<const u32x2 *>(codes + row[u] * P + run[u] * 8);
            b[u] = scales[row[u] * S + run[u] / 16];
        }
    }
#pragma unroll
    for (int u = 0; u < 4; u++) {
        if (first + u * 256 >= total) return;
        float v[8];
        f8_values8(c[u], b[u], v);
        store8<DT>(y + (row[u] * ldy + run[u] * 8) * item_bytes<DT>(), cols - run[u] * 8, v);
    }
}

// Weights, once per update: 16 lanes take a block of a row, mask it, quantise it and put it where the matrix instruction's lanes expect it.
template <int DT>
__global__ __launch_bounds__(256) void f8_pack_kernel(const uint16_t *__restrict__ W, const uint8_t *__restrict__ M, uint8_t *__restrict__ packed, int cout, int K, F8Dims t,
                                                      PackHeader hdr)
{
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<uint32_t *>(packed)[threadIdx.x] = threadIdx.x < kHdrWords ? hdr.w[threadIdx.x] : 0u;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int runs = 16 * t.S;                             // (with the blocks that pad the scale words)
    const long long row = i / runs;
    const int run = (int)(i - row * runs), k = run * 8, b = run / 16, mt = (int)(row / 32);
    if (mt >= t.Mt) return;
    const int n = row < cout ? K - k : 0;
    float v[8];
    load8<DT>(W + row * K + k, n, v);
    if (M != nullptr)
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (e < n && M[row * K + k + e] == 0) v[e] = 0.f;
    const uint32_t byte = f8_scale(row16_max(magnitude8(v)));
    if (k < t.P) {
        const size_t piece = ((size_t)mt * t.Ks + k / 64) * 2 + k / 16 % 2;
        *reinterpret_cast<u32x2 *>(packed + kHeaderBytes + piece * 1024 + (row % 32 + k / 32 % 2 * 32) * 16 + k % 16) = f8_codes8(v, byte);
    }
    if (run % 16 == 0) packed[f8_scales_at(t) + (((size_t)mt * t.Kq + b / 4) * 32 + row % 32) * 4 + b % 4] = (uint8_t)byte;
}

template <int DT>
__global__ __launch_bounds__(256) void f8_unpack_kernel(const uint8_t *__restrict__ packed, uint16_t *__restrict__ W, int cout, int K, F8Dims t)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int runs = t.P / 8;
    const long long row = i / runs;
    const int k = (int)(i - row * runs) * 8, b = k / 128, mt = (int)(row / 32);
    if (row >= cout) return;
    const size_t piece = ((size_t)mt * t.Ks + k / 64) * 2 + k / 16 % 2;
    const u32x2 c = *reinterpret_cast<const u32x2 *>(packed + kHeaderBytes + piece * 1024 + (row % 32 + k / 32 % 2 * 32) * 16 + k % 16);
    const uint32_t byte = packed[f8_scales_at(t) + (((size_t)mt * t.Kq + b / 4) * 32 + row % 32) * 4 + b % 4];
    float v[8];
    f8_values8(c, byte, v);
    store8<DT>(W + row * K + k, K - k, v);
}

// The same for weights that lie as [K][cout]: 128 rows of 64 columns at a time.  A thread holds four consecutive rows of eight columns, so that the elements of a column
// come out as whole words; the columns' largest magnitudes are joined over the lanes and, in LDS, over the waves; the words are turned in LDS (a column's 33 words
// apart: 64 banks), and leave 16 bytes at a time.
template <int DT>
__global__ __launch_bounds__(256) void f8_pack_turned_kernel(const uint16_t *__restrict__ W, const uint8_t *__restrict__ M, uint8_t *__restrict__ packed, int cout, int K,
                                                             F8Dims t, PackHeader hdr)
{
    __shared__ uint32_t words[64 * 33];
    __shared__ uint32_t largest[4][64];
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<uint32_t *>(packed)[threadIdx.x] = threadIdx.x < kHdrWords ? hdr.w[threadIdx.x] : 0u;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, run = tid % 8, quad = tid / 8;
    const int tiles = (cout + 63) / 64, kb = (int)(blockIdx.x / tiles), c0 = (int)(blockIdx.x - kb * tiles) * 64, c = c0 + run * 8;
    float v[4][8];
#pragma unroll
    for (int u = 0; u < 4; u++) {
        const int k = kb * 128 + quad * 4 + u, n = k < K ? cout - c : 0;
        load8<DT>(W + (size_t)k * cout + c, n, v[u]);
        if (M != nullptr)
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (e < n && M[(size_t)k * cout + c + e] == 0) v[u][e] = 0.f;
    }
    uint32_t m[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        m[e] = max(max(as_bits(v[0][e]) & 0x7FFFFFFFu, as_bits(v[1][e]) & 0x7FFFFFFFu), max(as_bits(v[2][e]) & 0x7FFFFFFFu, as_bits(v[3][e]) & 0x7FFFFFFFu));
        m[e] = max(m[e], (uint32_t)__builtin_amdgcn_mov_dpp((int)m[e], 0x128 /* eight lanes on in 16 */, 0xF, 0xF, true));
        const auto a = __builtin_amdgcn_permlane16_swap(m[e], m[e], false, false);
        m[e] = max((uint32_t)a[0], (uint32_t)a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(m[e], m[e], false, false);
        m[e] = max((uint32_t)b[0], (uint32_t)b[1]);
    }
    if (lane < 8)
#pragma unroll
        for (int e = 0; e < 8; e++) largest[wave][run * 8 + e] = m[e];
    __syncthreads();
    const auto column_scale = [&](int col) { return f8_scale(max(max(largest[0][col], largest[1][col]), max(largest[2][col], largest[3][col]))); };
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const uint32_t byte = column_scale(run * 8 + e), word = f8_codes4(v[0][e], v[1][e], v[2][e], v[3][e], f8_unit(byte));
        words[(run * 8 + e) * 33 + quad] = byte == 0xFFu ? 0u : word;
    }
    if (tid < 64 && c0 + tid < t.Mt * 32) {
        const int row = c0 + tid;
        uint8_t *const to = packed + f8_scales_at(t) + (((size_t)(row / 32) * t.Kq) * 32 + row % 32) * 4;
        to[(size_t)(kb / 4) * 128 + kb % 4] = (uint8_t)column_scale(tid);
        if (kb == t.KB - 1)
            for (int b = kb + 1; b < t.S; b++) to[(size_t)(b / 4) * 128 + b % 4] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; u++) {
        const int row = c0 + tid % 64, piece = tid / 64 + 4 * u, ks = kb * 2 + u;
        if (ks >= t.Ks || row >= t.Mt * 32) continue;
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] = words[(tid % 64) * 33 + piece * 4 + e];
        *reinterpret_cast<u32x4 *>(packed + kHeaderBytes + ((((size_t)(row / 32) * t.Ks + ks) * 2 + piece % 2) * 64 + row % 32 + piece / 2 % 2 * 32) * 16) = w;
    }
}

int f8_quantize(const void *x, int64_t rows, int cols, int64_t ldx, int dtype, uint8_t *codes, uint8_t *scales, hipStream_t s)
{
    const F8Dims t = f8_dims(1, cols);
    const unsigned runs = (unsigned)t.KB * 16;
    unsigned mul, sh;
    fast_div_setup(runs, &mul, &sh);
    const long long piece = piece_rows(runs / 4);
    const auto go = [&](auto kern) {
        for (long long at = 0; at < rows; at += piece) {
            const long long total = std::min(piece, (long long)rows - at) * runs;
            kern<<<dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, s>>>(static_cast<const char *>(x) + at * ldx * (dtype == SS_F32 ? 4 : 2), (long long)ldx,
                                                                              codes + at * t.P, scales + at * t.S, total, cols, runs, mul, sh);
        }
    };
    const auto pick = [&](auto wide, auto last) {
        constexpr bool WIDE = decltype(wide)::value, LAST = decltype(last)::value;
        dtype == SS_F16 ? go(f8_quantize_kernel<SS_F16, WIDE, LAST>) : dtype == SS_BF16 ? go(f8_quantize_kernel<SS_BF16, WIDE, LAST>) : go(f8_quantize_kernel<SS_F32, WIDE, LAST>);
    };
    if (cols < 8)
        pick(std::false_type{}, std::false_type{});
    else
        rows * (int64_t)cols * (dtype == SS_F32 ? 4 : 2) > 192ll << 20 ? pick(std::true_type{}, std::true_type{}) : pick(std::true_type{}, std::false_type{});
    return launched();
}

namespace {

int check_f8_desc(const ss_weight_desc *d)
{
    const int st = check_desc(d, false);
    if (st != SS_OK) return st;
    if (d->kh != 1 || d->kw != 1 || is_byte_type(d->dtype) || d->cin > kF8MostK) return SS_ERR_UNSUPPORTED;
    const F8Dims t = f8_dims(d->cout, d->cin);
    return (long long)t.Mt * t.Ks * 2048 < 1ll << 31 ? SS_OK : SS_ERR_UNSUPPORTED;
}

// rows x cols of an activation: SS_OK, or why it is refused
int check_rows(int64_t rows, int32_t cols, int64_t ld, int32_t dtype)
{
    if (rows < 0 || cols <= 0 || ld < cols || (dtype != SS_F16 && dtype != SS_BF16 && dtype != SS_F32)) return SS_ERR_INVALID_ARG;
    return rows <= INT32_MAX && cols <= kF8MostK && ld <= INT32_MAX ? SS_OK : SS_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_f8_quantize(const void *x, int64_t rows, int32_t cols, int64_t ldx, int32_t dtype, void *codes, void *scales, void *stream)
{
    const int st = check_rows(rows, cols, ldx, dtype);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!x || !codes || !scales || !aligned(x, dtype == SS_F32 ? 4 : 2) || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    return f8_quantize(x, rows, cols, ldx, dtype, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales), static_cast<hipStream_t>(stream));
}

extern "C" int ss_f8_dequantize(const void *codes, const void *scales, int64_t rows, int32_t cols, int32_t dtype, void *y, int64_t ldy, void *stream)
{
    const int st = check_rows(rows, cols, ldy, dtype);
    if (st != SS_OK) return st;
    if (rows == 0) return SS_OK;
    if (!y || !codes || !scales || !aligned(y, dtype == SS_F32 ? 4 : 2) || !aligned(codes, 16) || !aligned(scales, 4)) return SS_ERR_INVALID_ARG;
    const F8Dims t = f8_dims(1, cols);
    const unsigned runs = (unsigned)(cols + 7) / 8;
    unsigned mul, sh;
    fast_div_setup(runs, &mul, &sh);
    const long long piece = piece_rows((runs + 3) / 4);
    const auto go = [&](auto kern) {
        for (long long at = 0; at < rows; at += piece) {
            const long long total = std::min(piece, (long long)rows - at) * runs;
            kern<<<dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(
                static_cast<const uint8_t *>(codes) + at * t.P, static_cast<const uint8_t *>(scales) + at * t.S,
                static_cast<char *>(y) + at * ldy * (dtype == SS_F32 ? 4 : 2), (long long)ldy, total, cols, runs, mul, sh);
        }
    };
    dtype == SS_F16 ? go(f8_dequantize_kernel<SS_F16>) : dtype == SS_BF16 ? go(f8_dequantize_kernel<SS_BF16>) : go(f8_dequantize_kernel<SS_F32>);
    return launched();
}

extern "C" int ss_f8_packed_bytes(const ss_weight_desc *desc, size_t *packed_bytes)
{
    const int st = check_f8_desc(desc);
    if (st != SS_OK) return st;
    if (!packed_bytes) return SS_ERR_INVALID_ARG;
    *packed_bytes = f8_packed_size(f8_dims(desc->cout, desc->cin));
    return SS_OK;
}

extern "C" int ss_f8_pack(const ss_weight_desc *desc, const void *W, const uint8_t *M, int32_t transposed, void *packed, void *stream)
{
    const int st = check_f8_desc(desc);
    if (st != SS_OK) return st;
    if (!W || !packed || !aligned(W, 2) || !aligned(packed, 16) || (transposed != 0 && transposed != 1)) return SS_ERR_INVALID_ARG;
    const F8Dims t = f8_dims(desc->cout, desc->cin);
    TileDims td{};
    td.Mt = t.Mt;
    td.Ks = t.Ks;
    const PackHeader hdr = pack_header(kMagicF8, desc, td);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const long long blocks = transposed ? (long long)t.KB * ((desc->cout + 63) / 64) : ((long long)t.Mt * 32 * 16 * t.S + 255) / 256;
    if (blocks > 0x7FFFFFll) return SS_ERR_UNSUPPORTED;
    const auto go = [&](auto kern) {
        kern<<<dim3((unsigned)blocks), dim3(256), 0, s>>>(static_cast<const uint16_t *>(W), M, static_cast<uint8_t *>(packed), desc->cout, desc->cin, t, hdr);
    };
    if (transposed)
        desc->dtype == SS_F16 ? go(f8_pack_turned_kernel<SS_F16>) : go(f8_pack_turned_kernel<SS_BF16>);
    else
        desc->dtype == SS_F16 ? go(f8_pack_kernel<SS_F16>) : go(f8_pack_kernel<SS_BF16>);
    return launched();
}

extern "C" int ss_f8_unpack(const ss_weight_desc *desc, const void *packed, void *W, void *stream)
{
    const int st = check_f8_desc(desc);
    if (st != SS_OK) return st;
    if (!W || !packed || !aligned(W, 2) || !aligned(packed, 16)) return SS_ERR_INVALID_ARG;
    const F8Dims t = f8_dims(desc->cout, desc->cin);
    const long long blocks = ((long long)desc->cout * (t.P / 8) + 255) / 256;
    if (blocks > 0x7FFFFFll) return SS_ERR_UNSUPPORTED;
    const auto go = [&](auto kern) {
        kern<<<dim3((unsigned)blocks), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(static_cast<const uint8_t *>(packed), static_cast<uint16_t *>(W), desc->cout, desc->cin, t);
    };
    desc->dtype == SS_F16 ? go(f8_unpack_kernel<SS_F16>) : go(f8_unpack_kernel<SS_BF16>);
    return launched();
}
