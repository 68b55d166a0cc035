// What the pointwise kernels on block-scaled operands share: their arguments, the finishing and storing of tiles of sums, and launches with large LDS.
#ifndef SS_PW_TAIL_H_
#define SS_PW_TAIL_H_
#include "ss_mx4.h"
#include "ss_lds.h"
#include <type_traits>

namespace ss {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int N> using Int = std::integral_constant<int, N>;

struct PwArgs {
    const uint8_t *codes, *scales;         // quantised activation
    const uint8_t *w;                      // first weight tile
    const uint8_t *w_scales;               // first word of their scales
    const float *bias;
    const uint16_t *residual;
    uint16_t *y;
    long long ldr, ldy;
    int P, cout, K, act;
    bool stream;                           // the output passes the caches by
};

// Rows that a workgroup quantises itself.  A thread's runs are its workgroup's threads apart: `step_row` rows and `step_run` runs, or one row more and a row's runs less, so that only
// the first takes a division.
struct PwRowsArgs {
    const uint16_t *x;
    long long ldx;
    unsigned mul, sh;                      // division by a row's runs: 8 Ks in 4 bits, 16 KB in 8
    int step_row, step_run;                // the kernel's threads over and modulo the runs
    unsigned blocks;                       // workgroups that share the rows (the others take other output channels)
    int units;                             // units of output channels of a workgroup: 64 of them with one chunk, 32 with more
};

// The bias of a lane's 16 channels of the tile from channel o0 on; ALL: the tile ends within the matrix.
template <bool ALL>
__device__ __forceinline__ f32x16 tile_bias(const PwArgs &p, int o0, int half)
{
    f32x16 s = {};
    if (p.bias == nullptr) return s;
#pragma unroll
    for (int v = 0; v < 16; v++) {
        const int o = o0 + 8 * (v / 4) + 4 * half + v % 4;
        s[v] = ALL || o < p.cout ? p.bias[o] : 0.f;
    }
    return s;
}

// Is there a residual, is there none, or do the arguments tell?
enum { NO_RES = 0, RES = 1, MAYBE_RES = 2 };

// A tile's residual, as its output leaves: 16 bytes of a pixel to the lane.  (As runs of four channels, 8 bytes here and there: 96 -> 384 in 4 bits on 401408 rows 198 us instead of 153.)
template <bool ALL>
__device__ __forceinline__ void load_residual(const PwArgs &p, int o0, long long px0, int half, u32x4 (&from)[2])
{
    const int o = o0 + (int)(threadIdx.x / 16 % 2) * 16 + half * 8;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        from[q] = u32x4{};
        const long long at = px0 + 16 * q + threadIdx.x % 16;
        if (!ALL && at >= p.P) continue;
        const uint16_t *const src = p.residual + at * p.ldr + o;
        if (ALL || o + 8 <= p.cout)
            from[q] = reinterpret_cast<const Vec16 *>(src)->v;
        else
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (o + e < p.cout) from[q][e / 2] |= (uint32_t)src[e] << (16 * (e % 2));
    }
}

// A 32 x 32 tile of sums, finished: residual, activation, rounding.  A lane gets channels lane / 16 % 2 * 16 + half * 8 to 7 more of pixels lane % 16 and 16 more.  ALL: the
// tile ends within the matrix.  BIAS: it is not in the sums yet.
template <int DT, bool ALL, bool BIAS, int WITH>
__device__ __forceinline__ void finish_tile(const PwArgs &p, const f32x16 &acc, const f32x16 &bias, int o0, long long px0, int half, u32x4 (&run)[2])
{
    float z[16];
#pragma unroll
    for (int v = 0; v < 16; v++) z[v] = BIAS ? acc[v] + bias[v] : acc[v];
    if (WITH == RES || (WITH == MAYBE_RES && p.residual != nullptr)) {
        u32x4 from[2];
        load_residual<ALL>(p, o0, px0, half, from);
        // (the way back of the stores' trades, to the lane that has the sums)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t a = from[0][e], b = from[1][e];
            const auto s = __builtin_amdgcn_permlane16_swap(a, b, false, false);
            from[0][e] = s[0];
            from[1][e] = s[1];
        }
#pragma unroll
        for (int q = 0; q < 2; q++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const uint32_t a = from[q][e], b = from[q][2 + e];
                const auto s = __builtin_amdgcn_permlane32_swap(a, b, false, false);
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    z[8 * q + 4 * k + 2 * e] += widen<DT>((uint16_t)s[k]);
                    z[8 * q + 4 * k + 2 * e + 1] += widen<DT>((uint16_t)(s[k] >> 16));
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
    // A lane holds runs of four channels of one pixel, and a store of those would write 8 bytes here and there.  Its partner's runs come in first (16
    // bytes of a pixel to the lane, 32 to the two of them), then pixel 16 to 31's places in the first half of the channels are traded for pixel 0 to
    // 15's in the second: a store instruction then writes all 64 bytes of 16 pixels.
    uint32_t d[4][2];
#pragma unroll
    for (int q = 0; q < 4; q++) {
        d[q][0] = cvt_pack2<DT>(z[4 * q], z[4 * q + 1]);
        d[q][1] = cvt_pack2<DT>(z[4 * q + 2], z[4 * q + 3]);
    }
#pragma unroll
    for (int q = 0; q < 2; q++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const auto s = __builtin_amdgcn_permlane32_swap(d[2 * q][e], d[2 * q + 1][e], false, false);
            run[q][e] = s[0];
            run[q][2 + e] = s[1];
        }
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const uint32_t a = run[0][e], b = run[1][e];
        const auto s = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        run[0][e] = s[0];
        run[1][e] = s[1];
    }
}

// How an output leaves: by the caches, past them, or past them in whole lines where two tiles of 32 channels stand side by side.  (Whole lines where the caches do not put them
// together: 96 -> 384 on 401408 rows 98 -> 66 us; of 154 MB, which they do, 46 -> 49.  With a GELU the vector ALU has no time for the trade: 100 and 103.)
enum { KEPT = 0, PAST = 1, LINES = 2 };

template <bool STREAM>
__device__ __forceinline__ void store_run(uint16_t *dst, const u32x4 &v)
{
    if constexpr (STREAM)
        __builtin_nontemporal_store(v, &reinterpret_cast<Vec16 *>(dst)->v);
    else
        reinterpret_cast<Vec16 *>(dst)->v = v;
}

template <int DT, bool ALL, bool STREAM>
__device__ __forceinline__ void store_tile(const PwArgs &p, const u32x4 (&run)[2], int o0, long long px0, int lane)
{
    const int o = o0 + lane / 16 % 2 * 16 + lane / 32 * 8;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const long long to = px0 + 16 * q + lane % 16;
        if (!ALL && to >= p.P) continue;
        uint16_t *dst = p.y + to * p.ldy + o;
        if (ALL || o + 8 <= p.cout) {
            store_run<STREAM>(dst, run[q]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (o + e < p.cout) dst[e] = (uint16_t)(run[q][e / 2] >> (16 * (e % 2)));
        }
    }
}

// Two tiles of 64 channels side by side: every other eight pixels of the one are traded for the other's, so that a store writes all 128 bytes, a cache line, of 8 pixels.
__device__ __forceinline__ void store_pair(const PwArgs &p, const u32x4 (&left)[2], const u32x4 (&right)[2], int o0, long long px0, int lane)
{
    const bool upper = lane & 8;
    uint16_t *const dst = p.y + (px0 + lane % 8) * p.ldy + o0 + upper * 32 + lane / 16 % 2 * 16 + lane / 32 * 8;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        u32x4 low, high;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t a = left[q][e], b = right[q][e];
            const uint32_t from_a = (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x128, 0xF, 0xF, true), from_b = (uint32_t)__builtin_amdgcn_mov_dpp((int)b, 0x128, 0xF, 0xF, true);
            low[e] = upper ? from_b : a;
            high[e] = upper ? b : from_a;
        }
        store_run<true>(dst + 16 * q * p.ldy, low);
        store_run<true>(dst + (16 * q + 8) * p.ldy, high);
    }
}

// A wave's MI x NI tiles, from row tile mt0 and pixel px0 on.  BIAS: it is not in the sums yet.
template <int DT, int MI, int NI, bool ALL, bool BIAS, int OUT, int WITH = MAYBE_RES>
__device__ __forceinline__ void pw_store(const PwArgs &p, const f32x16 (&acc)[MI][NI], int mt0, long long px0, int lane)
{
    constexpr bool lines = MI == 2 && ALL && OUT == LINES;
    f32x16 bias[MI] = {};
    if constexpr (BIAS)
#pragma unroll
        for (int i = 0; i < MI; i++) bias[i] = tile_bias<ALL>(p, (mt0 + i) * 32, lane / 32);
#pragma unroll
    for (int j = 0; j < NI; j++) {
        u32x4 run[MI][2];
#pragma unroll
        for (int i = 0; i < MI; i++) {
            __builtin_amdgcn_sched_barrier(0);
            const int o0 = (mt0 + i) * 32;
            if (!ALL && o0 >= p.cout) break;
            finish_tile<DT, ALL, BIAS, WITH>(p, acc[i][j], bias[i], o0, px0 + j * 32, lane / 32, run[i]);
            if constexpr (!lines) store_tile<DT, ALL, OUT != KEPT>(p, run[i], o0, px0 + j * 32, lane);
        }
        if constexpr (lines) store_pair(p, run[0], run[1], mt0 * 32, px0 + j * 32, lane);
    }
}

// Waits until at most N of the wave's loads from memory are under way.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
}
template <auto KERNEL>
int launch_lds(long long blocks, int threads, size_t bytes, hipStream_t s, const PwArgs &a, const PwRowsArgs &r)
{
    if (blocks > 0x7FFFFFFFll) return SS_ERR_UNSUPPORTED;
    const int st = allow_lds<KERNEL>(bytes);
    if (st != SS_OK) return st;
    KERNEL<<<dim3((unsigned)blocks), dim3(threads), bytes, s>>>(a, r);
    return launched();
}

}  // namespace ss

#endif
