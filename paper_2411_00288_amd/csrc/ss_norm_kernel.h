// Norms before and after a block, fused with its gate, its residual scale and the residual sum; and their gradient.
//
//     u = post(h)            x_out = x + scale * gate * u            y = norm(x_out) * w + b
//
// post and norm: none, LayerNorm or RMS over the channels of a row.  A row lives in the registers of `LPR` lanes, 8 channels to the lane (NV runs of
// 8 in the widest rows), from its only read to its only write; means and sums of squares are fp32, the variance is the mean square of the
// differences from the mean.  Bound by memory: 401408 x 96, x, h and two outputs, LayerNorm, 61 us (5.0 TB/s), a copy's rate; calls of a few rows by their launch and one
// memory latency (4 x 4096 with both norms 3.6 us).
#ifndef SS_NORM_KERNEL_H_
#define SS_NORM_KERNEL_H_
#include "ss_mx4.h"
#include <algorithm>
#include <type_traits>

namespace ss {

struct NormArgs {
    const char *x, *h, *gate;
    const float *w, *b, *scale, *post_w, *post_b;
    char *x_out, *y;
    uint8_t *codes, *scales;
    long long ldx, ldh, ldx_out, ldy;
    int rows, cols, gate_cols, norm, post;
    float eps, post_eps;
    unsigned g_mul, g_sh;                  // a row's gate: row * g_mul >> g_sh
};

struct NormGradArgs {
    const char *dy, *x_out, *dx_out, *h, *gate;
    const float *w, *scale, *post_w, *post_b;
    char *dx, *dh, *dgate;
    float *part, *gate_part;               // [accumulator][workgroup][cols], [group][strip][gate_cols]
    long long lddy, ldx_out, lddx_out, ldh, lddx, lddh;
    int rows, cols, gate_cols, norm, post;
    float eps, post_eps;
    int groups, per_group, strips, per_strip;
    bool grouped;                          // a gate of several rows: its gradient is a sum over them
};

// ---------------------------------------------------------------------------------------------
// sums over the LPR lanes of a row; every lane gets the sum
// ---------------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)as_bits(v), CTRL, 0xF, 0xF, true));
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    v += dpp<0xB1>(v);                     // lane ^ 1
    v += dpp<0x4E>(v);                     // lane ^ 2
    v += dpp<0x141>(v);                    // the mirror image in 8 lanes
    v += dpp<0x140>(v);                    // the mirror image in 16
    if constexpr (LANES >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(as_bits(v), as_bits(v), false, false);
        v = as_float(p[0]) + as_float(p[1]);
    }
    if constexpr (LANES >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(as_bits(v), as_bits(v), false, false);
        v = as_float(p[0]) + as_float(p[1]);
    }
    return v;
}

// N sums at once.  Rows of several waves join theirs in LDS: `turn` alternates between two places, and a wave that writes one again has
// passed the barrier of the other, behind everyone's reads of the first.
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*shared)[2][LPR / 64 > 0 ? LPR / 64 : 1], int &turn)
{
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = lanes_sum < (LPR < 64 ? LPR : 64) > (v[i]);
    if constexpr (LPR > 64) {
        constexpr int WAVES = LPR / 64;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; i++) shared[turn][i][threadIdx.x % LPR / 64] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; i++) {
            v[i] = 0.f;
#pragma unroll
            for (int k = 0; k < WAVES; k++) v[i] += shared[turn][i][k];
        }
        turn ^= 1;
    }
}

// How a row's width meets the lanes' runs of 8: narrower than one, with a last run that is cut, or even; and even rows of tensors too large for the caches, whose
// lines are not kept (401408 x 96, gradient: 104 -> 94 us; of 4096 x 4096, which fit, 57 -> 60).
enum { NARROW = 0, CUT = 1, EVEN = 2, EVEN_LARGE = 3 };
constexpr bool even(int mode) { return mode >= EVEN; }

// One for a channel of the row, zero past its end.  (As a factor: values past the end are loaded as zeros, and what is subtracted from them is multiplied by
// this, so that they stay zeros without a comparison.)
template <int NV, int MODE>
struct Inside {
    float v[NV][even(MODE) ? 1 : 8];
    __device__ __forceinline__ Inside(const int (&c)[NV], int cols)
    {
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < (even(MODE) ? 1 : 8); e++) v[j][e] = c[j] + e < cols ? 1.f : 0.f;
    }
    __device__ __forceinline__ float at(int j, int e) const { return v[j][even(MODE) ? 0 : e]; }
};

// 1 / sqrt(q), within two units in the last place.  (The instruction alone takes no denormal numbers.)
__device__ __forceinline__ float reciprocal_root(float q)
{
    return q > 1e-36f ? __builtin_amdgcn_rsqf(q) : 1.f / sqrtf(q);
}

// v becomes its normalised row; the factor is returned.  `in`: the row is one; otherwise its values are zero and so is the factor.
template <int LPR, int NV, int MODE>
__device__ __forceinline__ float normalise(float (&v)[NV][8], const Inside<NV, MODE> &inside, float inv, bool layer, float eps, bool in,
                                           float (*shared)[2][LPR / 64 > 0 ? LPR / 64 : 1], int &turn)
{
    if (layer) {
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) s[0] += v[j][e];
        row_sums<LPR>(s, shared, turn);
        const float mean = s[0] * inv;
        if constexpr (even(MODE)) {
#pragma unroll
            for (int j = 0; j < NV; j++) {
                const float m = mean * inside.at(j, 0);
#pragma unroll
                for (int e = 0; e < 8; e++) v[j][e] -= m;
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) v[j][e] = __builtin_fmaf(-mean, inside.at(j, e), v[j][e]);
        }
    }
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < 8; e++) s[0] = __builtin_fmaf(v[j][e], v[j][e], s[0]);
    row_sums<LPR>(s, shared, turn);
    const float r = in ? reciprocal_root(__builtin_fmaf(s[0], inv, eps)) : 0.f;
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < 8; e++) v[j][e] *= r;
    return r;
}

// A vector of the channels, or `fill` where there is none; zero past the row's end.
template <int NV>
__device__ __forceinline__ void channel_vector(const float *p, const int (&c)[NV], int cols, float fill, float (&v)[NV][8])
{
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if (p != nullptr)
            load8<SS_F32>(p + c[j], cols - c[j], v[j]);
        else
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = c[j] + e < cols ? fill : 0.f;
    }
}

// A run of a row, the way its width allows.
template <int DT, int MODE>
__device__ __forceinline__ Run<DT> row_run(const char *row, int c, int n, int cols)
{
    if constexpr (MODE != NARROW)
        return load_wide<DT, MODE == EVEN_LARGE>(row, c, cols);
    else
        return load_run<DT>(row + (long long)c * item_bytes<DT>(), n);
}

template <int DT, int MODE>
__device__ __forceinline__ void row_values(Run<DT> r, int c, int n, int cols, float (&v)[8])
{
    if constexpr (MODE == CUT) place_wide<DT>(r, c, cols, n > 0);
    if constexpr (even(MODE)) {
#pragma unroll
        for (int k = 0; k < (DT == SS_F32 ? 2 : 1); k++) r.v[k] = n > 0 ? r.v[k] : u32x4{};
    }
    widen_run<DT>(r, v);
}

// The next rows are loaded while the current ones are worked on.
template <int DT, int LPR, int NV, bool MX4, bool POST, int MODE>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR) void norm_kernel(NormArgs p)
{
    constexpr int THREADS = LPR < 256 ? 256 : LPR, R = THREADS / LPR;
    constexpr int B = item_bytes<DT>();
    // (rows of 128 lanes: two to the workgroup, each with its own half of the waves)
    __shared__ float shared_all[R][2][2][LPR / 64 > 0 ? LPR / 64 : 1];
    auto *shared = shared_all[threadIdx.x / LPR];
    int turn = 0;
    const int lane = threadIdx.x % LPR;
    int c[NV];
#pragma unroll
    for (int j = 0; j < NV; j++) c[j] = (j * LPR + lane) * 8;
    const bool vector_gate = p.gate_cols > 1 || p.cols == 1;
    const Inside<NV, MODE> inside(c, p.cols);
    const float inv = 1.f / (float)p.cols;
    Run<DT> nx[NV], nh[NV], ng[NV];
    float one = 1.f;
    auto fetch = [&](long long row) {
        const long long at = min(row, (long long)p.rows - 1);
        const bool in = row < p.rows;
#pragma unroll
        for (int j = 0; j < NV; j++) nx[j] = row_run<DT, MODE>(p.x + at * p.ldx * B, c[j], in ? p.cols - c[j] : 0, p.cols);
        if (p.h == nullptr) return;
#pragma unroll
        for (int j = 0; j < NV; j++) nh[j] = row_run<DT, MODE>(p.h + at * p.ldh * B, c[j], in ? p.cols - c[j] : 0, p.cols);
        if (p.gate == nullptr) return;
        const long long g = (long long)(((unsigned long long)(unsigned)at * p.g_mul) >> p.g_sh);
        if (vector_gate) {
#pragma unroll
            for (int j = 0; j < NV; j++) ng[j] = row_run<DT, MODE>(p.gate + g * p.gate_cols * B, c[j], in ? p.cols - c[j] : 0, p.cols);
        } else {
            one = load1<DT>(p.gate + g * B);
        }
    };
    fetch((long long)blockIdx.x * R + threadIdx.x / LPR);
    float w[NV][8], b[NV][8], scale[NV][8], post_w[NV][8], post_b[NV][8];
    channel_vector<NV>(p.w, c, p.cols, 1.f, w);
    channel_vector<NV>(p.b, c, p.cols, 0.f, b);
    channel_vector<NV>(p.scale, c, p.cols, 1.f, scale);
    if constexpr (POST) {
        channel_vector<NV>(p.post_w, c, p.cols, 1.f, post_w);
        channel_vector<NV>(p.post_b, c, p.cols, 0.f, post_b);
    }
    for (long long base = (long long)blockIdx.x * R; base < p.rows; base += (long long)gridDim.x * R) {
        const long long row = base + threadIdx.x / LPR;
        int n[NV];
        float v[NV][8], u[NV][8], gate[NV][8];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            n[j] = row < p.rows ? p.cols - c[j] : 0;
            row_values<DT, MODE>(nx[j], c[j], n[j], p.cols, v[j]);
            if (p.h != nullptr) row_values<DT, MODE>(nh[j], c[j], n[j], p.cols, u[j]);
            if (p.gate != nullptr) {
                if (vector_gate)
                    row_values<DT, MODE>(ng[j], c[j], n[j], p.cols, gate[j]);
                else
#pragma unroll
                    for (int e = 0; e < 8; e++) gate[j][e] = one;
            }
        }
        fetch(row + (long long)gridDim.x * R);
        if (p.h != nullptr) {
            if constexpr (POST) {
                normalise<LPR, NV, MODE>(u, inside, inv, p.post == SS_NORM_LAYER, p.post_eps, row < p.rows, shared, turn);
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) u[j][e] = __builtin_fmaf(u[j][e], post_w[j][e], post_b[j][e]);
            }
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    // (past the row's end u is zero: post_w and post_b are)
                    float s = u[j][e] * scale[j][e];
                    if (p.gate != nullptr) s *= gate[j][e];
                    v[j][e] += s;
                }
#pragma unroll
            for (int j = 0; j < NV; j++) store8<DT>(p.x_out + (row * p.ldx_out + c[j]) * B, n[j], v[j]);
        }
        if (p.norm == SS_NORM_NONE) continue;
        normalise<LPR, NV, MODE>(v, inside, inv, p.norm == SS_NORM_LAYER, p.eps, row < p.rows, shared, turn);
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = __builtin_fmaf(v[j][e], w[j][e], b[j][e]);
#pragma unroll
        for (int j = 0; j < NV; j++) {
            if constexpr (MX4) {
                // four lanes hold a block
                const int KB = (p.cols + 31) / 32, S = (KB + 3) / 4 * 4, run = c[j] / 8;
#pragma unroll
                for (int e = 0; e < 8; e++) v[j][e] = e < n[j] ? v[j][e] : 0.f;
                const uint32_t byte = mx4_scale(quad_max(magnitude8(v[j])));
                if (row < p.rows && run < 4 * KB) *reinterpret_cast<uint32_t *>(p.codes + (row * KB * 4 + run) * 4) = mx4_codes8(v[j], byte);
                if (row < p.rows && run < 4 * S && run % 4 == 0) p.scales[row * S + run / 4] = (uint8_t)byte;
            } else {
                store8<DT>(p.y + (row * p.ldy + c[j]) * B, n[j], v[j]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
// With xh the normalised row, r its factor and g = dy * w:
//     t = dx_out + r (g - mean(g) - xh mean(g xh))          (RMS: without mean(g))
//     dx = t,  dw = sum dy xh,  db = sum dy,  dscale = sum t gate u,  dgate = sum t scale u,  du = t scale gate,  and the same through post.
// Statistics are found again from the rows, which have to be read anyway.  Sums over rows: a workgroup's own rows in registers, in their order,
// then its partial sums in the workspace, which norm_grad_sum_kernel adds in a fixed order: the same bits every time.
// 401408 x 96 without post norm 94 us (4.9 TB/s).  With a post norm the sums are a chain of five joins to a row, and five accumulators and four vectors leave one workgroup to
// the compute unit: 2049 x 1001 26 us, three rounds of rows at 2 to 3 us each, then the sums' launch (4 us); 4096 x 4096 in bfloat16 35 and 7 us.
enum { ACC_W = 0, ACC_B, ACC_SCALE, ACC_POST_W, ACC_POST_B, ACC_COUNT };

// Waves to the SIMD: what the registers of a kernel without post norm leave.
constexpr int grad_waves(int dt, bool vector_gate) { return dt == SS_F32 || vector_gate ? 3 : 4; }
constexpr int grad_threads(int lpr, bool post) { return lpr >= 512 ? lpr : post ? 512 : 256; }

template <int DT, int LPR, int NV, bool POST, bool VECTOR_GATE, int MODE>
__global__ __launch_bounds__(grad_threads(LPR, POST), LPR >= 512 || POST ? 0 : grad_waves(DT, VECTOR_GATE)) void norm_grad_kernel(NormGradArgs p)
{
    constexpr int THREADS = grad_threads(LPR, POST), R = THREADS / LPR;
    constexpr int B = item_bytes<DT>();
    __shared__ float shared_all[R][2][2][LPR / 64 > 0 ? LPR / 64 : 1];
    __shared__ float joined[R > 1 ? THREADS * 8 : 1];
    __shared__ float waves[THREADS / 64];
    auto *shared = shared_all[threadIdx.x / LPR];
    int turn = 0;
    const int lane = threadIdx.x % LPR, rg = threadIdx.x / LPR;
    int c[NV];
#pragma unroll
    for (int j = 0; j < NV; j++) c[j] = (j * LPR + lane) * 8;
    float acc[POST ? ACC_COUNT : ACC_SCALE + 1][NV][8] = {};
    const float inv = 1.f / (float)p.cols;
    const Inside<NV, MODE> inside(c, p.cols);

    // sums of the row groups' registers: put(first channel, how many, 8 values)
    auto join = [&](const float (&v)[NV][8], auto &&put) {
        if constexpr (R == 1) {
#pragma unroll
            for (int j = 0; j < NV; j++) put(c[j], p.cols - c[j], v[j]);
        } else {
            static_assert(NV == 1, "one run to the lane");
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; e++) joined[rg * LPR * 8 + e * LPR + lane] = v[0][e];
            __syncthreads();
            for (int col = threadIdx.x; col < p.cols; col += THREADS) {
                float s[8] = {};
#pragma unroll
                for (int k = 0; k < R; k++) s[0] += joined[k * LPR * 8 + col % 8 * LPR + col / 8];
                put(col, 1, s);
            }
        }
    };

    // The channels' vectors stay in registers where there is room for them.
    constexpr bool KEEP = LPR <= 512 && NV == 1;
    float w[NV][8], scale[NV][8], post_w[NV][8], post_b[NV][8];
    auto vectors = [&] {
        channel_vector<NV>(p.w, c, p.cols, 1.f, w);
        channel_vector<NV>(p.scale, c, p.cols, 1.f, scale);
        if constexpr (POST) {
            channel_vector<NV>(p.post_w, c, p.cols, 1.f, post_w);
            channel_vector<NV>(p.post_b, c, p.cols, 0.f, post_b);
        }
    };
    if constexpr (KEEP) vectors();

    const long long units = (long long)p.groups * p.strips;
    const long long u0 = units * blockIdx.x / gridDim.x, u1 = units * (blockIdx.x + 1) / gridDim.x;
    for (long long unit = u0; unit < u1; unit++) {
        const long long group = unit / p.strips, strip = unit - group * p.strips;
        const long long first = group * p.per_group + strip * p.per_strip;
        const long long last = group * p.per_group + min((long long)p.per_group, (strip + 1) * p.per_strip);
        float gate_acc[VECTOR_GATE ? NV : 1][8] = {}, gate_one = 0.f;
        Run<DT> nv[NV], nt[NV];
        // What the sums begin with is loaded while the rows before are worked on; what comes behind them, at their start.  (All of it ahead took more registers
        // than four waves have: 134 -> 156 us.)
        auto fetch = [&](long long base) {
            const long long row = base + rg, at = min(row, last - 1);
            if (p.norm != SS_NORM_NONE)
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    const int n = row < last ? p.cols - c[j] : 0;
                    nv[j] = row_run<DT, MODE>(p.x_out + at * p.ldx_out * B, c[j], n, p.cols);
                    nt[j] = row_run<DT, MODE>(p.dy + at * p.lddy * B, c[j], n, p.cols);
                }
        };
        if (first < last) fetch(first);
        for (long long base = first; base < last; base += R) {
            const long long row = base + rg;
            const bool in = row < last;
            if constexpr (!KEEP) vectors();
            int n[NV];
            float t[NV][8] = {}, v[NV][8], one = 1.f;
            Run<DT> rd[NV], rh[NV], rgate[VECTOR_GATE ? NV : 1];
            const long long at = min(row, last - 1), g = p.grouped ? group : at;
#pragma unroll
            for (int j = 0; j < NV; j++) {
                n[j] = in ? p.cols - c[j] : 0;
                rd[j] = rh[j] = Run<DT>{};
                if (p.norm != SS_NORM_NONE) {
                    row_values<DT, MODE>(nv[j], c[j], n[j], p.cols, v[j]);
                    row_values<DT, MODE>(nt[j], c[j], n[j], p.cols, t[j]);
                }
                if (p.dx_out != nullptr) rd[j] = row_run<DT, MODE>(p.dx_out + at * p.lddx_out * B, c[j], n[j], p.cols);
                if (p.h != nullptr) rh[j] = row_run<DT, MODE>(p.h + at * p.ldh * B, c[j], n[j], p.cols);
                if constexpr (VECTOR_GATE) rgate[j] = row_run<DT, MODE>(p.gate + g * p.gate_cols * B, c[j], n[j], p.cols);
            }
            if (!VECTOR_GATE && p.gate != nullptr) one = load1<DT>(p.gate + g * B);
            if constexpr (KEEP) fetch(base + R);           // (past the last: the last row again)
            if (p.norm != SS_NORM_NONE) {
                const bool layer = p.norm == SS_NORM_LAYER;
                const float r = normalise<LPR, NV, MODE>(v, inside, inv, layer, p.eps, in, shared, turn);
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        // (values past a row's end are zero, in all of its tensors and in w)
                        acc[ACC_W][j][e] = __builtin_fmaf(t[j][e], v[j][e], acc[ACC_W][j][e]);
                        acc[ACC_B][j][e] += t[j][e];
                        const float g = t[j][e] * w[j][e];
                        t[j][e] = g;
                        s[0] += g;
                        s[1] = __builtin_fmaf(g, v[j][e], s[1]);
                    }
                row_sums<LPR>(s, shared, turn);
                const float m0 = layer ? s[0] * inv : 0.f, m1 = s[1] * inv;
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) t[j][e] = r * __builtin_fmaf(-v[j][e], m1, __builtin_fmaf(-m0, inside.at(j, e), t[j][e]));
            }
            if (p.dx_out != nullptr) {
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    float d[8];
                    row_values<DT, MODE>(rd[j], c[j], n[j], p.cols, d);
#pragma unroll
                    for (int e = 0; e < 8; e++) t[j][e] += d[e];
                }
            }
#pragma unroll
            for (int j = 0; j < NV; j++) store8<DT>(p.dx + (row * p.lddx + c[j]) * B, n[j], t[j]);
            if (p.h != nullptr) {
                float hr = 0.f, hh[NV][8], gate[VECTOR_GATE ? NV : 1][8];
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    row_values<DT, MODE>(rh[j], c[j], n[j], p.cols, hh[j]);
                    if constexpr (VECTOR_GATE) row_values<DT, MODE>(rgate[j], c[j], n[j], p.cols, gate[j]);
                }
                if constexpr (POST) hr = normalise<LPR, NV, MODE>(hh, inside, inv, p.post == SS_NORM_LAYER, p.post_eps, in, shared, turn);
                float dg[VECTOR_GATE ? NV : 1][8], dg_one = 0.f, s[2] = {0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float u = POST ? __builtin_fmaf(hh[j][e], post_w[j][e], post_b[j][e]) : hh[j][e];
                        const float tu = t[j][e] * u, ts = t[j][e] * scale[j][e];
                        const float g = VECTOR_GATE ? gate[VECTOR_GATE ? j : 0][e] : one;
                        acc[ACC_SCALE][j][e] = __builtin_fmaf(tu, g, acc[ACC_SCALE][j][e]);
                        if constexpr (VECTOR_GATE)
                            dg[j][e] = ts * u;
                        else
                            dg_one = __builtin_fmaf(ts, u, dg_one);
                        const float du = ts * g;
                        if constexpr (POST) {
                            acc[ACC_POST_W][j][e] = __builtin_fmaf(du, hh[j][e], acc[ACC_POST_W][j][e]);
                            acc[ACC_POST_B][j][e] += du;
                            const float gg = du * post_w[j][e];
                            t[j][e] = gg;
                            s[0] += gg;
                            s[1] = __builtin_fmaf(gg, hh[j][e], s[1]);
                        } else {
                            t[j][e] = du;
                        }
                    }
                if constexpr (POST) {
                    row_sums<LPR>(s, shared, turn);
                    const float m0 = p.post == SS_NORM_LAYER ? s[0] * inv : 0.f, m1 = s[1] * inv;
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) t[j][e] = hr * __builtin_fmaf(-hh[j][e], m1, __builtin_fmaf(-m0, inside.at(j, e), t[j][e]));
                }
#pragma unroll
                for (int j = 0; j < NV; j++) store8<DT>(p.dh + (row * p.lddh + c[j]) * B, n[j], t[j]);
                if constexpr (VECTOR_GATE) {
#pragma unroll
                    for (int j = 0; j < NV; j++) {
                        if (p.grouped) {
#pragma unroll
                            for (int e = 0; e < 8; e++) gate_acc[j][e] += dg[j][e];
                        } else {
                            store8<DT>(p.dgate + (row * p.gate_cols + c[j]) * B, n[j], dg[j]);
                        }
                    }
                } else if (p.gate != nullptr) {
                    if (p.grouped) {
                        gate_one += dg_one;
                    } else {
                        float sum[1] = {dg_one};
                        row_sums<LPR>(sum, shared, turn);
                        if (in && lane == 0) store1<DT>(p.dgate + row * B, sum[0]);
                    }
                }
            }
            if constexpr (!KEEP)
                if (base + R < last) fetch(base + R);
        }
        if (p.grouped && p.gate != nullptr) {
            auto put = [&](int col, int n, const float (&v)[8]) {
                if (p.strips > 1)
                    store8<SS_F32>(p.gate_part + unit * p.gate_cols + col, n, v);
                else
                    store8<DT>(p.dgate + (group * p.gate_cols + col) * B, n, v);
            };
            if constexpr (VECTOR_GATE) {
                join(gate_acc, put);
            } else {
                gate_one = lanes_sum<64>(gate_one);
                __syncthreads();
                if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = gate_one;
                __syncthreads();
                float s[8] = {};
                for (int k = 0; k < THREADS / 64; k++) s[0] += waves[k];
                if (threadIdx.x == 0) put(0, 1, s);
            }
        }
    }
    const size_t at = (size_t)blockIdx.x * p.cols, step = (size_t)gridDim.x * p.cols;
    auto part = [&](int a, const float (&v)[NV][8]) { join(v, [&](int col, int n, const float (&s)[8]) { store8<SS_F32>(p.part + a * step + at + col, n, s); }); };
    if (p.norm != SS_NORM_NONE) {
        part(ACC_W, acc[ACC_W]);
        part(ACC_B, acc[ACC_B]);
    }
    if (p.h != nullptr) part(ACC_SCALE, acc[ACC_SCALE]);
    if constexpr (POST) {
        part(ACC_POST_W, acc[ACC_POST_W]);
        part(ACC_POST_B, acc[ACC_POST_B]);
    }
}

struct NormSumArgs {
    const float *part, *gate_part;
    float *out[ACC_COUNT];                 // those that are wanted, first
    int which[ACC_COUNT];                  // their accumulators
    char *dgate;
    int cols, parts, strips, wanted, tiles;
    long long gates;                       // elements of the gate's gradient that are still in `strips` parts, or 0
    int gate_cols;
};

constexpr int kSumColumns = 16;            // columns of a workgroup where 64 slices of the parts share them
constexpr int sum_columns(int parts) { return parts > 64 ? kSumColumns : 1024; }

// The workgroups' partial sums: 16 columns to the workgroup and 64 slices of the parts, or, of few parts, a column to the thread.  Behind those workgroups, one thread
// for an element of the gate's gradient.
template <int DT>
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(NormSumArgs p)
{
    __shared__ float s[64][kSumColumns + 1];
    const int columns = sum_columns(p.parts), blocks = p.tiles * p.wanted;
    if ((int)blockIdx.x < blocks) {
        const int a = blockIdx.x / p.tiles, tile = blockIdx.x - a * p.tiles;
        const float *const src = p.part + (size_t)p.which[a] * p.parts * p.cols;
        if (columns != kSumColumns) {
            const int col = tile * 1024 + threadIdx.x;
            if (col >= p.cols) return;
            float v = 0.f;
#pragma unroll 8
            for (int i = 0; i < p.parts; i++) v += src[(size_t)i * p.cols + col];
            p.out[a][col] = v;
            return;
        }
        const int col = tile * kSumColumns + threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
        float v = 0.f;
        if (col < p.cols) {
#pragma unroll 8
            for (int i = slice; i < p.parts; i += 64) v += src[(size_t)i * p.cols + col];
        }
        s[slice][threadIdx.x % kSumColumns] = v;
        __syncthreads();
        for (int half = 32; half > 0; half >>= 1) {
            if (slice < half) s[slice][threadIdx.x % kSumColumns] += s[slice + half][threadIdx.x % kSumColumns];
            __syncthreads();
        }
        if (slice == 0 && col < p.cols) p.out[a][col] = s[0][threadIdx.x];
        return;
    }
    const long long i = (long long)(blockIdx.x - blocks) * 1024 + threadIdx.x;
    if (i >= p.gates) return;
    const long long group = i / p.gate_cols, col = i - group * p.gate_cols;
    const float *src = p.gate_part + group * p.strips * p.gate_cols + col;
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < p.strips; k++) v += src[(long long)k * p.gate_cols];
    store1<DT>(p.dgate + i * item_bytes<DT>(), v);
}

// Lanes of a row (8 channels each), and with 1024 of them two runs to the lane.
struct RowShape {
    int lanes, runs;
};
inline RowShape row_shape(int cols)
{
    int lanes = 16;
    while (lanes < 1024 && lanes * 8 < cols) lanes *= 2;
    return {lanes, lanes * 8 < cols ? 2 : 1};
}

template <int M> using Mode = std::integral_constant<int, M>;

// bytes: what the call reads and writes, against the last-level cache's 256 MB
inline int width_mode(int cols, long long bytes) { return cols < 8 ? NARROW : cols % 8 ? CUT : bytes > 256ll << 20 ? EVEN_LARGE : EVEN; }

template <int DT>
void launch_norm(const NormArgs &a, bool mx4, bool post, hipStream_t s)
{
    const RowShape shape = row_shape(a.cols);
    const int threads = shape.lanes < 256 ? 256 : shape.lanes, r = threads / shape.lanes;
    const int cus = std::max(compute_units(), 1);
    // (as many workgroups as run at once: four waves to the SIMD with a post norm, five without)
    const unsigned grid = (unsigned)std::min<long long>(((long long)a.rows + r - 1) / r, (long long)cus * ((post ? 1024 : 1280) / threads));
    const auto go = [&](auto kern) { kern<<<dim3(grid), dim3(threads), 0, s>>>(a); };
    const auto pick = [&](auto m, auto ps, auto md) {
        constexpr bool MX4 = decltype(m)::value, POST = decltype(ps)::value;
        constexpr int MODE = decltype(md)::value;
        switch (shape.lanes) {
            case 16: go(norm_kernel<DT, 16, 1, MX4, POST, MODE>); break;
            case 32: if constexpr (MODE != NARROW) go(norm_kernel<DT, 32, 1, MX4, POST, MODE>); break;
            case 64: if constexpr (MODE != NARROW) go(norm_kernel<DT, 64, 1, MX4, POST, MODE>); break;
            case 128: if constexpr (MODE != NARROW) go(norm_kernel<DT, 128, 1, MX4, POST, MODE>); break;
            case 256: if constexpr (MODE != NARROW) go(norm_kernel<DT, 256, 1, MX4, POST, MODE>); break;
            case 512: if constexpr (MODE != NARROW) go(norm_kernel<DT, 512, 1, MX4, POST, MODE>); break;
            default:
                if constexpr (MODE != NARROW) shape.runs == 1 ? go(norm_kernel<DT, 1024, 1, MX4, POST, MODE>) : go(norm_kernel<DT, 1024, 2, MX4, POST, MODE>);
        }
    };
    const auto widths = [&](auto m, auto ps) {
        const int mode = width_mode(a.cols, (long long)a.rows * a.cols * item_bytes<DT>() * (a.h != nullptr ? 4 : 2));
        mode == NARROW ? pick(m, ps, Mode<NARROW>{}) : mode == CUT ? pick(m, ps, Mode<CUT>{}) : mode == EVEN ? pick(m, ps, Mode<EVEN>{}) : pick(m, ps, Mode<EVEN_LARGE>{});
    };
    const auto posts = [&](auto m) { post ? widths(m, std::true_type{}) : widths(m, std::false_type{}); };
    mx4 ? posts(std::true_type{}) : posts(std::false_type{});
}

template <int DT>
void launch_norm_grad(const NormGradArgs &a, bool post, int workgroups, hipStream_t s)
{
    const RowShape shape = row_shape(a.cols);
    const auto go = [&](auto kern) { kern<<<dim3(workgroups), dim3(grad_threads(shape.lanes, post)), 0, s>>>(a); };
    const auto pick = [&](auto ps, auto vg, auto md) {
        constexpr bool POST = decltype(ps)::value, VG = decltype(vg)::value;
        constexpr int MODE = decltype(md)::value;
        switch (shape.lanes) {
            case 16: go(norm_grad_kernel<DT, 16, 1, POST, VG, MODE>); break;
            case 32: if constexpr (MODE != NARROW) go(norm_grad_kernel<DT, 32, 1, POST, VG, MODE>); break;
            case 64: if constexpr (MODE != NARROW) go(norm_grad_kernel<DT, 64, 1, POST, VG, MODE>); break;
            case 128: if constexpr (MODE != NARROW) go(norm_grad_kernel<DT, 128, 1, POST, VG, MODE>); break;
            case 256: if constexpr (MODE != NARROW) go(norm_grad_kernel<DT, 256, 1, POST, VG, MODE>); break;
            case 512: if constexpr (MODE != NARROW) go(norm_grad_kernel<DT, 512, 1, POST, VG, MODE>); break;
            default: if constexpr (MODE != NARROW) shape.runs == 1 ? go(norm_grad_kernel<DT, 1024, 1, POST, VG, MODE>) : go(norm_grad_kernel<DT, 1024, 2, POST, VG, MODE>);
        }
    };
    const auto widths = [&](auto ps, auto vg) {
        const int mode = width_mode(a.cols, (long long)a.rows * a.cols * item_bytes<DT>() * (a.h != nullptr ? 6 : 4));
        mode == NARROW ? pick(ps, vg, Mode<NARROW>{}) : mode == CUT ? pick(ps, vg, Mode<CUT>{}) : mode == EVEN ? pick(ps, vg, Mode<EVEN>{}) : pick(ps, vg, Mode<EVEN_LARGE>{});
    };
    const auto gates = [&](auto ps) { a.gate != nullptr && (a.gate_cols > 1 || a.cols == 1) ? widths(ps, std::true_type{}) : widths(ps, std::false_type{}); };
    post ? gates(std::true_type{}) : gates(std::false_type{});
}

template <int DT>
void launch_norm_sum(const NormSumArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.tiles * a.wanted + (a.gates + 1023) / 1024)), block(1024);
    norm_grad_sum_kernel<DT><<<grid, block, 0, s>>>(a);
}

// (one translation unit to the type, ss_norm_*.hip, instantiates these)
#define SS_NORM_LAUNCHES(X, DT)                                                  \
    X template void launch_norm<DT>(const NormArgs &, bool, bool, hipStream_t);  \
    X template void launch_norm_grad<DT>(const NormGradArgs &, bool, int, hipStream_t); \
    X template void launch_norm_sum<DT>(const NormSumArgs &, hipStream_t);

}  // namespace ss

#endif
