// Group norm of channels-last images with its activation, and its gradient.  For image n and group g of C / G neighbouring channels, m = pixels * C / G values:
//
//     mean, var over the m values      r = 1 / sqrt(var + eps)      xh = (x - mean) r      z = xh w + b      y = act(z)
//
//     t = dy act'(z)      S0[n][c] = sum over pixels of t      S1[n][c] = sum of t xh      dw[c] = sum over n of S1,  db[c] = sum of S0
//     dx = r (w t - A - xh B),      A = sum over the group of w S0 / m,      B = sum of w S1 / m
//
// Images of any size: a kernel finds sums of each channel over a chunk of pixels, a second joins them for each image and group, a third applies what they give.  A channel's mean and
// sum of squared differences are found around its first value, and joined by the differences of means: no small difference of large sums.  All sums are in 32 bits, over
// the chunks in 64, in a fixed order.  Bound by memory, three times x forward (64 x 56 x 56 x 256 in bfloat16 57 us, 5.4 TB/s), five tensors backward (95 us, 5.4 TB/s), and by three launches: one image of
// 64 x 64 x 320 16 and 19 us.
#ifndef SS_GROUPNORM_KERNEL_H_
#define SS_GROUPNORM_KERNEL_H_
#include "ss_norm_kernel.h"

namespace ss {

struct GroupArgs {
    const char *x, *dy;
    char *out;                             // y, or dx
    const float *w, *b;
    float2 *stats;                         // [images][groups]: mean, r
    float2 *part;                          // [images][chunks][C]: mean and M2, or S0 and S1, of a chunk
    float2 *total;                         // backward: [images][C] S0 and S1, or NULL where one image's are dw and db
    float2 *coef;                          // backward: [images][groups] A and B
    float *dw, *db;
    long long ldx, lddy, ldout;
    int images, pixels, C, cg, groups, act, chunks, per_chunk;
    int lanes, slots, tiles;               // threads of a row (8 channels each), rows of a workgroup, column tiles
    unsigned cg_mul, cg_sh;                // a channel's group: c * cg_mul >> cg_sh
    float eps;
};

template <int ODT>
__device__ __forceinline__ float normal_cdf(float z)
{
    if constexpr (ODT == SS_F32) return 0.5f * erfcf(-0.70710678118654752f * z);
    const float h = __builtin_amdgcn_exp2f(log2_upper_tail<ODT == SS_F16 ? SS_F16 : SS_BF16>(fabsf(z)));
    return z < 0.f ? h : 1.f - h;
}

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }

// From 256 on in magnitude the exponentials are 0 or infinity, and sigmoid, Phi and both slopes 0 or 1, whatever z is: a factor z bounded there meets no 0 as an infinity, and the product is
// the limit.  (One instruction; it makes a number of a NaN, which the other factor keeps.)
constexpr float kActEnd = 256.f;
__device__ __forceinline__ float act_factor(float z, float end) { return __builtin_amdgcn_fmed3f(z, -kActEnd, end); }

template <int DT>
__device__ __forceinline__ float activate(float z, int act)
{
    if (act == SS_ACT_RELU) return floor_at(z, 0.f);
    if (act == SS_ACT_SILU) return act_factor(z, __builtin_inff()) * sigmoid(z);
    if (act == SS_ACT_GELU) {
        if constexpr (DT == SS_F32)
            return act_factor(z, __builtin_inff()) * normal_cdf<DT>(z);
        else
            return gelu_cdf<DT>(z);
    }
    return z;
}

// act'(z) where it has no corner.
template <int DT>
__device__ __forceinline__ float slope(float z, int act)
{
    const float f = act_factor(z, kActEnd);
    if (act == SS_ACT_SILU) {
        const float s = sigmoid(z);
        return s * __builtin_fmaf(f, 1.f - s, 1.f);
    }
    return __builtin_fmaf(f, 0.39894228040143268f * __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z), normal_cdf<DT>(z));
}

__device__ __forceinline__ int group_of(const GroupArgs &p, int c) { return (int)(((unsigned long long)(unsigned)c * p.cg_mul) >> p.cg_sh); }

// f(the activation, known at compile time): a thread's loops over its rows stand inside.
template <typename F>
__device__ __forceinline__ void with_act(int act, F &&f)
{
    if (act == SS_ACT_RELU)
        f(std::integral_constant<int, SS_ACT_RELU>{});
    else if (act == SS_ACT_SILU)
        f(std::integral_constant<int, SS_ACT_SILU>{});
    else if (act == SS_ACT_GELU)
        f(std::integral_constant<int, SS_ACT_GELU>{});
    else
        f(std::integral_constant<int, SS_ACT_NONE>{});
}

// The constants of eight channels from c on, of G groups (1, or up to 8): z = (x - mean) a + b.
template <int G>
struct Channels {
    float mean[G], r[G], a[8], b[8];
    const float *w;                        // of these channels, or NULL
    int left;                              // how many there are
    __device__ __forceinline__ Channels(const GroupArgs &p, int n, int c) : w(p.w != nullptr ? p.w + c : nullptr), left(p.C - c)
    {
        if (w != nullptr)
            load8<SS_F32>(w, left, a);
        else
#pragma unroll
            for (int e = 0; e < 8; e++) a[e] = 1.f;
        if (p.b != nullptr)
            load8<SS_F32>(p.b + c, left, b);
        else
#pragma unroll
            for (int e = 0; e < 8; e++) b[e] = 0.f;
#pragma unroll
        for (int e = 0; e < G; e++) {
            const float2 s = p.stats[(long long)n * p.groups + group_of(p, min(c + e, p.C - 1))];
            mean[e] = s.x;
            r[e] = s.y;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) a[e] *= r[e % G];
    }
};

// t = dy act'(z) of eight channels of a pixel, d = x - mean.
// A sum of 32 bits next to the corner of a ReLU may be on its wrong side, which is no small error of the gradient: where any of the eight is, they are summed in 64.
template <int DT, int ACT, int G>
__device__ __forceinline__ void before_act(const Channels<G> &k, const float (&d)[8], const float (&x)[8], const float (&dy)[8], float (&t)[8])
{
    if constexpr (ACT == SS_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = dy[e];
    } else if constexpr (ACT == SS_ACT_RELU) {
        float z[8], near = 1.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            z[e] = __builtin_fmaf(d[e], k.a[e], k.b[e]);
            near = fminf(near, fabsf(z[e]) - fmaxf(fabsf(k.b[e]) * 0x1p-20f, 0x1p-100f));
        }
        if (near <= 0.f) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const double w = k.w != nullptr && e < k.left ? k.w[e] : 1.f;
                const double exact = ((double)x[e] - (double)k.mean[e % G]) * (double)k.r[e % G] * w + (double)k.b[e];
                z[e] = exact > 0.0 ? 1.f : exact <= 0.0 ? 0.f : z[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = z[e] <= 0.f ? 0.f : dy[e];          // (a NaN in the group comes in by xh)
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) t[e] = dy[e] * slope<DT>(__builtin_fmaf(d[e], k.a[e], k.b[e]), ACT);
    }
}

// Where a thread works: eight channels from c on, of rows slot, slot + slots, ...
struct Place {
    int n, chunk, c, slot, count, first, last;
    bool idle;
};

__device__ __forceinline__ Place group_place(const GroupArgs &p)
{
    Place q;
    const int tile = (int)(blockIdx.x % (unsigned)p.tiles), unit = (int)(blockIdx.x / (unsigned)p.tiles);
    q.n = unit / p.chunks;
    q.chunk = unit - q.n * p.chunks;
    q.slot = (int)threadIdx.x / p.lanes;
    q.c = (tile * p.lanes + (int)threadIdx.x - q.slot * p.lanes) * 8;
    q.first = q.chunk * p.per_chunk;
    q.last = min(p.pixels, q.first + p.per_chunk);
    q.idle = q.slot >= p.slots || q.c >= p.C;
    q.count = q.idle ? 0 : max(0, (q.last - q.first - q.slot + p.slots - 1) / p.slots);
    return q;
}

// mean and M2 of n values, joined with those of k more
__device__ __forceinline__ void join_moments(float n, float &mean, float &m2, float k, float mean_k, float m2_k)
{
    const float total = n + k, d = mean_k - mean, f = total > 0.f ? k / total : 0.f;
    mean = __builtin_fmaf(d, f, mean);
    m2 = (m2 + m2_k) + d * d * (n * f);
}

constexpr int kGroupThreads = 256;

// Moments of each channel over a chunk.
template <int DT, int MODE>
__global__ __launch_bounds__(kGroupThreads) void group_moments_kernel(GroupArgs p)
{
    constexpr int U = 4, B = item_bytes<DT>();
    __shared__ float mean_s[8][kGroupThreads], m2_s[8][kGroupThreads];
    __shared__ int count_s[kGroupThreads];
    const Place q = group_place(p);
    const int n = q.idle ? 0 : p.C - q.c, t = threadIdx.x;
    float k[8] = {}, s1[8] = {}, s2[8] = {};
    if (q.count > 0) {
        const char *const image = p.x + (long long)q.n * p.pixels * p.ldx * B;
        for (int i = 0; i < q.count; i += U) {
            Run<DT> raw[U];
#pragma unroll
            for (int u = 0; u < U; u++) raw[u] = row_run<DT, MODE>(image + (q.first + q.slot + (long long)min(i + u, q.count - 1) * p.slots) * p.ldx * B, q.c, n, p.C);
#pragma unroll
            for (int u = 0; u < U; u++) {
                float v[8];
                row_values<DT, MODE>(raw[u], q.c, n, p.C, v);
                const float f = i + u < q.count ? 1.f : 0.f;
                if (i + u == 0)
#pragma unroll
                    for (int e = 0; e < 8; e++) k[e] = v[e];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float d = (v[e] - k[e]) * f;
                    s1[e] += d;
                    s2[e] = __builtin_fmaf(d, d, s2[e]);
                }
            }
        }
    }
    const float inv = q.count > 0 ? 1.f / (float)q.count : 0.f;
    int count = q.count;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float d = s1[e] * inv;
        s2[e] -= s1[e] * d;
        if (s2[e] < 0.f) s2[e] = 0.f;                     // (a NaN stays one)
        s1[e] = k[e] + d;
        mean_s[e][t] = s1[e];
        m2_s[e][t] = s2[e];
    }
    count_s[t] = count;
    for (int rows = p.slots; rows > 1;) {
        const int half = (rows + 1) / 2, other = t + half * p.lanes;
        __syncthreads();
        if (q.slot + half < rows) {
            const int more = count_s[other];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                join_moments((float)count, s1[e], s2[e], (float)more, mean_s[e][other], m2_s[e][other]);
                mean_s[e][t] = s1[e];
                m2_s[e][t] = s2[e];
            }
            count += more;
            count_s[t] = count;
        }
        rows = half;
    }
    if (q.slot != 0 || q.idle) return;
    float2 *const out = p.part + ((long long)q.n * p.chunks + q.chunk) * p.C + q.c;
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < n) out[e] = float2{s1[e], s2[e]};
}

template <int DT, int MODE>
__global__ __launch_bounds__(kGroupThreads) void group_apply_kernel(GroupArgs p)
{
    constexpr int U = 4, B = item_bytes<DT>();
    const Place q = group_place(p);
    if (q.count == 0) return;
    const int n = p.C - q.c;
    const Channels<8> k(p, q.n, q.c);
    const long long base = (long long)q.n * p.pixels + q.first + q.slot;
    with_act(p.act, [&](auto act) {
        for (int i = 0; i < q.count; i += U) {
            Run<DT> raw[U];
#pragma unroll
            for (int u = 0; u < U; u++) raw[u] = row_run<DT, MODE>(p.x + (base + (long long)min(i + u, q.count - 1) * p.slots) * p.ldx * B, q.c, n, p.C);
#pragma unroll
            for (int u = 0; u < U; u++) {
                float v[8];
                row_values<DT, MODE>(raw[u], q.c, n, p.C, v);
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = activate<DT>(__builtin_fmaf(v[e] - k.mean[e], k.a[e], k.b[e]), decltype(act)::value);
                if (i + u < q.count) store8<DT>(p.out + ((base + (long long)(i + u) * p.slots) * p.ldout + q.c) * B, n, v);
            }
        }
    });
}

// ---------------------------------------------------------------------------------------------
// gradient
// ---------------------------------------------------------------------------------------------
// S0 and S1 of each channel over a chunk.
template <int DT, int MODE>
__global__ __launch_bounds__(kGroupThreads) void group_sums_kernel(GroupArgs p)
{
    constexpr int U = 4, B = item_bytes<DT>();
    __shared__ float s0_s[8][kGroupThreads], s1_s[8][kGroupThreads];
    const Place q = group_place(p);
    const int n = q.idle ? 0 : p.C - q.c, t = threadIdx.x;
    float s0[8] = {}, s1[8] = {};
    if (q.count > 0) {
        const Channels<8> k(p, q.n, q.c);
        const long long base = (long long)q.n * p.pixels + q.first + q.slot;
        with_act(p.act, [&](auto act) {
            for (int i = 0; i < q.count; i += U) {
                Run<DT> rx[U], rd[U];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    const long long row = base + (long long)min(i + u, q.count - 1) * p.slots;
                    rx[u] = row_run<DT, MODE>(p.x + row * p.ldx * B, q.c, n, p.C);
                    rd[u] = row_run<DT, MODE>(p.dy + row * p.lddy * B, q.c, n, p.C);
                }
#pragma unroll
                for (int u = 0; u < U; u++) {
                    float x[8], dy[8], d[8], g[8];
                    row_values<DT, MODE>(rx[u], q.c, n, p.C, x);
                    row_values<DT, MODE>(rd[u], q.c, n, p.C, dy);
#pragma unroll
                    for (int e = 0; e < 8; e++) d[e] = x[e] - k.mean[e];
                    before_act<DT, decltype(act)::value>(k, d, x, dy, g);
                    if (i + u >= q.count) break;
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        s0[e] += g[e];
                        s1[e] = __builtin_fmaf(g[e], d[e], s1[e]);
                    }
                }
            }
        });
#pragma unroll
        for (int e = 0; e < 8; e++) s1[e] *= k.r[e];
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        s0_s[e][t] = s0[e];
        s1_s[e][t] = s1[e];
    }
    for (int rows = p.slots; rows > 1;) {
        const int half = (rows + 1) / 2, other = t + half * p.lanes;
        __syncthreads();
        if (q.slot + half < rows)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                s0_s[e][t] = s0[e] += s0_s[e][other];
                s1_s[e][t] = s1[e] += s1_s[e][other];
            }
        rows = half;
    }
    if (q.slot != 0 || q.idle) return;
    float2 *const out = p.part + ((long long)q.n * p.chunks + q.chunk) * p.C + q.c;
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (e < n) out[e] = float2{s0[e], s1[e]};
}

// dw and db: the images' sums, in 64 bits, however many there are; 16 channels to the workgroup and `SLICES` slices of the images.
template <int SLICES>
__device__ __forceinline__ void group_vectors(const GroupArgs &p, int block)
{
    __shared__ double2 s[SLICES][17];
    const int lane = threadIdx.x % 16, slice = threadIdx.x / 16, c = block * 16 + lane;
    double2 v = {0.0, 0.0};
    if (c < p.C)
#pragma unroll 4
        for (int n = slice; n < p.images; n += SLICES) {
            const float2 t = p.total[(long long)n * p.C + c];
            v.x += t.x;
            v.y += t.y;
        }
    s[slice][lane] = v;
    __syncthreads();
    if (slice != 0 || c >= p.C) return;
    double2 sum = {0.0, 0.0};
#pragma unroll 8
    for (int k = 0; k < SLICES; k++) {
        sum.x += s[k][lane].x;
        sum.y += s[k][lane].y;
    }
    if (p.dw != nullptr) p.dw[c] = (float)sum.y;
    if (p.db != nullptr) p.db[c] = (float)sum.x;
}

template <int DT, int MODE>
__global__ __launch_bounds__(kGroupThreads) void group_grad_kernel(GroupArgs p)
{
    constexpr int U = 4, B = item_bytes<DT>();
    const int vector_blocks = p.dw != nullptr || p.db != nullptr ? (p.C + 15) / 16 : 0, blocks = (int)gridDim.x - vector_blocks;
    if ((int)blockIdx.x >= blocks) return group_vectors<kGroupThreads / 16>(p, (int)blockIdx.x - blocks);           // uniform (workgroups behind those of the pass)
    const Place q = group_place(p);
    if (q.count == 0) return;
    const int n = p.C - q.c;
    const Channels<8> k(p, q.n, q.c);
    float c0[8], c1[8];                                    // dx = a t - r A - (r B) xh = a t + c0 + c1 d
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float2 coef = p.coef[(long long)q.n * p.groups + group_of(p, min(q.c + e, p.C - 1))];
        c0[e] = -k.r[e] * coef.x;
        c1[e] = -k.r[e] * k.r[e] * coef.y;
    }
    const long long base = (long long)q.n * p.pixels + q.first + q.slot;
    with_act(p.act, [&](auto act) {
        for (int i = 0; i < q.count; i += U) {
            Run<DT> rx[U], rd[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const long long row = base + (long long)min(i + u, q.count - 1) * p.slots;
                rx[u] = row_run<DT, MODE>(p.x + row * p.ldx * B, q.c, n, p.C);
                rd[u] = row_run<DT, MODE>(p.dy + row * p.lddy * B, q.c, n, p.C);
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                float x[8], dy[8], d[8], t[8];
                row_values<DT, MODE>(rx[u], q.c, n, p.C, x);
                row_values<DT, MODE>(rd[u], q.c, n, p.C, dy);
#pragma unroll
                for (int e = 0; e < 8; e++) d[e] = x[e] - k.mean[e];
                before_act<DT, decltype(act)::value>(k, d, x, dy, t);
#pragma unroll
                for (int e = 0; e < 8; e++) t[e] = __builtin_fmaf(d[e], c1[e], __builtin_fmaf(t[e], k.a[e], c0[e]));
                if (i + u < q.count) store8<DT>(p.out + ((base + (long long)(i + u) * p.slots) * p.ldout + q.c) * B, n, t);
            }
        }
    });
}

template <int DT>
void launch_group(const GroupArgs &a, int stage, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.images * a.chunks * a.tiles)), block(kGroupThreads);
    const auto pick = [&](auto md) {
        constexpr int MODE = decltype(md)::value;
        if (stage == 0) group_moments_kernel<DT, MODE><<<grid, block, 0, s>>>(a);
        if (stage == 1) group_apply_kernel<DT, MODE><<<grid, block, 0, s>>>(a);
        if (stage == 2) group_sums_kernel<DT, MODE><<<grid, block, 0, s>>>(a);
        if (stage == 3) group_grad_kernel<DT, MODE><<<dim3(grid.x + (a.dw != nullptr || a.db != nullptr ? (unsigned)((a.C + 15) / 16) : 0u)), block, 0, s>>>(a);
    };
    a.C < 8 ? pick(Mode<NARROW>{}) : a.C % 8 ? pick(Mode<CUT>{}) : pick(Mode<EVEN>{});
}

// (one translation unit to the type, ss_groupnorm_*.hip, instantiates this)
#define SS_GROUP_LAUNCHES(X, DT) X template void launch_group<DT>(const GroupArgs &, int, hipStream_t);

}  // namespace ss

#endif
