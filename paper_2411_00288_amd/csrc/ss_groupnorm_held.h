// Group norm of images that a workgroup can hold: one pass over the data.
//
// A workgroup takes one image's bundle of neighbouring groups, so many that a pixel's share is worth a memory access, and keeps it in registers from its only read to its only write: a
// thread holds eight channels of every R-th pixel.  The mean is found first and the squares of the differences from it then.  Sums go over the threads in LDS:
// first each channel's over the threads that hold it, then each group's over its channels.  Bundles of an image follow each other on one XCD, so that a line whose channels several
// of them share is read and written once.
// 64 images of 28 x 28 x 512 in bfloat16 24 us (4.2 TB/s), of 56 x 56 x 256, which takes 1024 threads and a compute unit for 200 KB, 46 to 53; the gradient of the former 45 us and 48 with
// the vectors' launch: two workgroups of 256 threads to the compute unit (216 registers a lane), memory read and written once and the vector ALU busy a tenth of the time, so that probably
// too few reads are in flight while sums are joined and rows written.  One image of 7 x 7 x 768 5.0 us.
#ifndef SS_GROUPNORM_HELD_H_
#define SS_GROUPNORM_HELD_H_
#include "ss_groupnorm_kernel.h"
#include "ss_lds.h"

namespace ss {

// The shape of a workgroup: its groups, their channels, threads of a pixel, pixels at a time, pixels of a thread.
struct HeldShape {
    int groups, width, lanes, slots, rows, threads, bundles;
};

constexpr int held_most_threads(bool backward) { return backward ? 512 : 1024; }
// Registers of a thread for data, in values of 16 bits: 16 rows of 8 values forward, and of two tensors backward.
constexpr int held_most_rows(int dt) { return dt == SS_F32 ? 8 : 16; }

// LDS of a workgroup, in floats, behind each other: the threads' values, the channels', the groups'.
inline size_t held_lds(const HeldShape &h, int values) { return ((size_t)values * (8 * (size_t)h.threads + (size_t)h.lanes * 8 + h.groups)) * sizeof(float); }

// N sums over the workgroup at once: v[i][e] of every thread -> channel[i * lanes * 8 + c] and group[i * groups + g], weighted by the channel's `weight`.  Entered and left behind a barrier.
template <int N, typename Weight>
__device__ __forceinline__ void held_sums(const HeldShape &h, int cg, const float (&v)[N][8], float *shared, float *channel, float *group, Weight &&weight)
{
    const int t = threadIdx.x, T = h.threads, lane = t % 64, wave = t / 64, waves = T / 64;
#pragma unroll
    for (int i = 0; i < N; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) shared[(i * 8 + e) * T + t] = v[i][e];
    __syncthreads();
    if (h.slots >= 32) {
        // a wave to the channel
        for (int c = wave; c < h.width; c += waves) {
            float s[N] = {};
            const float *const from = shared + (c % 8) * T + c / 8;
            for (int k = lane; k < h.slots; k += 64)
#pragma unroll
                for (int i = 0; i < N; i++) s[i] += from[i * 8 * T + k * h.lanes];
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float sum = lanes_sum<64>(s[i]);
                if (lane == 0) channel[i * h.lanes * 8 + c] = sum;
            }
        }
    } else {
        for (int c = t; c < h.width; c += T) {
            float s[N] = {};
            const float *const from = shared + (c % 8) * T + c / 8;
            for (int k = 0; k < h.slots; k++)
#pragma unroll
                for (int i = 0; i < N; i++) s[i] += from[i * 8 * T + k * h.lanes];
#pragma unroll
            for (int i = 0; i < N; i++) channel[i * h.lanes * 8 + c] = s[i];
        }
    }
    __syncthreads();
    if (cg <= 16) {
        for (int g = t; g < h.groups; g += T) {
            float s[N] = {};
            for (int c = g * cg; c < (g + 1) * cg; c++)
#pragma unroll
                for (int i = 0; i < N; i++) s[i] = __builtin_fmaf(weight(c), channel[i * h.lanes * 8 + c], s[i]);
#pragma unroll
            for (int i = 0; i < N; i++) group[i * h.groups + g] = s[i];
        }
    } else {
        for (int g = wave; g < h.groups; g += waves) {
            float s[N] = {};
            for (int c = g * cg + lane; c < (g + 1) * cg; c += 64)
#pragma unroll
                for (int i = 0; i < N; i++) s[i] = __builtin_fmaf(weight(c), channel[i * h.lanes * 8 + c], s[i]);
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float sum = lanes_sum<64>(s[i]);
                if (lane == 0) group[i * h.groups + g] = sum;
            }
        }
    }
    __syncthreads();
}

// The groups' sums of one value to the thread, where a thread's eight channels are of one group: v -> group[g].
__device__ __forceinline__ void held_group_sums(const HeldShape &h, int cg, float v, float *shared, float *group)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = h.threads / 64, per = cg / 8;
    shared[threadIdx.x] = v;
    __syncthreads();
    for (int g = wave; g < h.groups; g += waves) {
        float s = 0.f;
        for (int k = lane; k < h.slots * per; k += 64) {
            const int slot = k / per;
            s += shared[slot * h.lanes + g * per + k - slot * per];
        }
        s = lanes_sum<64>(s);
        if (lane == 0) group[g] = s;
    }
    __syncthreads();
}

struct HeldPlace {
    int n, c0, c, slot, left, rows;        // image, the bundle's first channel, the thread's, its pixel, its channels in the bundle, its pixels
};

// Row i of a thread: a uniform address and the lane's 32 bits (the shape sees to it that they are enough), so that a row in flight takes no registers for its address.
template <int DT>
__device__ __forceinline__ Run<DT> held_run(const char *image, long long ld, const HeldShape &h, const HeldPlace &q, int i, int C)
{
    constexpr int B = item_bytes<DT>();
    const unsigned lane_at = ((unsigned)q.slot * (unsigned)ld + (unsigned)min(q.c, C - 8)) * B;
    Run<DT> r;
    const char *const p = image + (long long)i * h.slots * ld * B + lane_at;
    if constexpr (DT == SS_F32) {
        r.v[0] = reinterpret_cast<const Vec32 *>(p)[0].v;
        r.v[1] = reinterpret_cast<const Vec32 *>(p)[1].v;
    } else {
        r.v[0] = reinterpret_cast<const Vec16 *>(p)->v;
    }
    return r;
}

__device__ __forceinline__ HeldPlace held_place(const GroupArgs &p, const HeldShape &h)
{
    HeldPlace q;
    const int total = (int)gridDim.x, xcd = (int)blockIdx.x % 8, id = xcd * (total / 8) + min(xcd, total % 8) + (int)blockIdx.x / 8;
    q.n = id / h.bundles;
    q.c0 = (id - q.n * h.bundles) * h.width;
    q.slot = (int)threadIdx.x / h.lanes;
    const int run = ((int)threadIdx.x - q.slot * h.lanes) * 8;
    q.c = q.c0 + run;
    q.left = min(h.width - run, p.C - q.c);                // (a last bundle may be narrower)
    q.rows = q.slot < h.slots && q.left > 0 ? max(0, (p.pixels - q.slot + h.slots - 1) / h.slots) : 0;
    return q;
}

// ONE: a thread's eight channels are of one group.
template <int DT, int NR, int MODE, bool ONE>
__global__ __launch_bounds__(held_most_threads(false)) void group_held_kernel(GroupArgs p, HeldShape h)
{
    constexpr int B = item_bytes<DT>(), G = ONE ? 1 : 8;
    extern __shared__ float smem[];
    const HeldPlace q = held_place(p, h);
    float *const channel = smem + 8 * h.threads, *const group = channel + h.lanes * 8;
    const char *const image = p.x + (long long)q.n * p.pixels * p.ldx * B;
    char *const out = p.out + (long long)q.n * p.pixels * p.ldout * B;
    const unsigned out_at = ((unsigned)q.slot * (unsigned)p.ldout + (unsigned)q.c) * B;
    Run<DT> raw[NR];
#pragma unroll
    for (int i = 0; i < NR; i++)
        if (i < q.rows) raw[i] = held_run<DT>(image, p.ldx, h, q, i, p.C);
    float w[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int c = min(q.c + e, p.C - 1);
        w[e] = p.w != nullptr ? p.w[c] : 1.f;
        b[e] = p.b != nullptr ? p.b[c] : 0.f;
    }
    const auto values = [&](int i, float (&v)[8]) { row_values<DT, MODE>(raw[i], q.c, q.left, p.C, v); };
    int g[G];                                              // groups in the bundle
#pragma unroll
    for (int e = 0; e < G; e++) g[e] = min(group_of(p, max(min(q.c + e, p.C - 1) - q.c0, 0)), h.groups - 1);
    const float inv = 1.f / ((float)p.pixels * (float)p.cg);
    float s[1][8] = {};
#pragma unroll
    for (int i = 0; i < NR; i++)
        if (i < q.rows) {
            float v[8];
            values(i, v);
#pragma unroll
            for (int e = 0; e < 8; e++) s[0][e] += v[e];
        }
    const auto sums = [&] {
        if constexpr (ONE)
            held_group_sums(h, p.cg, ((s[0][0] + s[0][1]) + (s[0][2] + s[0][3])) + ((s[0][4] + s[0][5]) + (s[0][6] + s[0][7])), smem, group);
        else
            held_sums<1>(h, p.cg, s, smem, channel, group, [](int) { return 1.f; });
    };
    sums();
    float mean[G];
#pragma unroll
    for (int e = 0; e < G; e++) mean[e] = group[g[e]] * inv;
    const int mine = (int)threadIdx.x;
    const float mean_out = mine < h.groups ? group[mine] * inv : 0.f;         // (a bundle has at most 32 groups)
#pragma unroll
    for (int e = 0; e < 8; e++) s[0][e] = 0.f;
#pragma unroll
    for (int i = 0; i < NR; i++)
        if (i < q.rows) {
            float v[8];
            values(i, v);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = v[e] - mean[e % G];
                s[0][e] = __builtin_fmaf(d, d, s[0][e]);
            }
        }
    sums();
    if (p.stats != nullptr && mine < h.groups) {
        const int at = group_of(p, q.c0) + mine;
        if (at < p.groups) p.stats[(long long)q.n * p.groups + at] = float2{mean_out, reciprocal_root(group[mine] * inv + p.eps)};
    }
    float r[G];
#pragma unroll
    for (int e = 0; e < G; e++) r[e] = reciprocal_root(group[g[e]] * inv + p.eps);
#pragma unroll
    for (int e = 0; e < 8; e++) w[e] *= r[e % G];
    with_act(p.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
#pragma unroll
        for (int i = 0; i < NR; i++)
            if (i < q.rows) {
                float v[8];
                values(i, v);
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = activate<DT>(__builtin_fmaf(v[e] - mean[e % G], w[e], b[e]), ACT);
                store8<DT>(out + (long long)i * h.slots * p.ldout * B + out_at, q.left, v);
            }
    });
}

template <int DT, int NR, int MODE, bool ONE>
__global__ __launch_bounds__(held_most_threads(true)) void group_held_grad_kernel(GroupArgs p, HeldShape h)
{
    constexpr int B = item_bytes<DT>(), G = ONE ? 1 : 8;
    extern __shared__ float smem[];
    const HeldPlace q = held_place(p, h);
    float *const channel = smem + 16 * h.threads, *const group = channel + 2 * h.lanes * 8;
    const char *const image = p.x + (long long)q.n * p.pixels * p.ldx * B, *const image_dy = p.dy + (long long)q.n * p.pixels * p.lddy * B;
    char *const out = p.out + (long long)q.n * p.pixels * p.ldout * B;
    const unsigned out_at = ((unsigned)q.slot * (unsigned)p.ldout + (unsigned)q.c) * B;
    Run<DT> rx[NR], rd[NR];
#pragma unroll
    for (int i = 0; i < NR; i++)
        if (i < q.rows) {
            rx[i] = held_run<DT>(image, p.ldx, h, q, i, p.C);
            rd[i] = held_run<DT>(image_dy, p.lddy, h, q, i, p.C);
        }
    const Channels<G> k(p, q.n, min(q.c, p.C - 1));
    int g[G];
#pragma unroll
    for (int e = 0; e < G; e++) g[e] = min(group_of(p, max(min(q.c + e, p.C - 1) - q.c0, 0)), h.groups - 1);
    const auto row_of = [&](int i, float (&x)[8], float (&d)[8]) {
        row_values<DT, MODE>(rx[i], q.c, q.left, p.C, x);
#pragma unroll
        for (int e = 0; e < 8; e++) d[e] = x[e] - k.mean[e % G];
    };
    float s[2][8] = {};
    with_act(p.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
#pragma unroll
        for (int i = 0; i < NR; i++)
            if (i < q.rows) {
                float x[8], d[8], dy[8], t[8];
                row_of(i, x, d);
                row_values<DT, MODE>(rd[i], q.c, q.left, p.C, dy);
                before_act<DT, ACT>(k, d, x, dy, t);
                if constexpr (ACT == SS_ACT_RELU) {        // (dy or nothing: it takes dy's place, its channels in theirs)
#pragma unroll
                    for (int e = 0; e < (DT == SS_F32 ? 8 : 4); e++) {
                        if constexpr (DT == SS_F32)
                            rd[i].v[e / 4][e % 4] = as_bits(t[e]);
                        else
                            rd[i].v[0][e] = cvt_pack2<DT>(t[2 * e], t[2 * e + 1]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    s[0][e] += t[e];
                    s[1][e] = __builtin_fmaf(t[e], d[e], s[1][e]);
                }
            }
    });
#pragma unroll
    for (int e = 0; e < 8; e++) s[1][e] *= k.r[e % G];
    held_sums<2>(h, p.cg, s, smem, channel, group, [&](int c) { return p.w != nullptr ? p.w[min(q.c0 + c, p.C - 1)] : 1.f; });
    for (int c = threadIdx.x; c < h.width && q.c0 + c < p.C; c += h.threads) {
        const float s0 = channel[c], s1 = channel[h.lanes * 8 + c];
        if (p.total != nullptr) {
            p.total[(long long)q.n * p.C + q.c0 + c] = float2{s0, s1};
        } else {
            if (p.dw != nullptr) p.dw[q.c0 + c] = s1;
            if (p.db != nullptr) p.db[q.c0 + c] = s0;
        }
    }
    const float inv = 1.f / ((float)p.pixels * (float)p.cg);
    float c0[G], c1[G];                                    // dx = a t - r A - (r B) xh = a t + c0 + c1 d
#pragma unroll
    for (int e = 0; e < G; e++) {
        c0[e] = -k.r[e] * (group[g[e]] * inv);
        c1[e] = -k.r[e] * k.r[e] * (group[h.groups + g[e]] * inv);
    }
    with_act(p.act, [&](auto act) {
        constexpr int ACT = decltype(act)::value;
#pragma unroll
        for (int i = 0; i < NR; i++)
            if (i < q.rows) {
                float x[8], d[8], dy[8], t[8];
                row_of(i, x, d);
                if constexpr (ACT == SS_ACT_RELU) {
                    widen_run<DT>(rd[i], t);
                } else {
                    row_values<DT, MODE>(rd[i], q.c, q.left, p.C, dy);
                    before_act<DT, ACT>(k, d, x, dy, t);
                }
#pragma unroll
                for (int e = 0; e < 8; e++) t[e] = __builtin_fmaf(d[e], c1[e % G], __builtin_fmaf(t[e], k.a[e], c0[e % G]));
                store8<DT>(out + (long long)i * h.slots * p.ldout * B + out_at, q.left, t);
            }
    });
}

template <auto KERNEL>
int launch_held_kernel(const GroupArgs &a, const HeldShape &h, size_t lds, hipStream_t s)
{
    const int st = allow_lds<KERNEL>(lds);
    if (st != SS_OK) return st;
    KERNEL<<<dim3((unsigned)(a.images * h.bundles)), dim3(h.threads), lds, s>>>(a, h);
    return launched();
}

template <int DT>
int launch_held(const GroupArgs &a, const HeldShape &h, bool backward, hipStream_t s)
{
    const size_t lds = held_lds(h, backward ? 2 : 1);
    const auto rows = [&](auto nr) {
        constexpr int NR = decltype(nr)::value;
        const auto pick = [&](auto md, auto one) -> int {
            constexpr int MODE = decltype(md)::value;
            constexpr bool ONE = decltype(one)::value;
            return backward ? launch_held_kernel<group_held_grad_kernel<DT, NR, MODE, ONE>>(a, h, lds, s) : launch_held_kernel<group_held_kernel<DT, NR, MODE, ONE>>(a, h, lds, s);
        };
        if (a.C % 8 || h.width % 8) return pick(Mode<CUT>{}, std::false_type{});
        return a.cg % 8 ? pick(Mode<EVEN>{}, std::false_type{}) : pick(Mode<EVEN>{}, std::true_type{});
    };
    if (h.rows <= 1) return rows(Mode<1>{});
    if (h.rows <= 2) return rows(Mode<2>{});
    if (h.rows <= 4) return rows(Mode<4>{});
    if (h.rows <= 8) return rows(Mode<8>{});
    if constexpr (held_most_rows(DT) >= 16) return rows(Mode<16>{});
    return SS_ERR_UNSUPPORTED;
}

#define SS_HELD_LAUNCHES(X, DT) X template int launch_held<DT>(const GroupArgs &, const HeldShape &, bool, hipStream_t);

}  // namespace ss

#endif
