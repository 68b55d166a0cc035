// Entry points of the group norm of channels-last images (kernels: ss_groupnorm_kernel.h and, where a workgroup holds its data, ss_groupnorm_held.h).
#include "ss_groupnorm_held.h"
#include "ss_conv_params.h"
#include <cmath>

namespace ss {

SS_GROUP_LAUNCHES(extern, SS_F16)
SS_GROUP_LAUNCHES(extern, SS_BF16)
SS_GROUP_LAUNCHES(extern, SS_F32)
SS_HELD_LAUNCHES(extern, SS_F16)
SS_HELD_LAUNCHES(extern, SS_BF16)
SS_HELD_LAUNCHES(extern, SS_F32)

namespace {

constexpr int kMostJoinThreads = 1024;

// Where a thread works that joins what the chunks of an image's group left: `lanes` threads side by side over its channels, `slices` of those over its chunks.
struct JoinPlace {
    int n, g, lanes, slices, lane, slice;
    __device__ __forceinline__ explicit JoinPlace(const GroupArgs &p)
    {
        n = (int)(blockIdx.x / (unsigned)p.groups);
        g = (int)blockIdx.x - n * p.groups;
        lanes = min(p.cg, (int)blockDim.x);
        slices = (int)blockDim.x / lanes;
        slice = (int)threadIdx.x / lanes;
        lane = (int)threadIdx.x - slice * lanes;
    }
};

// The workgroup's sum, in a fixed order.
__device__ __forceinline__ double join_sum(double v, double *shared)
{
#pragma unroll
    for (int step = 1; step < 64; step *= 2) v += __shfl_xor(v, step);
    __syncthreads();
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
    __syncthreads();
    double s = 0.0;
    for (int k = 0; k < (int)blockDim.x / 64; k++) s += shared[k];
    return s;
}

// An image's group: its chunks' and channels' moments together.  With a channel's mean d away from a value k of the group, over `rows` pixels, mean = k + sum of rows d / m and
// M2 = sum of (M2 + rows d^2) - m (mean - k)^2: in 64 bits, where neither the number of chunks nor the difference takes what 32 hold.
__global__ __launch_bounds__(kMostJoinThreads) void group_stats_kernel(GroupArgs p)
{
    __shared__ double shared[kMostJoinThreads / 64];
    const JoinPlace q(p);
    const float2 *const part = p.part + (long long)q.n * p.chunks * p.C + (long long)q.g * p.cg;
    const double m = (double)p.pixels * (double)p.cg, k = part[0].x;
    const double rows = p.per_chunk, last = p.pixels - (p.chunks - 1) * p.per_chunk;
    double s1 = 0.0, s2 = 0.0;
    if (q.slice < q.slices)
        for (int c = q.lane; c < p.cg; c += q.lanes)
#pragma unroll 8
            for (int chunk = q.slice; chunk < p.chunks; chunk += q.slices) {
                const float2 v = part[(long long)chunk * p.C + c];
                const double d = (double)v.x - k, t = (chunk + 1 < p.chunks ? rows : last) * d;
                s1 += t;
                s2 += __builtin_fma(t, d, (double)v.y);
            }
    s1 = join_sum(s1, shared);
    s2 = join_sum(s2, shared);
    const double d = s1 / m;
    double var = s2 / m - d * d;
    if (var < 0.0) var = 0.0;                              // (a NaN stays one)
    if (threadIdx.x == 0) p.stats[(long long)q.n * p.groups + q.g] = float2{(float)(k + d), reciprocal_root((float)(var + (double)p.eps))};
}

// An image's group: its channels' sums over the chunks, and A and B; in 64 bits, as many chunks as there may be.
__global__ __launch_bounds__(kMostJoinThreads) void group_coef_kernel(GroupArgs p)
{
    __shared__ double2 slice_s[kMostJoinThreads];
    __shared__ double shared[kMostJoinThreads / 64];
    const JoinPlace q(p);
    double a = 0.0, b = 0.0;
    for (int at = 0; at < p.cg; at += q.lanes) {           // (more than once: then there is one slice)
        const int i = at + q.lane, c = q.g * p.cg + i;
        const bool in = q.slice < q.slices && i < p.cg;
        const float2 *const part = p.part + (long long)q.n * p.chunks * p.C + c;
        double2 s = {0.0, 0.0};
        if (in)
#pragma unroll 8
            for (int k = q.slice; k < p.chunks; k += q.slices) {
                const float2 v = part[(long long)k * p.C];
                s.x += v.x;
                s.y += v.y;
            }
        if (q.slices > 1) {
            slice_s[threadIdx.x] = s;
            for (int left = q.slices; left > 1;) {
                const int half = (left + 1) / 2;
                __syncthreads();
                if (q.slice + half < left) {
                    const double2 o = slice_s[threadIdx.x + half * q.lanes];
                    s.x += o.x;
                    s.y += o.y;
                    slice_s[threadIdx.x] = s;
                }
                left = half;
            }
        }
        if (in && q.slice == 0) {
            p.total[(long long)q.n * p.C + c] = float2{(float)s.x, (float)s.y};
            const double w = p.w != nullptr ? p.w[c] : 1.f;
            a = __builtin_fma(w, s.x, a);
            b = __builtin_fma(w, s.y, b);
        }
    }
    a = join_sum(a, shared);
    b = join_sum(b, shared);
    const double m = (double)p.pixels * (double)p.cg;
    if (threadIdx.x == 0) p.coef[(long long)q.n * p.groups + q.g] = float2{(float)(a / m), (float)(b / m)};
}

// Threads that join a group's chunks: one to eight of its values.
int join_threads(const GroupArgs &a) { return (int)std::clamp<long long>(((long long)a.chunks * a.cg / 8 + 63) / 64 * 64, 64, kMostJoinThreads); }

template <int SLICES>
__global__ __launch_bounds__(SLICES * 16) void group_vectors_kernel(GroupArgs p) { group_vectors<SLICES>(p, (int)blockIdx.x); }

constexpr int kManyImages = 512;            // 32 to a thread of 16 slices

constexpr int kMostChannels = 16384;
constexpr int64_t kMostPixels = 1 << 24;   // (a group's values are counted in fp32)
constexpr int64_t kMostPitch = 1 << 19;    // (1024 pixels of it are 2^31 bytes, a lane's offset)

int check_group(const ss_groupnorm_desc *d, int64_t images, int64_t pixels)
{
    if (!d || d->channels <= 0 || d->groups <= 0 || d->channels % d->groups != 0 || d->reserved != 0) return SS_ERR_INVALID_ARG;
    if (d->dtype != SS_F16 && d->dtype != SS_BF16 && d->dtype != SS_F32) return SS_ERR_INVALID_ARG;
    if (d->act != SS_ACT_NONE && d->act != SS_ACT_RELU && d->act != SS_ACT_GELU && d->act != SS_ACT_SILU) return SS_ERR_INVALID_ARG;
    if (!(d->eps >= 0.f) || std::isinf(d->eps) || images < 0 || pixels < 0) return SS_ERR_INVALID_ARG;
    if (d->channels > kMostChannels || pixels > kMostPixels || images > INT32_MAX || images * std::max<int64_t>(pixels, 1) > INT32_MAX) return SS_ERR_UNSUPPORTED;
    return SS_OK;
}

bool rows_ok(const ss_groupnorm_desc *d, const void *p, int64_t ld) { return p && aligned(p, d->dtype == SS_F32 ? 4 : 2) && ld >= d->channels; }

constexpr int kGroupPasses = 96;            // the test hook's id of the passes

// A workgroup's share of an image where it can be held; threads = 0: it cannot.
HeldShape held_shape(const ss_groupnorm_desc *d, long long images, long long pixels, bool backward)
{
    HeldShape h{};
    const int C = d->channels, cg = C / d->groups, item = d->dtype == SS_F32 ? 4 : 2, most_rows = held_most_rows(d->dtype);
    const long long cus = std::max(compute_units(), 1);
    if (C < 8 || forced_tile() == kGroupPasses) return h;
    // Bundles of 64 bytes of a pixel and more, whose widths are whole runs of eight channels where the groups allow it (`unit` of them together); narrower ones, and then, of little to hold, any,
    // where that gives fewer workgroups than compute units.  (Any, of much: gradient of 128 x 56 x 56 x 96 200 us, in passes 93.)
    int unit = 8;
    while (unit > 1 && cg * (unit / 2) % 8 == 0) unit /= 2;
    for (int k = 0; k < 6; k++) {
        const int segment = 64 >> k % 3, together = k < 3 ? unit : 1;
        HeldShape s{};
        s.groups = std::max(1, (segment + cg * item - 1) / (cg * item));
        s.groups = std::min(d->groups, (s.groups + together - 1) / together * together);
        s.width = s.groups * cg;
        s.bundles = (d->groups + s.groups - 1) / s.groups;
        s.lanes = (s.width + 7) / 8;
        for (int threads = 256; threads <= held_most_threads(backward); threads *= 2) {
            if (s.lanes > threads) continue;
            const int slots = threads / s.lanes;
            const long long rows = (pixels + slots - 1) / slots;
            if (rows > most_rows) continue;
            s.threads = threads;
            s.slots = slots;
            s.rows = (int)rows;
            if (rows <= 4 || images * s.bundles >= cus) break;
        }
        if (s.threads == 0 || (h.threads != 0 && s.bundles <= h.bundles) || (k >= 3 && pixels * s.width * item > 16 << 10)) continue;
        h = s;
        if (images * s.bundles >= cus) return h;
    }
    // Few workgroups with much to hold: the passes share it between more.  (8 images of 112 x 112 x 64, 64 workgroups of 200 KB, 30 us and 17; 2 of 32 x 32 x 640, 32 of
    // 80 KB, 12 and 15.)
    if (pixels * h.width * item > 96 << 10) h.threads = 0;
    return h;
}

struct GroupPlan {
    GroupArgs a;
    HeldShape held;
    size_t total_at, coef_at, stats_at, bytes;
};

// Chunks: as many as give each compute unit eight workgroups, of at least eight rows to the thread and 32 in all, so that what they leave is at most an eighth of the data; for a group of many
// channels, which one workgroup joins, so many that they leave it 128 values to the thread at most; but of at most 512 rows to the thread, which adds them in 32 bits.  (Of eight rows of 2048
// channels the joins took most of the time: one image of 112 x 112 x 2048 in bfloat16 264 us and its gradient 173, in chunks of 32 rows and joined by more threads 40 and 53; 64 x 64 x 1280 in one group
// 1813 and 230, 41 and 53.)
GroupPlan group_plan(const ss_groupnorm_desc *d, long long images, long long pixels, bool backward)
{
    GroupPlan g{};
    GroupArgs &a = g.a;
    const long long cus = std::max(compute_units(), 1);
    a.images = (int)images;
    a.pixels = (int)pixels;
    a.C = d->channels;
    a.groups = d->groups;
    a.cg = d->channels / d->groups;
    a.act = d->act;
    a.eps = d->eps;
    fast_div_setup((unsigned)a.cg, &a.cg_mul, &a.cg_sh);
    a.lanes = std::min((a.C + 7) / 8, kGroupThreads);
    a.tiles = ((a.C + 7) / 8 + a.lanes - 1) / a.lanes;
    a.slots = kGroupThreads / a.lanes;
    const long long want = 8 * cus / (images * a.tiles), most = pixels / std::max(8ll * a.slots, 32ll), least = pixels / (512ll * a.slots);
    const long long chunks = std::max({1ll, least, std::min({want, most, 128ll * kMostJoinThreads / a.cg})});
    a.per_chunk = (int)((pixels + chunks - 1) / chunks);
    a.chunks = (int)((pixels + a.per_chunk - 1) / a.per_chunk);
    const auto up = [](size_t bytes) { return (bytes + 255) / 256 * 256; };
    g.total_at = up((size_t)images * a.chunks * a.C * sizeof(float2));
    g.coef_at = g.total_at + (backward ? up((size_t)images * a.C * sizeof(float2)) : 0);
    g.stats_at = g.coef_at + (backward ? up((size_t)images * a.groups * sizeof(float2)) : 0);
    g.bytes = g.stats_at + (backward ? 0 : (size_t)images * a.groups * sizeof(float2));
    g.held = held_shape(d, images, pixels, backward);
    if (g.held.threads != 0) {                              // only the images' sums, of several images
        g.total_at = 0;
        g.bytes = backward && images > 1 ? (size_t)images * a.C * sizeof(float2) : 0;
    }
    return g;
}

// A call in pieces of images, so that no launch has 2^32 threads: f(arguments of a piece).
template <typename F>
int in_pieces(const GroupPlan &g, int item, F &&f)
{
    const GroupArgs &all = g.a;
    const long long threads = g.held.threads != 0 ? (long long)g.held.threads * g.held.bundles : std::max((long long)kGroupThreads * all.chunks * all.tiles, (long long)kMostJoinThreads * all.groups);
    const long long piece = std::max(1ll, (1ll << 31) / threads);
    for (long long at = 0; at < all.images; at += piece) {
        GroupArgs a = all;
        a.images = (int)std::min(piece, all.images - at);
        a.x += at * a.pixels * a.ldx * item;
        if (a.dy != nullptr) a.dy += at * a.pixels * a.lddy * item;
        a.out += at * a.pixels * a.ldout * item;
        if (a.stats != nullptr) a.stats += at * a.groups;
        if (a.part != nullptr) a.part += at * a.chunks * a.C;
        if (a.total != nullptr) a.total += at * a.C;
        if (a.coef != nullptr) a.coef += at * a.groups;
        const int st = f(a, piece >= all.images);
        if (st != SS_OK) return st;
    }
    return SS_OK;
}

int launch(const GroupArgs &a, int dtype, int stage, hipStream_t s)
{
    dtype == SS_F16 ? launch_group<SS_F16>(a, stage, s) : dtype == SS_BF16 ? launch_group<SS_BF16>(a, stage, s) : launch_group<SS_F32>(a, stage, s);
    return launched();
}

int launch(const GroupArgs &a, const HeldShape &h, int dtype, bool backward, hipStream_t s)
{
    return dtype == SS_F16 ? launch_held<SS_F16>(a, h, backward, s) : dtype == SS_BF16 ? launch_held<SS_BF16>(a, h, backward, s) : launch_held<SS_F32>(a, h, backward, s);
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_groupnorm_workspace_bytes(const ss_groupnorm_desc *d, int64_t images, int64_t pixels, int32_t backward, size_t *bytes)
{
    const int st = check_group(d, images, pixels);
    if (st != SS_OK) return st;
    if (!bytes || (backward != 0 && backward != 1)) return SS_ERR_INVALID_ARG;
    *bytes = images == 0 || pixels == 0 ? 0 : group_plan(d, images, pixels, backward != 0).bytes;
    return SS_OK;
}

extern "C" int ss_groupnorm_fwd(const ss_groupnorm_desc *d, const void *x, int64_t ldx, int64_t images, int64_t pixels, const float *w, const float *b, void *y, int64_t ldy,
                                float *stats, void *workspace, size_t ws_bytes, void *stream)
{
    const int st = check_group(d, images, pixels);
    if (st != SS_OK) return st;
    if (!aligned(w, 4) || !aligned(b, 4) || !aligned(stats, 8)) return SS_ERR_INVALID_ARG;
    if (images == 0 || pixels == 0) return SS_OK;
    if (!rows_ok(d, x, ldx) || !rows_ok(d, y, ldy)) return SS_ERR_INVALID_ARG;
    if (ldx > kMostPitch || ldy > kMostPitch) return SS_ERR_UNSUPPORTED;
    GroupPlan g = group_plan(d, images, pixels, false);
    if (g.bytes > 0 && (!workspace || !aligned(workspace, 16) || ws_bytes < g.bytes)) return SS_ERR_WORKSPACE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    char *const ws = static_cast<char *>(workspace);
    GroupArgs &a = g.a;
    a.x = static_cast<const char *>(x);
    a.ldx = ldx;
    a.out = static_cast<char *>(y);
    a.ldout = ldy;
    a.w = w;
    a.b = b;
    a.part = reinterpret_cast<float2 *>(ws);
    a.stats = reinterpret_cast<float2 *>(stats);
    const int item = d->dtype == SS_F32 ? 4 : 2;
    if (g.held.threads != 0) {
        a.part = nullptr;
        return in_pieces(g, item, [&](const GroupArgs &p, bool) { return launch(p, g.held, d->dtype, false, s); });
    }
    if (!stats) a.stats = reinterpret_cast<float2 *>(ws + g.stats_at);
    return in_pieces(g, item, [&](const GroupArgs &p, bool) {
        int done = launch(p, d->dtype, 0, s);
        if (done != SS_OK) return done;
        group_stats_kernel<<<dim3((unsigned)(p.images * p.groups)), dim3(join_threads(p)), 0, s>>>(p);
        done = launched();
        return done != SS_OK ? done : launch(p, d->dtype, 1, s);
    });
}

extern "C" int ss_groupnorm_bwd(const ss_groupnorm_desc *d, const void *dy, int64_t lddy, const void *x, int64_t ldx, int64_t images, int64_t pixels, const float *stats,
                                const float *w, const float *b, void *dx, int64_t lddx, float *dw, float *db, void *workspace, size_t ws_bytes, void *stream)
{
    const int st = check_group(d, images, pixels);
    if (st != SS_OK) return st;
    if (!aligned(w, 4) || !aligned(b, 4) || !aligned(dw, 4) || !aligned(db, 4) || !aligned(stats, 8)) return SS_ERR_INVALID_ARG;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    GroupPlan g = group_plan(d, std::max<int64_t>(images, 1), std::max<int64_t>(pixels, 1), true);
    GroupArgs &a = g.a;
    a.dw = dw;
    a.db = db;
    const auto vectors = [&] {
        if (!dw && !db) return (int)SS_OK;
        const dim3 grid((unsigned)((a.C + 15) / 16));
        if (a.images < kManyImages)
            group_vectors_kernel<16><<<grid, dim3(256), 0, s>>>(a);
        else
            group_vectors_kernel<64><<<grid, dim3(1024), 0, s>>>(a);
        return launched();
    };
    if (images == 0 || pixels == 0) {                       // sums over nothing
        a.images = 0;
        return vectors();
    }
    if (!stats || !rows_ok(d, x, ldx) || !rows_ok(d, dy, lddy) || !rows_ok(d, dx, lddx)) return SS_ERR_INVALID_ARG;
    if (std::max({ldx, lddy, lddx}) > kMostPitch) return SS_ERR_UNSUPPORTED;
    if (g.bytes > 0 && (!workspace || !aligned(workspace, 16) || ws_bytes < g.bytes)) return SS_ERR_WORKSPACE;
    char *const ws = static_cast<char *>(workspace);
    a.x = static_cast<const char *>(x);
    a.ldx = ldx;
    a.dy = static_cast<const char *>(dy);
    a.lddy = lddy;
    a.out = static_cast<char *>(dx);
    a.ldout = lddx;
    a.w = w;
    a.b = b;
    a.stats = reinterpret_cast<float2 *>(const_cast<float *>(stats));
    const int item = d->dtype == SS_F32 ? 4 : 2;
    if (g.held.threads != 0) {
        if (images > 1) a.total = reinterpret_cast<float2 *>(ws + g.total_at);
        const int held = in_pieces(g, item, [&](const GroupArgs &p, bool) { return launch(p, g.held, d->dtype, true, s); });
        return held != SS_OK || images == 1 ? held : vectors();
    }
    a.part = reinterpret_cast<float2 *>(ws);
    a.total = reinterpret_cast<float2 *>(ws + g.total_at);
    a.coef = reinterpret_cast<float2 *>(ws + g.coef_at);
    bool joined = false;
    const int done = in_pieces(g, item, [&](GroupArgs &p, bool only) {
        int done = launch(p, d->dtype, 2, s);
        if (done != SS_OK) return done;
        group_coef_kernel<<<dim3((unsigned)(p.images * p.groups)), dim3(join_threads(p)), 0, s>>>(p);
        done = launched();
        if (done != SS_OK) return done;
        joined = only;
        if (!only) p.dw = p.db = nullptr;                  // (all pieces' sums, behind the last)
        return launch(p, d->dtype, 3, s);
    });
    return done != SS_OK || joined ? done : vectors();
}
