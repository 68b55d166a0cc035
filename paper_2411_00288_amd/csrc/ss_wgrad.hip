// Gradient of a pointwise (1x1) or linear layer's weights and bias:  dw[o][c] = sum_r dy[r][o] x[r][c],  db[o] = sum_r dy[r][o].
//
// The matrix instruction wants eight consecutive rows of a column side by side, and the rows lie with their channels side by side.  A thread loads eight rows of
// eight channels and turns them in registers: a word of the result takes one half from each of two rows (32 byte permutations for 64 values, and no
// row is read twice).  The eight columns are eight operands of the instruction, which go to LDS as they are, column e of all threads side by side, so that writes and
// reads meet no bank twice; the output's rows and columns come out in that order and are put right when they are stored.
//
// The sum over the rows is shared by as many workgroups as fill the chip, each of which leaves its part in 32 bits in the workspace; a second kernel adds them in
// their order, so that the same call gives the same bits.
//
// 96 -> 384 over 401408 rows 88 us (385 MB: 83 at 4.6 TB/s, and 6 for the parts), 1024 -> 256 over 12544 26 (a chunk's latencies and 28 MB of parts), 8192 -> 8192 over 8192 1090 (1.0
// PFLOP/s; 96 KB through LDS to a chunk).  Sums in 32 bits from 16-bit operands, whatever the forward pass multiplies: inside the 8-bit instruction eight products keep 13 bits.
#include "ss_mx4.h"
#include "ss_conv_params.h"
#include <type_traits>

namespace ss {
namespace {

constexpr int64_t kMostPitch = 1 << 23;    // (128 rows of it are 2^31 bytes)

// The kernels, by the ids of the test hook: tiles of 64 x 64, 128 x 128 and 256 x 256.
enum { WGRAD_64 = 90, WGRAD_128, WGRAD_256 };

struct WgradArgs {
    const uint16_t *dy, *x;
    float *sums;                           // [part][cout][cin]
    float *columns;                        // [part][cout], or NULL
    long long lddy, ldx, rows, per_part;
    int cout, cin, tiles_o, tiles_c, parts;
};

template <int DT>
__device__ __forceinline__ f32x16 mma16(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    if constexpr (DT == SS_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// sum + both halves of a word
template <int DT>
__device__ __forceinline__ float add_pair(uint32_t word, float sum)
{
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if constexpr (DT == SS_F16)
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, word), f16x2{1, 1}, sum, false);
    else
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, word), bf16x2{1, 1}, sum, false);
}

// Four waves of M x M tiles of 32 x 32, two by two: B = 64 M output and input channels, chunks of 128 / M rows, of which a thread of the first two waves holds
// 8 x 8 of dy, one of the others 8 x 8 of x.  WIDE: both have at least 8 channels.
template <int DT, int M, bool WIDE>
__global__ __launch_bounds__(256, M >= 4 ? 1 : 2) void wgrad_kernel(WgradArgs p)
{
    constexpr int B = 64 * M, KC = 128 / M, KG = KC / 8, CB = B / 8;
    __shared__ __attribute__((aligned(16))) u32x4 block_s[2][2][KG * B];       // [buffer][dy, x][eight rows][place]
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    // An XCD (workgroups b, b + 8, ...) makes neighbouring tiles of a part, whose rows it then has in its L2, in bands of eight tiles of output channels.
    const int tiles = p.tiles_o * p.tiles_c, total_tiles = tiles * p.parts, xcd = blockIdx.x % 8;
    const int id = xcd * (total_tiles / 8) + min(xcd, total_tiles % 8) + blockIdx.x / 8;
    const int part = id / tiles, tile = id - part * tiles, band = tile / (8 * p.tiles_c), high = min(8, p.tiles_o - band * 8), in_band = tile - band * 8 * p.tiles_c;
    const int o0 = (band * 8 + in_band % high) * B, c0 = in_band / high * B;
    const long long first = part * p.per_part, last = min(p.rows, first + p.per_part);

    // this thread's block
    const int which = wave / 2, cb = tid % 128 % CB, kg = tid % 128 / CB, cols = which ? p.cin : p.cout, col = (which ? c0 : o0) + cb * 8;
    const long long ld = which ? p.ldx : p.lddy;
    const uint16_t *const src = which ? p.x : p.dy;
    const bool inside = col < cols;
    const bool add_columns = p.columns != nullptr && which == 0 && c0 == 0;    // uniform
    Run<DT> even_v[8], odd_v[8];
    float total[8] = {};
    const unsigned column = (unsigned)min(col, cols - 8) * 2, lane_at = (unsigned)(kg * 8) * (unsigned)ld * 2 + column;
    const auto load = [&](long long at, Run<DT> (&v)[8]) {
        if constexpr (WIDE) {
            const long long from = min(at, last - 1);      // (past the last: its last row again)
            const int there = (int)min((long long)KC, last - from);
            const char *const origin = reinterpret_cast<const char *>(src + from * ld);
            if (there == KC) {                              // uniform
#pragma unroll
                for (int u = 0; u < 8; u++) v[u].v[0] = reinterpret_cast<const Vec16 *>(origin + u * ld * 2 + lane_at)->v;
            } else {
#pragma unroll
                for (int u = 0; u < 8; u++) v[u].v[0] = reinterpret_cast<const Vec16 *>(origin + ((unsigned)min(kg * 8 + u, there - 1) * (unsigned)ld * 2 + column))->v;
            }
        } else {
#pragma unroll
            for (int u = 0; u < 8; u++) {
                const long long row = at + kg * 8 + u;
                v[u] = load_run<DT>(src + row * ld + col, row < last ? cols - col : 0);
            }
        }
    };
    const auto put = [&](long long at, Run<DT> (&v)[8], int buffer) {
        if constexpr (WIDE) {
            if (at + KC > last || !inside || col + 8 > cols)
#pragma unroll
                for (int u = 0; u < 8; u++) place_wide<DT>(v[u], col, cols, at + kg * 8 + u < last && inside);
        }
#pragma unroll
        for (int e = 0; e < 8; e++) {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint32_t low = v[2 * j].v[0][e / 2], high = v[2 * j + 1].v[0][e / 2];
                w[j] = __builtin_amdgcn_perm(high, low, e % 2 ? 0x07060302u : 0x05040100u);
            }
            block_s[buffer][which][kg * B + e * CB + cb] = w;
            if (add_columns)
#pragma unroll
                for (int j = 0; j < 4; j++) total[e] = add_pair<DT>(w[j], total[e]);
        }
    };
    f32x16 acc[M][M] = {};
    // Two chunks are on their way while one is multiplied.  Past the last their last row comes again, and zeros are multiplied: with a branch around the loads, or around their
    // use, a load waits for the ones before it.
    const auto chunk = [&](long long at, Run<DT> (&next)[8], Run<DT> (&after)[8], auto buffer) {
        constexpr int N = decltype(buffer)::value;
        lds_barrier();
        load(at + 2 * KC, after);
        __builtin_amdgcn_sched_barrier(0);                  // (the compiler moves them behind the products)
        u32x4 a[2][M], b[2][M];
        const auto operands = [&](int s) {
            const int from = (2 * s + lane / 32) * B + lane % 32;
#pragma unroll
            for (int i = 0; i < M; i++) {
                a[s % 2][i] = block_s[N][0][from + (wave / 2 * M + i) * 32];
                b[s % 2][i] = block_s[N][1][from + (wave % 2 * M + i) * 32];
            }
        };
        operands(0);
        put(at + KC, next, N ^ 1);                          // (zeros past the last)
#pragma unroll
        for (int s = 0; s < KC / 16; s++) {
            if (s + 1 < KC / 16) operands(s + 1);
#pragma unroll
            for (int i = 0; i < M; i++)
#pragma unroll
                for (int j = 0; j < M; j++) acc[i][j] = mma16<DT>(a[s % 2][i], b[s % 2][j], acc[i][j]);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * M, 0);                 // the first operands, and then, between two matrix instructions each, some of the others
#pragma unroll
        for (int i = 0; i < M * M * KC / 16; i++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
        }
    };
    load(first, even_v);
    load(first + KC, odd_v);
    put(first, even_v, 0);
    for (long long at = first; at < last; at += 2 * KC) {
        chunk(at, odd_v, even_v, std::integral_constant<int, 0>{});
        chunk(at + KC, even_v, odd_v, std::integral_constant<int, 1>{});
    }
    // The tile's sums leave by LDS, 64 rows at a time, so that a store writes neighbouring channels of a row.
    constexpr int PAD = M < 4 ? 1 : 0, PITCH = 8 * (CB + PAD);
    float *const out = p.sums + (long long)part * p.cout * p.cin, *const sums_s = reinterpret_cast<float *>(block_s);
#pragma unroll
    for (int i = 0; i < M; i++) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < M; j++) {
            const int place = (wave % 2 * M + j) * 32 + lane % 32;
#pragma unroll
            for (int e = 0; e < 16; e++)
                sums_s[(wave / 2 * 32 + 8 * (e / 4) + 4 * (lane / 32) + e % 4) * PITCH + place / CB * (CB + PAD) + place % CB] = acc[i][j][e];
        }
        __syncthreads();
        constexpr int ROWS = 1024 / B;                      // rows at a time, four channels to the thread
        const int c = tid % (B / 4) * 4, left = p.cin - c0 - c;
        const float *const from = sums_s + c % 8 * (CB + PAD) + c / 8;
#pragma unroll
        for (int k = 0; k < 64 / ROWS; k++) {
            const int row = k * ROWS + tid / (B / 4), place = (row / 32 * M + i) * 32 + row % 32, o = o0 + place % CB * 8 + place / CB;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = from[row * PITCH + e * (CB + PAD)];
            if (o >= p.cout) continue;
            float *const to = out + (long long)o * p.cin + c0 + c;
            if (left >= 4)
                reinterpret_cast<Vec32 *>(to)->v = __builtin_bit_cast(u32x4, v);
            else
#pragma unroll
                for (int e = 0; e < 3; e++)
                    if (e < left) to[e] = v[e];
        }
    }
    if (p.columns == nullptr || c0 != 0) return;            // uniform
    __syncthreads();
    float *const column_s = reinterpret_cast<float *>(block_s);                // [eight rows][channel]
    if (which == 0)
#pragma unroll
        for (int e = 0; e < 8; e++) column_s[kg * B + cb * 8 + e] = total[e];
    __syncthreads();
    for (int o = tid; o < B && o0 + o < p.cout; o += 256) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < KG; k++) s += column_s[k * B + o];
        p.columns[(long long)part * p.cout + o0 + o] = s;
    }
}

struct JoinArgs {
    const float *sums, *columns;
    float *dw, *db;
    long long n;                           // elements of dw
    int parts, cout;
    unsigned blocks;                       // workgroups of dw
};

// The parts, added in a fixed order: four of a row's values to the thread and, of many parts, 16 slices of them, joined in LDS.  Behind those workgroups the bias's, 16 columns to the
// workgroup and 16 slices.
template <bool MANY>
__global__ __launch_bounds__(256) void wgrad_join_kernel(JoinArgs p)
{
    __shared__ f32x4 s[16][17];
    const int c = threadIdx.x % 16, slice = threadIdx.x / 16;
    if (blockIdx.x < p.blocks) {
        const long long i = MANY ? ((long long)blockIdx.x * 16 + c) * 4 : ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
        const int n = (int)min(4ll, p.n - i);
        const bool whole = p.n % 4 == 0;
        f32x4 v = {};
        if (n > 0) {
            if (whole) {
#pragma unroll 8
                for (int k = MANY ? slice : 0; k < p.parts; k += MANY ? 16 : 1) v += *reinterpret_cast<const f32x4 *>(p.sums + k * p.n + i);
            } else {
                for (int k = MANY ? slice : 0; k < p.parts; k += MANY ? 16 : 1)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (e < n) v[e] += p.sums[k * p.n + i + e];
            }
        }
        if constexpr (MANY) {
            s[slice][c] = v;
            __syncthreads();
            if (slice != 0) return;
            v = f32x4{};
#pragma unroll
            for (int k = 0; k < 16; k++) v += s[k][c];
        }
        if (n == 4)
            reinterpret_cast<Vec32 *>(p.dw + i)->v = __builtin_bit_cast(u32x4, v);
        else
            for (int e = 0; e < n; e++) p.dw[i + e] = v[e];
        return;
    }
    const int col = (int)(blockIdx.x - p.blocks) * 16 + c;
    float v = 0.f;
    if (col < p.cout)
#pragma unroll 4
        for (int k = slice; k < p.parts; k += 16) v += p.columns[(long long)k * p.cout + col];
    s[slice][c][0] = v;
    __syncthreads();
    if (slice != 0 || col >= p.cout) return;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 16; k++) sum += s[k][c][0];
    p.db[col] = sum;
}

struct WgradPlan {
    int m, parts;                          // tiles of a wave in each direction
    long long per_part;
    size_t columns_at, bytes;              // (the parts' sums stand first, where there are several)
};

// Tiles of 256 x 256 for matrices of two of them to the compute unit (8192 -> 8192 over 8192 rows 1090 us, in tiles of 128 x 128 1290; 4096 -> 4096 320 and 310), of 64 x 64 for narrow
// ones (64 -> 256 over 200704 rows 33 us, in tiles of 128 x 128 40) and short sums (1024 -> 1024 over 2048 rows 21 and 25, 300 -> 77 over 1000 11 and 18; 1024 ->
// 256 over 12544 27 and 27; 96 -> 384 over 401408 143 and 87).  Parts of at least 256 rows, until two workgroups of each compute unit, one of the largest tiles, have
// work (512 -> 128 over 50176 rows in tiles of 64 x 64, 128, 256, 512 and 1024 workgroups: 50, 31, 27 and 32 us).
WgradPlan wgrad_plan(const ss_weight_desc *d, long long rows)
{
    WgradPlan w{};
    const long long cus = std::max(compute_units(), 1);
    const auto tiles = [&](int b) { return (long long)((d->cout + b - 1) / b) * ((d->cin + b - 1) / b); };
    const int forced = forced_tile();
    w.m = tiles(256) >= 2 * cus ? 4 : std::min(d->cout, d->cin) <= 64 || tiles(128) * ((rows + 63) / 64) <= 8 * cus ? 1 : 2;
    if (forced >= WGRAD_64 && forced <= WGRAD_256) w.m = 1 << (forced - WGRAD_64);
    const long long t = tiles(64 * w.m), chunk = 128 / w.m;
    const long long want = forced_split() > 0 ? forced_split() : std::max(1ll, std::min((w.m == 4 ? 1 : 2) * cus / t, rows / 256));
    w.per_part = ((rows + want - 1) / want + chunk - 1) / chunk * chunk;
    w.parts = (int)((rows + w.per_part - 1) / w.per_part);
    w.columns_at = w.parts > 1 ? ((size_t)w.parts * d->cout * d->cin * 4 + 255) / 256 * 256 : 0;
    w.bytes = w.columns_at + (size_t)w.parts * d->cout * 4;
    return w;
}

int check_wgrad(const ss_weight_desc *d, int64_t rows)
{
    const int st = check_desc(d, false);
    if (st != SS_OK) return st;
    if (d->kh != 1 || d->kw != 1 || is_byte_type(d->dtype)) return SS_ERR_UNSUPPORTED;
    if (rows < 0) return SS_ERR_INVALID_ARG;
    return rows <= INT32_MAX ? SS_OK : SS_ERR_UNSUPPORTED;
}

template <int DT>
int launch_wgrad(const WgradArgs &a, int m, hipStream_t s)
{
    const long long blocks = (long long)a.parts * a.tiles_o * a.tiles_c;
    if (blocks > 0xFFFFFFll) return SS_ERR_UNSUPPORTED;
    const auto go = [&](auto kern) { kern<<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a); };
    const auto pick = [&](auto wide) {
        constexpr bool WIDE = decltype(wide)::value;
        m == 1 ? go(wgrad_kernel<DT, 1, WIDE>) : m == 2 ? go(wgrad_kernel<DT, 2, WIDE>) : go(wgrad_kernel<DT, 4, WIDE>);
    };
    a.cout >= 8 && a.cin >= 8 ? pick(std::true_type{}) : pick(std::false_type{});
    return launched();
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_pw_wgrad_workspace_bytes(const ss_weight_desc *desc, int64_t rows, size_t *bytes)
{
    const int st = check_wgrad(desc, rows);
    if (st != SS_OK) return st;
    if (!bytes) return SS_ERR_INVALID_ARG;
    *bytes = rows > 0 ? wgrad_plan(desc, rows).bytes : 0;
    return SS_OK;
}

extern "C" int ss_pw_wgrad(const ss_weight_desc *desc, const void *dy, int64_t lddy, const void *x, int64_t ldx, int64_t rows, float *dw, float *db, void *workspace,
                           size_t ws_bytes, void *stream)
{
    int st = check_wgrad(desc, rows);
    if (st != SS_OK) return st;
    if (!dw || !aligned(dw, 4) || !aligned(db, 4)) return SS_ERR_INVALID_ARG;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    JoinArgs j{};
    j.dw = dw;
    j.db = db;
    j.n = (long long)desc->cout * desc->cin;
    j.cout = desc->cout;
    const auto join = [&](bool weights) {
        const bool many = j.parts >= 16 && j.n <= 1 << 28;     // (a thread to 64 / 256 of a value: fewer than 2^32)
        j.blocks = weights ? (unsigned)((j.n + (many ? 63 : 1023)) / (many ? 64 : 1024)) : 0u;
        const unsigned grid = j.blocks + (db ? (unsigned)((desc->cout + 15) / 16) : 0u);
        if (grid == 0) return (int)SS_OK;
        if (many)
            wgrad_join_kernel<true><<<dim3(grid), dim3(256), 0, s>>>(j);
        else
            wgrad_join_kernel<false><<<dim3(grid), dim3(256), 0, s>>>(j);
        return launched();
    };
    if (rows == 0) return join(true);                       // sums over no rows
    if (lddy < desc->cout || ldx < desc->cin) return SS_ERR_INVALID_ARG;
    if (lddy > kMostPitch || ldx > kMostPitch) return SS_ERR_UNSUPPORTED;
    if (!dy || !x || !aligned(dy, 2) || !aligned(x, 2)) return SS_ERR_INVALID_ARG;
    const WgradPlan w = wgrad_plan(desc, rows);
    if (!workspace || !aligned(workspace, 16) || ws_bytes < w.bytes) return SS_ERR_WORKSPACE;
    WgradArgs a{};
    a.dy = static_cast<const uint16_t *>(dy);
    a.x = static_cast<const uint16_t *>(x);
    a.sums = w.parts > 1 ? static_cast<float *>(workspace) : dw;
    a.columns = db ? reinterpret_cast<float *>(static_cast<char *>(workspace) + w.columns_at) : nullptr;
    a.lddy = lddy;
    a.ldx = ldx;
    a.rows = rows;
    a.per_part = w.per_part;
    a.cout = desc->cout;
    a.cin = desc->cin;
    a.tiles_o = (desc->cout + 64 * w.m - 1) / (64 * w.m);
    a.tiles_c = (desc->cin + 64 * w.m - 1) / (64 * w.m);
    a.parts = w.parts;
    st = desc->dtype == SS_F16 ? launch_wgrad<SS_F16>(a, w.m, s) : launch_wgrad<SS_BF16>(a, w.m, s);
    if (st != SS_OK) return st;
    j.sums = a.sums;
    j.columns = a.columns;
    j.parts = w.parts;
    return w.parts > 1 || db ? join(w.parts > 1) : SS_OK;
}
