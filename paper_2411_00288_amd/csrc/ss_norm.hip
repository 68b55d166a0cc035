// Norms before and after a block, fused with its gate, its residual scale and the residual sum; and their gradient.
//
//     u = post(h)            x_out = x + scale * gate * u            y = norm(x_out) * w + b
//
// post and norm: none, LayerNorm or RMS over the channels of a row.  A row lives in the registers of `LPR` lanes, 8 channels to the lane (NV runs of
// 8 in the widest rows), from its only read to its only write; means and sums of squares are fp32, the variance is the mean square of the
// differences from the mean.  Bound by memory.
#include "ss_mx4.h"
#include "ss_conv_params.h"
#include <algorithm>
#include <cmath>

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

// v becomes its normalised row; the factor is returned.  Places past the row stay zero.
template <int LPR, int NV>
__device__ __forceinline__ float normalise(float (&v)[NV][8], const int (&n)[NV], int cols, bool layer, float eps, float (*shared)[2][LPR / 64 > 0 ? LPR / 64 : 1],
                                           int &turn)
{
    if (layer) {
        float s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) s[0] += v[j][e];
        row_sums<LPR>(s, shared, turn);
        const float mean = s[0] / (float)cols;
#pragma unroll
        for (int j = 0; j < NV; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = e < n[j] ? v[j][e] - mean : 0.f;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < 8; e++) s[0] = __builtin_fmaf(v[j][e], v[j][e], s[0]);
    row_sums<LPR>(s, shared, turn);
    const float r = 1.f / sqrtf(s[0] / (float)cols + eps);
#pragma unroll
    for (int j = 0; j < NV; j++)
#pragma unroll
        for (int e = 0; e < 8; e++) v[j][e] = e < n[j] ? v[j][e] * r : 0.f;
    return r;
}

// A vector of the channels, or `fill` where there is none.
template <int NV>
__device__ __forceinline__ void channel_vector(const float *p, const int (&c)[NV], int cols, float fill, float (&v)[NV][8])
{
#pragma unroll
    for (int j = 0; j < NV; j++) {
        if (p != nullptr)
            load8<SS_F32>(p + c[j], cols - c[j], v[j]);
        else
#pragma unroll
            for (int e = 0; e < 8; e++) v[j][e] = fill;
    }
}

template <int DT, int LPR, int NV, bool MX4>
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
    float w[NV][8], b[NV][8], scale[NV][8], post_w[NV][8], post_b[NV][8];
    channel_vector<NV>(p.w, c, p.cols, 1.f, w);
    channel_vector<NV>(p.b, c, p.cols, 0.f, b);
    channel_vector<NV>(p.scale, c, p.cols, 1.f, scale);
    channel_vector<NV>(p.post_w, c, p.cols, 1.f, post_w);
    channel_vector<NV>(p.post_b, c, p.cols, 0.f, post_b);
    for (long long base = (long long)blockIdx.x * R; base < p.rows; base += (long long)gridDim.x * R) {
        const long long row = base + threadIdx.x / LPR;
        int n[NV];
        float v[NV][8];
#pragma unroll
        for (int j = 0; j < NV; j++) {
            n[j] = row < p.rows ? p.cols - c[j] : 0;
            load8<DT>(p.x + (row * p.ldx + c[j]) * B, n[j], v[j]);
        }
        if (p.h != nullptr) {
            float u[NV][8];
#pragma unroll
            for (int j = 0; j < NV; j++) load8<DT>(p.h + (row * p.ldh + c[j]) * B, n[j], u[j]);
            float gate[NV][8];
            const long long g = (long long)(((unsigned long long)(unsigned)row * p.g_mul) >> p.g_sh);
#pragma unroll
            for (int j = 0; j < NV; j++) {
                if (p.gate_cols > 1 || p.cols == 1) {
                    if (p.gate != nullptr) load8<DT>(p.gate + (g * p.gate_cols + c[j]) * B, n[j], gate[j]);
                } else if (p.gate != nullptr) {
                    const float one = n[j] > 0 ? load1<DT>(p.gate + g * B) : 0.f;
#pragma unroll
                    for (int e = 0; e < 8; e++) gate[j][e] = one;
                }
            }
            if (p.post != SS_NORM_NONE) {
                normalise<LPR, NV>(u, n, p.cols, p.post == SS_NORM_LAYER, p.post_eps, shared, turn);
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) u[j][e] = __builtin_fmaf(u[j][e], post_w[j][e], post_b[j][e]);
            }
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    float s = u[j][e] * scale[j][e];
                    if (p.gate != nullptr) s *= gate[j][e];
                    v[j][e] = e < n[j] ? v[j][e] + s : 0.f;
                }
#pragma unroll
            for (int j = 0; j < NV; j++) store8<DT>(p.x_out + (row * p.ldx_out + c[j]) * B, n[j], v[j]);
        }
        if (p.norm == SS_NORM_NONE) continue;
        normalise<LPR, NV>(v, n, p.cols, p.norm == SS_NORM_LAYER, p.eps, shared, turn);
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
enum { ACC_W = 0, ACC_B, ACC_SCALE, ACC_POST_W, ACC_POST_B, ACC_COUNT };

template <int DT, int LPR, int NV, bool POST>
__global__ __launch_bounds__(LPR < 256 ? 256 : LPR) void norm_grad_kernel(NormGradArgs p)
{
    constexpr int THREADS = LPR < 256 ? 256 : LPR, R = THREADS / LPR;
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
    const bool vector_gate = p.gate != nullptr && (p.gate_cols > 1 || p.cols == 1);

    // sums of the row groups' registers, to dst[0 .. cols)
    auto join = [&](const float (&v)[NV][8], auto &&put) {
        if constexpr (R == 1) {
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (c[j] + e < p.cols) put(c[j] + e, v[j][e]);
        } else {
            static_assert(NV == 1, "one run to the lane");
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; e++) joined[rg * LPR * 8 + c[0] + e] = v[0][e];
            __syncthreads();
            for (int col = threadIdx.x; col < p.cols; col += THREADS) {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < R; k++) s += joined[k * LPR * 8 + col];
                put(col, s);
            }
        }
    };

    const long long units = (long long)p.groups * p.strips;
    const long long u0 = units * blockIdx.x / gridDim.x, u1 = units * (blockIdx.x + 1) / gridDim.x;
    for (long long unit = u0; unit < u1; unit++) {
        const long long group = unit / p.strips, strip = unit - group * p.strips;
        const long long first = group * p.per_group + strip * p.per_strip;
        const long long last = group * p.per_group + min((long long)p.per_group, (strip + 1) * p.per_strip);
        float gate_acc[NV][8] = {}, gate_one = 0.f;
        for (long long base = first; base < last; base += R) {
            const long long row = base + rg;
            const bool in = row < last;
            int n[NV];
            float t[NV][8] = {};
#pragma unroll
            for (int j = 0; j < NV; j++) n[j] = in ? p.cols - c[j] : 0;
            if (p.norm != SS_NORM_NONE) {
                float v[NV][8], w[NV][8];
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    load8<DT>(p.x_out + (row * p.ldx_out + c[j]) * B, n[j], v[j]);
                    load8<DT>(p.dy + (row * p.lddy + c[j]) * B, n[j], t[j]);
                }
                channel_vector<NV>(p.w, c, p.cols, 1.f, w);
                const bool layer = p.norm == SS_NORM_LAYER;
                float r = normalise<LPR, NV>(v, n, p.cols, layer, p.eps, shared, turn);
                float s[2] = {0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float dy = e < n[j] ? t[j][e] : 0.f, xh = e < n[j] ? v[j][e] : 0.f;
                        acc[ACC_W][j][e] = __builtin_fmaf(dy, xh, acc[ACC_W][j][e]);
                        acc[ACC_B][j][e] += dy;
                        const float g = e < n[j] ? dy * w[j][e] : 0.f;
                        t[j][e] = g;
                        s[0] += g;
                        s[1] = __builtin_fmaf(g, xh, s[1]);
                    }
                row_sums<LPR>(s, shared, turn);
                const float m0 = layer ? s[0] * inv : 0.f, m1 = s[1] * inv;
#pragma unroll
                for (int j = 0; j < NV; j++)
#pragma unroll
                    for (int e = 0; e < 8; e++) t[j][e] = e < n[j] ? r * (t[j][e] - m0 - v[j][e] * m1) : 0.f;
            }
            if (p.dx_out != nullptr) {
                float d[NV][8];
#pragma unroll
                for (int j = 0; j < NV; j++) {
                    load8<DT>(p.dx_out + (row * p.lddx_out + c[j]) * B, n[j], d[j]);
#pragma unroll
                    for (int e = 0; e < 8; e++) t[j][e] += d[j][e];
                }
            }
#pragma unroll
            for (int j = 0; j < NV; j++) store8<DT>(p.dx + (row * p.lddx + c[j]) * B, n[j], t[j]);
            if (p.h == nullptr) continue;

            float hh[NV][8], scale[NV][8], gate[NV][8];
            float hr = 0.f;
#pragma unroll
            for (int j = 0; j < NV; j++) load8<DT>(p.h + (row * p.ldh + c[j]) * B, n[j], hh[j]);
            channel_vector<NV>(p.scale, c, p.cols, 1.f, scale);
            const long long g = p.grouped ? group : row;
#pragma unroll
            for (int j = 0; j < NV; j++) {
                if (vector_gate) {
                    load8<DT>(p.gate + (g * p.gate_cols + c[j]) * B, n[j], gate[j]);
                } else {
                    const float one = p.gate != nullptr && n[j] > 0 ? load1<DT>(p.gate + g * B) : 1.f;
#pragma unroll
                    for (int e = 0; e < 8; e++) gate[j][e] = one;
                }
            }
            float post_w[NV][8], post_b[NV][8];
            if constexpr (POST) {
                channel_vector<NV>(p.post_w, c, p.cols, 1.f, post_w);
                channel_vector<NV>(p.post_b, c, p.cols, 0.f, post_b);
                hr = normalise<LPR, NV>(hh, n, p.cols, p.post == SS_NORM_LAYER, p.post_eps, shared, turn);
            }
            float dg[NV][8], s[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NV; j++)
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const bool valid = e < n[j];
                    const float u = POST ? __builtin_fmaf(hh[j][e], post_w[j][e], post_b[j][e]) : hh[j][e];
                    const float tu = valid ? t[j][e] * u : 0.f;
                    acc[ACC_SCALE][j][e] += valid ? tu * gate[j][e] : 0.f;
                    dg[j][e] = valid ? tu * scale[j][e] : 0.f;
                    const float du = valid ? t[j][e] * scale[j][e] * gate[j][e] : 0.f;
                    if constexpr (POST) {
                        acc[ACC_POST_W][j][e] = __builtin_fmaf(du, hh[j][e], acc[ACC_POST_W][j][e]);
                        acc[ACC_POST_B][j][e] += du;
                        const float gg = valid ? du * post_w[j][e] : 0.f;
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
                    for (int e = 0; e < 8; e++) t[j][e] = hr * (t[j][e] - m0 - hh[j][e] * m1);
            }
#pragma unroll
            for (int j = 0; j < NV; j++) store8<DT>(p.dh + (row * p.lddh + c[j]) * B, n[j], t[j]);
            if (p.gate != nullptr) {
                if (p.grouped) {
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            if (vector_gate) gate_acc[j][e] += dg[j][e];
                            else gate_one += dg[j][e];
                        }
                } else if (vector_gate) {
#pragma unroll
                    for (int j = 0; j < NV; j++) store8<DT>(p.dgate + (row * p.gate_cols + c[j]) * B, n[j], dg[j]);
                } else {
                    float one[1] = {0.f};
#pragma unroll
                    for (int j = 0; j < NV; j++)
#pragma unroll
                        for (int e = 0; e < 8; e++) one[0] += dg[j][e];
                    row_sums<LPR>(one, shared, turn);
                    if (in && lane == 0) store1<DT>(p.dgate + row * B, one[0]);
                }
            }
        }
        if (p.grouped && p.gate != nullptr) {
            auto put = [&](int col, float v) {
                if (p.strips > 1)
                    p.gate_part[unit * p.gate_cols + col] = v;
                else
                    store1<DT>(p.dgate + (group * p.gate_cols + col) * B, v);
            };
            if (vector_gate) {
                join(gate_acc, put);
            } else {
                gate_one = lanes_sum<64>(gate_one);
                __syncthreads();
                if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = gate_one;
                __syncthreads();
                float s = 0.f;
                for (int k = 0; k < THREADS / 64; k++) s += waves[k];
                if (threadIdx.x == 0) put(0, s);
            }
        }
    }
    const size_t at = (size_t)blockIdx.x * p.cols, step = (size_t)gridDim.x * p.cols;
    auto part = [&](int a, const float (&v)[NV][8]) { join(v, [&](int col, float s) { p.part[a * step + at + col] = s; }); };
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
    float *out[ACC_COUNT];
    char *dgate;
    int cols, parts, strips, column_tiles;
    long long gates;                       // elements of the gate's gradient that are still in `strips` parts, or 0
    int gate_cols;
};

// 16 columns to the workgroup, 64 slices of the partial sums; behind those workgroups, one thread for an element of the gate's gradient.
template <int DT>
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(NormSumArgs p)
{
    __shared__ float s[64][17];
    const int tiles = p.column_tiles * ACC_COUNT;
    if ((int)blockIdx.x < tiles) {
        const int a = blockIdx.x / p.column_tiles, col = (blockIdx.x - a * p.column_tiles) * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
        if (p.out[a] == nullptr) return;                 // uniform
        float v = 0.f;
        if (col < p.cols) {
            const float *src = p.part + (size_t)a * p.parts * p.cols + col;
#pragma unroll 8
            for (int i = slice; i < p.parts; i += 64) v += src[(size_t)i * p.cols];
        }
        s[slice][threadIdx.x % 16] = v;
        __syncthreads();
        for (int half = 32; half > 0; half >>= 1) {
            if (slice < half) s[slice][threadIdx.x % 16] += s[slice + half][threadIdx.x % 16];
            __syncthreads();
        }
        if (slice == 0 && col < p.cols) p.out[a][col] = s[0][threadIdx.x];
        return;
    }
    const long long i = (long long)(blockIdx.x - tiles) * 1024 + threadIdx.x;
    if (i >= p.gates) return;
    const long long group = i / p.gate_cols, col = i - group * p.gate_cols;
    const float *src = p.gate_part + group * p.strips * p.gate_cols + col;
    float v = 0.f;
    for (int k = 0; k < p.strips; k++) v += src[(long long)k * p.gate_cols];
    store1<DT>(p.dgate + i * item_bytes<DT>(), v);
}

namespace {

constexpr int kMaxCols = 16384;

// Lanes of a row (8 channels each), and with 1024 of them two runs to the lane.
struct RowShape {
    int lanes, runs;
};
RowShape row_shape(int cols)
{
    int lanes = 16;
    while (lanes < 1024 && lanes * 8 < cols) lanes *= 2;
    return {lanes, lanes * 8 < cols ? 2 : 1};
}

int row_threads(const RowShape &s) { return std::max(256, s.lanes); }

template <int DT, bool MX4>
void launch_norm(const NormArgs &a, hipStream_t s)
{
    const RowShape shape = row_shape(a.cols);
    const int threads = row_threads(shape), r = threads / shape.lanes;
    const int cus = std::max(compute_units(), 1);
    const unsigned grid = (unsigned)std::min<long long>(((long long)a.rows + r - 1) / r, (long long)cus * (2048 / threads));
    const auto go = [&](auto kern) { kern<<<dim3(grid), dim3(threads), 0, s>>>(a); };
    switch (shape.lanes) {
        case 16: go(norm_kernel<DT, 16, 1, MX4>); break;
        case 32: go(norm_kernel<DT, 32, 1, MX4>); break;
        case 64: go(norm_kernel<DT, 64, 1, MX4>); break;
        case 128: go(norm_kernel<DT, 128, 1, MX4>); break;
        case 256: go(norm_kernel<DT, 256, 1, MX4>); break;
        case 512: go(norm_kernel<DT, 512, 1, MX4>); break;
        default: shape.runs == 1 ? go(norm_kernel<DT, 1024, 1, MX4>) : go(norm_kernel<DT, 1024, 2, MX4>);
    }
}

struct GradPlan {
    int workgroups, groups, per_group, strips, per_strip;
    bool grouped;
    size_t part, gate_part;                // floats
};

// How the rows are shared out.  A workgroup leaves one partial sum per column and accumulator behind, so it gets at least eight rows' worth
// once there are 64 workgroups, and no more of them are made than run at once.  A gate of several rows gives strips that do not cross a
// group, so that a strip's sum is a part of one gate's gradient.
GradPlan grad_plan(const ss_norm_desc &d, long long rows, long long groups, int gate_cols)
{
    GradPlan g{};
    const RowShape shape = row_shape(d.cols);
    const int threads = row_threads(shape), r = threads / shape.lanes;
    const long long cus = std::max(compute_units(), 1);
    const long long most = std::min(std::max(64ll, rows / 8), cus * std::max(1, 1024 / threads));
    const long long target = std::max(1ll, std::min((rows + r - 1) / r, most));
    g.grouped = gate_cols > 0 && groups < rows;
    g.groups = g.grouped ? (int)groups : 1;
    g.per_group = (int)(rows / g.groups);
    const long long want = std::max(1ll, std::min((target + g.groups - 1) / g.groups, ((long long)g.per_group + r - 1) / r));
    g.per_strip = (int)((g.per_group + want - 1) / want);
    g.strips = g.per_strip > 0 ? (g.per_group + g.per_strip - 1) / g.per_strip : 1;
    g.workgroups = (int)std::min<long long>((long long)g.groups * g.strips, target * 2);
    g.part = (size_t)ACC_COUNT * g.workgroups * d.cols;
    g.gate_part = g.grouped && g.strips > 1 ? (size_t)g.groups * g.strips * gate_cols : 0;
    return g;
}

template <int DT>
void launch_grad(const NormGradArgs &a, int workgroups, hipStream_t s)
{
    const RowShape shape = row_shape(a.cols);
    const int threads = row_threads(shape);
    const auto go = [&](auto kern) { kern<<<dim3(workgroups), dim3(threads), 0, s>>>(a); };
    const auto pick = [&](auto post) {
        constexpr bool POST = decltype(post)::value;
        switch (shape.lanes) {
            case 16: go(norm_grad_kernel<DT, 16, 1, POST>); break;
            case 32: go(norm_grad_kernel<DT, 32, 1, POST>); break;
            case 64: go(norm_grad_kernel<DT, 64, 1, POST>); break;
            case 128: go(norm_grad_kernel<DT, 128, 1, POST>); break;
            case 256: go(norm_grad_kernel<DT, 256, 1, POST>); break;
            case 512: go(norm_grad_kernel<DT, 512, 1, POST>); break;
            default: shape.runs == 1 ? go(norm_grad_kernel<DT, 1024, 1, POST>) : go(norm_grad_kernel<DT, 1024, 2, POST>);
        }
    };
    a.post != SS_NORM_NONE && a.h != nullptr ? pick(std::true_type{}) : pick(std::false_type{});
}

bool norm_kind(int k) { return k == SS_NORM_NONE || k == SS_NORM_LAYER || k == SS_NORM_RMS; }

int check_norm(const ss_norm_desc *d, int64_t rows, int64_t groups, int32_t gate_cols)
{
    if (!d || d->cols <= 0 || !norm_kind(d->norm) || !norm_kind(d->post)) return SS_ERR_INVALID_ARG;
    if (d->dtype != SS_F16 && d->dtype != SS_BF16 && d->dtype != SS_F32) return SS_ERR_INVALID_ARG;
    if (!(d->eps >= 0.f) || !(d->post_eps >= 0.f) || std::isinf(d->eps) || std::isinf(d->post_eps)) return SS_ERR_INVALID_ARG;
    if (rows < 0 || gate_cols < 0) return SS_ERR_INVALID_ARG;
    if (gate_cols != 0 && gate_cols != 1 && gate_cols != d->cols) return SS_ERR_INVALID_ARG;
    if (gate_cols != 0 && rows > 0 && (groups <= 0 || rows % groups != 0)) return SS_ERR_INVALID_ARG;
    return d->cols <= kMaxCols && rows <= INT32_MAX ? SS_OK : SS_ERR_UNSUPPORTED;
}

// A tensor of rows: there (or allowed to be absent), on an element's boundary, with a pitch that holds a row.
bool rows_ok(const ss_norm_desc *d, const void *p, int64_t ld, bool needed)
{
    if (!p) return !needed;
    return aligned(p, d->dtype == SS_F32 ? 4 : 2) && ld >= d->cols && ld <= INT32_MAX;
}

}  // namespace
}  // namespace ss

using namespace ss;

extern "C" int ss_norm_fwd(const ss_norm_desc *d, const ss_norm_io *io, void *stream)
{
    if (!io) return SS_ERR_INVALID_ARG;
    const int st = check_norm(d, io->rows, io->groups, io->gate ? io->gate_cols : 0);
    if (st != SS_OK) return st;
    const bool mx4 = io->codes != nullptr || io->scales != nullptr, norm = d->norm != SS_NORM_NONE;
    if (io->gate && io->gate_cols == 0) return SS_ERR_INVALID_ARG;
    if (!io->h && (io->x_out || io->gate || io->scale || d->post != SS_NORM_NONE)) return SS_ERR_INVALID_ARG;
    if (!norm && (io->y || mx4 || !io->h)) return SS_ERR_INVALID_ARG;
    if (io->rows == 0) return SS_OK;
    if (!rows_ok(d, io->x, io->ldx, true) || !rows_ok(d, io->h, io->ldh, false) || !rows_ok(d, io->x_out, io->ldx_out, io->h != nullptr) ||
        !rows_ok(d, io->y, io->ldy, norm && !mx4) || (mx4 && (io->y || !io->codes || !io->scales || !aligned(io->codes, 16) || !aligned(io->scales, 4))) ||
        (io->gate && !aligned(io->gate, d->dtype == SS_F32 ? 4 : 2)))
        return SS_ERR_INVALID_ARG;
    for (const float *v : {io->w, io->b, io->scale, io->post_w, io->post_b})
        if (!aligned(v, 4)) return SS_ERR_INVALID_ARG;
    NormArgs a{};
    a.x = static_cast<const char *>(io->x); a.h = static_cast<const char *>(io->h); a.gate = static_cast<const char *>(io->gate);
    a.w = io->w; a.b = io->b; a.scale = io->scale; a.post_w = io->post_w; a.post_b = io->post_b;
    a.x_out = static_cast<char *>(io->x_out); a.y = static_cast<char *>(io->y);
    a.codes = static_cast<uint8_t *>(io->codes); a.scales = static_cast<uint8_t *>(io->scales);
    a.ldx = io->ldx; a.ldh = io->ldh; a.ldx_out = io->ldx_out; a.ldy = io->ldy;
    a.rows = (int)io->rows; a.cols = d->cols; a.gate_cols = io->gate_cols; a.norm = d->norm; a.post = d->post;
    a.eps = d->eps; a.post_eps = d->post_eps;
    fast_div_setup(io->gate ? (unsigned)(io->rows / io->groups) : 1u, &a.g_mul, &a.g_sh);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const auto go = [&](auto m) {
        constexpr bool MX4 = decltype(m)::value;
        d->dtype == SS_F16 ? launch_norm<SS_F16, MX4>(a, s) : d->dtype == SS_BF16 ? launch_norm<SS_BF16, MX4>(a, s) : launch_norm<SS_F32, MX4>(a, s);
    };
    mx4 ? go(std::true_type{}) : go(std::false_type{});
    return launched();
}

extern "C" int ss_norm_bwd_workspace_bytes(const ss_norm_desc *d, int64_t rows, int64_t groups, int32_t gate_cols, size_t *bytes)
{
    const int st = check_norm(d, rows, groups, gate_cols);
    if (st != SS_OK) return st;
    if (!bytes) return SS_ERR_INVALID_ARG;
    const GradPlan g = grad_plan(*d, rows, groups, gate_cols);
    *bytes = rows == 0 ? 0 : (g.part + g.gate_part) * sizeof(float);
    return SS_OK;
}

extern "C" int ss_norm_bwd(const ss_norm_desc *d, const ss_norm_grad_io *io, void *workspace, size_t ws_bytes, void *stream)
{
    if (!io) return SS_ERR_INVALID_ARG;
    const int st = check_norm(d, io->rows, io->groups, io->gate ? io->gate_cols : 0);
    if (st != SS_OK) return st;
    const bool norm = d->norm != SS_NORM_NONE, post = d->post != SS_NORM_NONE;
    if (io->gate && io->gate_cols == 0) return SS_ERR_INVALID_ARG;
    if (!io->h && (io->dh || io->gate || io->scale || post)) return SS_ERR_INVALID_ARG;
    if ((!norm && (io->dy || io->dw || io->db || !io->dx_out)) || (io->dscale && !io->h) || (io->dgate && !io->gate) || (io->gate && !io->dgate) ||
        ((io->dpost_w || io->dpost_b) && !(post && io->h)))
        return SS_ERR_INVALID_ARG;
    for (const float *v : {io->w, io->scale, io->post_w, io->post_b, (const float *)io->dw, (const float *)io->db, (const float *)io->dscale, (const float *)io->dpost_w,
                           (const float *)io->dpost_b})
        if (!aligned(v, 4)) return SS_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    NormSumArgs sum{};
    sum.out[ACC_W] = io->dw; sum.out[ACC_B] = io->db; sum.out[ACC_SCALE] = io->dscale; sum.out[ACC_POST_W] = io->dpost_w; sum.out[ACC_POST_B] = io->dpost_b;
    sum.cols = d->cols;
    sum.column_tiles = (d->cols + 15) / 16;
    bool any = false;
    for (const float *o : sum.out) any = any || o;
    const auto finish = [&](long long gates) {
        const dim3 grid((unsigned)(sum.column_tiles * ACC_COUNT + (gates + 1023) / 1024)), block(1024);
        sum.gates = gates;
        const auto go = [&](auto kern) { kern<<<grid, block, 0, s>>>(sum); };
        d->dtype == SS_F16 ? go(norm_grad_sum_kernel<SS_F16>) : d->dtype == SS_BF16 ? go(norm_grad_sum_kernel<SS_BF16>) : go(norm_grad_sum_kernel<SS_F32>);
        return launched();
    };
    if (io->rows == 0) return any ? finish(0) : SS_OK;   // sums over no rows
    if (!rows_ok(d, io->dy, io->lddy, norm) || !rows_ok(d, io->x_out, io->ldx_out, norm) || !rows_ok(d, io->dx_out, io->lddx_out, false) ||
        !rows_ok(d, io->h, io->ldh, false) || !rows_ok(d, io->dx, io->lddx, true) || !rows_ok(d, io->dh, io->lddh, io->h != nullptr) ||
        (io->gate && (!aligned(io->gate, d->dtype == SS_F32 ? 4 : 2) || !aligned(io->dgate, d->dtype == SS_F32 ? 4 : 2))))
        return SS_ERR_INVALID_ARG;
    const GradPlan g = grad_plan(*d, io->rows, io->groups, io->gate ? io->gate_cols : 0);
    if (!workspace || !aligned(workspace, 16) || ws_bytes < (g.part + g.gate_part) * sizeof(float)) return SS_ERR_WORKSPACE;
    NormGradArgs a{};
    a.dy = static_cast<const char *>(io->dy); a.x_out = static_cast<const char *>(io->x_out); a.dx_out = static_cast<const char *>(io->dx_out);
    a.h = static_cast<const char *>(io->h); a.gate = static_cast<const char *>(io->gate);
    a.w = io->w; a.scale = io->scale; a.post_w = io->post_w; a.post_b = io->post_b;
    a.dx = static_cast<char *>(io->dx); a.dh = static_cast<char *>(io->dh); a.dgate = static_cast<char *>(io->dgate);
    a.part = static_cast<float *>(workspace);
    a.gate_part = a.part + g.part;
    a.lddy = io->lddy; a.ldx_out = io->ldx_out; a.lddx_out = io->lddx_out; a.ldh = io->ldh; a.lddx = io->lddx; a.lddh = io->lddh;
    a.rows = (int)io->rows; a.cols = d->cols; a.gate_cols = io->gate ? io->gate_cols : 0; a.norm = d->norm; a.post = d->post;
    a.eps = d->eps; a.post_eps = d->post_eps;
    a.groups = g.groups; a.per_group = g.per_group; a.strips = g.strips; a.per_strip = g.per_strip; a.grouped = g.grouped;
    d->dtype == SS_F16 ? launch_grad<SS_F16>(a, g.workgroups, s) : d->dtype == SS_BF16 ? launch_grad<SS_BF16>(a, g.workgroups, s) : launch_grad<SS_F32>(a, g.workgroups, s);
    const int started = launched();
    if (started != SS_OK) return started;
    const long long gates = g.gate_part ? (long long)g.groups * a.gate_cols : 0;
    if (!any && gates == 0) return SS_OK;
    sum.part = a.part; sum.gate_part = a.gate_part; sum.dgate = a.dgate;
    sum.parts = g.workgroups; sum.strips = g.strips; sum.gate_cols = a.gate_cols;
    return finish(gates);
}
