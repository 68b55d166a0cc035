// Entry points of the norms around a block (kernels: ss_norm_kernel.h).
#include "ss_norm_kernel.h"
#include "ss_conv_params.h"
#include <cmath>

namespace ss {

SS_NORM_LAUNCHES(extern, SS_F16)
SS_NORM_LAUNCHES(extern, SS_BF16)
SS_NORM_LAUNCHES(extern, SS_F32)

namespace {

constexpr int kMaxCols = 16384;

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
    const int threads = grad_threads(shape.lanes, d.post != SS_NORM_NONE), r = threads / shape.lanes;
    const long long cus = std::max(compute_units(), 1);
    const bool post = d.post != SS_NORM_NONE;
    const int resident = post ? 512 : 256 * grad_waves(d.dtype, gate_cols > 1);          // threads of a compute unit
    const long long most = std::min(std::max(64ll, rows / 8), cus * std::max(1, resident / threads));
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

bool norm_kind(int k) { return k == SS_NORM_NONE || k == SS_NORM_LAYER || k == SS_NORM_RMS; }

int check_norm(const ss_norm_desc *d, int64_t rows, int64_t groups, int32_t gate_cols)
{
    if (!d || d->cols <= 0 || !norm_kind(d->norm) || !norm_kind(d->post)) return SS_ERR_INVALID_ARG;
    if (d->dtype != SS_F16 && d->dtype != SS_BF16 && d->dtype != SS_F32) return SS_ERR_INVALID_ARG;
    if (!(d->eps >= 0.f) || !(d->post_eps >= 0.f) || std::isinf(d->eps) || std::isinf(d->post_eps)) return SS_ERR_INVALID_ARG;
    if (rows < 0 || gate_cols < 0) return SS_ERR_INVALID_ARG;
    if (gate_cols != 0 && gate_cols != 1 && gate_cols != d->cols) return SS_ERR_INVALID_ARG;
    if (gate_cols != 0 && (rows > 0 ? groups <= 0 || rows % groups != 0 : groups < 0)) return SS_ERR_INVALID_ARG;
    return d->cols <= kMaxCols && rows <= INT32_MAX && (gate_cols == 0 || groups <= INT32_MAX) ? SS_OK : SS_ERR_UNSUPPORTED;
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
    if (!norm && (io->y || mx4 || !io->h || io->w || io->b)) return SS_ERR_INVALID_ARG;
    if (d->post == SS_NORM_NONE && (io->post_w || io->post_b)) return SS_ERR_INVALID_ARG;
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
    const bool post = io->h && d->post != SS_NORM_NONE;
    d->dtype == SS_F16 ? launch_norm<SS_F16>(a, mx4, post, s) : d->dtype == SS_BF16 ? launch_norm<SS_BF16>(a, mx4, post, s) : launch_norm<SS_F32>(a, mx4, post, s);
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
    if ((!norm && (io->dy || io->w || io->dw || io->db || !io->dx_out)) || (!post && (io->post_w || io->post_b)) || (io->dscale && !io->h) || (io->dgate && !io->gate) || (io->gate && !io->dgate) ||
        ((io->dpost_w || io->dpost_b) && !(post && io->h)))
        return SS_ERR_INVALID_ARG;
    for (const float *v : {io->w, io->scale, io->post_w, io->post_b, (const float *)io->dw, (const float *)io->db, (const float *)io->dscale, (const float *)io->dpost_w,
                           (const float *)io->dpost_b})
        if (!aligned(v, 4)) return SS_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    NormSumArgs sum{};
    float *const outs[ACC_COUNT] = {io->dw, io->db, io->dscale, io->dpost_w, io->dpost_b};       // (in the order of the accumulators)
    for (int a = 0; a < ACC_COUNT; a++)
        if (outs[a]) {
            sum.out[sum.wanted] = outs[a];
            sum.which[sum.wanted++] = a;
        }
    sum.cols = d->cols;
    const auto finish = [&](long long gates) {
        sum.gates = gates;
        sum.tiles = (d->cols + sum_columns(sum.parts) - 1) / sum_columns(sum.parts);
        d->dtype == SS_F16 ? launch_norm_sum<SS_F16>(sum, s) : d->dtype == SS_BF16 ? launch_norm_sum<SS_BF16>(sum, s) : launch_norm_sum<SS_F32>(sum, s);
        return launched();
    };
    if (io->rows == 0) {                                        // sums over no rows
        const long long gates = io->gate ? io->groups * (long long)io->gate_cols : 0;
        if (io->dgate && !aligned(io->dgate, d->dtype == SS_F32 ? 4 : 2)) return SS_ERR_INVALID_ARG;
        if (gates > INT32_MAX) return SS_ERR_UNSUPPORTED;       // (a thread to the element)
        sum.dgate = static_cast<char *>(io->dgate);
        sum.gate_cols = io->gate_cols;
        return sum.wanted || gates ? finish(gates) : SS_OK;
    }
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
    d->dtype == SS_F16 ? launch_norm_grad<SS_F16>(a, post, g.workgroups, s)
                       : d->dtype == SS_BF16 ? launch_norm_grad<SS_BF16>(a, post, g.workgroups, s) : launch_norm_grad<SS_F32>(a, post, g.workgroups, s);
    const int started = launched();
    if (started != SS_OK) return started;
    const long long gates = g.gate_part ? (long long)g.groups * a.gate_cols : 0;
    if (!sum.wanted && gates == 0) return SS_OK;
    sum.part = a.part; sum.gate_part = a.gate_part; sum.dgate = a.dgate;
    sum.parts = g.workgroups; sum.strips = g.strips; sum.gate_cols = a.gate_cols;
    return finish(gates);
}
