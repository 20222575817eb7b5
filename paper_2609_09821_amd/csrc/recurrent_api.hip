// recurrent_api.hip -- C ABI of a recurrent policy's blocks: argument checks on the host,
// then the launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/instantmimic.h"
#include "recurrent.h"

using namespace im;

namespace {

constexpr int64_t MAX_ROWS = (int64_t)1 << 30, MAX_WIDTH = 1 << 20;

im_status invalid(const char *msg) { return api_fail(IM_ERR_INVALID_ARG, msg); }
im_status unsupported(const char *msg) { return api_fail(IM_ERR_UNSUPPORTED, msg); }
im_status launched(hipError_t e, const char *what) { return e == hipSuccess ? IM_OK : api_hip_fail(e, what); }

bool is_dtype(int32_t t) { return t == IM_DTYPE_F32 || t == IM_DTYPE_BF16; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// What every call on [n][d] rows asks of them.
im_status check_rows(int64_t n, int64_t d, int32_t dtype)
{
    if (n < 0 || d < 1) return invalid("n must be >= 0 and the rows' width >= 1");
    if (n > MAX_ROWS) return unsupported("more than 2^30 rows");
    if (!is_dtype(dtype)) return invalid("dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16");
    return IM_OK;
}

// A matrix [n][d] in 8 bits.
im_status check_block8(const im_block8 *b, int64_t n, int64_t d)
{
    if (b->rows != 1 && b->rows != IM_BLOCK8) return invalid("block8: rows must be 1 or 128");
    if (b->ld_q < IM_BLOCK8_PAD(d) || b->ld_q % 16 != 0)
        return invalid("block8: ld_q must be a multiple of 16 and >= d rounded up to 128");
    if (b->ld_scale < ceil_div(d, IM_BLOCK8)) return invalid("block8: ld_scale must be >= ceil(d / 128)");
    if (n > 0 && (!b->q || !b->scale)) return invalid("NULL block8 buffer");
    if (!aligned(b->q, 16)) return invalid("block8: q must be 16-byte aligned");
    return IM_OK;
}

im_status check_workspace(const void *ws, int64_t have, int64_t need, uintptr_t align)
{
    if (need > 0 && (!ws || have < need)) return invalid("workspace NULL or too small");
    if (need > 0 && !aligned(ws, align)) return invalid("workspace not aligned");
    return IM_OK;
}

int64_t pad16(int64_t x) { return (x + 15) & ~(int64_t)15; }

// Sections of im_block_linear_grad's workspace: dy in 8 bits and transposed, the column sums of
// 128 rows each, the parts of dw.
struct GradSpace {
    int64_t q, scale, tq, tscale, sums, part, bytes;
    int splits;
};
GradSpace grad_space(int64_t n, int64_t in, int64_t out)
{
    GradSpace g{};
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += pad16(bytes);
        return here;
    };
    g.splits = linear8_splits(out, in, ceil_div(n, IM_BLOCK8));
    g.q = take(n * IM_BLOCK8_PAD(out));
    g.scale = take(n * ceil_div(out, IM_BLOCK8));
    g.tq = take(out * IM_BLOCK8_PAD(n));
    g.tscale = take(out * ceil_div(n, IM_BLOCK8));
    g.sums = take(ceil_div(n, IM_BLOCK8) * out * (int64_t)sizeof(float));
    g.part = take(g.splits > 1 ? g.splits * out * ((in + 3) / 4 * 4) * (int64_t)sizeof(float) : 0);
    g.bytes = at;
    return g;
}

im_status check_layer8(int64_t n, int64_t in, int64_t out, int32_t dtype)
{
    im_status s = check_rows(n, in, dtype);
    if (s != IM_OK) return s;
    if (out < 1) return invalid("out must be >= 1");
    if (in > MAX_WIDTH || out > MAX_WIDTH || in * out > MAX_ROWS)
        return unsupported("in or out above 2^20, or in * out above 2^30");
    return IM_OK;
}

// Strides of [T][n][d] values of which no two lie at one place.
bool apart(int64_t T, int64_t n, int64_t d, int64_t st, int64_t ld)
{
    if (st < 0 || ld < 0) return false;
    if (T < 2) return n < 2 || ld >= d;
    if (n < 2) return st >= d;
    return (ld >= d && st >= (n - 1) * ld + d) || (st >= d && ld >= (T - 1) * st + d);
}

// Checks that the scan and its gradient share.
im_status check_scan(int64_t T, int64_t n, int64_t d, int32_t dtype, const void *term, const void *trunc,
                     int64_t ld_flags)
{
    if (T < 0 || n < 0 || d < 1) return invalid("T and n must be >= 0 and d >= 1");
    if (T > MAX_ROWS || n > MAX_ROWS || d > MAX_ROWS) return unsupported("T, n or d above 2^30");
    if (n * d > ((int64_t)1 << 31)) return unsupported("more than 2^31 states");
    if (!is_dtype(dtype)) return invalid("dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16");
    if ((term || trunc) && T > 1 && ld_flags < n) return invalid("ld_flags must be >= n");
    return IM_OK;
}

// Chunks of a scan, and the bytes of their maps.
int64_t plan_scan(ScanArgs &a, void *workspace)
{
    a.chunk = std::max<int64_t>(scan_chunk(a.T, a.n, a.d), 1);
    a.chunks = std::max<int64_t>(ceil_div(a.T, a.chunk), 1);
    a.maps = (float *)workspace;
    return a.chunks > 1 ? a.chunks * 2 * a.n * a.d * (int64_t)sizeof(float) : 0;
}

}  // namespace

extern "C" {

im_status im_block_store(const void *x, int64_t ld_x, int32_t dtype, int64_t n, int64_t d, const im_block8 *c,
                          const im_block8 *t, void *stream)
{
    im_status s = check_rows(n, d, dtype);
    if (s != IM_OK) return s;
    if (d > MAX_WIDTH) return unsupported("d above 2^20");
    if (!c && !t) return invalid("NULL block8: neither c nor t");
    if (c && (s = check_block8(c, n, d)) != IM_OK) return s;
    if (t && (s = check_block8(t, d, n)) != IM_OK) return s;
    if (c && t && c->rows != t->rows) return invalid("block8: c and t must have the same rows");
    if (ld_x < d) return invalid("ld_x must be >= d");
    if (n == 0) return IM_OK;
    if (!x) return invalid("NULL x");
    StoreArgs a{};
    a.x = x;
    a.ld_x = ld_x;
    a.n = n;
    a.d = d;
    a.c = mat8(c);
    a.t = mat8(t);
    return launched(launch_block8_store(a, dtype == IM_DTYPE_F32, (hipStream_t)stream), "block_store launch");
}

im_status im_block_load(const im_block8 *c, int64_t n, int64_t d, void *x, int64_t ld_x, int32_t dtype,
                         void *stream)
{
    im_status s = check_rows(n, d, dtype);
    if (s != IM_OK) return s;
    if (d > MAX_WIDTH) return unsupported("d above 2^20");
    if (!c) return invalid("NULL block8");
    if ((s = check_block8(c, n, d)) != IM_OK) return s;
    if (ld_x < d) return invalid("ld_x must be >= d");
    if (n == 0) return IM_OK;
    if (!x) return invalid("NULL x");
    return launched(launch_block8_load(mat8(c), n, d, x, ld_x, dtype == IM_DTYPE_F32, (hipStream_t)stream),
                    "block_load launch");
}

im_status im_rms_norm(const im_rms *p, void *stream)
{
    if (!p) return invalid("NULL im_rms");
    im_status s = check_rows(p->n, p->d, p->dtype);
    if (s != IM_OK) return s;
    if (p->d > IM_NORM_MAX_WIDTH) return unsupported("d above IM_NORM_MAX_WIDTH");
    if (!(p->eps >= 0.0f)) return invalid("eps must be >= 0");
    if (p->ld_x < p->d || (p->residual && p->ld_residual < p->d) || (p->h && p->ld_h < p->d) ||
        (p->y && p->ld_y < p->d))
        return invalid("ld_x, ld_residual, ld_h and ld_y must be >= d");
    if (p->y8 && (s = check_block8(p->y8, p->n, p->d)) != IM_OK) return s;
    if (p->y8 && p->y8->rows != 1) return invalid("block8: y8's rows must be 1");
    if (p->n == 0) return IM_OK;
    if (!p->h && !p->y && !p->y8 && !p->rstd) return invalid("no output asked for");
    if (p->h && p->h == p->y) return invalid("h and y are one array");
    if (!p->x) return invalid("NULL x");
    RmsArgs a{};
    a.n = p->n;
    a.d = (int)p->d;
    a.eps = p->eps;
    a.inv_d = 1.0f / (float)p->d;
    a.x = p->x;
    a.ld_x = p->ld_x;
    a.res = p->residual;
    a.ld_res = p->ld_residual;
    a.gamma = p->gamma;
    a.h = p->h;
    a.ld_h = p->ld_h;
    a.y = p->y;
    a.ld_y = p->ld_y;
    a.rstd = p->rstd;
    a.y8 = mat8(p->y8);
    return launched(launch_rms(a, p->dtype == IM_DTYPE_F32, (hipStream_t)stream), "rms_norm launch");
}

int64_t im_rms_norm_grad_workspace(int64_t n, int64_t d)
{
    if (n < 0 || n > MAX_ROWS || d < 1 || d > IM_NORM_MAX_WIDTH) return -1;
    return rms_grad_blocks(n, d) * d * (int64_t)sizeof(float);
}

im_status im_rms_norm_grad(const im_rms_grad *p, void *stream)
{
    if (!p) return invalid("NULL im_rms_grad");
    im_status s = check_rows(p->n, p->d, p->dtype);
    if (s != IM_OK) return s;
    if (p->d > IM_NORM_MAX_WIDTH) return unsupported("d above IM_NORM_MAX_WIDTH");
    if (p->ld_dy < p->d || p->ld_h < p->d || (p->dh && p->ld_dh < p->d) || (p->dx && p->ld_dx < p->d))
        return invalid("ld_dy, ld_h, ld_dh and ld_dx must be >= d");
    if (p->n > 0 && (!p->dy || !p->h || !p->rstd)) return invalid("NULL dy, h or rstd");
    if (p->n > 0 && !p->dx && !p->dgamma) return invalid("no output asked for");
    s = check_workspace(p->workspace, p->workspace_bytes, p->dgamma ? im_rms_norm_grad_workspace(p->n, p->d) : 0, 4);
    if (s != IM_OK) return s;
    if (p->n == 0 && !p->dgamma) return IM_OK;
    RmsGradArgs a{};
    a.n = p->n;
    a.d = (int)p->d;
    a.inv_d = 1.0f / (float)p->d;
    a.dy = p->dy;
    a.ld_dy = p->ld_dy;
    a.h = p->h;
    a.ld_h = p->ld_h;
    a.dh = p->dh;
    a.ld_dh = p->ld_dh;
    a.gamma = p->gamma;
    a.rstd = p->rstd;
    a.dx = p->dx;
    a.ld_dx = p->ld_dx;
    a.dgamma = p->dgamma;
    a.part = p->dgamma ? (float *)p->workspace : nullptr;
    return launched(launch_rms_grad(a, p->dtype == IM_DTYPE_F32, (hipStream_t)stream), "rms_norm_grad launch");
}

im_status im_block_linear(const im_layer8 *p, void *stream)
{
    if (!p) return invalid("NULL im_layer8");
    im_status s = check_layer8(p->n, p->in, p->out, p->y_dtype);
    if (s != IM_OK) return s;
    if (!p->x || !p->w) return invalid("NULL block8: x or w");
    if ((s = check_block8(p->x, p->n, p->in)) != IM_OK || (s = check_block8(p->w, p->out, p->in)) != IM_OK) return s;
    if (p->y && p->ld_y < p->out) return invalid("ld_y must be >= out");
    if (p->y8 && (s = check_block8(p->y8, p->n, p->out)) != IM_OK) return s;
    if (p->y8 && p->y8->rows != 1) return invalid("block8: y8's rows must be 1");
    if (p->n == 0) return IM_OK;
    if (!p->y && !p->y8) return invalid("no output asked for");
    Linear8Args a{};
    a.n = p->n;
    a.out = p->out;
    a.steps = ceil_div(p->in, IM_BLOCK8);
    a.q = mat8(p->x);
    a.p = mat8(p->w);
    a.bias = p->bias;
    a.relu = p->relu != 0;
    a.y = p->y;
    a.ld_y = p->ld_y;
    a.y_f32 = p->y_dtype == IM_DTYPE_F32;
    a.y8 = mat8(p->y8);
    a.splits = 1;
    return launched(launch_linear8(a, (hipStream_t)stream), "block_linear launch");
}

int64_t im_block_linear_grad_workspace(int64_t n, int64_t in, int64_t out)
{
    if (n < 0 || n > MAX_ROWS || in < 1 || in > MAX_WIDTH || out < 1 || out > MAX_WIDTH ||
        in * out > MAX_ROWS)
        return -1;
    return grad_space(n, in, out).bytes;
}

im_status im_block_linear_grad(const im_layer8_grad *p, void *stream)
{
    if (!p) return invalid("NULL im_layer8_grad");
    im_status s = check_layer8(p->n, p->in, p->out, p->dtype);
    if (s != IM_OK) return s;
    const bool sums = p->dw || p->db;
    if (!p->dx && !sums && p->n > 0) return invalid("no output asked for");
    if (p->ld_dy < p->out || (p->y && p->ld_y < p->out) || (p->dx && p->ld_dx < p->in) ||
        (p->dw && p->ld_dw < p->in))
        return invalid("ld_dy and ld_y must be >= out, ld_dx and ld_dw >= in");
    if (p->n > 0 && !p->dy) return invalid("NULL dy");
    if (p->dx && !p->wt) return invalid("NULL block8: wt");
    if (p->dx && (s = check_block8(p->wt, p->in, p->out)) != IM_OK) return s;
    // no rows: x^T has no values, and dw is zero
    if (p->dw && p->n > 0 && !p->xt) return invalid("NULL block8: xt");
    if (p->dw && p->n > 0 && (s = check_block8(p->xt, p->in, p->n)) != IM_OK) return s;
    const GradSpace g = grad_space(p->n, p->in, p->out);
    // the parts, which come last, are dw's: without it `in` does not count
    s = check_workspace(p->workspace, p->workspace_bytes, p->dw ? g.bytes : g.part, 16);
    if (s != IM_OK) return s;
    if (p->n == 0 && !sums) return IM_OK;
    const hipStream_t st = (hipStream_t)stream;
    const bool f32 = p->dtype == IM_DTYPE_F32;
    char *ws = (char *)p->workspace;
    StoreArgs a{};
    a.x = p->dy;
    a.ld_x = p->ld_dy;
    a.y = p->y;
    a.ld_y = p->ld_y;
    a.n = p->n;
    a.d = p->out;
    if (p->dx)
        a.c = Mat8{(uint8_t *)ws + g.q, (uint8_t *)ws + g.scale, IM_BLOCK8_PAD(p->out), ceil_div(p->out, IM_BLOCK8), 0};
    if (p->dw) a.t = Mat8{(uint8_t *)ws + g.tq, (uint8_t *)ws + g.tscale, IM_BLOCK8_PAD(p->n), ceil_div(p->n, IM_BLOCK8), 0};
    if (p->db) a.sums = (float *)(ws + g.sums);
    hipError_t e = hipSuccess;
    if (p->n > 0) e = launch_block8_store(a, f32, st);
    Linear8Args dx{}, dw{};
    if (p->dx && p->n > 0) {
        dx.n = p->n;
        dx.out = p->in;
        dx.steps = ceil_div(p->out, IM_BLOCK8);
        dx.q = a.c;
        dx.p = mat8(p->wt);
        dx.y = p->dx;
        dx.ld_y = p->ld_dx;
        dx.y_f32 = f32;
        dx.splits = 1;
    }
    if (p->dw) {
        dw.n = p->out;
        dw.out = p->in;
        dw.steps = ceil_div(p->n, IM_BLOCK8);
        dw.q = a.t;
        if (p->n > 0) dw.p = mat8(p->xt);
        dw.y = p->dw;
        dw.ld_y = p->ld_dw;
        dw.y_f32 = 1;
        dw.splits = g.splits;
        if (g.splits > 1) dw.part = (float *)(ws + g.part);
    }
    if (e == hipSuccess)
        e = launch_linear8_grad(dx, dw, ColumnSums{a.sums, ceil_div(p->n, IM_BLOCK8), p->out, p->db}, st);
    return launched(e, "block_linear_grad launch");
}

int64_t im_gated_scan_workspace(int64_t T, int64_t n, int64_t d)
{
    if (T < 0 || T > MAX_ROWS || n < 0 || n > MAX_ROWS || d < 1 || d > MAX_ROWS || n * d > ((int64_t)1 << 31)) return -1;
    return scan_workspace_bound(T, n, d);
}

im_status im_gated_scan(const im_scan *p, void *stream)
{
    if (!p) return invalid("NULL im_scan");
    im_status s = check_scan(p->T, p->n, p->d, p->dtype, p->terminated, p->truncated, p->ld_flags);
    if (s != IM_OK) return s;
    if (p->n == 0) return IM_OK;
    ScanArgs a{};
    a.T = p->T;
    a.n = p->n;
    a.d = p->d;
    s = check_workspace(p->workspace, p->workspace_bytes, plan_scan(a, p->workspace), 16);
    if (s != IM_OK) return s;
    if (p->T > 0) {
        if (!apart(p->T, p->n, p->d, p->st_h, p->ld_h)) return invalid("h: steps or rows overlap");
        if (p->st_gate < 0 || p->ld_gate < 0 || p->st_x < 0 || p->ld_x < 0) return invalid("negative stride");
        if (!p->gate || !p->x || !p->h) return invalid("NULL gate, x or h");
    }
    if (p->T == 0 && !p->state_out) return IM_OK;
    a.gate = p->gate;
    a.st_gate = p->st_gate;
    a.ld_gate = p->ld_gate;
    a.x = p->x;
    a.st_x = p->st_x;
    a.ld_x = p->ld_x;
    a.term = p->terminated;
    a.trunc = p->truncated;
    a.ld_flags = p->ld_flags;
    a.state = p->state;
    a.h = p->h;
    a.st_h = p->st_h;
    a.ld_h = p->ld_h;
    a.state_out = p->state_out;
    a.keep = p->keep;
    return launched(launch_scan(a, false, p->dtype == IM_DTYPE_F32, (hipStream_t)stream), "gated_scan launch");
}

im_status im_gated_scan_grad(const im_scan_grad *p, void *stream)
{
    if (!p) return invalid("NULL im_scan_grad");
    im_status s = check_scan(p->T, p->n, p->d, p->dtype, p->terminated, p->truncated, p->ld_flags);
    if (s != IM_OK) return s;
    if (p->n == 0) return IM_OK;
    ScanArgs a{};
    a.T = p->T;
    a.n = p->n;
    a.d = p->d;
    s = check_workspace(p->workspace, p->workspace_bytes, plan_scan(a, p->workspace), 16);
    if (s != IM_OK) return s;
    if (p->T > 0) {
        if (!apart(p->T, p->n, p->d, p->st_dgate, p->ld_dgate) || !apart(p->T, p->n, p->d, p->st_dx, p->ld_dx))
            return invalid("dgate or dx: steps or rows overlap");
        if (p->st_dh < 0 || p->ld_dh < 0 || p->st_gate < 0 || p->ld_gate < 0 || p->st_x < 0 || p->ld_x < 0)
            return invalid("negative stride");
        if (!p->dh || !p->gate || !p->x || !p->keep || !p->dgate || !p->dx)
            return invalid("NULL dh, gate, x, keep, dgate or dx");
    }
    if (p->T == 0 && !p->dstate_out) return IM_OK;
    a.gate = p->gate;
    a.st_gate = p->st_gate;
    a.ld_gate = p->ld_gate;
    a.x = p->x;
    a.st_x = p->st_x;
    a.ld_x = p->ld_x;
    a.term = p->terminated;
    a.trunc = p->truncated;
    a.ld_flags = p->ld_flags;
    a.state = p->dstate;
    a.state_out = p->dstate_out;
    a.keep = const_cast<float *>(p->keep);
    a.dh = p->dh;
    a.st_dh = p->st_dh;
    a.ld_dh = p->ld_dh;
    a.dgate = p->dgate;
    a.st_dgate = p->st_dgate;
    a.ld_dgate = p->ld_dgate;
    a.dx = p->dx;
    a.st_dx = p->st_dx;
    a.ld_dx = p->ld_dx;
    return launched(launch_scan(a, true, p->dtype == IM_DTYPE_F32, (hipStream_t)stream), "gated_scan_grad launch");
}

}  // extern "C"
