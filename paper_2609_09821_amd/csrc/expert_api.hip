// expert_api.hip -- C ABI of the layers of experts: argument checks on the host,
// then the launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/instantmimic.h"
#include "expert.h"

using namespace im;

namespace {

constexpr int64_t MAX_ROWS = (int64_t)1 << 30, MAX_WIDTH = 1 << 20;

im_status invalid(const char *msg) { return api_fail(IM_ERR_INVALID_ARG, msg); }
im_status unsupported(const char *msg) { return api_fail(IM_ERR_UNSUPPORTED, msg); }
im_status launched(hipError_t e, const char *what) { return e == hipSuccess ? IM_OK : api_hip_fail(e, what); }

bool is_dtype(int32_t t) { return t == IM_DTYPE_F32 || t == IM_DTYPE_BF16; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What every call on [n][d] rows asks of them.
im_status check_rows(int64_t n, int64_t d, int32_t dtype)
{
    if (n < 0 || d < 1) return invalid("n must be >= 0 and the rows' width >= 1");
    if (n > MAX_ROWS) return unsupported("more than 2^30 rows");
    if (!is_dtype(dtype)) return invalid("dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16");
    return IM_OK;
}

im_status check_checkpoint(const im_checkpoint *c, int64_t n, int64_t d)
{
    if (n > 0 && (!c->q || !c->scale)) return invalid("NULL checkpoint buffer");
    if (c->ld_q < d || c->ld_scale < ceil_div(d, CKPT_BLOCK))
        return invalid("checkpoint: ld_q must be >= d and ld_scale >= ceil(d / 32)");
    return IM_OK;
}

bool aligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

im_status check_workspace(const void *ws, int64_t have, int64_t need, uintptr_t align)
{
    if (need > 0 && (!ws || have < need)) return invalid("workspace NULL or too small");
    if (need > 0 && !aligned(ws, align)) return invalid("workspace not aligned");
    return IM_OK;
}

im_status checkpoint_call(bool store, void *x, int64_t ld_x, int32_t dtype, int64_t n, int64_t d,
                          const im_checkpoint *c, void *stream)
{
    im_status s = check_rows(n, d, dtype);
    if (s != IM_OK) return s;
    if (d > ((int64_t)1 << 30)) return unsupported("rows of more than 2^30 values");
    if (!c) return invalid("NULL checkpoint");
    if ((s = check_checkpoint(c, n, d)) != IM_OK) return s;
    if (ld_x < d) return invalid("ld_x must be >= d");
    if (n == 0) return IM_OK;
    if (!x) return invalid("NULL x");
    return launched(launch_checkpoint(store, x, ld_x, dtype == IM_DTYPE_F32, n, d, *c, (hipStream_t)stream),
                    "checkpoint launch");
}

// What the layer and its gradient ask alike.
im_status check_layer(int64_t n, int32_t E, int32_t in, int32_t out, int32_t dtype, const int32_t *offsets)
{
    im_status s = check_rows(n, in, dtype);
    if (s != IM_OK) return s;
    if (out < 1 || E < 1) return invalid("out and n_experts must be >= 1");
    if (E > IM_MAX_EXPERTS) return unsupported("n_experts above IM_MAX_EXPERTS");
    if (in > MAX_WIDTH || out > MAX_WIDTH || (int64_t)in * out > MAX_ROWS)
        return unsupported("in or out above 2^20, or in * out above 2^30");
    if (dtype != IM_DTYPE_BF16) return unsupported("expert layers are bf16 only");
    // a launch has fewer than 2^32 threads, in tiles of 64 x 64 at the least
    const int64_t wide = ceil_div(in > out ? in : out, 128);
    if ((n / 128 + E + 1) * wide >= (1 << 21)) return unsupported("more than 2^21 tiles of 128 rows and columns");
    if (!offsets) return invalid("NULL offsets");
    return IM_OK;
}

int64_t pad4(int64_t x) { return (x + 3) & ~(int64_t)3; }

}  // namespace

extern "C" {

int64_t im_group_rows_workspace(int64_t n, int32_t n_experts)
{
    if (n < 0 || n > MAX_ROWS || n_experts < 1 || n_experts > IM_MAX_EXPERTS) return -1;
    const int64_t blocks = group_blocks(n);
    return blocks > 1 ? blocks * (n_experts + 1) * (int64_t)sizeof(int32_t) : 0;
}

im_status im_group_rows(const int32_t *expert, int64_t n, int32_t n_experts, int32_t *offsets, int32_t *rows,
                        void *workspace, int64_t workspace_bytes, void *stream)
{
    if (n < 0 || n_experts < 1) return invalid("n must be >= 0 and n_experts >= 1");
    if (n > MAX_ROWS) return unsupported("more than 2^30 rows");
    if (n_experts > IM_MAX_EXPERTS) return unsupported("n_experts above IM_MAX_EXPERTS");
    if (!offsets || (n > 0 && (!expert || !rows))) return invalid("NULL expert, offsets or rows");
    const im_status s = check_workspace(workspace, workspace_bytes, im_group_rows_workspace(n, n_experts), 4);
    if (s != IM_OK) return s;
    return launched(launch_group_rows(expert, n, n_experts, offsets, rows, (int32_t *)workspace,
                                      (hipStream_t)stream),
                    "group_rows launch");
}

im_status im_checkpoint_store(const void *x, int64_t ld_x, int32_t dtype, int64_t n, int64_t d,
                              const im_checkpoint *c, void *stream)
{
    return checkpoint_call(true, const_cast<void *>(x), ld_x, dtype, n, d, c, stream);
}

im_status im_checkpoint_load(const im_checkpoint *c, int64_t n, int64_t d, void *x, int64_t ld_x, int32_t dtype,
                             void *stream)
{
    return checkpoint_call(false, x, ld_x, dtype, n, d, c, stream);
}

im_status im_layer_norm(const im_norm *p, void *stream)
{
    if (!p) return invalid("NULL im_norm");
    im_status s = check_rows(p->n, p->d, p->dtype);
    if (s != IM_OK) return s;
    if (p->d > IM_NORM_MAX_WIDTH) return unsupported("d above IM_NORM_MAX_WIDTH");
    if (!(p->eps >= 0.0f)) return invalid("eps must be >= 0");
    if (p->ld_x < p->d || p->ld_y < p->d) return invalid("ld_x and ld_y must be >= d");
    if (p->checkpoint && (s = check_checkpoint(p->checkpoint, p->n, p->d)) != IM_OK) return s;
    if (p->n == 0) return IM_OK;
    if (!p->x || !p->y) return invalid("NULL x or y");
    NormArgs a{};
    a.n = p->n;
    a.d = (int)p->d;
    a.eps = p->eps;
    a.inv_d = 1.0f / (float)p->d;
    a.x = p->x;
    a.ld_x = p->ld_x;
    a.gamma = p->gamma;
    a.beta = p->beta;
    a.y = p->y;
    a.ld_y = p->ld_y;
    a.mean = p->mean;
    a.rstd = p->rstd;
    if (p->checkpoint) a.c = *p->checkpoint;
    return launched(launch_norm(a, p->dtype == IM_DTYPE_F32, (hipStream_t)stream), "layer_norm launch");
}

int64_t im_layer_norm_grad_workspace(int64_t n, int64_t d)
{
    if (n < 0 || n > MAX_ROWS || d < 1 || d > IM_NORM_MAX_WIDTH) return -1;
    return norm_grad_blocks(n, d) * 2 * d * (int64_t)sizeof(float);
}

im_status im_layer_norm_grad(const im_norm_grad *p, void *stream)
{
    if (!p) return invalid("NULL im_norm_grad");
    im_status s = check_rows(p->n, p->d, p->dtype);
    if (s != IM_OK) return s;
    if (p->d > IM_NORM_MAX_WIDTH) return unsupported("d above IM_NORM_MAX_WIDTH");
    if (p->ld_dy < p->d || (p->x && p->ld_x < p->d) || (p->dx && p->ld_dx < p->d))
        return invalid("ld_dy, ld_x and ld_dx must be >= d");
    if (!p->x && p->checkpoint && (s = check_checkpoint(p->checkpoint, p->n, p->d)) != IM_OK) return s;
    if (p->n > 0 && (!p->dy || !p->mean || !p->rstd || (!p->x && !p->checkpoint)))
        return invalid("NULL dy, mean, rstd, or neither x nor a checkpoint");
    const bool sums = p->dgamma || p->dbeta;
    if (!p->dx && !sums && p->n > 0) return invalid("no output asked for");
    s = check_workspace(p->workspace, p->workspace_bytes, sums ? im_layer_norm_grad_workspace(p->n, p->d) : 0, 4);
    if (s != IM_OK) return s;
    if (p->n == 0 && !sums) return IM_OK;
    NormGradArgs a{};
    a.n = p->n;
    a.d = (int)p->d;
    a.inv_d = 1.0f / (float)p->d;
    a.dy = p->dy;
    a.ld_dy = p->ld_dy;
    a.x = p->x;
    a.ld_x = p->ld_x;
    if (!p->x && p->checkpoint) a.c = *p->checkpoint;
    a.gamma = p->gamma;
    a.mean = p->mean;
    a.rstd = p->rstd;
    a.dx = p->dx;
    a.ld_dx = p->ld_dx;
    a.dgamma = p->dgamma;
    a.dbeta = p->dbeta;
    a.part = sums ? (float *)p->workspace : nullptr;
    return launched(launch_norm_grad(a, p->dtype == IM_DTYPE_F32, (hipStream_t)stream), "layer_norm_grad launch");
}

im_status im_expert_linear(const im_expert_layer *p, void *stream)
{
    if (!p) return invalid("NULL im_expert_layer");
    im_status s = check_layer(p->n, p->n_experts, p->in, p->out, p->dtype, p->offsets);
    if (s != IM_OK) return s;
    if (!is_dtype(p->y_dtype)) return invalid("y_dtype must be IM_DTYPE_F32 or IM_DTYPE_BF16");
    if (p->ld_x < p->in || p->ld_w < p->in || p->ld_y < p->out)
        return invalid("ld_x and ld_w must be >= in and ld_y >= out");
    if (p->n == 0) return IM_OK;
    if (!p->x || !p->w || !p->y) return invalid("NULL x, w or y");
    ExpertArgs a{};
    a.offsets = p->offsets;
    a.rows = p->rows;
    a.E = p->n_experts;
    a.n = (int)p->n;
    a.in = p->in;
    a.out = p->out;
    a.x = (const uint16_t *)p->x;
    a.ld_x = p->ld_x;
    a.w = (const uint16_t *)p->w;
    a.ld_w = p->ld_w;
    a.bias = p->bias;
    a.relu = p->relu != 0;
    a.y = p->y;
    a.ld_y = p->ld_y;
    a.y_f32 = p->y_dtype == IM_DTYPE_F32;
    return launched(launch_expert_linear(a, (hipStream_t)stream), "expert_linear launch");
}

int64_t im_expert_linear_grad_workspace(int64_t n, int32_t n_experts, int32_t in, int32_t out)
{
    if (n < 0 || n > MAX_ROWS || n_experts < 1 || n_experts > IM_MAX_EXPERTS || in < 1 || in > MAX_WIDTH ||
        out < 1 || out > MAX_WIDTH)
        return -1;
    const int64_t teams = std::max(1, expert_grad_teams(n, n_experts, in, out));
    return 2 * teams * (out * pad4(in) + out) * (int64_t)sizeof(float);
}

im_status im_expert_linear_grad(const im_expert_layer_grad *p, void *stream)
{
    if (!p) return invalid("NULL im_expert_layer_grad");
    im_status s = check_layer(p->n, p->n_experts, p->in, p->out, p->dtype, p->offsets);
    if (s != IM_OK) return s;
    const bool need_x = p->dw || (p->dx && p->relu_x), sums = p->dw || p->db;
    if (!p->dx && !sums && p->n > 0) return invalid("no output asked for");
    if (sums && p->n_experts * ceil_div(p->in, 64) * ceil_div(p->out, 64) >= (1 << 24))
        return unsupported("more than 2^24 tiles of 64 x 64 in all experts' weights");
    if (p->ld_dy < p->out || (p->x && p->ld_x < p->in) || (p->dx && (p->ld_dx < p->in || p->ld_w < p->in)) ||
        (p->dw && p->ld_dw < p->in))
        return invalid("ld_dy must be >= out; ld_x, ld_w, ld_dx and ld_dw >= in");
    if (need_x && !p->x && p->checkpoint && (s = check_checkpoint(p->checkpoint, p->n, p->in)) != IM_OK) return s;
    if (p->n > 0 && (!p->dy || (p->dx && !p->w) || (need_x && !p->x && !p->checkpoint)))
        return invalid("NULL dy or w, or neither x nor a checkpoint");
    s = check_workspace(p->workspace, p->workspace_bytes,
                        sums ? im_expert_linear_grad_workspace(p->n, p->n_experts, p->in, p->out) : 0, 16);
    if (s != IM_OK) return s;
    if (p->n == 0 && !sums) return IM_OK;
    ExpertArgs a{};
    a.offsets = p->offsets;
    a.rows = p->rows;
    a.E = p->n_experts;
    a.n = (int)p->n;
    a.in = p->in;
    a.out = p->out;
    a.x = (const uint16_t *)p->x;
    a.ld_x = p->ld_x;
    if (!p->x && p->checkpoint) a.c = *p->checkpoint;
    a.w = (const uint16_t *)p->w;
    a.ld_w = p->ld_w;
    a.relu = p->relu_x != 0;
    a.dy = (const uint16_t *)p->dy;
    a.ld_dy = p->ld_dy;
    a.dx = (uint16_t *)p->dx;
    a.ld_dx = p->ld_dx;
    a.dw = p->dw;
    a.ld_dw = p->ld_dw;
    a.db = p->db;
    if (sums) {
        a.part = (float *)p->workspace;
        a.part_db = a.part + 2 * (int64_t)expert_grad_teams(p->n, p->n_experts, p->in, p->out) * p->out * pad4(p->in);
    }
    return launched(launch_expert_grad(a, (hipStream_t)stream), "expert_linear_grad launch");
}

}  // extern "C"
