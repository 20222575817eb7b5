// expert.h -- argument blocks and host launchers of the layers of experts
// (expert_kernels.hip, norm_kernels.hip), shared with their C ABI (expert_api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/instantmimic.h"

namespace im {

// Message of the calling thread's last failure (api.hip); returns s.
im_status api_fail(im_status s, const char *msg);
im_status api_hip_fail(hipError_t e, const char *what);

// Values of a checkpoint that share a scale.
constexpr int CKPT_BLOCK = 32;

struct NormArgs {
    int64_t n;
    int d;
    float eps, inv_d;
    const void *x;
    int64_t ld_x;
    const float *gamma, *beta;   // null: 1 and 0
    void *y;
    int64_t ld_y;
    float *mean, *rstd;          // null: not written
    im_checkpoint c;             // q null: none
};
hipError_t launch_norm(const NormArgs &a, bool f32, hipStream_t s);

struct NormGradArgs {
    int64_t n;
    int d;
    float inv_d;
    const void *dy;
    int64_t ld_dy;
    const void *x;               // null: from the checkpoint
    int64_t ld_x;
    im_checkpoint c;
    const float *gamma;          // null: 1
    const float *mean, *rstd;
    void *dx;                    // null: not wanted
    int64_t ld_dx;
    float *dgamma, *dbeta;       // null: not wanted
    float *part;                 // [norm_grad_blocks][2][d]; null: neither is wanted
};
int64_t norm_grad_blocks(int64_t n, int64_t d);
hipError_t launch_norm_grad(const NormGradArgs &a, bool f32, hipStream_t s);

hipError_t launch_checkpoint(bool store, void *x, int64_t ld_x, bool f32, int64_t n, int64_t d,
                             const im_checkpoint &c, hipStream_t s);

// Rows by expert: blocks of a launch over n rows; where there are several, their counts are
// left in `count`, [blocks][n_experts + 1].
int64_t group_blocks(int64_t n);
hipError_t launch_group_rows(const int32_t *expert, int64_t n, int n_experts, int32_t *offsets,
                             int32_t *rows, int32_t *count, hipStream_t s);

struct ExpertArgs {
    const int32_t *offsets, *rows;   // rows null: the identity
    int E;
    int n;
    int in, out;
    const uint16_t *x;               // [n][in] bf16 (null: from q, scale)
    int64_t ld_x;
    im_checkpoint c;
    const uint16_t *w;               // [E][out][in]
    int64_t ld_w;
    const float *bias;               // [E][out] or null
    int relu;                        // forward: of y; gradient: x is a ReLU's output
    void *y;                         // [n][out]
    int64_t ld_y;
    int y_f32;
    const uint16_t *dy;              // [n][out]
    int64_t ld_dy;
    uint16_t *dx;                    // [n][in]
    int64_t ld_dx;
    float *dw;                       // [E][out][in], null: not wanted
    int64_t ld_dw;
    float *db;                       // [E][out], null: not wanted
    // weight gradient: parts of the experts that several teams' runs share, 2 slots a team of
    // [out][in4] (in4 = in rounded up to 4) and of [out]
    float *part, *part_db;
};
hipError_t launch_expert_linear(const ExpertArgs &a, hipStream_t s);
// Teams of blocks among which the weight gradient's rows are divided (0: one for each expert).
int expert_grad_teams(int64_t n, int n_experts, int in, int out);
hipError_t launch_expert_grad(const ExpertArgs &a, hipStream_t s);

}  // namespace im
