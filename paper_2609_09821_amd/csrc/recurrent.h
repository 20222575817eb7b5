// recurrent.h -- argument blocks and host launchers of a recurrent policy's blocks
// (block8_kernels.hip, linear8_kernels.hip, rms_kernels.hip, scan_kernels.hip), shared
// with their C ABI (recurrent_api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/instantmimic.h"

namespace im {

// Message of the calling thread's last failure (api.hip); returns s.
im_status api_fail(im_status s, const char *msg);
im_status api_hip_fail(hipError_t e, const char *what);

// A matrix in 8 bits as the kernels take it: row r's scales are at (r >> shift) * ld_scale.
struct Mat8 {
    uint8_t *q, *scale;     // q null: none
    int64_t ld_q, ld_scale;
    int shift;              // 0: a scale for each row, 7: for 128 rows
};
inline Mat8 mat8(const im_block8 *b)
{
    if (!b) return Mat8{};
    return Mat8{b->q, b->scale, b->ld_q, b->ld_scale, b->rows == IM_BLOCK8 ? 7 : 0};
}

struct StoreArgs {
    const void *x;
    int64_t ld_x;
    const void *y;           // not null: x counts as 0 where not y > 0
    int64_t ld_y;
    int64_t n, d;
    Mat8 c, t;
    float *sums;             // [ceil(n / 128)][d]: column sums of each 128 rows, or null
};
hipError_t launch_block8_store(const StoreArgs &a, bool f32, hipStream_t s);
hipError_t launch_block8_load(const Mat8 &c, int64_t n, int64_t d, void *x, int64_t ld_x, bool f32, hipStream_t s);

struct RmsArgs {
    int64_t n;
    int d;
    float eps, inv_d;
    const void *x;
    int64_t ld_x;
    const void *res;         // null: none
    int64_t ld_res;
    const float *gamma;      // null: 1
    void *h;                 // null: not written, as y, rstd, y8
    int64_t ld_h;
    void *y;
    int64_t ld_y;
    float *rstd;
    Mat8 y8;
};
hipError_t launch_rms(const RmsArgs &a, bool f32, hipStream_t s);

struct RmsGradArgs {
    int64_t n;
    int d;
    float inv_d;
    const void *dy;
    int64_t ld_dy;
    const void *h;
    int64_t ld_h;
    const void *dh;          // null: none
    int64_t ld_dh;
    const float *gamma;      // null: 1
    const float *rstd;
    void *dx;                // null: not wanted
    int64_t ld_dx;
    float *dgamma;           // null: not wanted
    float *part;             // [rms_grad_blocks][d]
};
int64_t rms_grad_blocks(int64_t n, int64_t d);
hipError_t launch_rms_grad(const RmsGradArgs &a, bool f32, hipStream_t s);

// sums[col] = the sum of part[row][col] over the rows, in float64 in a fixed order.
struct ColumnSums {
    const float *part;
    int64_t rows, d;
    float *sums;             // null: not wanted
};
hipError_t launch_column_sums(const ColumnSums &c, hipStream_t s);

// C[q][p] = sum_k Q[q][k] P[p][k]: rows of Q are y's rows, rows of P its columns.
struct Linear8Args {
    int64_t n, out;          // rows and columns of y
    int64_t steps;           // blocks of 128 along k
    Mat8 q, p;
    const float *bias;       // null: none
    int relu;
    void *y;                 // null: not written
    int64_t ld_y;
    int y_f32;
    Mat8 y8;
    float *part;             // parts of y where k is split: [splits][n][out4]
    int splits;
};
// `splits` parts of k pay for a float y of few tiles and a long k.
int linear8_splits(int64_t n, int64_t out, int64_t steps);
hipError_t launch_linear8(const Linear8Args &a, hipStream_t s);
// A layer's gradients: dx and dw (y null: not wanted; dw in its splits) and db's column sums.
hipError_t launch_linear8_grad(const Linear8Args &dx, const Linear8Args &dw, const ColumnSums &c, hipStream_t s);

struct ScanArgs {
    int64_t T, n, d;
    const void *gate, *x;
    int64_t st_gate, ld_gate, st_x, ld_x;
    const uint8_t *term, *trunc;   // null: none
    int64_t ld_flags;
    const float *state;            // null: 0
    void *h;
    int64_t st_h, ld_h;
    float *state_out, *keep;       // null: not wanted
    // gradient alone: dh; keep is an input, state and state_out are dstate and dstate_out
    const void *dh;
    int64_t st_dh, ld_dh;
    void *dgate, *dx;
    int64_t st_dgate, ld_dgate, st_dx, ld_dx;
    // steps of a chunk, chunks, and each chunk's map of the state: [chunks][2][n d]
    int64_t chunk, chunks;
    float *maps;
};
// Steps of a chunk, a multiple of IM_SCAN_KEEP; T or more: one chunk.
int64_t scan_chunk(int64_t T, int64_t n, int64_t d);
// Bytes of the maps that any call of at most T steps, n envs and d values takes.
int64_t scan_workspace_bound(int64_t T, int64_t n, int64_t d);
hipError_t launch_scan(const ScanArgs &a, bool grad, bool f32, hipStream_t s);

}  // namespace im
