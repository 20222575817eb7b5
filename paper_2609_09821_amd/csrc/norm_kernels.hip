// norm_kernels.hip -- layer norm, its gradient and the 8-bit checkpoint of an
// activation.  All three read each value once and are bound by HBM.
//
// A row belongs to a team of T lanes that holds it in registers, eight
// consecutive values a lane and chunk of 8 T columns: T = 4 .. 64 lanes for rows
// up to 8 T values (several rows a wavefront, so that narrow rows leave no lane
// idle), NC chunks of a wavefront up to 2048, and a block of 256 threads above,
// whose sums meet in LDS.  Four lanes then hold one 32-block of a checkpoint.
#include <algorithm>
#include <type_traits>

#include "expert.h"
#include "rows.h"

namespace im {

constexpr int NORM_NT = 256;

// Sum over the team.  T = 256: over the block, through `lds` (8 floats, the two
// halves used in turn, so that one barrier a sum is enough).
template <int T>
__device__ __forceinline__ float row_sum(float x, float *lds, int &half)
{
    if constexpr (T <= 64) {
        return team_sum<T>(x);
    } else {
        x = team_sum<64>(x);
        float *b = lds + 4 * half;
        half ^= 1;
        if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = x;
        __syncthreads();
        return (b[0] + b[1]) + (b[2] + b[3]);
    }
}

// Rows per block and pass, and a block's loop over them: every thread of a
// wavefront (of a block for T = 256) makes the same passes.
template <int T>
struct Team {
    static constexpr int ROWS = NORM_NT / T;
    __device__ static int lane() { return threadIdx.x % T; }
    __device__ static int64_t first() { return (int64_t)blockIdx.x * ROWS + threadIdx.x / T; }
};

// ---------------------------------------------------------------------------
// y = (x - mean) rstd gamma + beta, the variance about the mean (two passes over
// the registers: no cancellation), optionally the checkpoint of x.
// ---------------------------------------------------------------------------
template <typename E, int T, int NC, bool CK>
__global__ __launch_bounds__(NORM_NT) void norm_kernel(NormArgs a)
{
    __shared__ float lds[8];
    int half = 0;
    const int lane = Team<T>::lane();
    const int64_t step = (int64_t)gridDim.x * Team<T>::ROWS;
    int nv[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) nv[c] = a.d - (c * T + lane) * 8;
    // gamma and beta stay in registers over the rows where they are few
    constexpr bool KEEP = NC <= 2;
    float ga[KEEP ? NC : 1][8], be[KEEP ? NC : 1][8];
    auto affine = [&](int c, float *g, float *b) {
        const int col = (c * T + lane) * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) g[k] = 1.0f, b[k] = 0.0f;
        if (a.gamma) load8(a.gamma + col, nv[c], g);
        if (a.beta) load8(a.beta + col, nv[c], b);
    };
    if constexpr (KEEP)
#pragma unroll
        for (int c = 0; c < NC; ++c) affine(c, ga[c], be[c]);

    // the wavefront's first row decides (teams of one wavefront stay together)
    const int64_t lead = T <= 64 ? Team<T>::first() - (threadIdx.x & 63) / (T <= 64 ? T : 64) : Team<T>::first();
    const int64_t ofs = Team<T>::first() - lead;
    for (int64_t r0 = lead; r0 < a.n; r0 += step) {
        const int64_t r = r0 + ofs;
        const bool on = r < a.n;
        float v[NC][8];
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            load8((const E *)a.x + r * a.ld_x + (c * T + lane) * 8, on ? nv[c] : 0, v[c]);
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[c][k];
        }
        const float mean = row_sum<T>(s, lds, half) * a.inv_d;
        float q = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float t = k < nv[c] ? v[c][k] - mean : 0.0f;
                q = fmaf(t, t, q);
            }
        const float rstd = 1.0f / sqrtf(row_sum<T>(q, lds, half) * a.inv_d + a.eps);
        if (on && lane == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * T + lane) * 8;
            if constexpr (CK) {
                const int scale = ckpt_scale(ckpt_top(v[c]));
                if (on && nv[c] > 0) {
                    store8_bytes(a.c.q + r * a.c.ld_q + col, nv[c], ckpt_pack(v[c], scale));
                    if ((lane & 3) == 0) a.c.scale[r * a.c.ld_scale + (col >> 5)] = (uint8_t)scale;
                }
            }
            float g[8], b[8], y[8];
            if constexpr (KEEP) {
#pragma unroll
                for (int k = 0; k < 8; ++k) g[k] = ga[c][k], b[k] = be[c][k];
            } else {
                affine(c, g, b);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = fmaf((v[c][k] - mean) * rstd, g[k], b[k]);
            if (on) store8((E *)a.y + r * a.ld_y + col, nv[c], y);
        }
    }
}

// ---------------------------------------------------------------------------
// The gradient.  Each thread sums its columns' dgamma and dbeta over the rows of
// its team; the block's teams meet at the end and leave one row of partial sums,
// which norm_grad_sum_kernel adds up in float64 in the blocks' order.
// ---------------------------------------------------------------------------
template <typename E, int T, int NC, bool CK>
__global__ __launch_bounds__(NORM_NT) void norm_grad_kernel(NormGradArgs a)
{
    constexpr int W = (T < 64 ? T : 64) * NC * 8;    // columns of a wavefront
    __shared__ float lds[T <= 64 ? 4 * W : 8];
    int half = 0;
    const int lane = Team<T>::lane();
    const int64_t step = (int64_t)gridDim.x * Team<T>::ROWS;
    int nv[NC];
    float ga[NC][8], dg[NC][8], db[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * T + lane) * 8;
        nv[c] = a.d - col;
#pragma unroll
        for (int k = 0; k < 8; ++k) ga[c][k] = 1.0f, dg[c][k] = 0.0f, db[c][k] = 0.0f;
        if (a.gamma) load8(a.gamma + col, nv[c], ga[c]);
    }
    const int64_t lead = T <= 64 ? Team<T>::first() - (threadIdx.x & 63) / (T <= 64 ? T : 64) : Team<T>::first();
    const int64_t ofs = Team<T>::first() - lead;
    for (int64_t r0 = lead; r0 < a.n; r0 += step) {
        const int64_t r = r0 + ofs;
        const bool on = r < a.n;
        const float mean = on ? a.mean[r] : 0.0f, rstd = on ? a.rstd[r] : 0.0f;
        float h[NC][8], dy[NC][8];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * T + lane) * 8, m = on ? nv[c] : 0;
            load8((const E *)a.dy + r * a.ld_dy + col, m, dy[c]);
            if constexpr (CK) {
                u32x2_r q = load8_bytes(a.c.q + r * a.c.ld_q + col, m);
                const int scale = m > 0 ? a.c.scale[r * a.c.ld_scale + (col >> 5)] : 0;
                ckpt_unpack(q, scale, h[c]);
            } else {
                load8((const E *)a.x + r * a.ld_x + col, m, h[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // columns past the width have dy = 0; their h is held at 0 too
                h[c][k] = k < nv[c] ? (h[c][k] - mean) * rstd : 0.0f;
                const float g = dy[c][k] * ga[c][k];
                s1 += g;
                s2 = fmaf(g, h[c][k], s2);
                dg[c][k] = fmaf(dy[c][k], h[c][k], dg[c][k]);
                db[c][k] += dy[c][k];
            }
        if (a.dx) {
            s1 = row_sum<T>(s1, lds, half) * a.inv_d;
            s2 = row_sum<T>(s2, lds, half) * a.inv_d;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = rstd * (dy[c][k] * ga[c][k] - s1 - h[c][k] * s2);
                if (on) store8((E *)a.dx + r * a.ld_dx + (c * T + lane) * 8, nv[c], o);
            }
        }
    }
    if (!a.part) return;
    // one block alone: its sums are the result
    const bool alone = gridDim.x == 1;
    float *sums[2] = {alone ? a.dgamma : a.part + (int64_t)blockIdx.x * 2 * a.d,
                      alone ? a.dbeta : a.part + ((int64_t)blockIdx.x * 2 + 1) * a.d};
    if constexpr (T <= 64) {
        // teams of a wavefront, then the four wavefronts in order
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            auto &v = p ? db : dg;
            __syncthreads();
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float t = v[c][k];
#pragma unroll
                    for (int m = T; m < 64; m *= 2) t += __shfl_xor(t, m);
                    if ((threadIdx.x & 63) < T) lds[(threadIdx.x >> 6) * W + (c * T + lane) * 8 + k] = t;
                }
            __syncthreads();
            if (sums[p])
                for (int i = threadIdx.x; i < W && i < a.d; i += NORM_NT)
                    sums[p][i] = (lds[i] + lds[W + i]) + (lds[2 * W + i] + lds[3 * W + i]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (sums[0]) store8(sums[0] + (c * T + lane) * 8, nv[c], dg[c]);
            if (sums[1]) store8(sums[1] + (c * T + lane) * 8, nv[c], db[c]);
        }
    }
}

// Column sums of the partial rows: 64 columns a block, wavefront w takes rows w,
// w + 16, ...; the wavefronts' sums meet in LDS in order.
constexpr int NORM_SUM_WAVES = 16;
__global__ __launch_bounds__(64 * NORM_SUM_WAVES) void norm_grad_sum_kernel(const float *part, int rows, int d,
                                                                            float *dgamma, float *dbeta)
{
    __shared__ double lds[NORM_SUM_WAVES][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;
    double s = 0.0;
    if (col < 2 * d)
#pragma unroll 8
        for (int r = w; r < rows; r += NORM_SUM_WAVES) s += (double)part[(int64_t)r * 2 * d + col];
    lds[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < 2 * d) {
        for (int k = 1; k < NORM_SUM_WAVES; ++k) s += lds[k][lane];
        if (col < d) {
            if (dgamma) dgamma[col] = (float)s;
        } else if (dbeta) {
            dbeta[col - d] = (float)s;
        }
    }
}

template <int V>
using Int = std::integral_constant<int, V>;

// Calls f(T, NC) for rows of d values.
template <typename F>
void by_width(int64_t d, F &&f)
{
    if (d <= 32) f(Int<4>(), Int<1>());
    else if (d <= 64) f(Int<8>(), Int<1>());
    else if (d <= 128) f(Int<16>(), Int<1>());
    else if (d <= 256) f(Int<32>(), Int<1>());
    else if (d <= 512) f(Int<64>(), Int<1>());
    else if (d <= 1024) f(Int<64>(), Int<2>());
    else if (d <= 1536) f(Int<64>(), Int<3>());
    else if (d <= 2048) f(Int<64>(), Int<4>());
    else if (d <= 4096) f(Int<256>(), Int<2>());
    else f(Int<256>(), Int<4>());
}

// Rows that a block takes in one pass.
static int64_t pass_rows(int64_t d)
{
    int64_t t = 4;
    while (t < 64 && 8 * t < d) t *= 2;
    return NORM_NT / (d > 2048 ? 256 : t);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

hipError_t launch_norm(const NormArgs &a, bool f32, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n, pass_rows(a.d)), 256 * 8);
    auto go = [&](auto t, auto nc) {
        constexpr int T = decltype(t)::value, NC = decltype(nc)::value;
        const dim3 g((unsigned)blocks), b(NORM_NT);
        if (f32) {
            if (a.c.q) norm_kernel<float, T, NC, true><<<g, b, 0, s>>>(a);
            else norm_kernel<float, T, NC, false><<<g, b, 0, s>>>(a);
        } else {
            if (a.c.q) norm_kernel<uint16_t, T, NC, true><<<g, b, 0, s>>>(a);
            else norm_kernel<uint16_t, T, NC, false><<<g, b, 0, s>>>(a);
        }
    };
    by_width(a.d, go);
    return hipGetLastError();
}

// Few rows go to one block, which needs no second launch (4 us of the host): up to 8 passes.
// Else four passes a block at least, and four blocks a CU at most (two: 262144 x 64 and
// narrower stay as fast, 524288 x 512 takes 318 us for 262; eight: 302).
int64_t norm_grad_blocks(int64_t n, int64_t d)
{
    if (n <= 8 * pass_rows(d)) return 1;
    return std::max<int64_t>(1, std::min<int64_t>(ceil_div(n, 4 * pass_rows(d)), 1024));
}

hipError_t launch_norm_grad(const NormGradArgs &a, bool f32, hipStream_t s)
{
    const int64_t blocks = norm_grad_blocks(a.n, a.d);
    auto go = [&](auto t, auto nc) {
        constexpr int T = decltype(t)::value, NC = decltype(nc)::value;
        const dim3 g((unsigned)blocks), b(NORM_NT);
        if (f32) {
            if (a.x) norm_grad_kernel<float, T, NC, false><<<g, b, 0, s>>>(a);
            else norm_grad_kernel<float, T, NC, true><<<g, b, 0, s>>>(a);
        } else {
            if (a.x) norm_grad_kernel<uint16_t, T, NC, false><<<g, b, 0, s>>>(a);
            else norm_grad_kernel<uint16_t, T, NC, true><<<g, b, 0, s>>>(a);
        }
    };
    by_width(a.d, go);
    if (a.part && blocks > 1)
        norm_grad_sum_kernel<<<dim3((unsigned)ceil_div(2 * a.d, 64)), dim3(64 * NORM_SUM_WAVES), 0, s>>>(
            a.part, (int)blocks, a.d, a.dgamma, a.dbeta);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Checkpoints alone.  A team of T lanes walks a row in chunks of 8 T columns.
// ---------------------------------------------------------------------------
template <typename E, int T, bool STORE>
__global__ __launch_bounds__(NORM_NT) void ckpt_kernel(E *x, int64_t ld_x, int64_t n, int64_t d, im_checkpoint c)
{
    const int lane = threadIdx.x % T;
    const int64_t step = (int64_t)gridDim.x * (NORM_NT / T);
    const int64_t row0 = (int64_t)blockIdx.x * (NORM_NT / T) + threadIdx.x / T;
    for (int64_t r = row0; r < n; r += step) {
        E *xr = x + r * ld_x;
        int8_t *qr = c.q + r * c.ld_q;
        uint8_t *sr = c.scale + r * c.ld_scale;
        // a quad's lanes are on one 32-block and pass together
        for (int64_t b = 0; b < d; b += 8 * T) {
            const int64_t col = b + lane * 8;
            const int nv = (int)(d - col < 8 ? d - col : 8);
            float v[8];
            if constexpr (STORE) {
                load8(xr + col, nv, v);
                const int scale = ckpt_scale(ckpt_top(v));
                if (nv > 0) {
                    store8_bytes(qr + col, nv, ckpt_pack(v, scale));
                    if ((lane & 3) == 0) sr[col >> 5] = (uint8_t)scale;
                }
            } else if (nv > 0) {
                ckpt_unpack(load8_bytes(qr + col, nv), sr[col >> 5], v);
                store8(xr + col, nv, v);
            }
        }
    }
}

hipError_t launch_checkpoint(bool store, void *x, int64_t ld_x, bool f32, int64_t n, int64_t d,
                             const im_checkpoint &c, hipStream_t s)
{
    auto go = [&](auto t) {
        constexpr int T = decltype(t)::value;
        const dim3 g((unsigned)std::min<int64_t>(ceil_div(n, NORM_NT / T), 256 * 16)), b(NORM_NT);
        if (f32) {
            if (store) ckpt_kernel<float, T, true><<<g, b, 0, s>>>((float *)x, ld_x, n, d, c);
            else ckpt_kernel<float, T, false><<<g, b, 0, s>>>((float *)x, ld_x, n, d, c);
        } else {
            if (store) ckpt_kernel<uint16_t, T, true><<<g, b, 0, s>>>((uint16_t *)x, ld_x, n, d, c);
            else ckpt_kernel<uint16_t, T, false><<<g, b, 0, s>>>((uint16_t *)x, ld_x, n, d, c);
        }
    };
    if (d <= 32) go(Int<4>());
    else if (d <= 64) go(Int<8>());
    else if (d <= 128) go(Int<16>());
    else if (d <= 256) go(Int<32>());
    else go(Int<64>());
    return hipGetLastError();
}

}  // namespace im
