// norm_kernels.hip -- layer norm, its gradient and the 8-bit checkpoint of an
// activation.  All three read each value once and are bound by HBM.
//
// A row belongs to a team of T lanes that holds it in registers, eight consecutive
// values a lane: 4 .. 64 lanes (several rows a wavefront, so that narrow rows leave
// few lanes idle) or 2 .. 16 wavefronts of a block, whose sums meet in LDS.  Four
// lanes then hold one 32-block of a checkpoint.  Up to four pieces a lane, on fewer
// lanes, hold more registers: the gradient of 29296 rows of 4096 bf16 from their
// checkpoint took 155 us so and takes 118, of 117187 rows of 1024 123 and 112, of 96000
// of 2500 674 and 297; of 446096 rows of 538 floats 470 and 487 (back to back from a
// graph).
#include <algorithm>
#include <type_traits>

#include "expert.h"
#include "rows.h"

namespace im {

constexpr int NORM_NT = 256;
template <int T>
constexpr int norm_threads = T > NORM_NT ? T : NORM_NT;

// Sum over the team.  Teams of several wavefronts: through `lds` (one float a wavefront, in
// two halves used in turn, so that one barrier a sum is enough), in the wavefronts' order.
template <int T>
__device__ __forceinline__ float row_sum(float x, float *lds, int &half)
{
    if constexpr (T <= 64) {
        return team_sum<T>(x);
    } else {
        x = team_sum<64>(x);
        float *b = lds + norm_threads<T> / 64 * half;
        half ^= 1;
        if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = x;
        __syncthreads();
        b += threadIdx.x / T * (T / 64);
        float s = b[0];
#pragma unroll
        for (int w = 1; w < T / 64; ++w) s += b[w];
        return s;
    }
}

// Rows per block and pass, and a block's loop over them: every thread of a
// wavefront (of a block for teams of several) makes the same passes: as its first row does.
template <int T>
struct Team {
    static constexpr int ROWS = norm_threads<T> / T;
    __device__ static int lane() { return threadIdx.x % T; }
    __device__ static int offset() { return T <= 64 ? (threadIdx.x & 63) / T : threadIdx.x / T; }
    __device__ static int64_t lead() { return (int64_t)blockIdx.x * ROWS + threadIdx.x / T - offset(); }
};

// ---------------------------------------------------------------------------
// y = (x - mean) rstd gamma + beta, the variance about the mean (two passes over
// the registers: no cancellation), optionally the checkpoint of x.  65536 x 1024 bf16
// with the checkpoint: 62 us, 338 MB at 5.4 TB/s; one row of 1024 floats: 2.1 us, the
// latency of a load, two sums and a store; 3478260 x 69 bf16 231 us, 4.3 TB/s.
// ---------------------------------------------------------------------------
template <typename E, int T, int W, bool CK>
__global__ __launch_bounds__(norm_threads<T>) void norm_kernel(NormArgs a)
{
    typedef RowPiece<W> P;
    __shared__ float lds[2 * norm_threads<T> / 64];
    int half = 0;
    const int64_t step = (int64_t)gridDim.x * Team<T>::ROWS, lead = Team<T>::lead();
    const int ofs = Team<T>::offset();
    P pc;
    pc.init(Team<T>::lane() * 8, a.d);
    // the next row is on its way while this one is worked on
    auto fetch = [&](int64_t r) { return load_raw((const E *)a.x + r * a.ld_x, pc, r < a.n); };
    auto next = fetch(lead + ofs);
    float ga[8], be[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) ga[k] = 1.0f, be[k] = 0.0f;
    if (a.gamma) unpack8(load_raw(a.gamma, pc, true), ga);
    if (a.beta) unpack8(load_raw(a.beta, pc, true), be);
    for (int64_t r0 = lead; r0 < a.n; r0 += step) {
        const int64_t r = r0 + ofs;
        const bool on = r < a.n;
        float v[8], s = 0.0f, q = 0.0f;
        unpack8(next, v);
        if (r0 + step < a.n) next = fetch(r + step);
#pragma unroll
        for (int k = 0; k < 8; ++k) s += W == EVEN || pc.own(k) ? v[k] : 0.0f;    // lanes past the row hold zeros
        const float mean = row_sum<T>(s, lds, half) * a.inv_d;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float t = pc.own(k) ? v[k] - mean : 0.0f;
            q = fmaf(t, t, q);
        }
        const float rstd = 1.0f / sqrtf(row_sum<T>(q, lds, half) * a.inv_d + a.eps);
        if (on && Team<T>::lane() == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        if constexpr (CK) store_bytes(a.c.q + r * a.c.ld_q, a.c.scale + r * a.c.ld_scale, pc, on, v);
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = fmaf((v[k] - mean) * rstd, ga[k], be[k]);
        if (on) store_piece((E *)a.y + r * a.ld_y, pc, y);
    }
}

// ---------------------------------------------------------------------------
// The gradient.  Each thread sums its columns' dgamma and dbeta over the rows of
// its team; the block's teams meet at the end and leave one row of partial sums,
// which norm_grad_sum_kernel adds up in float64 in the blocks' order: no atomics, the
// same bits in every run.  524288 x 512 bf16 from a checkpoint: 254 us with 8 for the
// sum, 1.35 GB at 5.3 TB/s; without the next row's loads in flight 18 us more.  Odd widths
// that fill little more than half of a team are bound by its instructions (538: 3.9 TB/s,
// 69: 3.6).
// ---------------------------------------------------------------------------
template <typename E, int T, int W, bool CK>
__global__ __launch_bounds__(norm_threads<T>) void norm_grad_kernel(NormGradArgs a)
{
    typedef RowPiece<W> P;
    constexpr int G = T <= 64 ? 4 : norm_threads<T> / T;    // wavefronts or teams whose sums meet
    constexpr int C = T * 8, WAVES = norm_threads<T> / 64;
    __shared__ float lds[G > 1 ? G * C : 2 * WAVES];
    int half = 0;
    const int64_t step = (int64_t)gridDim.x * Team<T>::ROWS, lead = Team<T>::lead();
    const int ofs = Team<T>::offset();
    P pc;
    pc.init(Team<T>::lane() * 8, a.d);
    // the next row is on its way while this one is worked on
    decltype(load_raw((const E *)0, pc, true)) next_dy, next_x;
    RawBytes next_q;
    float next_mean, next_rstd;
    auto fetch = [&](int64_t r) {
        const bool on = r < a.n;
        next_mean = on ? a.mean[r] : 0.0f, next_rstd = on ? a.rstd[r] : 0.0f;
        next_dy = load_raw((const E *)a.dy + r * a.ld_dy, pc, on);
        if constexpr (CK) next_q = load_bytes(a.c.q + r * a.c.ld_q, a.c.scale + r * a.c.ld_scale, pc, on);
        else next_x = load_raw((const E *)a.x + r * a.ld_x, pc, on);
    };
    fetch(lead + ofs);
    float ga[8], dg[8], db[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) ga[k] = 1.0f, dg[k] = 0.0f, db[k] = 0.0f;
    if (a.gamma) unpack8(load_raw(a.gamma, pc, true), ga);
    for (int64_t r0 = lead; r0 < a.n; r0 += step) {
        const int64_t r = r0 + ofs;
        const bool on = r < a.n;
        const float mean = next_mean, rstd = next_rstd;
        float h[8], dy[8], s1 = 0.0f, s2 = 0.0f;
        unpack8(next_dy, dy);
        if constexpr (CK) unpack8(next_q, pc, h);
        else unpack8(next_x, h);
        fetch(r + step);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            h[k] = (h[k] - mean) * rstd;
            const float t = W == EVEN || pc.own(k) ? dy[k] : 0.0f;    // lanes past the row hold zeros
            const float g = t * ga[k];
            s1 += g;
            s2 = fmaf(g, h[k], s2);
            dg[k] = fmaf(t, h[k], dg[k]);
            db[k] += t;
        }
        if (a.dx) {
            s1 = row_sum<T>(s1, lds, half) * a.inv_d;
            s2 = row_sum<T>(s2, lds, half) * a.inv_d;
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = rstd * (dy[k] * ga[k] - s1 - h[k] * s2);
            if (on) store_piece((E *)a.dx + r * a.ld_dx, pc, o);
        }
    }
    if (!a.part) return;
    // one block alone: its sums are the result
    const bool alone = gridDim.x == 1;
    float *sums[2] = {alone ? a.dgamma : a.part + (int64_t)blockIdx.x * 2 * a.d,
                      alone ? a.dbeta : a.part + ((int64_t)blockIdx.x * 2 + 1) * a.d};
    if constexpr (G > 1) {
        // teams of a wavefront, then wavefronts or teams in order
        constexpr int V = T < 64 ? 64 : T;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float t = p ? db[k] : dg[k];
#pragma unroll
                for (int m = T; m < 64; m *= 2) t += __shfl_xor(t, m);
                if (threadIdx.x % V < T && pc.own(k)) lds[threadIdx.x / V * C + pc.at + k] = t;
            }
            __syncthreads();
            if (sums[p])
                for (int i = threadIdx.x; i < a.d; i += NORM_NT) {
                    const float t = lds[i] + lds[C + i];
                    sums[p][i] = G == 2 ? t : t + (lds[2 * C + i] + lds[3 * C + i]);
                }
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (pc.own(k)) {
                if (sums[0]) sums[0][pc.at + k] = dg[k];
                if (sums[1]) sums[1][pc.at + k] = db[k];
            }
    }
}

// Column sums of the partial rows: 64 columns a block, wavefront w takes rows w,
// w + 16, ...; the wavefronts' sums meet in LDS in order.  1024 rows of 512: 8 us, of
// which most is the latency of 64 loads in turn by each of few blocks.
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

// Lanes of a team for rows of d values.
static int64_t team_lanes(int64_t d)
{
    int64_t t = 4;
    while (8 * t < d) t *= 2;
    return t;
}

// Calls f(T, W) for rows of d values, T up to MOST lanes (which walk longer rows).
template <int MOST, int T = 4, typename F>
void by_width(int64_t d, F &&f)
{
    if constexpr (T < MOST)
        if (8 * T < d) return by_width<MOST, 2 * T>(d, f);
    if constexpr (T == 4) f(Int<T>(), Int<NARROW>());
    else d % 8 ? f(Int<T>(), Int<ODD>()) : f(Int<T>(), Int<EVEN>());
}
constexpr int NORM_LANES = IM_NORM_MAX_WIDTH / 8;

// Threads of a block, and rows that it takes in one pass.
static int64_t block_threads(int64_t d) { return std::max<int64_t>(NORM_NT, team_lanes(d)); }
static int64_t pass_rows(int64_t d) { return block_threads(d) / team_lanes(d); }

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

hipError_t launch_norm(const NormArgs &a, bool f32, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n, pass_rows(a.d)), 256 * 32 * NORM_NT / block_threads(a.d));
    auto go = [&](auto t, auto w) {
        constexpr int T = decltype(t)::value, W = decltype(w)::value;
        const dim3 g((unsigned)blocks), b(norm_threads<T>);
        if (f32) {
            if (a.c.q) norm_kernel<float, T, W, true><<<g, b, 0, s>>>(a);
            else norm_kernel<float, T, W, false><<<g, b, 0, s>>>(a);
        } else {
            if (a.c.q) norm_kernel<uint16_t, T, W, true><<<g, b, 0, s>>>(a);
            else norm_kernel<uint16_t, T, W, false><<<g, b, 0, s>>>(a);
        }
    };
    by_width<NORM_LANES>(a.d, go);
    return hipGetLastError();
}

// Few rows go to one block, which needs no second launch (4 us of the host): up to 8 passes.
// Else four passes a block at least, and four blocks of 256 threads a CU at most (with five,
// which bf16 allows, 524288 x 512 takes 270 us for 257).
int64_t norm_grad_blocks(int64_t n, int64_t d)
{
    if (n <= 8 * pass_rows(d)) return 1;
    return std::min(ceil_div(n, 4 * pass_rows(d)), 1024 * NORM_NT / block_threads(d));
}

hipError_t launch_norm_grad(const NormGradArgs &a, bool f32, hipStream_t s)
{
    const int64_t blocks = norm_grad_blocks(a.n, a.d);
    auto go = [&](auto t, auto w) {
        constexpr int T = decltype(t)::value, W = decltype(w)::value;
        const dim3 g((unsigned)blocks), b(norm_threads<T>);
        if (f32) {
            if (a.x) norm_grad_kernel<float, T, W, false><<<g, b, 0, s>>>(a);
            else norm_grad_kernel<float, T, W, true><<<g, b, 0, s>>>(a);
        } else {
            if (a.x) norm_grad_kernel<uint16_t, T, W, false><<<g, b, 0, s>>>(a);
            else norm_grad_kernel<uint16_t, T, W, true><<<g, b, 0, s>>>(a);
        }
    };
    by_width<NORM_LANES>(a.d, go);
    if (a.part && blocks > 1)
        norm_grad_sum_kernel<<<dim3((unsigned)ceil_div(2 * a.d, 64)), dim3(64 * NORM_SUM_WAVES), 0, s>>>(
            a.part, (int)blocks, a.d, a.dgamma, a.dbeta);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Checkpoints alone.  A team of up to CKPT_LANES lanes walks a row in chunks of 8 T columns.
// 262144 x 1024 bf16: 146 us to store, 140 us to restore, 814 MB each way.
// ---------------------------------------------------------------------------
constexpr int CKPT_LANES = 64;
template <typename E, int T, int W, bool STORE>
__global__ __launch_bounds__(NORM_NT) void ckpt_kernel(E *x, int64_t ld_x, int64_t n, int64_t d, im_checkpoint c)
{
    static_assert(T <= CKPT_LANES && NORM_NT % T == 0, "whole teams in a block, each in one wavefront");
    const int lane = threadIdx.x % T;
    const int64_t step = (int64_t)gridDim.x * (NORM_NT / T);
    const int64_t row0 = (int64_t)blockIdx.x * (NORM_NT / T) + threadIdx.x / T;
    for (int64_t r = row0; r < n; r += step) {
        E *xr = x + r * ld_x;
        int8_t *qr = c.q + r * c.ld_q;
        uint8_t *sr = c.scale + r * c.ld_scale;
        // a quad's lanes are on one 32-block and pass together
        for (int64_t b = 0; b < d; b += 8 * T) {
            RowPiece<W> p;
            p.init((int)b + lane * 8, (int)d);
            float v[8];
            if constexpr (STORE) {
                unpack8(load_raw((const E *)xr, p, true), v);
                store_bytes(qr, sr, p, true, v);
            } else {
                unpack8(load_bytes(qr, sr, p, true), p, v);
                store_piece(xr, p, v);
            }
        }
    }
}

hipError_t launch_checkpoint(bool store, void *x, int64_t ld_x, bool f32, int64_t n, int64_t d,
                             const im_checkpoint &c, hipStream_t s)
{
    auto go = [&](auto t, auto w) {
        constexpr int T = decltype(t)::value, W = decltype(w)::value;
        const dim3 g((unsigned)std::min<int64_t>(ceil_div(n, NORM_NT / T), 256 * 64)), b(NORM_NT);
        if (f32) {
            if (store) ckpt_kernel<float, T, W, true><<<g, b, 0, s>>>((float *)x, ld_x, n, d, c);
            else ckpt_kernel<float, T, W, false><<<g, b, 0, s>>>((float *)x, ld_x, n, d, c);
        } else {
            if (store) ckpt_kernel<uint16_t, T, W, true><<<g, b, 0, s>>>((uint16_t *)x, ld_x, n, d, c);
            else ckpt_kernel<uint16_t, T, W, false><<<g, b, 0, s>>>((uint16_t *)x, ld_x, n, d, c);
        }
    };
    by_width<CKPT_LANES>(d, go);
    return hipGetLastError();
}

}  // namespace im
