// rms_kernels.hip -- root-mean-square norm of a residual stream and its gradient.  Each
// value is read once; bound by HBM.  Rows in teams of lanes as the layer norm's (team.h).
#include <algorithm>

#include "block8.h"
#include "recurrent.h"
#include "team.h"

namespace im {

// A piece's bytes to a row in 8 bits: the scale from the largest magnitude of the lanes on one
// 128-block (16, or the whole of a smaller team).  A lane writes the eight bytes of its own
// columns, zeros from the d-th on, and small teams walk on to the block's end.  The whole team
// calls.
template <int T, int W>
__device__ __forceinline__ void store_block8(const Mat8 &c, int64_t r, int d, const RowPiece<W> &pc, bool on,
                                             const float *v)
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, pc.own(k) ? magnitude(v[k]) : 0);
    const int s = block8_scale(lanes_max<T < 16 ? T : 16>(top));
    if (!on) return;
    // a piece that ends its row holds the columns from col on at its end
    u32x2_r q = block8_pack(v, s, W == NARROW ? pc.hi : 8);
    if constexpr (W != EVEN) {
        const uint64_t w = pc.lo >= 8 ? 0 : (q[0] | (uint64_t)q[1] << 32) >> (8 * pc.lo);
        q = u32x2_r{(uint32_t)w, (uint32_t)(w >> 32)};
    } else if (!pc.any()) {
        q = u32x2_r{0, 0};
    }
    const int pad = (d + 127) / 128 * 128;
    uint8_t *row = c.q + r * c.ld_q;
    if (pc.col < pad) *(u32x2_r *)(row + pc.col) = q;
    if constexpr (T < 16)
        for (int at = pc.col + 8 * T; at < pad; at += 8 * T) *(u32x2_r *)(row + at) = u32x2_r{0, 0};
    if ((pc.col & 127) == 0 && pc.col < d) c.scale[r * c.ld_scale + (pc.col >> 7)] = (uint8_t)s;
}

// ---------------------------------------------------------------------------
// h = x + residual, y = h rstd gamma from the unrounded sum.  65536 x 1024 bf16 with the residual, h
// and 8 bits out: 94 us, 471 MB at 5.0 TB/s; one row of 1024 floats: 1.9 us, the latency of a load, a
// sum and a store.
// ---------------------------------------------------------------------------
template <typename E, int T, int W, bool RES>
__global__ __launch_bounds__(norm_threads<T>) void rms_kernel(RmsArgs a)
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
    auto fetch_res = [&](int64_t r) { return load_raw((const E *)a.res + r * a.ld_res, pc, RES && r < a.n); };
    auto next = fetch(lead + ofs);
    auto next_res = fetch_res(lead + ofs);
    float ga[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) ga[k] = 1.0f;
    if (a.gamma) unpack8(load_raw(a.gamma, pc, true), ga);
    for (int64_t r0 = lead; r0 < a.n; r0 += step) {
        const int64_t r = r0 + ofs;
        const bool on = r < a.n;
        float v[8], q = 0.0f;
        unpack8(next, v);
        if constexpr (RES) {
            float t[8];
            unpack8(next_res, t);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += t[k];
        }
        if (r0 + step < a.n) {
            next = fetch(r + step);
            if constexpr (RES) next_res = fetch_res(r + step);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float t = W == EVEN || pc.own(k) ? v[k] : 0.0f;     // lanes past the row hold zeros
            q = fmaf(t, t, q);
        }
        const float rstd = 1.0f / sqrtf(row_sum<T>(q, lds, half) * a.inv_d + a.eps);
        if (on && Team<T>::lane() == 0 && a.rstd) a.rstd[r] = rstd;
        if (on && a.h) store_piece((E *)a.h + r * a.ld_h, pc, v);
        float y[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = v[k] * rstd * ga[k];
        if (on && a.y) store_piece((E *)a.y + r * a.ld_y, pc, y);
        if (a.y8.q) store_block8<T, W>(a.y8, r, a.d, pc, on, y);
    }
}

hipError_t launch_rms(const RmsArgs &a, bool f32, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n, pass_rows(a.d)), 256 * 32 * NORM_NT / block_threads(a.d));
    auto go = [&](auto t, auto w) {
        constexpr int T = decltype(t)::value, W = decltype(w)::value;
        const dim3 g((unsigned)blocks), b(norm_threads<T>);
        if (f32) {
            if (a.res) rms_kernel<float, T, W, true><<<g, b, 0, s>>>(a);
            else rms_kernel<float, T, W, false><<<g, b, 0, s>>>(a);
        } else {
            if (a.res) rms_kernel<uint16_t, T, W, true><<<g, b, 0, s>>>(a);
            else rms_kernel<uint16_t, T, W, false><<<g, b, 0, s>>>(a);
        }
    };
    by_width<NORM_LANES>(a.d, go);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The gradient: dx = dh + rstd (g - u sum (g u) / d), u = h rstd, g = dy gamma.  Each thread
// sums its columns' dgamma over its team's rows; the teams meet at the end and leave one row of
// partial sums a block, added up in float64 in a fixed order.  524288 x 512 bf16 with dh: 423 us
// and 6 for the sums, 2.15 GB at 5.0 TB/s; 4097 x 361 floats: 5.8 and 3.2 us, few rows a block and the
// second launch.
// ---------------------------------------------------------------------------
template <typename E, int T, int W, bool RES>
__global__ __launch_bounds__(norm_threads<T>) void rms_grad_kernel(RmsGradArgs a)
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
    decltype(load_raw((const E *)0, pc, true)) next_dy, next_h, next_dh;
    float next_rstd;
    auto fetch = [&](int64_t r) {
        const bool on = r < a.n;
        next_rstd = on ? a.rstd[r] : 0.0f;
        next_dy = load_raw((const E *)a.dy + r * a.ld_dy, pc, on);
        next_h = load_raw((const E *)a.h + r * a.ld_h, pc, on);
        if constexpr (RES) next_dh = load_raw((const E *)a.dh + r * a.ld_dh, pc, on);
    };
    fetch(lead + ofs);
    float ga[8], dg[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) ga[k] = 1.0f, dg[k] = 0.0f;
    if (a.gamma) unpack8(load_raw(a.gamma, pc, true), ga);
    for (int64_t r0 = lead; r0 < a.n; r0 += step) {
        const int64_t r = r0 + ofs;
        const bool on = r < a.n;
        const float rstd = next_rstd;
        float u[8], dy[8], dh[8], s = 0.0f;
        unpack8(next_dy, dy);
        unpack8(next_h, u);
        if constexpr (RES) {
            unpack8(next_dh, dh);
            // has arrived before the sum's barrier: where dx is dh, another wavefront may then store
            // the columns that two pieces of an odd row share
            asm volatile("" ::"v"(dh[0]), "v"(dh[7]));
        }
        fetch(r + step);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u[k] *= rstd;
            const float t = W == EVEN || pc.own(k) ? dy[k] : 0.0f;    // lanes past the row hold zeros
            dg[k] = fmaf(t, u[k], dg[k]);
            s = fmaf(t * ga[k], u[k], s);
        }
        if (a.dx) {
            s = row_sum<T>(s, lds, half) * a.inv_d;
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                o[k] = rstd * (dy[k] * ga[k] - u[k] * s);
                if constexpr (RES) o[k] += dh[k];
            }
            if (on) store_piece((E *)a.dx + r * a.ld_dx, pc, o);
        }
    }
    if (!a.part) return;
    // one block alone: its sums are the result
    float *sums = gridDim.x == 1 ? a.dgamma : a.part + (int64_t)blockIdx.x * a.d;
    if constexpr (G > 1) {
        // teams of a wavefront, then wavefronts or teams in order
        constexpr int V = T < 64 ? 64 : T;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float t = dg[k];
#pragma unroll
            for (int m = T; m < 64; m *= 2) t += __shfl_xor(t, m);
            if (threadIdx.x % V < T && pc.own(k)) lds[threadIdx.x / V * C + pc.at + k] = t;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.d; i += NORM_NT) {
            const float t = lds[i] + lds[C + i];
            sums[i] = G == 2 ? t : t + (lds[2 * C + i] + lds[3 * C + i]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (pc.own(k)) sums[pc.at + k] = dg[k];
    }
}

// As the layer norm's gradient: few rows in one block and one launch, up to 8 passes; else four
// passes a block at least and four blocks of 256 threads a CU at most.
int64_t rms_grad_blocks(int64_t n, int64_t d)
{
    if (n <= 8 * pass_rows(d)) return 1;
    return std::min(ceil_div(n, 4 * pass_rows(d)), 1024 * NORM_NT / block_threads(d));
}

hipError_t launch_rms_grad(const RmsGradArgs &a, bool f32, hipStream_t s)
{
    const int64_t blocks = rms_grad_blocks(a.n, a.d);
    auto go = [&](auto t, auto w) {
        constexpr int T = decltype(t)::value, W = decltype(w)::value;
        const dim3 g((unsigned)blocks), b(norm_threads<T>);
        if (f32) {
            if (a.dh) rms_grad_kernel<float, T, W, true><<<g, b, 0, s>>>(a);
            else rms_grad_kernel<float, T, W, false><<<g, b, 0, s>>>(a);
        } else {
            if (a.dh) rms_grad_kernel<uint16_t, T, W, true><<<g, b, 0, s>>>(a);
            else rms_grad_kernel<uint16_t, T, W, false><<<g, b, 0, s>>>(a);
        }
    };
    by_width<NORM_LANES>(a.d, go);
    if (a.part && blocks > 1) return launch_column_sums(ColumnSums{a.part, blocks, a.d, a.dgamma}, s);
    return hipGetLastError();
}

}  // namespace im
