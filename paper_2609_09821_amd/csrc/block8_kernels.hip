// block8_kernels.hip -- a matrix in 8 bits: stored, as it lies and transposed, and
// restored.  Each value is read once; bound by HBM.
#include <algorithm>
#include <type_traits>

#include "block8.h"
#include "recurrent.h"

namespace im {

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------
// Stores.  A block of 256 threads takes 128 rows x 128 columns: thread (g, l) = (t / 16,
// t % 16) holds eight values of each of the rows 8 g .. 8 g + 7, columns 8 l .. 8 l + 7, in
// registers.  A row's block is 16 neighbouring lanes; a column's meets in LDS, as does the
// whole tile's where it has one scale.  The transposed bytes are put together from a thread's
// eight rows and pass through LDS, so that both outputs leave in whole 128-byte blocks.
// C, TR: which outputs; SQUARE: one scale a tile; MASK: x counts as 0 where not y > 0.
// ---------------------------------------------------------------------------
constexpr int ST_PITCH = 128 + 16;      // bytes of a transposed column in LDS
template <typename E, bool C, bool TR, bool SQUARE, bool MASK>
__global__ __launch_bounds__(256) void block8_store_kernel(StoreArgs a, int64_t col_tiles, int64_t tiles)
{
    __shared__ __attribute__((aligned(16))) uint8_t bytes[TR ? 128 * ST_PITCH : 16];
    __shared__ uint32_t tops[16][128];
    __shared__ float sums[16][128];
    const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile / col_tiles * 128, c0 = tile % col_tiles * 128;
        const int64_t col = c0 + 8 * l;
        const int nv = (int)min((int64_t)8, a.d - col);      // columns, may be none
        const int rows = (int)min((int64_t)128, a.n - r0);
        float v[8][8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int r = 8 * g + k;
            const int have = r < rows ? nv : 0;
            load8((const E *)a.x + (r0 + r) * a.ld_x + col, have, v[k]);
            if constexpr (MASK) {
                float y[8];
                load8((const E *)a.y + (r0 + r) * a.ld_y + col, have, y);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] = y[j] > 0.0f ? v[k][j] : 0.0f;
            }
        }
        // largest magnitudes of the rows, of the columns
        uint32_t across[8], down[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) across[k] = down[k] = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t m = magnitude(v[k][j]);
                across[k] = max(across[k], m);
                down[j] = max(down[j], m);
            }
        if (a.sums) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) s += v[k][j];
                sums[g][8 * l + j] = s;
            }
        }
        if constexpr (TR || SQUARE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) tops[g][8 * l + j] = down[j];
        }
        if (TR || SQUARE || a.sums) __syncthreads();
        if (a.sums && threadIdx.x < 128 && c0 + threadIdx.x < a.d) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) s += sums[k][threadIdx.x];
            a.sums[r0 / 128 * a.d + c0 + threadIdx.x] = s;
        }
        int whole = 0;
        if constexpr (SQUARE) {
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) m = max(m, tops[k][threadIdx.x & 127]), m = max(m, tops[k + 8][threadIdx.x & 127]);
#pragma unroll
            for (int b = 1; b < 64; b *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, b));
            // the wavefronts' two halves of the columns
            __syncthreads();
            if ((threadIdx.x & 63) == 0) tops[0][threadIdx.x >> 6] = m;
            __syncthreads();
            whole = block8_scale(max(tops[0][0], tops[0][1]));
        }
        if constexpr (C) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = 8 * g + k;
                const int s = SQUARE ? whole : block8_scale(lanes_max<16>(across[k]));
                if (r >= rows) continue;
                *(u32x2_r *)(a.c.q + (r0 + r) * a.c.ld_q + col) = block8_pack(v[k], s, nv);
                if (!SQUARE && l == 0) a.c.scale[(r0 + r) * a.c.ld_scale + c0 / 128] = (uint8_t)s;
            }
            if (SQUARE && threadIdx.x == 0) a.c.scale[r0 / 128 * a.c.ld_scale + c0 / 128] = (uint8_t)whole;
        }
        if constexpr (TR) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int s = whole;
                if constexpr (!SQUARE) {
                    uint32_t m = 0;
#pragma unroll
                    for (int k = 0; k < 16; ++k) m = max(m, tops[k][8 * l + j]);
                    s = block8_scale(m);
                    if (g == 0 && j < nv) a.t.scale[(col + j) * a.t.ld_scale + r0 / 128] = (uint8_t)s;
                }
                float w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = v[k][j];
                *(u32x2_r *)(bytes + (8 * l + j) * ST_PITCH + 8 * g) = block8_pack(w, s, min(max(rows - 8 * g, 0), 8));
            }
            if (SQUARE && threadIdx.x == 0) a.t.scale[c0 / 128 * a.t.ld_scale + r0 / 128] = (uint8_t)whole;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = u * 32 + (threadIdx.x >> 3), at = threadIdx.x % 8 * 16;
                if (c0 + c < a.d)
                    *(u32x4_r *)(a.t.q + (c0 + c) * a.t.ld_q + r0 + at) = *(const u32x4_r *)(bytes + c * ST_PITCH + at);
            }
        }
        if (tile + gridDim.x < tiles) __syncthreads();
    }
}

template <typename E>
static void store_by(const StoreArgs &a, int64_t cols, int64_t tiles, hipStream_t s)
{
    // the loop over tiles is for more than a launch can have
    const dim3 g((unsigned)std::min<int64_t>(tiles, 1 << 22));
    const bool square = (a.c.q ? a.c.shift : a.t.shift) != 0, mask = a.y != nullptr;
    auto go = [&](auto c, auto t) {
        constexpr bool C = decltype(c)::value, T = decltype(t)::value;
        // only a gradient is masked, and its blocks lie along rows
        if (square) block8_store_kernel<E, C, T, true, false><<<g, dim3(256), 0, s>>>(a, cols, tiles);
        else if (mask) block8_store_kernel<E, C, T, false, true><<<g, dim3(256), 0, s>>>(a, cols, tiles);
        else block8_store_kernel<E, C, T, false, false><<<g, dim3(256), 0, s>>>(a, cols, tiles);
    };
    const std::true_type yes;
    const std::false_type no;
    if (a.c.q && a.t.q) go(yes, yes);
    else if (a.c.q) go(yes, no);
    else if (a.t.q) go(no, yes);
    else if (mask) block8_store_kernel<E, false, false, false, true><<<g, dim3(256), 0, s>>>(a, cols, tiles);
    else block8_store_kernel<E, false, false, false, false><<<g, dim3(256), 0, s>>>(a, cols, tiles);
}

hipError_t launch_block8_store(const StoreArgs &a, bool f32, hipStream_t s)
{
    const int64_t cols = ceil_div(a.d, 128);
    const int64_t tiles = ceil_div(a.n, 128) * cols;
    if (f32) store_by<float>(a, cols, tiles, s);
    else store_by<uint16_t>(a, cols, tiles, s);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Restores: 16 lanes a block of 128 values.
// ---------------------------------------------------------------------------
template <typename E>
__global__ __launch_bounds__(256) void block8_load_kernel(Mat8 c, int64_t n, int64_t d, E *x, int64_t ld_x)
{
    const int64_t cols = (d + 127) / 128, all = n * cols;
    for (int64_t b = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); b < all; b += (int64_t)gridDim.x * 16) {
        const int64_t r = b / cols, k = b - r * cols, col = k * 128 + (threadIdx.x & 15) * 8;
        const int nv = (int)min((int64_t)8, d - col);
        if (nv <= 0) continue;
        const u32x2_r q = *(const u32x2_r *)(c.q + r * c.ld_q + col);
        float v[8];
        block8_unpack(q, c.scale[(r >> c.shift) * c.ld_scale + k], v);
        store8(x + r * ld_x + col, nv, v);
    }
}

hipError_t launch_block8_load(const Mat8 &c, int64_t n, int64_t d, void *x, int64_t ld_x, bool f32, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(ceil_div(n, 16) * ceil_div(d, 128), 256 * 64);
    const dim3 g((unsigned)blocks), b(256);
    if (f32) block8_load_kernel<float><<<g, b, 0, s>>>(c, n, d, (float *)x, ld_x);
    else block8_load_kernel<uint16_t><<<g, b, 0, s>>>(c, n, d, (uint16_t *)x, ld_x);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Column sums of partial rows: 64 columns a block, wavefront w takes rows w, w + 16, ..;
// the wavefronts' sums meet in LDS in order.
// ---------------------------------------------------------------------------
constexpr int SUM_WAVES = 16;
__global__ __launch_bounds__(64 * SUM_WAVES) void column_sums_kernel(const float *part, int64_t rows, int64_t d,
                                                                     float *sums)
{
    __shared__ double lds[SUM_WAVES][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (col < d)
#pragma unroll 8
        for (int64_t r = w; r < rows; r += SUM_WAVES) s += (double)part[r * d + col];
    lds[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < d) {
        for (int k = 1; k < SUM_WAVES; ++k) s += lds[k][lane];
        sums[col] = (float)s;
    }
}

hipError_t launch_column_sums(const float *part, int64_t rows, int64_t d, float *sums, hipStream_t s)
{
    column_sums_kernel<<<dim3((unsigned)ceil_div(d, 64)), dim3(64 * SUM_WAVES), 0, s>>>(part, rows, d, sums);
    return hipGetLastError();
}

}  // namespace im
