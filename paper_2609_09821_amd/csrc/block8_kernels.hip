// block8_kernels.hip -- a matrix in 8 bits: stored, as it lies and transposed, and
// restored.  Each value is read once; bound by HBM.
#include <algorithm>
#include <type_traits>

#include "block8.h"
#include "recurrent.h"

namespace im {

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------
// Stores.  A block takes 128 rows x 128 columns: thread (g, l) = (t / 16, t % 16) holds eight
// values of each of the rows 4 g .. 4 g + 3, columns 8 l .. 8 l + 7, in registers.  A row's block
// is 16 neighbouring lanes; a column's meets in LDS, as does the whole tile's where it has one scale.
// The transposed bytes are put together from a thread's four rows and pass through LDS, so that
// both outputs leave in whole 128-byte blocks.
// 65536 x 512 bf16 with a mask, both outputs and column sums: 46 us, 202 MB at 4.4 TB/s; 4095 x 1024 both
// ways 10.2 us, one tile a CU from load to store.  With 256 threads of eight rows, which hold twice the
// registers, 57 and 12 us.  Loads without branches in whole tiles gained nothing (49 and 10.2 us).
// C, TR: which outputs; SQUARE: one scale a tile; MASK: x counts as 0 where not y > 0.
// ---------------------------------------------------------------------------
constexpr int ST_NT = 512, ST_ROWS = 4, ST_GROUPS = ST_NT / 16;
constexpr int ST_PITCH = 128 + 16;      // bytes of a transposed column in LDS
constexpr int ST_WORDS = 128 + 2;       // words of a row group's columns
// A column's place in LDS: the lanes of a row group, which hold each eighth column, are neighbours
// (column by column they meet in few banks: 4095 x 1024 bf16 both ways 11.4 us for 10.2).
__device__ __forceinline__ int column_of(int place) { return (place & 15) * 8 + (place >> 4); }
static_assert(ST_ROWS * ST_GROUPS == 128, "whole tiles");
template <typename E, bool C, bool TR, bool SQUARE, bool MASK>
__global__ __launch_bounds__(ST_NT) void block8_store_kernel(StoreArgs a, int64_t col_tiles, int64_t tiles)
{
    __shared__ __attribute__((aligned(16))) uint8_t bytes[TR ? 128 * ST_PITCH : 16];
    __shared__ uint32_t tops[TR || SQUARE ? ST_GROUPS : 1][ST_WORDS];
    __shared__ float sums[ST_GROUPS][ST_WORDS];
    const int g = threadIdx.x >> 4, l = threadIdx.x & 15;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t r0 = tile / col_tiles * 128, c0 = tile % col_tiles * 128;
        const int64_t col = c0 + 8 * l;
        const int nv = (int)min((int64_t)8, a.d - col);      // columns, may be none
        const int rows = (int)min((int64_t)128, a.n - r0);
        float v[ST_ROWS][8];
#pragma unroll
        for (int k = 0; k < ST_ROWS; ++k) {
            const int r = ST_ROWS * g + k;
            load8((const E *)a.x + (r0 + r) * a.ld_x + col, r < rows ? nv : 0, v[k]);
        }
        if constexpr (MASK) {
            float y[ST_ROWS][8];
#pragma unroll
            for (int k = 0; k < ST_ROWS; ++k) {
                const int r = ST_ROWS * g + k;
                load8((const E *)a.y + (r0 + r) * a.ld_y + col, r < rows ? nv : 0, y[k]);
            }
#pragma unroll
            for (int k = 0; k < ST_ROWS; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] = y[k][j] > 0.0f ? v[k][j] : 0.0f;
        }
        // largest magnitudes and sums of the thread's part of each column
        if (TR || SQUARE || a.sums) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t top = 0;
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < ST_ROWS; ++k) top = max(top, magnitude(v[k][j])), s += v[k][j];
                if constexpr (TR || SQUARE) tops[g][16 * j + l] = top;
                if (a.sums) sums[g][16 * j + l] = s;
            }
            __syncthreads();
        }
        // of whole columns, by four threads each; a magnitude goes in the first of its column's words
        const int place = threadIdx.x >> 2, part = threadIdx.x & 3;
        const int64_t own = c0 + column_of(place);
        if (a.sums) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < ST_GROUPS / 4; ++k) s += sums[part * (ST_GROUPS / 4) + k][place];
            s = team_sum<4>(s);
            if (part == 0 && own < a.d) a.sums[r0 / 128 * a.d + own] = s;
        }
        if constexpr (TR || SQUARE) {
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < ST_GROUPS / 4; ++k) m = max(m, tops[part * (ST_GROUPS / 4) + k][place]);
            m = quad_max(m);
            if constexpr (SQUARE) {
#pragma unroll
                for (int b = 4; b < 64; b *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, b));
            } else if (part == 0 && own < a.d) {
                a.t.scale[own * a.t.ld_scale + r0 / 128] = (uint8_t)block8_scale(m);
            }
            __syncthreads();
            if (SQUARE ? (threadIdx.x & 63) == 0 : part == 0) tops[0][SQUARE ? threadIdx.x >> 6 : place] = m;
            __syncthreads();
        }
        int whole = 0;
        if constexpr (SQUARE) {
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < ST_NT / 64; ++k) m = max(m, tops[0][k]);
            whole = block8_scale(m);
        }
        if constexpr (TR) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int s = SQUARE ? whole : block8_scale(tops[0][16 * j + l]);
                float w[ST_ROWS];
#pragma unroll
                for (int k = 0; k < ST_ROWS; ++k) w[k] = v[k][j];
                *(uint32_t *)(bytes + (16 * j + l) * ST_PITCH + ST_ROWS * g) = block8_pack4(w, s, rows - ST_ROWS * g);
            }
            if (SQUARE && threadIdx.x == 0) a.t.scale[c0 / 128 * a.t.ld_scale + r0 / 128] = (uint8_t)whole;
        }
        if constexpr (C) {
#pragma unroll
            for (int k = 0; k < ST_ROWS; ++k) {
                const int r = ST_ROWS * g + k;
                int s = whole;
                if constexpr (!SQUARE) {
                    uint32_t top = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[k][j]));
                    s = block8_scale(lanes_max<16>(top));
                }
                if (r >= rows) continue;
                *(u32x2_r *)(a.c.q + (r0 + r) * a.c.ld_q + col) = block8_pack(v[k], s, nv);
                if (!SQUARE && l == 0) a.c.scale[(r0 + r) * a.c.ld_scale + c0 / 128] = (uint8_t)s;
            }
            if (SQUARE && threadIdx.x == 0) a.c.scale[r0 / 128 * a.c.ld_scale + c0 / 128] = (uint8_t)whole;
        }
        if constexpr (TR) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 128 * 8 / ST_NT; ++u) {
                const int c = u * (ST_NT / 8) + (threadIdx.x >> 3), at = threadIdx.x % 8 * 16;
                const int64_t to = c0 + column_of(c);
                if (to < a.d)
                    *(u32x4_r *)(a.t.q + to * a.t.ld_q + r0 + at) = *(const u32x4_r *)(bytes + c * ST_PITCH + at);
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
        if (square) block8_store_kernel<E, C, T, true, false><<<g, dim3(ST_NT), 0, s>>>(a, cols, tiles);
        else if (mask) block8_store_kernel<E, C, T, false, true><<<g, dim3(ST_NT), 0, s>>>(a, cols, tiles);
        else block8_store_kernel<E, C, T, false, false><<<g, dim3(ST_NT), 0, s>>>(a, cols, tiles);
    };
    const std::true_type yes;
    const std::false_type no;
    if (a.c.q && a.t.q) go(yes, yes);
    else if (a.c.q) go(yes, no);
    else if (a.t.q) go(no, yes);
    else if (mask) block8_store_kernel<E, false, false, false, true><<<g, dim3(ST_NT), 0, s>>>(a, cols, tiles);
    else block8_store_kernel<E, false, false, false, false><<<g, dim3(ST_NT), 0, s>>>(a, cols, tiles);
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
// Restores: 16 lanes a block of 128 values.  65536 x 1024 to bf16: 31 us, 202 MB at 6.5 TB/s, of which the
// caches still hold what was stored just before.
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

__global__ __launch_bounds__(64 * COLUMN_SUM_WAVES) void column_sums_kernel(ColumnSums c)
{
    __shared__ double lds[COLUMN_SUM_WAVES][64];
    column_sums(c.part, c.rows, c.d, c.sums, blockIdx.x, lds);
}

hipError_t launch_column_sums(const ColumnSums &c, hipStream_t s)
{
    column_sums_kernel<<<dim3((unsigned)ceil_div(c.d, 64)), dim3(64 * COLUMN_SUM_WAVES), 0, s>>>(c);
    return hipGetLastError();
}

}  // namespace im
