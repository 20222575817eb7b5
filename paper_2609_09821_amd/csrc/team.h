// team.h -- rows in registers: a row belongs to a team of T lanes, eight consecutive values a
// lane, for the norms' kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/instantmimic.h"
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

template <int V>
using Int = std::integral_constant<int, V>;

// Lanes of a team for rows of d values.
inline int64_t team_lanes(int64_t d)
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
inline int64_t block_threads(int64_t d) { return std::max<int64_t>(NORM_NT, team_lanes(d)); }
inline int64_t pass_rows(int64_t d) { return block_threads(d) / team_lanes(d); }

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace im
