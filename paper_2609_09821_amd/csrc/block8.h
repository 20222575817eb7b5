// block8.h -- arithmetic of matrices in 8 bits (im_block8) and loads and stores of eight
// values, for the kernels of a recurrent policy's blocks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rows.h"

namespace im {

// Eight values of a row, zeros from the nv-th on.
__device__ __forceinline__ void load8(const uint16_t *p, int nv, float *v) { unpack8(load8_bits(p, nv), v); }
__device__ __forceinline__ void load8(const float *p, int nv, float *v)
{
    if (nv >= 8) {
        const f32x4_r a = *(const f32x4_a4 *)p, b = *(const f32x4_a4 *)(p + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = a[k], v[4 + k] = b[k];
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k < nv ? p[k] : 0.0f;
    }
}
__device__ __forceinline__ void store8(uint16_t *p, int nv, const float *v) { store8_bits(p, nv, pack8(v)); }
__device__ __forceinline__ void store8(float *p, int nv, const float *v)
{
    if (nv >= 8) {
        const f32x4_r a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        *(f32x4_a4 *)p = a;
        *(f32x4_a4 *)(p + 4) = b;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < nv) p[k] = v[k];
    }
}

// Scale of a block from the bits of its largest magnitude (as an integer: NaNs above
// infinity above the finite ones).  The magnitude is m 2^(E - 127) with m in [1, 2) and
// 448 is 1.75 2^8: the exponent less 8, one more for m > 1.75.
__device__ __forceinline__ int block8_scale(uint32_t top)
{
    const int e = (int)(top >> 23);
    if (e == 255) return 255;
    return max(e - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}

// 2^(127 - scale) for the scales 0 .. 247 of finite blocks.
__device__ __forceinline__ float block8_inverse(int scale) { return __uint_as_float((uint32_t)(254 - scale) << 23); }

// Four values as e4m3 at a block's scale: the product is exact or far below e4m3's smallest
// value, so that the conversion's rounding to nearest even is the only one.  nv: values that
// exist, may be none; zeros after them.
__device__ __forceinline__ uint32_t block8_pack4(const float *v, int scale, int nv)
{
    uint32_t w = 0x7F7F7F7Fu;
    if (scale != 255) {
        const float s = block8_inverse(scale);
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * s, v[1] * s, 0, false);
        w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * s, v[3] * s, lo, true);
    }
    return nv >= 4 ? w : nv <= 0 ? 0 : w & ((1u << (8 * nv)) - 1);
}
__device__ __forceinline__ u32x2_r block8_pack(const float *v, int scale, int nv)
{
    return u32x2_r{block8_pack4(v, scale, nv), block8_pack4(v + 4, scale, nv - 4)};
}

// Eight restored values.  The scale's power of two is subnormal for scale 0.
__device__ __forceinline__ void block8_unpack(u32x2_r q, int scale, float *v)
{
    const float s = scale == 255 ? __builtin_nanf("") : ldexpf(1.0f, scale - 127);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v[4 * k] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 0) * s;
        v[4 * k + 1] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 1) * s;
        v[4 * k + 2] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 2) * s;
        v[4 * k + 3] = __builtin_amdgcn_cvt_f32_fp8((int)q[k], 3) * s;
    }
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Largest of T lanes' words (4, 8 or 16, aligned), in each.
template <int T>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x)
{
    x = quad_max(x);
    if constexpr (T >= 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));
    if constexpr (T >= 16) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));
    return x;
}

// Column sums of partial rows by a block of 1024: 64 columns, wavefront w takes rows w, w + 16, ..;
// the wavefronts' sums meet in LDS in order.
constexpr int COLUMN_SUM_WAVES = 16;
__device__ __forceinline__ void column_sums(const float *part, int64_t rows, int64_t d, float *sums, int64_t block,
                                            double (*lds)[64])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = block * 64 + lane;
    double s = 0.0;
    if (col < d)
#pragma unroll 8
        for (int64_t r = w; r < rows; r += COLUMN_SUM_WAVES) s += (double)part[r * d + col];
    lds[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < d) {
        for (int k = 1; k < COLUMN_SUM_WAVES; ++k) s += lds[k][lane];
        sums[col] = (float)s;
    }
}

}  // namespace im
