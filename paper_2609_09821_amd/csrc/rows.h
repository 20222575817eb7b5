// rows.h -- loads and stores of eight consecutive values of a row and the
// 8-bit checkpoint's arithmetic, for the kernels of the layers of experts.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_math.h"

namespace im {

// Vectors at the alignment of their elements' type: gfx950 loads and stores them
// at any address, so rows of odd widths take the same instructions as aligned ones.
typedef unsigned int u32x4_r __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_r __attribute__((ext_vector_type(2)));
typedef u32x4_r u32x4_a4 __attribute__((aligned(4)));
typedef u32x4_r u32x4_a2 __attribute__((aligned(2)));
typedef u32x2_r u32x2_a1 __attribute__((aligned(1)));
typedef float f32x4_r __attribute__((ext_vector_type(4)));
typedef f32x4_r f32x4_a4 __attribute__((aligned(4)));

// The first nv (0..8 or more) of the eight values at p, zeros for the others.
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

// Eight bf16 as four words.
__device__ __forceinline__ u32x4_r load8_bits(const uint16_t *p, int nv)
{
    if (nv >= 8) return *(const u32x4_a2 *)p;
    uint32_t h[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = k < nv ? p[k] : 0;
    u32x4_r r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = h[2 * k] | (h[2 * k + 1] << 16);
    return r;
}

__device__ __forceinline__ void unpack8(u32x4_r r, float *v)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[2 * k] = __uint_as_float(r[k] << 16);
        v[2 * k + 1] = __uint_as_float(r[k] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ void load8(const uint16_t *p, int nv, float *v) { unpack8(load8_bits(p, nv), v); }

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

__device__ __forceinline__ void store8_bits(uint16_t *p, int nv, u32x4_r r)
{
    if (nv >= 8) {
        *(u32x4_a2 *)p = r;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < nv) p[k] = (uint16_t)(r[k >> 1] >> (16 * (k & 1)));
    }
}

__device__ __forceinline__ u32x4_r pack8(const float *v)
{
    const u32x4_r r = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                       pack_bf16x2(v[6], v[7])};
    return r;
}

__device__ __forceinline__ void store8(uint16_t *p, int nv, const float *v) { store8_bits(p, nv, pack8(v)); }

// Eight int8 as two words (signed bytes in order).
__device__ __forceinline__ u32x2_r load8_bytes(const int8_t *p, int nv)
{
    if (nv >= 8) return *(const u32x2_a1 *)p;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < nv) w[k >> 2] |= (uint32_t)(uint8_t)p[k] << (8 * (k & 3));
    const u32x2_r r = {w[0], w[1]};
    return r;
}

__device__ __forceinline__ void store8_bytes(int8_t *p, int nv, u32x2_r r)
{
    if (nv >= 8) {
        *(u32x2_a1 *)p = r;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < nv) p[k] = (int8_t)(r[k >> 2] >> (8 * (k & 3)));
    }
}

// Scale of a block from the bits of its largest magnitude (as an integer: NaNs
// above infinity above the finite ones): the biased exponent, one more where the
// magnitude would round to 128 steps, 255 for a block that is not finite.
__device__ __forceinline__ int ckpt_scale(uint32_t top)
{
    const int b = (int)(top >> 23);
    if (b == 255) return 255;
    const bool up = rintf(ldexpf(__uint_as_float(top), 133 - b)) > 127.0f;
    return b + (up && b < 254 ? 1 : 0);
}

// Eight values as signed bytes at a finite block's scale.
__device__ __forceinline__ u32x2_r ckpt_pack(const float *v, int scale)
{
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        float t = rintf(ldexpf(v[k], 133 - scale));
        t = fminf(fmaxf(t, -127.0f), 127.0f);   // NaN in a block of scale 255: -127, restored as NaN
        w[k >> 2] |= ((uint32_t)(int)t & 0xFFu) << (8 * (k & 3));
    }
    const u32x2_r r = {w[0], w[1]};
    return r;
}

// The step is a power of two (subnormal below scale 7): every product is exact.
__device__ __forceinline__ void ckpt_unpack(u32x2_r r, int scale, float *v)
{
    const float s = scale == 255 ? __builtin_nanf("") : ldexpf(1.0f, scale - 133);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)(int8_t)(r[k >> 2] >> (8 * (k & 3))) * s;
}

template <int CTRL>
__device__ __forceinline__ float dpp_swap(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// Sum over each aligned group of T lanes (4..64), in every lane, in a fixed
// order: pairs by quad permutes, then mirrored halves and rows (the partial sums
// are equal within the half that is mirrored).
template <int T>
__device__ __forceinline__ float team_sum(float x)
{
    x += dpp_swap<0xB1>(x);                      // lanes 1 0 3 2 of a quad
    x += dpp_swap<0x4E>(x);                      // 2 3 0 1
    if constexpr (T >= 8) x += dpp_swap<0x141>(x);    // half rows mirrored
    if constexpr (T >= 16) x += dpp_swap<0x140>(x);   // rows mirrored
    if constexpr (T >= 32) x += __shfl_xor(x, 16);
    if constexpr (T >= 64) x += __shfl_xor(x, 32);
    return x;
}

// Largest of four lanes' words, in each.
__device__ __forceinline__ uint32_t quad_max(uint32_t x)
{
    uint32_t t = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true);
    x = x > t ? x : t;
    t = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true);
    return x > t ? x : t;
}

// Bits of the largest magnitude of a 32-block whose four quarters a quad's lanes hold.
__device__ __forceinline__ uint32_t ckpt_top(const float *v)
{
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t b = __float_as_uint(v[k]) & 0x7FFFFFFFu;
        m = m > b ? m : b;
    }
    return quad_max(m);
}

}  // namespace im
