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

// The eight consecutive values of a row of d that a lane holds: of the columns col .. col + 7,
// or, where the row ends inside them, its last eight, from column `at` on.  The `lo` values
// before col are then its neighbour's as well; both compute and store them, the same bits, and
// only one counts them in a sum.  So a row of any width is loaded and stored in whole pieces;
// value by value, up to seven loads that wait for each other would hold up the whole row.
// Widths of whole pieces (EVEN) need none of this: with it the gradient of 524288 x 512 from a
// checkpoint takes 264 us for 255, restoring 262144 x 1024 155 us for 140 (storing is alike).  A
// row of fewer than eight values is read value by value (NARROW: may be one).
enum RowWidth { EVEN, ODD, NARROW };
template <int W>
struct RowPiece {
    int col, at, lo, hi;
    __device__ __forceinline__ void init(int column, int d)
    {
        col = column;
        at = max(0, min(col, d - 8));
        lo = min(col - at, 8);
        hi = W == NARROW ? min(d, 8) : 8;
    }
    __device__ __forceinline__ bool any() const { return lo < 8; }
    __device__ __forceinline__ bool own(int k) const
    {
        return W == EVEN ? any() : k >= lo && (W != NARROW || k < hi);
    }
    // a 32-block of a checkpoint begins at col, and the values before are of another
    __device__ __forceinline__ bool split() const { return W != EVEN && lo > 0 && lo < 8 && (col & 31) == 0; }
    __device__ __forceinline__ bool whole() const { return W != NARROW || hi == 8; }
};

struct Raw32 {
    f32x4_r a, b;
};

template <int W>
__device__ __forceinline__ Raw32 load_raw(const float *row, const RowPiece<W> &c, bool on)
{
    Raw32 r = {};
    if (on && c.any()) {
        const float *p = row + c.at;
        if (c.whole()) {
            r.a = *(const f32x4_a4 *)p;
            r.b = *(const f32x4_a4 *)(p + 4);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k < c.hi) r.a[k] = p[k];
                if (k + 4 < c.hi) r.b[k] = p[k + 4];
            }
        }
    }
    return r;
}

template <int W>
__device__ __forceinline__ u32x4_r load_raw(const uint16_t *row, const RowPiece<W> &c, bool on)
{
    u32x4_r r = {0, 0, 0, 0};
    if (on && c.any()) r = c.whole() ? *(const u32x4_a2 *)(row + c.at) : load8_bits(row + c.at, c.hi);
    return r;
}

template <int W>
__device__ __forceinline__ u32x2_r load_raw(const int8_t *row, const RowPiece<W> &c, bool on)
{
    u32x2_r r = {0, 0};
    if (on && c.any()) r = c.whole() ? *(const u32x2_a1 *)(row + c.at) : load8_bytes(row + c.at, c.hi);
    return r;
}

__device__ __forceinline__ void unpack8(const Raw32 &r, float *v)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = r.a[k], v[4 + k] = r.b[k];
}

template <int W>
__device__ __forceinline__ void store_piece(float *row, const RowPiece<W> &c, const float *v)
{
    if (!c.any()) return;
    float *p = row + c.at;
    if (c.whole()) {
        const f32x4_r a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        *(f32x4_a4 *)p = a;
        *(f32x4_a4 *)(p + 4) = b;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < c.hi) p[k] = v[k];
    }
}

template <int W>
__device__ __forceinline__ void store_piece(uint16_t *row, const RowPiece<W> &c, const float *v)
{
    if (!c.any()) return;
    if (c.whole()) *(u32x4_a2 *)(row + c.at) = pack8(v);
    else store8_bits(row + c.at, c.hi, pack8(v));
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
__device__ __forceinline__ float ckpt_step(int scale)
{
    return scale == 255 ? __builtin_nanf("") : ldexpf(1.0f, scale - 133);
}
__device__ __forceinline__ float ckpt_value(u32x2_r r, int k) { return (float)(int8_t)(r[k >> 2] >> (8 * (k & 3))); }
__device__ __forceinline__ void ckpt_unpack(u32x2_r r, int scale, float *v)
{
    const float s = ckpt_step(scale);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = ckpt_value(r, k) * s;
}

// A piece of a checkpoint: its bytes, its block's scale, and that of the block before if split.
struct RawBytes {
    u32x2_r q;
    int scale, before;
};
template <int W>
__device__ __forceinline__ RawBytes load_bytes(const int8_t *q, const uint8_t *scale, const RowPiece<W> &c,
                                               bool on)
{
    RawBytes r = {load_raw(q, c, on), 0, 0};
    if (on && c.any()) {
        r.scale = scale[c.col >> 5];
        if (c.split()) r.before = scale[c.at >> 5];
    }
    return r;
}
template <int W>
__device__ __forceinline__ void unpack8(RawBytes r, const RowPiece<W> &c, float *v)
{
    // the unpacking stays here: in the branch that loads, where the compiler would begin it, it
    // would wait for the load
    asm("" : "+v"(r.q[0]), "+v"(r.q[1]));
    ckpt_unpack(r.q, r.scale, v);
    if (c.split()) {
        const float s = ckpt_step(r.before);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < c.lo) v[k] = ckpt_value(r.q, k) * s;
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp_swap(float x)
{
    return __builtin_bit_cast(
        float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
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
    // odd rows of one register against even rows of another: the sum is in both
    if constexpr (T >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (T >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
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

// A piece's values to a row of a checkpoint: the scale from the largest magnitude of a 32-block,
// whose four quarters a quad's lanes hold, and the bytes.  The bytes before col are stored by the
// neighbour alone, whose block can be another.  The whole quad calls.
template <int W>
__device__ __forceinline__ void store_bytes(int8_t *q, uint8_t *scale, const RowPiece<W> &c, bool on,
                                            const float *v)
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t b = c.own(k) ? __float_as_uint(v[k]) & 0x7FFFFFFFu : 0;
        top = top > b ? top : b;
    }
    const int s = ckpt_scale(quad_max(top));
    if (!on || !c.any()) return;
    const u32x2_r r = ckpt_pack(v, s);
    if (W == EVEN || (c.lo == 0 && c.whole())) {
        *(u32x2_a1 *)(q + c.at) = r;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (c.own(k)) q[c.at + k] = (int8_t)(r[k >> 2] >> (8 * (k & 3)));
    }
    if ((c.col & 31) == 0) scale[c.col >> 5] = (uint8_t)s;
}

}  // namespace im
