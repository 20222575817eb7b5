// linear8_kernels.hip -- products of matrices in 8 bits on MFMA: C[q][p] = sum_k Q[q][k] P[p][k].
//   forward  q = row,    p = output, k = input    Q = x, P = w
//   dx       q = row,    p = input,  k = output   Q = dy, P = w^T
//   dw       q = output, p = input,  k = row      Q = dy^T, P = x^T
// All three read both operands along k, in whole blocks of 128 (rows are padded with
// zeros).  MFMA accumulators give a lane one q and four consecutive p per register group.
//
// The bytes become bf16 with their block's scale, exactly, and are multiplied by
// v_mfma_f32_32x32x16_bf16: every sum is one of fp32, for outputs of all types.  The matrix cores' 8-bit
// instructions (v_mfma_scale_f32_32x32x64_f8f6f4, v_mfma_f32_32x32x16_fp8_fp8) run at twice the rate,
// but add the products of eight neighbouring k to 14 bits from the largest one's exponent down before
// they add the sum in fp32 (found by adding one small product to a large one): sums of normal values
// are then off by 1.4e-5 of their norm, a hundred times what fp32 loses, and a small product beside
// a large one is lost whole.  To bf16 they took 81 us of 65536 rows 1024 -> 1024 where fp32's sums take
// 126 to 132 (hipBLASLt's product of bf16 matrices of that size 133), of one row 4.9 and 6.3.
#include <algorithm>
#include <type_traits>

#include "block8.h"
#include "recurrent.h"

namespace im {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
#define IM_LDS3 __attribute__((address_space(3)))

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int V>
using Int = std::integral_constant<int, V>;

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Copies 16 bytes a lane to LDS at `to` (the same in every lane) + 16 lane.
__device__ __forceinline__ void copy_to_lds(const void *from, char *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)from,
                                     (IM_LDS3 uint32_t *)to, 16, 0, 0);
}

// Copies a byte a lane, as a word, to `to` + 4 lane.
__device__ __forceinline__ void copy_byte_to_lds(const void *from, char *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)from,
                                     (IM_LDS3 uint32_t *)to, 1, 0, 0);
}

// All but the wavefront's N last loads are done, and its LDS accesses.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// Waits for a step that `later` steps of L loads each follow (M of them at most).
template <int L, int M>
__device__ __forceinline__ void wait_for_step(int later)
{
    if constexpr (M > 0) {
        if (later >= M) wait_loads<M * L>();
        else wait_for_step<L, M - 1>(later);
    } else {
        wait_loads<0>();
    }
}

// The block meets; LDS accesses stay on their side.
__device__ __forceinline__ void meet()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Eight e4m3 values times the scale's power of two as bf16: exact, but for values below 2^-126.
__device__ __forceinline__ bf16x8_t widen8(uint32_t lo, uint32_t hi, float scale)
{
    const bf16x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false),
                           __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)};
    return __builtin_bit_cast(bf16x8_t, v);
}

// Bits of four values as a vector.
__device__ __forceinline__ u32x4_r bits4(const f32x16_t &a, int g)
{
    return u32x4_r{__float_as_uint(a[4 * g]), __float_as_uint(a[4 * g + 1]), __float_as_uint(a[4 * g + 2]),
                   __float_as_uint(a[4 * g + 3])};
}

// ---------------------------------------------------------------------------
// Tiles.  A block of WP x WQ wavefronts forms BP x BQ of C, a wavefront TP x TQ MFMA tiles.
// K steps of 128 bytes go through a ring of NS stages in LDS by direct loads, NS - 1 steps
// ahead, their scales as a word a row after them; a step has one barrier.  Direct loads write
// 64 consecutive 16-byte pieces, so a stage has no padding: pieces are permuted in their row
// instead, so that 16 rows' pieces of one k cover all banks.
//
// 65536 rows 1024 -> 1024 to bf16: 126 us, 1.09 PFLOP/s, 136 with all arrays out of HBM; to fp32 152 and 156.
// A 256 x 256 tile has a CU for itself, so that nothing multiplies while it stores.
// dw of 65536 rows 1024 -> 512: 76 us in 16 parts and 8 to join them; tiles of 256 x 256,
// 256 x 128 and eight wavefronts a tile are no faster (82, 85, 79).
// ---------------------------------------------------------------------------
template <int WP_, int WQ_, int TP_, int TQ_, int NS_>
struct TileShape {
    static constexpr int WP = WP_, WQ = WQ_, TP = TP_, TQ = TQ_, NS = NS_;
    static constexpr int NT = 64 * WP * WQ, WAVES = WP * WQ, BP = 32 * WP * TP, BQ = 32 * WQ * TQ;
    static constexpr int UP = BP * 8 / NT, UQ = BQ * 8 / NT;             // 16-byte pieces of a thread
    static constexpr int US = ((BP + BQ + 63) / 64 + WAVES - 1) / WAVES;      // scales of a thread
    static constexpr int L = UP + UQ + US;                               // direct loads of a step
    static constexpr int Q_AT = BP * 128, S_AT = Q_AT + BQ * 128, STAGE = S_AT + US * WAVES * 256;
    static constexpr int LDO = 128 + 16, OUT = 32 * LDO;                 // bytes of a wavefront's 32 output rows
    static constexpr bool WHOLE = TP == 4 || (TP == 1 && WP == 4);       // a y8 block's columns meet
    static constexpr int LDS = std::max(NS * STAGE, WAVES * OUT + (TP == 1 && WP == 4 ? TQ * WAVES * 128 : 0));
    // piece c of row r lies at c ^ perm(r)
    __device__ static int perm(int r) { return r >> 1 & 7; }
    static_assert(UP * NT == BP * 8 && UQ * NT == BQ * 8, "whole pieces");
};

template <typename S>
__device__ __forceinline__ void tile_run(const Linear8Args &a, int p_tiles, int tiles, int id, char *lds)
{
    constexpr int TP = S::TP, TQ = S::TQ, BP = S::BP, BQ = S::BQ, NS = S::NS;
    const int lane = threadIdx.x & 63, wave = wave_id();
    const int split = id / tiles, tile = id % tiles;
    const int64_t p0 = (int64_t)(tile % p_tiles) * BP, q0 = (int64_t)(tile / p_tiles) * BQ;
    const int wp = wave % S::WP * TP * 32, wq = wave / S::WP * TQ * 32;
    const int64_t k0 = a.steps * split / a.splits;
    const int nk = (int)(a.steps * (split + 1) / a.splits - k0);

    // Addresses of this thread's pieces and scales.  Rows past the last read the last one: their
    // sums are not stored.
    const uint8_t *from[S::UP + S::UQ], *sfrom[S::US];
#pragma unroll
    for (int u = 0; u < S::UP + S::UQ; ++u) {
        const bool q = u >= S::UP;
        const int r = ((q ? u - S::UP : u) * S::WAVES + wave) * 8 + lane / 8;
        const int c = (lane & 7) ^ S::perm(r);
        const Mat8 &m = q ? a.q : a.p;
        const int64_t row = min((q ? q0 : p0) + r, (q ? a.n : a.out) - 1);
        from[u] = m.q + row * m.ld_q + k0 * 128 + c * 16;
    }
#pragma unroll
    for (int u = 0; u < S::US; ++u) {
        const int r = (u * S::WAVES + wave) * 64 + lane;
        const bool q = r >= BP;
        const Mat8 &m = q ? a.q : a.p;
        const int64_t row = min(q ? q0 + min(r - BP, BQ - 1) : p0 + r, (q ? a.n : a.out) - 1);
        sfrom[u] = m.scale + (row >> m.shift) * m.ld_scale + k0;
    }
    auto copy = [&](int u, int kt, char *st) {
        if (u < S::UP + S::UQ) copy_to_lds(from[u] + kt * 128, st + (u * S::WAVES + wave) * 1024);
        else copy_byte_to_lds(sfrom[u - S::UP - S::UQ] + kt,
                              st + S::S_AT + ((u - S::UP - S::UQ) * S::WAVES + wave) * 256);
    };
    for (int kt = 0; kt < NS - 1 && kt < nk; ++kt)
#pragma unroll
        for (int u = 0; u < S::L; ++u) copy(u, kt, lds + kt * S::STAGE);
    // 16 bytes of one of 32 rows: half h of the wavefront takes piece 2 s + h
    auto piece = [&](const char *at, int row, int s) {
        const int r = row + (lane & 31);
        return *(const u32x4_r *)(at + r * 128 + (((2 * s + (lane >> 5)) ^ S::perm(r)) << 4));
    };
    // The sums start from the bias.  Columns past the last are copies of it, which leave their rows'
    // largest magnitudes as they are.
    f32x16_t acc[TP][TQ];
    const int half = lane >> 5, l32 = lane & 31;
    if (a.bias && p0 + BP <= a.out) {
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4_r b = *(const f32x4_a4 *)(a.bias + p0 + wp + 32 * i + 8 * g + 4 * half);
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][0][4 * g + k] = b[k];
            }
    } else {
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int64_t col = p0 + wp + 32 * i + 8 * (k / 4) + 4 * half + k % 4;
                acc[i][0][k] = a.bias ? a.bias[min(col, a.out - 1)] : 0.0f;
            }
    }
#pragma unroll
    for (int j = 1; j < TQ; ++j)
#pragma unroll
        for (int i = 0; i < TP; ++i) acc[i][j] = acc[i][0];
    auto multiply = [&](int kt, bool more) {
        const char *st = lds + kt % NS * S::STAGE;
        char *ahead = lds + (kt + NS - 1) % NS * S::STAGE;
        const int *sc = (const int *)(st + S::S_AT);
        int sp[TP], sq[TQ];
#pragma unroll
        for (int i = 0; i < TP; ++i) sp[i] = sc[wp + 32 * i + (lane & 31)];
#pragma unroll
        for (int j = 0; j < TQ; ++j) sq[j] = sc[BP + wq + 32 * j + (lane & 31)];
        // the pieces of a substep are read before the one before it is multiplied
        u32x4_r bp[2][TP], bq[2][TQ];
        auto read = [&](int s) {
#pragma unroll
            for (int i = 0; i < TP; ++i) bp[s & 1][i] = piece(st, wp + 32 * i, s);
#pragma unroll
            for (int j = 0; j < TQ; ++j) bq[s & 1][j] = piece(st + S::Q_AT, wq + 32 * j, s);
        };
        read(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (s + 1 < 4) read(s + 1);
            if (more)
#pragma unroll
                for (int u = S::L * s / 4; u < S::L * (s + 1) / 4; ++u) copy(u, kt + NS - 1, ahead);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8_t fp[TP], fq[TQ];
#pragma unroll
                for (int i = 0; i < TP; ++i)
                    fp[i] = widen8(bp[s & 1][i][2 * h], bp[s & 1][i][2 * h + 1],
                                   __uint_as_float((uint32_t)sp[i] << 23));
#pragma unroll
                for (int j = 0; j < TQ; ++j)
                    fq[j] = widen8(bq[s & 1][j][2 * h], bq[s & 1][j][2 * h + 1],
                                   __uint_as_float((uint32_t)sq[j] << 23));
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int j = 0; j < TQ; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[i], fq[j], acc[i][j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int kt = 0;
    for (; kt + NS - 1 < nk; ++kt) {
        wait_loads<(NS - 2) * S::L>();
        meet();
        multiply(kt, true);
    }
    for (; kt < nk; ++kt) {
        wait_for_step<S::L, NS - 2>(nk - 1 - kt);
        meet();
        multiply(kt, false);
    }

    // Outputs: lane l holds q = wq + 32 j + l % 32, p = wp + 32 i + 8 g + 4 (l / 32) + 0..3.  They leave
    // through a part of LDS of the wavefront's own, in pieces of 16 bytes, up to 128 of a row.
    meet();
    char *mine = lds + wave * S::OUT, *to = mine + l32 * S::LDO + 4 * half;
    // Of each row in `mine` row_bytes to y's rows of ld bytes, from byte `col` on, up to byte `end`;
    // values of `unit` bytes.
    auto leave = [&](auto row_bytes, char *y, int64_t ld, int j, int64_t col, int64_t end, int unit) {
        constexpr int LANES = decltype(row_bytes)::value / 16, ROWS = 64 / LANES;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int u = 0; u < 32 / ROWS; ++u) {
            const int r = u * ROWS + lane / LANES, c = lane % LANES * 16;
            const u32x4_r v = *(const u32x4_r *)(mine + r * S::LDO + c);
            const int64_t row = q0 + wq + 32 * j + r;
            const int64_t nv = end - col - c;
            if (row >= a.n || nv <= 0) continue;
            char *at = y + row * ld + col + c;
            if (nv >= 16) {
                *(u32x4_a2 *)at = v;
            } else if (unit == 2) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (2 * k < nv) ((uint16_t *)at)[k] = (uint16_t)(v[k / 2] >> (16 * (k & 1)));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (4 * k < nv) ((uint32_t *)at)[k] = v[k];
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
        if (a.relu)
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[i][j][k] = __builtin_elementwise_maximum(acc[i][j][k], 0.0f);   // NaN stays
        // A block of y8 is a wavefront's columns or, with one tile a wavefront, those of four.
        if constexpr (S::WHOLE) {
            if (a.y8.q) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) top = max(top, magnitude(acc[i][j][k]));
                top = max(top, (uint32_t)__shfl_xor((int)top, 32));
                if constexpr (TP == 1) {
                    uint32_t *tops = (uint32_t *)(lds + S::WAVES * S::OUT) + j * S::WAVES * 32;
                    tops[wave * 32 + l32] = top;
                    meet();
#pragma unroll
                    for (int w = 0; w < 4; ++w) top = max(top, tops[(wave / 4 * 4 + w) * 32 + l32]);
                }
                const int s = block8_scale(top);
                const int64_t row = q0 + wq + 32 * j + l32, col = p0 + wp;
                if (half == 0 && col % 128 == 0 && row < a.n && col < a.out)
                    a.y8.scale[row * a.y8.ld_scale + col / 128] = (uint8_t)s;
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float v[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                        const int64_t nv = a.out - col - (32 * i + 8 * g + 4 * half);
                        *(uint32_t *)(to + 32 * i + 8 * g) = block8_pack4(v, s, (int)max(min(nv, (int64_t)4), (int64_t)0));
                    }
                leave(Int<32 * TP>(), (char *)a.y8.q, a.y8.ld_q, j, col, (a.out + 127) / 128 * 128, 4);
            }
        }
        if (!a.y) continue;
        if (a.y_f32) {
            char *y = (char *)a.y;
            int64_t ld = a.ld_y * 4;
            if (a.part) {
                ld = (a.out + 3) / 4 * 16;
                y = (char *)a.part + split * a.n * ld;
            }
#pragma unroll
            for (int i = 0; i < TP; ++i) {
#pragma unroll
                for (int g = 0; g < 4; ++g) *(u32x4_r *)(mine + l32 * S::LDO + 32 * g + 16 * half) = bits4(acc[i][j], g);
                leave(Int<128>(), y, ld, j, (p0 + wp + 32 * i) * 4, a.out * 4, 4);
            }
        } else {
            constexpr int PAIR = TP % 2 ? 1 : 2;
#pragma unroll
            for (int i = 0; i < TP; i += PAIR) {
#pragma unroll
                for (int h = 0; h < PAIR; ++h)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x16_t &c = acc[i + h][j];
                        *(u32x2_r *)(mine + l32 * S::LDO + 64 * h + 16 * g + 8 * half) =
                            u32x2_r{pack_bf16x2(c[4 * g], c[4 * g + 1]), pack_bf16x2(c[4 * g + 2], c[4 * g + 3])};
                    }
                leave(Int<64 * PAIR>(), (char *)a.y, a.ld_y * 2, j, (p0 + wp + 32 * i) * 2, a.out * 2, 2);
            }
        }
    }
}

template <typename S>
__global__ __launch_bounds__(S::NT, 2) void linear8_tile_kernel(Linear8Args a, int p_tiles, int tiles)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    tile_run<S>(a, p_tiles, tiles, xcd_order(blockIdx.x, gridDim.x), lds);
}

// Two products side by side in one launch, a layer's gradients.
template <typename S>
__global__ __launch_bounds__(S::NT, 2) void linear8_two_kernel(Linear8Args a, int a_tiles, int a_blocks, Linear8Args b,
                                                              int b_p_tiles, int b_tiles)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int id = xcd_order(blockIdx.x, gridDim.x);
    if (id < a_blocks) tile_run<S>(a, a_tiles, a_blocks, id, lds);
    else tile_run<S>(b, b_p_tiles, b_tiles, id - a_blocks, lds);
}

// Parts of a product to y, in their order.  The blocks after the first `blocks` add up column
// sums instead (column_sums: 64 columns a block).
__global__ __launch_bounds__(1024) void linear8_join_kernel(Linear8Args a, int blocks, const float *part, int64_t rows,
                                                            int64_t d, float *sums)
{
    __shared__ double lds[COLUMN_SUM_WAVES][64];
    if ((int)blockIdx.x >= blocks) {
        column_sums(part, rows, d, sums, blockIdx.x - blocks, lds);
        return;
    }
    const int64_t ld = (a.out + 3) / 4 * 4, quads = ld / 4, all = a.n * quads;
    for (int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x; i < all; i += (int64_t)blocks * 1024) {
        const int64_t row = i / quads, col = (i - row * quads) * 4;
        const float *p = a.part + row * ld + col;
        f32x4_r s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (int k = 0; k < a.splits; ++k) s += *(const f32x4_r *)(p + (int64_t)k * a.n * ld);
        float *y = (float *)a.y + row * a.ld_y + col;
        if (col + 4 <= a.out) {
            *(f32x4_a4 *)y = s;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + k < a.out) y[k] = s[k];
        }
    }
}

// Sides of tiles, by us of n rows 1024 -> 1024 (361 -> 512 in brackets), replayed from a graph:
//   to bf16       n 1          2048         4096         8192         16384        65536
//     64 x 64      6.3 (4.2)    9.4 (4.7)   17.0 (5.8)   30.9 (10.0)  56.1 (17.7)  206 (61.8)
//     128 x 128   10.2 (6.0)   11.8 (6.9)   13.2 (7.3)   21.0 (8.3)   36.8 (12.0)  136 (34.9)
//     256 x 256   24.2 (11.6)  26.2 (13.2)  27.0 (13.5)  29.9 (14.3)  34.3 (16.0)  126 (34.4)
//   to 8 bits     n 1           2048         8192         16384        65536
//     128 x 32    7.1 (4.8)   14.0 (5.4)   49.0 (17.1)
//     128 x 128  11.4 (7.0)   12.4 (7.6)   21.1 (8.5)   36.1 (12.0)  141 (40.2)
//     256 x 256  26.7 (14.7)               30.3 (16.4)  35.0 (17.7)  123 (37.1)
// Of fewer than 256 tiles the smaller ones pay; 128 x 32 while each has a CU.
typedef TileShape<2, 2, 1, 1, 4> Tile64;      // 64 x 64, three steps ahead
typedef TileShape<2, 2, 1, 1, 2> Tile64Many;  // four blocks a CU beside each other
typedef TileShape<2, 2, 2, 2, 2> Tile128;     // 128 x 128, two blocks a CU
typedef TileShape<1, 4, 4, 1, 2> TileRows;    // the same, wavefronts of whole blocks of y8
typedef TileShape<4, 1, 1, 1, 4> TileFlat;    // 128 x 32, four wavefronts a block of y8
typedef TileShape<2, 4, 4, 2, 2> Tile256;     // 256 x 256

static int64_t tiles_of(int64_t n, int64_t out, int side) { return ceil_div(n, side) * ceil_div(out, side); }

// Few tiles of 128 x 128 leave CUs without one.
static bool few_tiles(int64_t n, int64_t out) { return tiles_of(n, out, 128) < 256; }

// Parts of dw, of tiles of 128 x 128 or 64 x 64, two a CU of the larger ones at most.  A part has four steps
// at least, of 64 x 64 eight where the tiles alone fill the CUs.
static int64_t large_splits(int64_t n, int64_t out, int64_t steps)
{
    return std::max<int64_t>(1, std::min<int64_t>(512 / tiles_of(n, out, 128), steps / 4));
}

// The larger ones where their parts come to 400.  Both gradients by us of rows, in and out, bf16, from a
// graph, with 64 x 64 below 256 parts, 400 and 512:
//   2000 x 1024 x 1024   36.8  28.4  28.4       4096 x 1024 x 512    37.6   33.9   33.8
//   16384 x 361 x 512    48.6  44.3  43.5       16384 x 361 x 1024   67.1   67.4   64.9
//   8192 x 538 x 1024    54.4  54.8  51.6       65536 x 361 x 1024    185    187    216
// 1024 x 1024 x 1024 in parts of four steps 22.3, of eight (no second part, no joining) 18.6.
// From 129 tiles on whole numbers of parts may come to less than 400 at any length: they are larger from 4096
// rows on, and where the tiles alone fill the CUs from three steps on.  By 64 x 64 and 128 x 128 of n rows:
//   n                  128           300           1024          2048          4096          16384        65536
//   1408 -> 1536                                 27.1 / 38.8   41.1 / 50.9   75.0 / 68.7   244 / 196    942 / 661
//   1536 -> 2048                                 37.6 / 43.8   45.6 / 58.4   84.9 / 81.7   286 / 255   1112 / 882
//   2048 -> 2304   24.5 / 27.7   38.5 / 32.4   48.7 / 45.3   73.6 / 67.0    116 / 110    408 / 364   1660 / 1358
static bool large_parts(int64_t n, int64_t out, int64_t steps)
{
    const int64_t tiles = tiles_of(n, out, 128);
    return tiles * large_splits(n, out, steps) >= 400 || (tiles >= 256 && steps > 2) || (tiles >= 128 && steps >= 32);
}

int linear8_splits(int64_t n, int64_t out, int64_t steps)
{
    if (large_parts(n, out, steps)) return (int)large_splits(n, out, steps);
    const int64_t tiles = tiles_of(n, out, 64);
    return (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, steps / (tiles >= 256 ? 8 : 4)));
}

template <typename S>
static void tile_by(const Linear8Args &a, hipStream_t s)
{
    const int64_t p_tiles = ceil_div(a.out, S::BP), tiles = p_tiles * ceil_div(a.n, S::BQ);
    const dim3 g((unsigned)(tiles * a.splits)), b(S::NT);
    linear8_tile_kernel<S><<<g, b, 0, s>>>(a, (int)p_tiles, (int)tiles);
}

template <typename S>
static void two_by(const Linear8Args &dx, const Linear8Args &dw, hipStream_t s)
{
    const int64_t ap = ceil_div(dx.out, S::BP), at = ap * ceil_div(dx.n, S::BQ);
    const int64_t bp = ceil_div(dw.out, S::BP), bt = bp * ceil_div(dw.n, S::BQ);
    const dim3 g((unsigned)(at + bt * dw.splits)), b(S::NT);
    linear8_two_kernel<S><<<g, b, 0, s>>>(dx, (int)ap, (int)at, dw, (int)bp, (int)bt);
}

static void join(const Linear8Args &a, const ColumnSums &c, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n * ceil_div(a.out, 4), 1024), 256 * 4);
    linear8_join_kernel<<<dim3((unsigned)(blocks + (c.sums ? ceil_div(c.d, 64) : 0))), dim3(1024), 0, s>>>(
        a, (int)blocks, c.part, c.rows, c.d, c.sums);
}

hipError_t launch_linear8(const Linear8Args &a, hipStream_t s)
{
    if (few_tiles(a.n, a.out) && !a.y8.q) {
        tile_by<Tile64>(a, s);
        return hipGetLastError();
    }
    // parts of rows with fewer than 2^21 tiles
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 20) / ceil_div(a.out, 128)) * 128;
    for (int64_t r = 0; r < a.n; r += most) {
        Linear8Args b = a;
        b.n = std::min(most, a.n - r);
        b.q.q += r * a.q.ld_q;
        b.q.scale += (r >> a.q.shift) * a.q.ld_scale;
        if (a.y) b.y = (char *)a.y + r * a.ld_y * (a.y_f32 ? 4 : 2);
        if (a.y8.q) b.y8.q += r * a.y8.ld_q, b.y8.scale += r * a.y8.ld_scale;
        if (tiles_of(b.n, b.out, 256) >= 256) tile_by<Tile256>(b, s);
        else if (a.y8.q && ceil_div(b.n, 32) * ceil_div(b.out, 128) <= 256) tile_by<TileFlat>(b, s);
        else if (a.y8.q) tile_by<TileRows>(b, s);
        else tile_by<Tile128>(b, s);
    }
    return hipGetLastError();
}

// dx (y null: not wanted), then dw's parts joined beside the column sums.
hipError_t launch_linear8_grad(const Linear8Args &dx, const Linear8Args &dw, const ColumnSums &c, hipStream_t s)
{
    hipError_t e = hipSuccess;
    const bool with_dx = dx.y != nullptr, small = dw.y && !large_parts(dw.n, dw.out, dw.steps);
    if (with_dx && small && few_tiles(dx.n, dx.out)) {
        const int64_t blocks = tiles_of(dx.n, dx.out, 64) + tiles_of(dw.n, dw.out, 64) * dw.splits;
        // of more than two blocks a CU: 4095 x 361 x 1024 30.5 and 28.2 us, 8192 x 361 x 512 34.1 and 31.9,
        // 256 x 361 x 1024, which has fewer, 14.4 and 15.3
        if (blocks > 512) two_by<Tile64Many>(dx, dw, s);
        else two_by<Tile64>(dx, dw, s);
        e = hipGetLastError();
    } else {
        if (with_dx) e = launch_linear8(dx, s);
        if (e == hipSuccess && dw.y) {
            if (small) tile_by<Tile64>(dw, s);
            else tile_by<Tile128>(dw, s);
            e = hipGetLastError();
        }
    }
    if (e != hipSuccess) return e;
    if (dw.y && dw.part) {
        join(dw, c, s);
        return hipGetLastError();
    }
    return c.sums ? launch_column_sums(c, s) : e;
}

}  // namespace im
