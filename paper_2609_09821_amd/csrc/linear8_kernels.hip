// linear8_kernels.hip -- products of matrices in 8 bits on MFMA: C[q][p] = sum_k Q[q][k] P[p][k].
//   forward  q = row,    p = output, k = input    Q = x, P = w
//   dx       q = row,    p = input,  k = output   Q = dy, P = w^T
//   dw       q = output, p = input,  k = row      Q = dy^T, P = x^T
// All three read both operands along k, in whole blocks of 128 (rows are padded with
// zeros).  MFMA accumulators give a lane one q and four consecutive p per register group.
//
// Outputs in bf16: v_mfma_scale_f32_32x32x64_f8f6f4, which multiplies each operand's
// row by its own power of two, so that scales cost no instruction besides their load.  It adds
// the products of eight neighbouring k to 14 bits from the largest one's exponent down, and only
// these sums in fp32 (found by adding one small product to a large one; v_mfma_f32_32x32x16_fp8_fp8
// gives the same bits): sums of normal values are off by 1.4e-5 of their norm, a hundredth of
// what an output in bf16 loses.  Outputs in fp32 would lose by it, and in 8 bits values next to the
// middle of two steps would go to the other one (8.9e-4 of the norm): there the bytes become bf16
// with their block's scale (exact) and are multiplied by v_mfma_f32_32x32x16_bf16, at half the rate.
#include <algorithm>
#include <type_traits>

#include "block8.h"
#include "recurrent.h"

namespace im {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
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

__device__ __forceinline__ i32x8_t join(u32x4_r lo, u32x4_r hi)
{
    return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// acc += (a 2^(sa - 127)) (b 2^(sb - 127)) over 64 k.  A lane holds 32 bytes of one row of each
// operand, its k by the half of the wavefront; both operands are read alike, so that which k is
// of no matter, and a row has one scale over all 128 k of a block.
__device__ __forceinline__ f32x16_t mfma8(i32x8_t a, i32x8_t b, f32x16_t acc, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 0, 0, 0, sa, 0, sb);
}

// The same of 16 rows each and 128 k, 32 bytes of a row in each of its four lanes; sa in byte A.
template <int A>
__device__ __forceinline__ f32x4_t mfma8_16(i32x8_t a, i32x8_t b, f32x4_t acc, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, A, sa, 0, sb);
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
// 65536 rows 1024 -> 1024 to bf16: 80 us, 1.72 PFLOP/s (hipBLASLt with one scale for each operand and no
// bias 87), 97 with all arrays out of HBM; 59 without the outputs, of which HBM takes 27 alone: a 256 x 256
// tile has a CU for itself, so that nothing multiplies while it stores.  Two blocks of 256 x 128 a CU store
// beside each other's products but load more (88 us).
// To fp32: 144 us.  dw of 65536 rows 1024 -> 512: 76 us in 16 parts and 8 to join them; tiles of 256 x 256,
// 256 x 128 and eight wavefronts a tile are no faster (82, 85, 79), and rows of x^T that lie a multiple
// of 64 KB apart cost 10 us.
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

template <typename S, bool WIDE>
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
        auto more_copies = [&](int s, int of) {
            if (more)
#pragma unroll
                for (int u = S::L * s / of; u < S::L * (s + 1) / of; ++u) copy(u, kt + NS - 1, ahead);
        };
        read(0);
        if constexpr (WIDE) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s + 1 < 4) read(s + 1);
                more_copies(s, 4);
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
        } else {
            u32x4_r cp[TP], cq[TQ];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                read(2 * s + 1);
#pragma unroll
                for (int i = 0; i < TP; ++i) cp[i] = bp[0][i];
#pragma unroll
                for (int j = 0; j < TQ; ++j) cq[j] = bq[0][j];
                i32x8_t fp[TP], fq[TQ];
#pragma unroll
                for (int i = 0; i < TP; ++i) fp[i] = join(cp[i], bp[1][i]);
#pragma unroll
                for (int j = 0; j < TQ; ++j) fq[j] = join(cq[j], bq[1][j]);
                if (s + 1 < 2) read(2 * s + 2);
                more_copies(s, 2);
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int j = 0; j < TQ; ++j) acc[i][j] = mfma8(fp[i], fq[j], acc[i][j], sp[i], sq[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
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
        if constexpr (WIDE && S::WHOLE) {
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
        if (WIDE && a.y_f32) {
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

template <typename S, bool WIDE>
__global__ __launch_bounds__(S::NT, 2) void linear8_tile_kernel(Linear8Args a, int p_tiles, int tiles)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    tile_run<S, WIDE>(a, p_tiles, tiles, xcd_order(blockIdx.x, gridDim.x), lds);
}

// Two products side by side in one launch, a layer's gradients: the second one is wide.
template <typename S, bool WIDE>
__global__ __launch_bounds__(S::NT, 2) void linear8_two_kernel(Linear8Args a, int a_tiles, int a_blocks, Linear8Args b,
                                                              int b_p_tiles, int b_tiles)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    const int id = xcd_order(blockIdx.x, gridDim.x);
    if (id < a_blocks) tile_run<S, WIDE>(a, a_tiles, a_blocks, id, lds);
    else tile_run<S, true>(b, b_p_tiles, b_tiles, id - a_blocks, lds);
}

// ---------------------------------------------------------------------------
// Panels.  With many rows, an output in bf16 and a k that fits, a block keeps 128 columns of P, all
// their k, in LDS and its wavefronts walk over the rows of Q by themselves, 64 at a time, without a
// barrier: Q's fragments come straight into registers, a step of 128 k ahead, also across the end of
// a tile, so that one wavefront's outputs leave while others multiply.  A block for each CU; the
// panels of one run of rows are neighbours in an L2.
//
// A wavefront's tile is 128 p x 64 q in MFMA tiles of 16 x 16 (v_mfma_scale_f32_16x16x128_f8f6f4):
// four lanes then hold one row of Q.  Bound by the CU's vector cache, to which each 16 bytes that a
// lane loads are an access: so scales are loaded four steps at a time and outputs pass through LDS.
// 65536 rows 1024 -> 1024: 84 us, 90 with all arrays out of HBM.  Weights in registers, rows in LDS: 113.
// ---------------------------------------------------------------------------
constexpr int PANEL_STEPS = 8, PANEL_WAVES = 8, PANEL_ROWS = 64;
__global__ __launch_bounds__(64 * PANEL_WAVES, 1) void linear8_panel_kernel(Linear8Args a, int panels, int streams)
{
    constexpr int TP = 8, TQ = PANEL_ROWS / 16, LDO = 128 + 16;
    __shared__ __attribute__((aligned(1024))) char lds[PANEL_STEPS * 16384];
    __shared__ __attribute__((aligned(16))) char outs[PANEL_WAVES][16 * LDO];
    __shared__ int pscale[PANEL_STEPS][16][2];      // byte i % 4 of word i / 4: row 16 i + lane's
    __shared__ float bias[128];
    const int lane = threadIdx.x & 63, wave = wave_id(), l16 = lane & 15, grp = lane >> 4;
    const int place = blockIdx.x >> 3, panel = place % panels;
    const int stream = place / panels * 8 + (blockIdx.x & 7);
    if (place / panels * 8 >= streams) return;
    const int64_t p0 = (int64_t)panel * 128;
    const int steps = (int)a.steps;
    for (int u = wave; u < steps * 16; u += PANEL_WAVES) {
        const int r = (u & 15) * 8 + lane / 8, c = (lane & 7) ^ (r >> 1 & 7);
        const int64_t row = min(p0 + r, a.out - 1);
        copy_to_lds(a.p.q + row * a.p.ld_q + (u >> 4) * 128 + c * 16, lds + u * 1024);
    }
    for (int u = threadIdx.x; u < steps * 32; u += 64 * PANEL_WAVES) {
        int v = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = min(p0 + 64 * (u & 1) + 16 * i + (u >> 1 & 15), a.out - 1);
            v |= a.p.scale[(row >> a.p.shift) * a.p.ld_scale + (u >> 5)] << (8 * i);
        }
        pscale[u >> 5][u >> 1 & 15][u & 1] = v;
    }
    if (threadIdx.x < 128) bias[threadIdx.x] = a.bias ? a.bias[min(p0 + threadIdx.x, a.out - 1)] : 0.0f;
    wait_loads<0>();
    __syncthreads();

    const int64_t tiles = (a.n + PANEL_ROWS - 1) / PANEL_ROWS, stride = (int64_t)streams * PANEL_WAVES;
    int64_t tile = (int64_t)stream * PANEL_WAVES + wave;
    if (tile >= tiles) return;
    // Q: 16 bytes grp and 4 + grp of a step of the rows 16 j + l16
    u32x4_r bq[2][TQ][2];
    // the scales of row `lane`: bytes of the steps 0..3, and of the last four (steps 4..7)
    uint32_t scale[2], next_scale[2] = {0, 0};
    // part j of step kt of tile t; rows past the last read the last one: their sums are not stored
    auto fetch = [&](int set, int64_t t, int kt, int j) {
        const int64_t q0 = t * PANEL_ROWS;
        const int last = (int)min((int64_t)PANEL_ROWS, a.n - q0) - 1;
        const uint8_t *base = a.q.q + q0 * a.q.ld_q + kt * 128;
        const uint32_t off = (uint32_t)min(16 * j + l16, last) * (uint32_t)a.q.ld_q + grp * 16;
        bq[set][j][0] = *(const u32x4_r *)(base + off);
        bq[set][j][1] = *(const u32x4_r *)(base + off + 64);
        if (j == 0 && kt == 0) {
            const uint8_t *s = a.q.scale + ((q0 + min(lane, last)) >> a.q.shift) * a.q.ld_scale;
            if (steps >= 4) {
                typedef uint32_t u32_a1 __attribute__((aligned(1)));
                next_scale[0] = *(const u32_a1 *)s;
                next_scale[1] = *(const u32_a1 *)(s + steps - 4) >> (8 * (8 - steps) & 31);
            } else {
                next_scale[0] = s[0];
                if (steps > 1) next_scale[0] |= s[1] << 8;
                if (steps > 2) next_scale[0] |= s[2] << 16;
            }
        }
    };
    f32x4_t acc[TP][TQ];
    auto start = [&] {
        scale[0] = next_scale[0], scale[1] = next_scale[1];
#pragma unroll
        for (int i = 0; i < TP; ++i) {
            const f32x4_t b = *(const f32x4_t *)(bias + 16 * i + 4 * grp);
#pragma unroll
            for (int j = 0; j < TQ; ++j) acc[i][j] = b;
        }
    };
    // a step's products; more(i): work beside those of the i-th tile of P
    auto multiply = [&](int set, int kt, auto more) {
        const char *st = lds + kt * 16384;
        const int sp[2] = {pscale[kt][l16][0], pscale[kt][l16][1]};
        // the scale of row 16 j + l16 in all four lanes of the row
        const uint32_t own = scale[kt >> 2] >> (8 * (kt & 3));
        const auto x = __builtin_amdgcn_permlane16_swap(own, own, false, false);
        const auto even = __builtin_amdgcn_permlane32_swap(x[0], x[0], false, false);
        const auto odd = __builtin_amdgcn_permlane32_swap(x[1], x[1], false, false);
        const int s4[TQ] = {(int)even[0], (int)odd[0], (int)even[1], (int)odd[1]};
        // piece c of a row at c ^ (row / 2 mod 8)
        auto piece = [&](int i, int k) {
            return *(const u32x4_r *)(st + (16 * i + l16) * 128 + (((4 * k + grp) ^ (l16 >> 1)) << 4));
        };
#pragma unroll
        for (int i = 0; i < TP; ++i) {
            const i32x8_t fp = join(piece(i, 0), piece(i, 1));
            more(i);
#pragma unroll
            for (int j = 0; j < TQ; ++j) {
                const i32x8_t fq = join(bq[set][j][0], bq[set][j][1]);
                if (i % 4 == 0) acc[i][j] = mfma8_16<0>(fp, fq, acc[i][j], sp[i / 4], s4[j]);
                if (i % 4 == 1) acc[i][j] = mfma8_16<1>(fp, fq, acc[i][j], sp[i / 4], s4[j]);
                if (i % 4 == 2) acc[i][j] = mfma8_16<2>(fp, fq, acc[i][j], sp[i / 4], s4[j]);
                if (i % 4 == 3) acc[i][j] = mfma8_16<3>(fp, fq, acc[i][j], sp[i / 4], s4[j]);
            }
        }
    };
    // A lane's sums of a 16 x 16 tile are p = 4 grp + 0..3 of one q.  16 rows x 64 columns at a time leave
    // through the wavefront's own LDS, 128 bytes of a row.
    auto store = [&](int64_t t) {
        char *mine = outs[wave];
#pragma unroll
        for (int j = 0; j < TQ; ++j)
#pragma unroll
            for (int i0 = 0; i0 < TP; i0 += 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4_t v = acc[i0 + i][j];
                    if (a.relu)
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = __builtin_elementwise_maximum(v[k], 0.0f);      // NaN stays
                    *(u32x2_r *)(mine + l16 * LDO + 32 * i + 8 * grp) = u32x2_r{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int r = u * 8 + lane / 8, c = lane % 8 * 8;
                    const u32x4_r o = *(const u32x4_r *)(mine + r * LDO + c * 2);
                    const int64_t row = t * PANEL_ROWS + 16 * j + r, col = p0 + 16 * i0 + c;
                    if (row < a.n)
                        store8_bits((uint16_t *)a.y + row * a.ld_y + col, (int)min((int64_t)8, a.out - col), o);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
    };
    int kt = 0, next_kt = 0;
    int64_t next_tile = tile;
#pragma unroll
    for (int j = 0; j < TQ; ++j) fetch(0, tile, 0, j);
    while (true) {
#pragma unroll
        for (int set = 0; set < 2; ++set) {
            if (++next_kt == steps) next_kt = 0, next_tile += stride;
            if (next_tile >= tiles) next_tile = tile;      // after the last step: read again, not used
            if (kt == 0) start();
            multiply(set, kt, [&](int i) {
                if (i < TQ) fetch(set ^ 1, next_tile, next_kt, i);
            });
            if (++kt == steps) {
                store(tile);
                kt = 0;
                tile += stride;
                if (tile >= tiles) return;
            }
        }
    }
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
//   to bf16       n 2048        4096         16384        65536
//     64 x 64     7.3 (4.1)   12.6 (4.9)   41.6 (14.3)  145 (47.5)
//     128 x 128   9.0 (5.8)   10.4 (6.3)   23.9 (9.6)   83.0 (28.0)
//     256 x 256  15.5 (9.4)   16.5 (9.6)   23.3 (11.8)  76.6 (25.7)
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

// Products in bf16, summed in fp32 throughout.
static bool wide(const Linear8Args &a) { return (a.y && a.y_f32) || a.y8.q; }

static int64_t tiles_of(int64_t n, int64_t out, int side) { return ceil_div(n, side) * ceil_div(out, side); }

// Few tiles of 128 x 128 leave CUs without one.
static bool few_tiles(int64_t n, int64_t out) { return tiles_of(n, out, 128) < 256; }

// Panels or tiles, by us of n rows to bf16, inputs and outputs out of HBM (panels / tiles):
//   n                 16384        65536        131072       262144
//   1024 -> 1024   29.8 / 27.1  89.8 / 96.6  163 / 183    315 / 356
//    361 -> 512    16.3 / 11.1  30.7 / 30.0  55.8 / 56.3  102 / 109
//    512 -> 69     15.6 /  6.6  18.8 / 19.6  26.3 / 35.7  45.3 / 65.6
// Panels pay from more than two tiles for each wavefront on, a single panel already from half a one.
static bool in_panels(const Linear8Args &a)
{
    const int64_t panels = ceil_div(a.out, 128), tiles = ceil_div(a.n, PANEL_ROWS) * panels;
    const bool enough = tiles > 2 * 256 * PANEL_WAVES || (panels == 1 && a.n >= 65536);
    return enough && !wide(a) && a.steps <= PANEL_STEPS && panels <= 32 && a.q.ld_q < (1 << 24);
}

// Parts of dw: of tiles of 128 x 128 where they come to 400 (two a CU at most), else of 64 x 64.  A part
// has four steps at least, eight where the tiles alone fill the CUs.  Both gradients by us of rows, in and
// out, bf16, from a graph, with 64 x 64 below 256 parts, 400 and 512:
//   2000 x 1024 x 1024   33.6  27.3  27.5       4096 x 1024 x 512    35.4   31.7   31.9
//   16384 x 361 x 512    43.8  39.4  39.4       16384 x 361 x 1024   59.0   58.9   57.2
//   8192 x 538 x 1024    47.4  47.5  45.7       65536 x 361 x 1024    165    165    196
// 1024 x 1024 x 1024 in parts of four steps 20.4, of eight (no second part, no joining) 17.6.
static bool large_parts(int64_t n, int64_t out, int64_t splits) { return tiles_of(n, out, 128) * splits >= 400; }

int linear8_splits(int64_t n, int64_t out, int64_t steps)
{
    const int64_t large = std::max<int64_t>(1, std::min<int64_t>(512 / tiles_of(n, out, 128), steps / 4));
    if (large_parts(n, out, large)) return (int)large;
    const int64_t tiles = tiles_of(n, out, 64);
    return (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, steps / (tiles >= 256 ? 8 : 4)));
}

template <typename S>
static void tile_by(const Linear8Args &a, hipStream_t s)
{
    const int64_t p_tiles = ceil_div(a.out, S::BP), tiles = p_tiles * ceil_div(a.n, S::BQ);
    const dim3 g((unsigned)(tiles * a.splits)), b(S::NT);
    if (wide(a)) linear8_tile_kernel<S, true><<<g, b, 0, s>>>(a, (int)p_tiles, (int)tiles);
    else linear8_tile_kernel<S, false><<<g, b, 0, s>>>(a, (int)p_tiles, (int)tiles);
}

template <typename S>
static void two_by(const Linear8Args &dx, const Linear8Args &dw, hipStream_t s)
{
    const int64_t ap = ceil_div(dx.out, S::BP), at = ap * ceil_div(dx.n, S::BQ);
    const int64_t bp = ceil_div(dw.out, S::BP), bt = bp * ceil_div(dw.n, S::BQ);
    const dim3 g((unsigned)(at + bt * dw.splits)), b(S::NT);
    if (wide(dx)) linear8_two_kernel<S, true><<<g, b, 0, s>>>(dx, (int)ap, (int)at, dw, (int)bp, (int)bt);
    else linear8_two_kernel<S, false><<<g, b, 0, s>>>(dx, (int)ap, (int)at, dw, (int)bp, (int)bt);
}

static void join(const Linear8Args &a, const ColumnSums &c, hipStream_t s)
{
    const int64_t blocks = std::min<int64_t>(ceil_div(a.n * ceil_div(a.out, 4), 1024), 256 * 4);
    linear8_join_kernel<<<dim3((unsigned)(blocks + (c.sums ? ceil_div(c.d, 64) : 0))), dim3(1024), 0, s>>>(
        a, (int)blocks, c.part, c.rows, c.d, c.sums);
}

hipError_t launch_linear8(const Linear8Args &a, hipStream_t s)
{
    if (in_panels(a)) {
        const int panels = (int)ceil_div(a.out, 128), streams = 8 * (32 / panels);
        linear8_panel_kernel<<<dim3(256), dim3(64 * PANEL_WAVES), 0, s>>>(a, panels, streams);
        return hipGetLastError();
    }
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
    const bool with_dx = dx.y != nullptr, small = dw.y && !large_parts(dw.n, dw.out, dw.splits);
    if (with_dx && small && few_tiles(dx.n, dx.out)) {
        const int64_t blocks = tiles_of(dx.n, dx.out, 64) + tiles_of(dw.n, dw.out, 64) * dw.splits;
        // of more than two blocks a CU: 4095 x 361 x 1024 29.8 and 27.9 us, 8192 x 361 x 512 34.0 and 31.2,
        // 256 x 361 x 1024, which has fewer, 12.5 and 13.8
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
