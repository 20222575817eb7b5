// expert_kernels.hip -- layers of experts: rows grouped by expert, and the
// products of each row with its own expert's weights, on MFMA.
//
// A product's rows are places of the grouping: expert e has the places
// offsets[e] .. offsets[e + 1] - 1, and place p is row rows[p] of the matrices,
// which stay in the rows' own order: kernels gather whole rows as they load a
// tile and scatter whole rows as they store one, so no sorted copy is made.
// The host does not know the group sizes: a launch has as many tiles as any
// sizes could need, and each block finds its expert from the offsets.
#include <algorithm>
#include <type_traits>

#include "expert.h"
#include "rows.h"

namespace im {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef short v4s_t __attribute__((ext_vector_type(4)));
#define IM_LDS3 __attribute__((address_space(3)))

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------------------
// Rows by expert.  A wavefront takes consecutive rows, 64 at a time: lanes of one
// expert find each other by a ballot for each bit of the expert's number, the
// first of them adds their count to the wavefront's counter of that expert, and
// a lane's rank is the counter plus the matching lanes below it.  No two lanes
// write a counter at a time, so the order is the rows' own, whatever the timing.
// Blocks of GROUP_NT threads; one block alone up to GROUP_ONE rows (its counts
// stay in LDS), else a counting launch leaves [block][expert] counts and every
// block of the second launch adds up those before it.
// ---------------------------------------------------------------------------
constexpr int GROUP_NT = 1024, GROUP_WAVES = GROUP_NT / 64;
constexpr int64_t GROUP_BLOCKS = 256;

// rows of a block, a multiple of GROUP_NT
static int64_t group_rows_of(int64_t n) { return ceil_div(std::max<int64_t>(n, 1), GROUP_BLOCKS * GROUP_NT) * GROUP_NT; }
int64_t group_blocks(int64_t n) { return ceil_div(std::max<int64_t>(n, 1), group_rows_of(n)); }

// The lanes with this lane's value v (< 2^bits).
__device__ __forceinline__ uint64_t same_lanes(int v, int bits)
{
    uint64_t m = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const uint64_t t = __ballot((v >> b) & 1);
        m &= ((v >> b) & 1) ? t : ~t;
    }
    return m;
}

struct GroupArgs {
    const int32_t *expert;
    int n, E, bits;      // values 0..E fit in `bits`
    int rows_block;
    int32_t *offsets, *rows, *count;   // count [blocks][E + 1]
};

// A row's expert, E for a row without one.
__device__ __forceinline__ int group_of(const GroupArgs &g, int i)
{
    const int e = g.expert[i];
    return (uint32_t)e < (uint32_t)g.E ? e : g.E;
}

// Adds up the block's rows: cnt[w][e] the number of wavefront w's rows of e.
__device__ __forceinline__ void group_count(const GroupArgs &g, int *cnt, int first, int last)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < GROUP_WAVES * (g.E + 1); i += GROUP_NT) cnt[i] = 0;
    __syncthreads();
    // another lane of the wavefront may have written it last: read it every time
    volatile int *mine = cnt + w * (g.E + 1);
    const int per = g.rows_block / GROUP_WAVES;
    const int b = first + w * per, e = min(b + per, last);
    for (int i0 = b; i0 < e; i0 += 64) {
        const bool on = i0 + lane < e;
        const int v = on ? group_of(g, i0 + lane) : g.E + 1;
        const uint64_t m = same_lanes(v, g.bits);
        if (on && (m & ((1ull << lane) - 1)) == 0) mine[v] = mine[v] + __popcll(m);
    }
    __syncthreads();
}

// Places of the block's rows; cnt[w][e] holds the place of wavefront w's first row of e.
__device__ __forceinline__ void group_place(const GroupArgs &g, int *cnt, int first, int last)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    // another lane of the wavefront may have written it last: read it every time
    volatile int *mine = cnt + w * (g.E + 1);
    const int per = g.rows_block / GROUP_WAVES;
    const int b = first + w * per, e = min(b + per, last);
    for (int i0 = b; i0 < e; i0 += 64) {
        const bool on = i0 + lane < e;
        const int v = on ? group_of(g, i0 + lane) : g.E + 1;
        const uint64_t m = same_lanes(v, g.bits);
        const uint64_t below = m & ((1ull << lane) - 1);
        if (on) {
            const int at = mine[v];
            g.rows[at + __popcll(below)] = i0 + lane;
            if (below == 0) mine[v] = at + __popcll(m);
        }
    }
}

__global__ __launch_bounds__(GROUP_NT) void group_count_kernel(GroupArgs g)
{
    extern __shared__ int cnt[];
    const int first = blockIdx.x * g.rows_block, last = min(first + g.rows_block, g.n);
    group_count(g, cnt, first, last);
    for (int e = threadIdx.x; e <= g.E; e += GROUP_NT) {
        int s = 0;
        for (int w = 0; w < GROUP_WAVES; ++w) s += cnt[w * (g.E + 1) + e];
        g.count[(int64_t)blockIdx.x * (g.E + 1) + e] = s;
    }
}

// MANY: blocks after group_count_kernel; else one block for all rows.
template <bool MANY>
__global__ __launch_bounds__(GROUP_NT) void group_place_kernel(GroupArgs g)
{
    extern __shared__ int cnt[];          // [GROUP_WAVES][E + 1], then [E + 2] starts
    int *start = cnt + GROUP_WAVES * (g.E + 1);
    const int first = blockIdx.x * g.rows_block, last = min(first + g.rows_block, g.n);
    group_count(g, cnt, first, last);
    // of each expert: the rows in all blocks (start) and in the blocks before this one
    // (a thread's own experts: e = thread, E + 1 <= GROUP_NT + 1 of them)
    int before[2] = {0, 0};
    for (int e = threadIdx.x, k = 0; e <= g.E; e += GROUP_NT, ++k) {
        int all = 0;
        if constexpr (MANY) {
#pragma unroll 8
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const int c = g.count[(int64_t)b * (g.E + 1) + e];
                if (b == (int)blockIdx.x) before[k] = all;
                all += c;
            }
        } else {
            for (int w = 0; w < GROUP_WAVES; ++w) all += cnt[w * (g.E + 1) + e];
        }
        start[e] = all;
    }
    __syncthreads();
    // exclusive sums over the experts, by the first wavefront
    if (threadIdx.x < 64) {
        int carry = 0;
        for (int e0 = 0; e0 <= g.E; e0 += 64) {
            const int e = e0 + threadIdx.x;
            const int v = e <= g.E ? start[e] : 0;
            int s = v;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int t = __shfl_up(s, d);
                s += (int)threadIdx.x >= d ? t : 0;
            }
            if (e <= g.E) start[e] = carry + s - v;
            carry += __shfl(s, 63);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x, k = 0; e <= g.E; e += GROUP_NT, ++k) {
        if (blockIdx.x == 0) g.offsets[e] = start[e];
        int at = start[e] + before[k];
        for (int w = 0; w < GROUP_WAVES; ++w) {
            const int c = cnt[w * (g.E + 1) + e];
            cnt[w * (g.E + 1) + e] = at;
            at += c;
        }
    }
    __syncthreads();
    group_place(g, cnt, first, last);
}

hipError_t launch_group_rows(const int32_t *expert, int64_t n, int n_experts, int32_t *offsets, int32_t *rows,
                             int32_t *count, hipStream_t s)
{
    GroupArgs g{};
    g.expert = expert;
    g.n = (int)n;
    g.E = n_experts;
    while ((1 << g.bits) <= n_experts + 1) ++g.bits;
    g.rows_block = (int)group_rows_of(n);
    g.offsets = offsets;
    g.rows = rows;
    g.count = count;
    const unsigned blocks = (unsigned)group_blocks(n);
    const size_t lds = ((size_t)GROUP_WAVES * (n_experts + 1) + n_experts + 1) * sizeof(int);
    if (blocks > 1) {
        group_count_kernel<<<dim3(blocks), dim3(GROUP_NT), lds, s>>>(g);
        group_place_kernel<true><<<dim3(blocks), dim3(GROUP_NT), lds, s>>>(g);
    } else {
        group_place_kernel<false><<<dim3(1), dim3(GROUP_NT), lds, s>>>(g);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Which expert's places a tile covers.
// ---------------------------------------------------------------------------
struct Piece {
    int e;         // its expert; E: the places without one; -1: no such tile
    int first;     // first place
    int count;     // places (<= unit)
    int index;     // the tile's number among its expert's
    int of;        // tiles of its expert
};

// Tile t when each expert's places are cut into tiles of `unit` places (the last one
// shorter), the places without an expert after them if REST.  Every lane of the
// wavefront calls it with the same t; offsets are held within [0, n].  EVEN: an expert's
// tiles are of one size, a multiple of 64 places.
template <bool REST, bool EVEN>
__device__ __forceinline__ Piece find_piece(const int32_t *offsets, int E, int n, int t, int unit)
{
    const int lane = threadIdx.x & 63;
    Piece p{-1, 0, 0, 0, 0};
    int carry = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const int e = e0 + lane;
        int a = 0, b = 0;
        if (e < E || (REST && e == E)) {
            a = min(max(offsets[e], 0), n);
            b = e < E ? min(max(offsets[e + 1], a), n) : n;
        }
        const int k = (b - a + unit - 1) / unit;
        int s = k;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int u = __shfl_up(s, d);
            s += lane >= d ? u : 0;
        }
        const uint64_t hit = __ballot(carry + s > t);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            const int la = __builtin_amdgcn_readlane(a, l), lb = __builtin_amdgcn_readlane(b, l);
            p.e = e0 + l;
            p.of = __builtin_amdgcn_readlane(k, l);
            p.index = t - (carry + __builtin_amdgcn_readlane(s, l) - p.of);
            const int size = EVEN ? ((lb - la + p.of - 1) / p.of + 63) / 64 * 64 : unit;
            p.first = min(la + p.index * size, lb);
            p.count = min(size, lb - p.first);
            return p;
        }
        carry += __builtin_amdgcn_readlane(s, 63);
    }
    return p;
}

// Row at place p, -1 where `rows` holds none.
__device__ __forceinline__ int row_at(const ExpertArgs &a, int p)
{
    const int r = a.rows ? a.rows[p] : p;
    return (uint32_t)r < (uint32_t)a.n ? r : -1;
}

// ---------------------------------------------------------------------------
// The products.  All three are C[q][p] = sum_k Q[q][k] P[p][k]:
//   forward  q = row,    p = output, k = input    P = W_e    (k along its rows)
//   dx       q = row,    p = input,  k = output   P = W_e^T  (k across its rows)
//   dw       q = output, p = input,  k = row      Q = dy^T, P = x^T (k across)
// A block of WP x WQ wavefronts forms BP x BQ of C, a wavefront TP x TQ tiles of
// v_mfma_f32_32x32x16_bf16, whose accumulator gives a lane one q and four
// consecutive p per register group.  K steps of 64 through two LDS stages, the
// next step's loads in flight in registers while a step is multiplied.
//
// A tile with k along its rows lies in LDS rows of 72 bf16 (144 bytes: fragment
// reads meet no bank twice); one with k across lies as in memory, [64 k][columns],
// in rows of 32 more columns, and its fragments are read transposed (in every
// 16-lane group, lane 4j+q addresses row k0+j, columns c0+4q.., and lane l receives
// rows k0..k0+3 of column c0+l).
// ---------------------------------------------------------------------------
enum { OP_FORWARD, OP_DX, OP_DW };

constexpr int BK = 64;

// LDS elements of a tile of C columns (rows) and 64 k.
constexpr int along_lds(int rows) { return rows * (BK + 8); }
constexpr int across_lds(int cols) { return BK * (cols + 32); }

// 16-byte pieces of a tile with k along its rows: thread t holds piece t % 8 of
// the rows t / 8 + c NT / 8.
template <int R, int NT>
struct AlongTile {
    static constexpr int C = R * 8 / NT;
    const uint16_t *p[C];
    u32x4_r v[C];
    // row(i): the address of row i of the tile (one that can be read, for all i < R)
    template <typename F>
    __device__ __forceinline__ void init(F row)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) p[c] = row(threadIdx.x / 8 + c * (NT / 8)) + (threadIdx.x & 7) * 8;
    }
    // K step kt of K values
    __device__ __forceinline__ void load(int kt, int K)
    {
        if ((kt + 1) * BK <= K) {
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = *(const u32x4_a2 *)(p[c] + kt * BK);
        } else {
            const int nv = K - kt * BK - (threadIdx.x & 7) * 8;
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = load8_bits(p[c] + kt * BK, nv);
        }
    }
    __device__ __forceinline__ void store(uint16_t *lds) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c)
            *(u32x4_r *)(lds + (threadIdx.x / 8 + c * (NT / 8)) * (BK + 8) + (threadIdx.x & 7) * 8) = v[c];
    }
};

// A fragment (8 consecutive k of 32 rows) of such a tile: lane l row l % 32, k + 8 (l / 32)..
__device__ __forceinline__ bf16x8_t along_frag(const uint16_t *lds, int row, int k)
{
    const int lane = threadIdx.x & 63;
    return *(const bf16x8_t *)(lds + (row + (lane & 31)) * (BK + 8) + k + 8 * (lane >> 5));
}

// A tile of 64 k rows of N columns: thread t holds the 16-byte piece t % (N / 8) of
// rows t / (N / 8) + c NT / (N / 8).
template <int N, int NT>
struct AcrossTile {
    static constexpr int PR = N / 8, C = BK * PR / NT;
    u32x4_r v[C];
    __device__ static int piece() { return threadIdx.x % PR; }
    __device__ static int krow(int c) { return threadIdx.x / PR + c * (NT / PR); }
    // row(i): the address of k row i of the step, null for none; nv: valid columns from
    // this thread's piece on
    template <typename F>
    __device__ __forceinline__ void load(F row, int nv)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const uint16_t *p = row(krow(c));
            v[c] = load8_bits(p + piece() * 8, p ? nv : 0);
        }
    }
    __device__ __forceinline__ void store(uint16_t *lds) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) *(u32x4_r *)(lds + krow(c) * (N + 32) + piece() * 8) = v[c];
    }
};

// The same from a checkpoint: bytes and scales are held until the store, which
// restores the values (exact in bf16).
template <int N, int NT>
struct AcrossCkpt {
    static constexpr int PR = N / 8, C = BK * PR / NT;
    u32x2_r v[C];
    int scale[C];
    __device__ static int piece() { return threadIdx.x % PR; }
    __device__ static int krow(int c) { return threadIdx.x / PR + c * (NT / PR); }
    // row(i): k row i's index, negative for none; col: the tile's first column
    template <typename F>
    __device__ __forceinline__ void load(const im_checkpoint &q, F row, int col, int nv)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int r = row(krow(c));
            const int m = r >= 0 ? nv : 0;
            const int at = col + piece() * 8;
            v[c] = load8_bytes(q.q + (int64_t)r * q.ld_q + at, m);
            scale[c] = m > 0 ? q.scale[(int64_t)r * q.ld_scale + (at >> 5)] : 0;
        }
    }
    __device__ __forceinline__ void store(uint16_t *lds) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float f[8];
            ckpt_unpack(v[c], scale[c], f);
            *(u32x4_r *)(lds + krow(c) * (N + 32) + piece() * 8) = pack8(f);
        }
    }
};

template <int N>
__device__ __forceinline__ bf16x8_t across_frag(const uint16_t *lds, int col, int k)
{
    const int lane = threadIdx.x & 63, gi = lane >> 4, si = lane & 15;
    const uint16_t *p = lds + (k + 8 * (gi >> 1) + (si >> 2)) * (N + 32) + col + 16 * (gi & 1) + 4 * (si & 3);
    const v4s_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((IM_LDS3 v4s_t *)p);
    const v4s_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((IM_LDS3 v4s_t *)(p + 4 * (N + 32)));
    const short v8[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8_t, v8);
}

template <int OP, int WP, int WQ, int TP, int TQ>
struct Tile {
    static constexpr int NT = 64 * WP * WQ, BP = 32 * WP * TP, BQ = 32 * WQ * TQ;
    static constexpr int P_LDS = OP == OP_FORWARD ? along_lds(BP) : across_lds(BP);
    static constexpr int Q_LDS = OP == OP_DW ? across_lds(BQ) : along_lds(BQ);
    static constexpr int STAGE = P_LDS + Q_LDS;
    static constexpr int LDO = BP + 8;      // epilogue rows
    static constexpr int LDS = 2 * STAGE > BQ * LDO || OP == OP_DW ? 2 * STAGE : BQ * LDO;
};

template <int TP, int TQ>
__device__ __forceinline__ void clear(f32x16_t (&acc)[TP][TQ])
{
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
        for (int j = 0; j < TQ; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
}

// ---------------------------------------------------------------------------
// Forward and input gradient: C rows are places.  Blocks p-tile fastest, blocks of
// one XCD consecutive: the tiles that read one set of rows share an L2.
// ---------------------------------------------------------------------------
template <int OP, int WP, int WQ, int TP, int TQ>
__global__ __launch_bounds__(64 * WP * WQ) void expert_rows_kernel(ExpertArgs a, int p_tiles)
{
    using T = Tile<OP, WP, WQ, TP, TQ>;
    constexpr int NT = T::NT, BP = T::BP, BQ = T::BQ;
    __shared__ __attribute__((aligned(16))) uint16_t lds[T::LDS];
    __shared__ int row_of[BQ];
    const int id = xcd_order(blockIdx.x, gridDim.x);
    const Piece pc = find_piece<true, false>(a.offsets, a.E, a.n, id / p_tiles, BQ);
    if (pc.e < 0) return;
    const int p0 = id % p_tiles * BP;
    const int NP = OP == OP_FORWARD ? a.out : a.in, K = OP == OP_FORWARD ? a.in : a.out;
    for (int i = threadIdx.x; i < BQ; i += NT) row_of[i] = i < pc.count ? row_at(a, pc.first + i) : -1;
    __syncthreads();

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wp = wave % WP * TP * 32, wq = wave / WP * TQ * 32;
    f32x16_t acc[TP][TQ];
    clear(acc);
    if (pc.e < a.E) {
        const uint16_t *q = OP == OP_FORWARD ? a.x : a.dy;
        const int64_t ldq = OP == OP_FORWARD ? a.ld_x : a.ld_dy;
        const uint16_t *w = a.w + (int64_t)pc.e * a.out * a.ld_w;
        AlongTile<BQ, NT> tq;
        // rows past the tile's last read row 0: their sums are not stored
        tq.init([&](int i) { return q + (int64_t)max(row_of[i], 0) * ldq; });
        const int nk = (K + BK - 1) / BK;
        auto multiply = [&](const uint16_t *ps, const uint16_t *qs) {
#pragma unroll
            for (int s = 0; s < BK; s += 16) {
                bf16x8_t fp[TP], fq[TQ];
#pragma unroll
                for (int i = 0; i < TP; ++i) {
                    if constexpr (OP == OP_FORWARD) fp[i] = along_frag(ps, wp + 32 * i, s);
                    else fp[i] = across_frag<BP>(ps, wp + 32 * i, s);
                }
#pragma unroll
                for (int j = 0; j < TQ; ++j) fq[j] = along_frag(qs, wq + 32 * j, s);
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int j = 0; j < TQ; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[i], fq[j], acc[i][j], 0, 0, 0);
            }
        };
        auto loop = [&](auto &tp, auto load_p) {
            load_p(0);
            tq.load(0, K);
            tp.store(lds);
            tq.store(lds + T::P_LDS);
            __syncthreads();
            if (nk > 1) load_p(1), tq.load(1, K);
            for (int kt = 0; kt < nk; ++kt) {
                const uint16_t *st = lds + (kt & 1) * T::STAGE;
                multiply(st, st + T::P_LDS);
                if (kt + 1 < nk) {
                    uint16_t *nx = lds + (~kt & 1) * T::STAGE;
                    tp.store(nx);
                    tq.store(nx + T::P_LDS);
                }
                if (kt + 2 < nk) load_p(kt + 2), tq.load(kt + 2, K);
                __syncthreads();
            }
        };
        if constexpr (OP == OP_FORWARD) {
            AlongTile<BP, NT> tp;
            tp.init([&](int i) { return w + (int64_t)min(p0 + i, NP - 1) * a.ld_w; });
            loop(tp, [&](int kt) { tp.load(kt, K); });
        } else {
            AcrossTile<BP, NT> tp;
            const int nv = NP - p0 - tp.piece() * 8;
            loop(tp, [&](int kt) {
                tp.load([&](int k) { return kt * BK + k < K ? w + (int64_t)(kt * BK + k) * a.ld_w + p0 : nullptr; }, nv);
            });
        }
    }

    // lane l: place wq + 32 j + l % 32, features wp + 32 i + 8 g + 4 (l / 32) + 0..3
    const bool has = pc.e < a.E;
    auto finish = [&](int f, f32x4_r v) {
        if constexpr (OP == OP_FORWARD) {
            if (a.bias && has) {
                const float *b = a.bias + (int64_t)pc.e * a.out + f;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] += f + k < NP ? b[k] : 0.0f;
            }
            if (a.relu)
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = v[k] < 0.0f ? 0.0f : v[k];   // NaN stays
        }
        return v;
    };
    if (OP == OP_FORWARD && a.y_f32) {
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
            const int r = row_of[wq + 32 * j + (lane & 31)];
            if (r < 0) continue;
            float *y = (float *)a.y + (int64_t)r * a.ld_y;
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int f = p0 + wp + 32 * i + 8 * g + 4 * (lane >> 5);
                    const f32x4_r v = finish(f, f32x4_r{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                                                        acc[i][j][4 * g + 3]});
                    if (f + 4 <= NP) {
                        *(f32x4_a4 *)(y + f) = v;
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (f + k < NP) y[f + k] = v[k];
                    }
                }
        }
        return;
    }
    // bf16 rows meet in LDS and leave in 16-byte pieces (the last K step ended at a barrier)
#pragma unroll
    for (int j = 0; j < TQ; ++j)
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int f = wp + 32 * i + 8 * g + 4 * (lane >> 5);
                const f32x4_r v = finish(p0 + f, f32x4_r{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                                                         acc[i][j][4 * g + 3]});
                const u32x2_r o = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                *(u32x2_r *)(lds + (wq + 32 * j + (lane & 31)) * T::LDO + f) = o;
            }
    __syncthreads();
#pragma unroll 4
    for (int t = tid; t < BQ * (BP / 8); t += NT) {
        const int i = t / (BP / 8), f = t % (BP / 8) * 8;
        const int r = row_of[i], nv = NP - p0 - f;
        if (r < 0 || nv <= 0) continue;
        u32x4_r o = *(const u32x4_r *)(lds + i * T::LDO + f);
        if constexpr (OP == OP_FORWARD) {
            store8_bits((uint16_t *)a.y + (int64_t)r * a.ld_y + p0 + f, nv, o);
        } else {
            if (a.relu) {
                // keep the values whose input is positive
                uint32_t keep = 0;
                if (a.x) {
                    const u32x4_r h = load8_bits(a.x + (int64_t)r * a.ld_x + p0 + f, nv);
                    float x[8];
                    unpack8(h, x);
#pragma unroll
                    for (int k = 0; k < 8; ++k) keep |= (x[k] > 0.0f ? 1u : 0u) << k;
                } else {
                    const u32x2_r h = load8_bytes(a.c.q + (int64_t)r * a.c.ld_q + p0 + f, nv);
                    const bool nan = a.c.scale[(int64_t)r * a.c.ld_scale + ((p0 + f) >> 5)] == 255;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        keep |= ((int8_t)(h[k >> 2] >> (8 * (k & 3))) > 0 && !nan ? 1u : 0u) << k;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    o[k] &= ((keep >> (2 * k)) & 1 ? 0x0000FFFFu : 0u) | ((keep >> (2 * k + 1)) & 1 ? 0xFFFF0000u : 0u);
            }
            store8_bits(a.dx + (int64_t)r * a.ld_dx + p0 + f, nv, o);
        }
    }
}

// ---------------------------------------------------------------------------
// Weight gradient.  An expert's rows are cut into pieces of at most a.piece; a
// block forms BQ outputs x BP inputs of one piece.  The blocks of the first inputs
// also form db: dy times a fragment of ones.
// ---------------------------------------------------------------------------
template <int WP, int WQ, int TP, int TQ, bool CK>
__global__ __launch_bounds__(64 * WP * WQ) void expert_dw_kernel(ExpertArgs a, int p_tiles, int q_tiles)
{
    using T = Tile<OP_DW, WP, WQ, TP, TQ>;
    constexpr int NT = T::NT, BP = T::BP, BQ = T::BQ;
    __shared__ __attribute__((aligned(16))) uint16_t lds[T::LDS];
    const int id = xcd_order(blockIdx.x, gridDim.x);
    const int piece = id / (p_tiles * q_tiles);
    const Piece pc = find_piece<false, true>(a.offsets, a.E, a.n, piece, a.piece);
    if (pc.e < 0) return;
    const int p0 = id % p_tiles * BP, q0 = id / p_tiles % q_tiles * BQ;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wp = wave % WP * TP * 32, wq = wave / WP * TQ * 32;
    const bool with_db = a.db && p0 == 0 && wp == 0;
    const int K = pc.count, nk = (K + BK - 1) / BK;

    AcrossTile<BQ, NT> tq;
    std::conditional_t<CK, AcrossCkpt<BP, NT>, AcrossTile<BP, NT>> tp;
    // rows of the step after the one that is being loaded
    int rq[tq.C], rp[tp.C];
    auto rows_of = [&](int kt) {
#pragma unroll
        for (int c = 0; c < tq.C; ++c) {
            const int k = kt * BK + tq.krow(c);
            rq[c] = k < K ? row_at(a, pc.first + k) : -1;
        }
#pragma unroll
        for (int c = 0; c < tp.C; ++c) {
            const int k = kt * BK + tp.krow(c);
            rp[c] = k < K ? row_at(a, pc.first + k) : -1;
        }
    };
    const int nvq = a.out - q0 - tq.piece() * 8, nvp = a.dw ? a.in - p0 - tp.piece() * 8 : 0;
    auto load = [&]() {
        int c = 0;
        tq.load([&](int) { const int r = rq[c++]; return r >= 0 ? a.dy + (int64_t)r * a.ld_dy + q0 : nullptr; }, nvq);
        c = 0;
        if constexpr (CK) {
            tp.load(a.c, [&](int) { return rp[c++]; }, p0, nvp);
        } else {
            tp.load([&](int) { const int r = rp[c++]; return r >= 0 ? a.x + (int64_t)r * a.ld_x + p0 : nullptr; }, nvp);
        }
    };

    f32x16_t acc[TP][TQ], sums[1][TQ];
    clear(acc);
    clear(sums);
    bf16x8_t ones;
#pragma unroll
    for (int k = 0; k < 8; ++k) ones[k] = (__bf16)1.0f;
    if (nk > 0) {
        rows_of(0);
        load();
        if (nk > 1) rows_of(1);
        tp.store(lds);
        tq.store(lds + T::P_LDS);
        __syncthreads();
        if (nk > 1) load();
        if (nk > 2) rows_of(2);
    }
    for (int kt = 0; kt < nk; ++kt) {
        const uint16_t *ps = lds + (kt & 1) * T::STAGE, *qs = ps + T::P_LDS;
#pragma unroll
        for (int s = 0; s < BK; s += 16) {
            bf16x8_t fp[TP], fq[TQ];
#pragma unroll
            for (int i = 0; i < TP; ++i) fp[i] = across_frag<BP>(ps, wp + 32 * i, s);
#pragma unroll
            for (int j = 0; j < TQ; ++j) fq[j] = across_frag<BQ>(qs, wq + 32 * j, s);
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int j = 0; j < TQ; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[i], fq[j], acc[i][j], 0, 0, 0);
            if (with_db)
#pragma unroll
                for (int j = 0; j < TQ; ++j)
                    sums[0][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, fq[j], sums[0][j], 0, 0, 0);
        }
        if (kt + 1 < nk) {
            uint16_t *nx = lds + (~kt & 1) * T::STAGE;
            tp.store(nx);
            tq.store(nx + T::P_LDS);
        }
        if (kt + 2 < nk) load();
        if (kt + 3 < nk) rows_of(kt + 3);
        __syncthreads();
    }

    const int in4 = (a.in + 3) & ~3;
    const bool alone = pc.of == 1;
    float *c = alone ? a.dw + (int64_t)pc.e * a.out * a.ld_dw : a.part + (int64_t)piece * a.out * in4;
    float *db = alone ? a.db + (int64_t)pc.e * a.out : a.part_db + (int64_t)piece * a.out;
    const int64_t ldc = alone ? a.ld_dw : in4;
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
        const int o = q0 + wq + 32 * j + (lane & 31);
        if (o >= a.out) continue;
        if (with_db && lane < 32) db[o] = sums[0][j][0];
        if (!a.dw) continue;
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int f = p0 + wp + 32 * i + 8 * g + 4 * (lane >> 5);
                const f32x4_r v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                if (f + 4 <= a.in) {
                    *(f32x4_a4 *)(c + o * ldc + f) = v;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (f + k < a.in) c[o * ldc + f + k] = v[k];
                }
            }
    }
}

// dw and db of the experts whose rows were not one piece: the pieces' sums in
// order, zeros without a piece.  blockIdx.y: the expert; x over [out][in4 / 4], then
// [out] of db.
__global__ __launch_bounds__(256) void expert_dw_sum_kernel(ExpertArgs a)
{
    const int e = blockIdx.y, lane = threadIdx.x & 63;
    // pieces of the experts before e, and of e (every wavefront for itself)
    int before = 0, mine = 0;
    for (int e0 = 0; e0 <= e; e0 += 64) {
        const int j = e0 + lane;
        int k = 0;
        if (j <= e) {
            const int f = min(max(a.offsets[j], 0), a.n), l = min(max(a.offsets[j + 1], f), a.n);
            k = (l - f + a.piece - 1) / a.piece;
        }
        if (j == e) mine = k;
        else before += k;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        before += __shfl_xor(before, d);
        mine += __shfl_xor(mine, d);
    }
    if (mine == 1) return;
    const int in4 = (a.in + 3) & ~3, q = in4 / 4;
    const int64_t size = (int64_t)a.out * q, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < size) {
        if (!a.dw) return;
        const int o = (int)(t / q), f = (int)(t % q) * 4;
        f32x4_r s = {0.0f, 0.0f, 0.0f, 0.0f};
        const float *p = a.part + ((int64_t)before * a.out + o) * in4 + f;
        for (int k = 0; k < mine; ++k) s += *(const f32x4_r *)(p + (int64_t)k * a.out * in4);
        float *c = a.dw + ((int64_t)e * a.out + o) * a.ld_dw + f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (f + k < a.in) c[k] = s[k];
    } else if (a.db && t - size < a.out) {
        const int o = (int)(t - size);
        float s = 0.0f;
        for (int k = 0; k < mine; ++k) s += a.part_db[((int64_t)before + k) * a.out + o];
        a.db[(int64_t)e * a.out + o] = s;
    }
}

template <int OP, int WP, int WQ, int TP, int TQ>
static void rows_go(const ExpertArgs &a, hipStream_t s)
{
    using T = Tile<OP, WP, WQ, TP, TQ>;
    const int p_tiles = (int)ceil_div(OP == OP_FORWARD ? a.out : a.in, T::BP);
    // any group sizes: whole tiles, and a shorter one for each expert and for the rest
    const int64_t tiles = a.n / T::BQ + std::min<int64_t>(a.E + 1, a.n);
    expert_rows_kernel<OP, WP, WQ, TP, TQ><<<dim3((unsigned)(tiles * p_tiles)), dim3(T::NT), 0, s>>>(a, p_tiles);
}

hipError_t launch_expert_linear(const ExpertArgs &a, hipStream_t s)
{
    rows_go<OP_FORWARD, 2, 2, 2, 2>(a, s);
    return hipGetLastError();
}

constexpr int DW_TILE = 128;

int expert_piece_rows(int64_t n, int n_experts, int in, int out)
{
    const int64_t tiles = ceil_div(in, DW_TILE) * ceil_div(out, DW_TILE);
    const int64_t pieces = std::max<int64_t>(1, ceil_div(512, tiles));
    return (int)(ceil_div(std::max<int64_t>(ceil_div(n, pieces), 1024), 64) * 64);
}

int64_t expert_pieces(int64_t n, int n_experts, int in, int out)
{
    return n / expert_piece_rows(n, n_experts, in, out) + std::min<int64_t>(n_experts, n);
}

hipError_t launch_expert_grad(const ExpertArgs &a, hipStream_t s)
{
    if (a.dx && a.n > 0) rows_go<OP_DX, 2, 2, 2, 2>(a, s);
    if (a.dw || a.db) {
        const int p_tiles = a.dw ? (int)ceil_div(a.in, DW_TILE) : 1, q_tiles = (int)ceil_div(a.out, DW_TILE);
        const int64_t pieces = expert_pieces(a.n, a.E, a.in, a.out);
        const dim3 g((unsigned)(pieces * p_tiles * q_tiles));
        if (pieces > 0) {
            if (a.x || !a.dw) expert_dw_kernel<2, 2, 2, 2, false><<<g, dim3(256), 0, s>>>(a, p_tiles, q_tiles);
            else expert_dw_kernel<2, 2, 2, 2, true><<<g, dim3(256), 0, s>>>(a, p_tiles, q_tiles);
        }
        const int64_t work = (int64_t)a.out * ((a.in + 3) / 4) + a.out;
        expert_dw_sum_kernel<<<dim3((unsigned)ceil_div(work, 256), a.E), dim3(256), 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace im
