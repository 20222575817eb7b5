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
// Blocks of GROUP_NT threads; one block alone up to GROUP_ONE rows (its counts stay in
// LDS), else a counting launch leaves [block][expert] counts and every block of the second
// launch adds up those before it.  us in one launch and in two, replayed from a graph: 2048
// rows of 64 experts 6.0, 7.4; 4096 rows 9.0, 7.5 (of 1024 experts 16.7, 20.2); 6000 rows 11.9,
// 7.7.  The bound counts the 4 us that a second launch costs the host where there is no graph.
// 262144 rows of 64 experts: 3.5 us to count, 7.6 to place.
// ---------------------------------------------------------------------------
constexpr int GROUP_NT = 1024, GROUP_WAVES = GROUP_NT / 64;
constexpr int64_t GROUP_BLOCKS = 256, GROUP_ONE = 4096;

// rows of a block, a multiple of GROUP_NT
static int64_t group_rows_of(int64_t n)
{
    const int64_t blocks = n <= GROUP_ONE ? 1 : GROUP_BLOCKS;
    return ceil_div(std::max<int64_t>(n, 1), blocks * GROUP_NT) * GROUP_NT;
}
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
    extern __shared__ int cnt[];          // [GROUP_WAVES][E + 1], then of each expert:
    int *start = cnt + GROUP_WAVES * (g.E + 1);      // the rows in all blocks, then the first place
    int *before = start + g.E + 1;                   // the rows in the blocks before this one
    const int first = blockIdx.x * g.rows_block, last = min(first + g.rows_block, g.n);
    for (int e = threadIdx.x; e <= g.E; e += GROUP_NT) start[e] = before[e] = 0;
    group_count(g, cnt, first, last);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if constexpr (MANY) {
        // wavefront w adds up blocks w, w + 16, .. (whole numbers: their order does not matter)
        for (int e = lane; e <= g.E; e += 64) {
            int all = 0, less = 0;
#pragma unroll 8
            for (int b = w; b < (int)gridDim.x; b += GROUP_WAVES) {
                const int c = g.count[(int64_t)b * (g.E + 1) + e];
                all += c;
                less += b < (int)blockIdx.x ? c : 0;
            }
            atomicAdd(&start[e], all);
            atomicAdd(&before[e], less);
        }
    } else {
        for (int e = threadIdx.x; e <= g.E; e += GROUP_NT) {
            int all = 0;
            for (int v = 0; v < GROUP_WAVES; ++v) all += cnt[v * (g.E + 1) + e];
            start[e] = all;
        }
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
    for (int e = threadIdx.x; e <= g.E; e += GROUP_NT) {
        if (blockIdx.x == 0) g.offsets[e] = start[e];
        int at = start[e] + before[e];
        for (int v = 0; v < GROUP_WAVES; ++v) {
            const int c = cnt[v * (g.E + 1) + e];
            cnt[v * (g.E + 1) + e] = at;
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
    const size_t lds = (size_t)(GROUP_WAVES + 2) * (n_experts + 1) * sizeof(int);
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
};

// Tile t when each expert's places are cut into tiles of `unit` places (the last one
// shorter), the places without an expert after them.  Every lane of the wavefront
// calls it with the same t; offsets are held within [0, n].
__device__ __forceinline__ Piece find_piece(const int32_t *offsets, int E, int n, int t, int unit)
{
    const int lane = threadIdx.x & 63;
    Piece p{-1, 0, 0};
    int carry = 0;
    for (int e0 = 0; e0 <= E; e0 += 64) {
        const int e = e0 + lane;
        int a = 0, b = 0;
        if (e <= E) {
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
            const int index = t - (carry + __builtin_amdgcn_readlane(s, l) - __builtin_amdgcn_readlane(k, l));
            p.first = la + index * unit;
            p.count = min(unit, lb - p.first);
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
// consecutive p per register group.
//
// K steps of BK go through a ring of NS stages in LDS.  Operands whose rows are 16-byte
// aligned are copied into it by direct loads (16 bytes a lane, no registers between),
// NS - 1 steps ahead; others (odd row strides) pass through D sets of registers, D steps
// ahead.  A step waits for its own loads only (vmcnt counts the later ones) and has
// one barrier.
//
// A direct load writes 64 consecutive 16-byte pieces, so a stage has no padding;
// pieces are permuted in their row instead, by the address that each lane loads:
//   k along: rows of BK values, piece c of row r at c ^ (r / (128 / BK)) mod (BK / 8):
//     16 rows' pieces of one k cover all banks;
//   k across: rows of N columns, 64-byte quarters permuted by the row: the four rows x
//     64 bytes that a half wavefront reads transposed cover all banks (in every 16-lane
//     group, lane 4j+q addresses row k0+j, columns c0+4q.., and lane l receives rows
//     k0..k0+3 of column c0+l).
// ---------------------------------------------------------------------------
// dx alone, or masked by its input being positive (bf16 or a checkpoint)
enum { OP_FORWARD, OP_DX, OP_DX_X, OP_DX_CKPT };

__device__ const uint4 zero_piece = {0, 0, 0, 0};

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

// The block meets; LDS accesses stay on their side.
__device__ __forceinline__ void meet()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
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

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Rows at any address, with an end inside a piece: the load takes eight values that end at
// the row's end at the latest (`back` values before the piece), always, so that loads need
// no branches, and end_of_row shifts them down, zeros after them, when they are stored.
// nv: values of the row from the piece's first on, also none or fewer.  A row shorter than
// eight values is read one by one (NARROW).
__device__ __forceinline__ int window_back(int nv) { return 8 - min(nv, 8); }
__device__ __forceinline__ u32x4_r end_of_row(u32x4_r r, int nv)
{
    uint64_t lo = r[0] | (uint64_t)r[1] << 32, hi = r[2] | (uint64_t)r[3] << 32;
    const int gone = 8 - max(min(nv, 8), 0), s = 16 * (gone & 3);
    if (gone >= 4) lo = hi, hi = 0;
    if (gone == 8) lo = 0;
    if (s) lo = lo >> s | hi << (64 - s), hi >>= s;
    const u32x4_r o = {(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
    return o;
}
__device__ __forceinline__ u32x2_r end_of_row(u32x2_r r, int nv)
{
    const int gone = 8 - max(min(nv, 8), 0);
    const uint64_t w = gone == 8 ? 0 : (r[0] | (uint64_t)r[1] << 32) >> (8 * gone);
    return u32x2_r{(uint32_t)w, (uint32_t)(w >> 32)};
}

// A tile of R rows with k along them.  Thread t holds pieces u of the rows row(u).
template <int R, int NT, int BK, int D>
struct AlongTile {
    static constexpr int PITCH = BK * 2, SLOTS = BK / 8, U = R * PITCH / (NT * 16), BYTES = R * PITCH;
    static_assert(U * NT * 16 == BYTES, "whole pieces");
    const uint16_t *p[U];
    u32x4_r v[D][U];
    __device__ static int row(int u)
    {
        return (u * (NT / 64) + wave_id()) * (64 / SLOTS) + (threadIdx.x & 63) / SLOTS;
    }
    __device__ static int perm(int r) { return BK == 32 ? (r >> 2) & 3 : (r >> 1) & 7; }
    __device__ static int col() { return (((int)threadIdx.x & (SLOTS - 1)) ^ perm(row(0))) * 8; }
    // at(i): the address of row i of the tile (one that can be read, for all i < R)
    template <typename F>
    __device__ __forceinline__ void init(F at)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) p[u] = at(row(u)) + col();
    }
    // piece u of a step of BK values
    __device__ __forceinline__ void copy(int u, int kt, char *lds)
    {
        copy_to_lds(p[u] + kt * BK, lds + (u * (NT / 64) + wave_id()) * 1024);
    }
    // a step (also one past the last) of K values in all, through register set d
    template <bool NARROW>
    __device__ __forceinline__ void load(int d, int kt, int K)
    {
        const int nv = K - kt * BK - col();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint16_t *at = p[u] + kt * BK;
            v[d][u] = NARROW ? load8_bits(at, nv) : *(const u32x4_a2 *)(at - window_back(nv));
        }
    }
    template <bool NARROW>
    __device__ __forceinline__ void store(int d, int kt, int K, char *lds) const
    {
        const bool end = !NARROW && (kt + 1) * BK > K;
        const int nv = K - kt * BK - col();
#pragma unroll
        for (int u = 0; u < U; ++u)
            *(u32x4_r *)(lds + (u * (NT / 64) + wave_id()) * 1024 + (threadIdx.x & 63) * 16) =
                end ? end_of_row(v[d][u], nv) : v[d][u];
    }
    // 8 consecutive k (of substep s) of 32 rows: lane l row l % 32, k + 8 (l / 32)..
    __device__ static bf16x8_t frag(const char *lds, int row, int s)
    {
        const int lane = threadIdx.x & 63, r = lane & 31;
        const int at = r * PITCH + (((lane >> 5) ^ perm(r)) << 4);
        return *(const bf16x8_t *)(lds + row * PITCH + (at ^ (s << 5)));
    }
};

// A tile of BK k rows of N columns, of which the thread's nv columns from its own first one
// on exist.
template <int N, int NT, int BK, int D>
struct AcrossTile {
    static constexpr int PITCH = N * 2, SLOTS = N / 8, U = BK * PITCH / (NT * 16), BYTES = BK * PITCH;
    static_assert(U * NT * 16 == BYTES, "whole pieces");
    u32x4_r v[D][U];
    __device__ static int krow(int u) { return ((u * (NT / 64) + wave_id()) * 64 + (threadIdx.x & 63)) / SLOTS; }
    // quarter permutation of row k; the same for the rows of one thread
    __device__ static int perm(int k) { return N >= 128 ? k & 3 : (k >> 1) & 1; }
    __device__ static int col() { return (((int)threadIdx.x & (SLOTS - 1)) ^ (perm(krow(0)) << 2)) * 8; }
    // Piece u from `from`, the address of this thread's first column in k row krow(u), null
    // for none.  A piece that holds a valid column is read whole: 16 aligned bytes lie in one
    // page, and what they hold past the row's end meets columns that are not stored.
    __device__ __forceinline__ void copy(int u, const uint16_t *from, char *lds)
    {
        copy_to_lds(from ? (const void *)from : (const void *)&zero_piece, lds + (u * (NT / 64) + wave_id()) * 1024);
    }
    // through register set d; at(u): that address, whatever nv; whole: all threads' nv >= 8
    template <bool NARROW, typename F>
    __device__ __forceinline__ void load(int d, F at, int nv)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint16_t *p = at(u);
            v[d][u] = NARROW ? load8_bits(p, p ? nv : 0)
                             : *(const u32x4_a2 *)(p ? p - window_back(nv) : (const uint16_t *)&zero_piece);
        }
    }
    template <bool NARROW>
    __device__ __forceinline__ void store(int d, int nv, bool whole, char *lds) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u)
            *(u32x4_r *)(lds + (u * (NT / 64) + wave_id()) * 1024 + (threadIdx.x & 63) * 16) =
                NARROW || whole ? v[d][u] : end_of_row(v[d][u], nv);
    }
    __device__ static bf16x8_t frag(const char *lds, int col, int s)
    {
        const int lane = threadIdx.x & 63, gi = lane >> 4, si = lane & 15;
        const int k = 8 * (gi >> 1) + (si >> 2);
        const char *p = lds + (s * 16 + k) * PITCH + (((col >> 5) ^ perm(k)) << 6) + 32 * (gi & 1) + 8 * (si & 3);
        const v4s_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((IM_LDS3 v4s_t *)p);
        const v4s_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((IM_LDS3 v4s_t *)(p + 4 * PITCH));
        const short v8[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8_t, v8);
    }
};

// The same from a checkpoint through registers: bytes and scales are held until the
// store, which restores the values (exact in bf16).
template <int N, int NT, int BK, int D>
struct AcrossCkpt : AcrossTile<N, NT, BK, 1> {
    using B = AcrossTile<N, NT, BK, 1>;
    u32x2_r q[D][B::U];
    int scale[D][B::U];
    // row(u): the index of k row krow(u), negative for none; col: this thread's first column
    template <bool NARROW, typename F>
    __device__ __forceinline__ void load(int d, const im_checkpoint &c, F row, int col, int nv)
    {
#pragma unroll
        for (int u = 0; u < B::U; ++u) {
            const int64_t r = row(u);
            const int8_t *p = c.q + r * c.ld_q + col;
            if constexpr (NARROW) q[d][u] = load8_bytes(p, r >= 0 ? nv : 0);
            else q[d][u] = *(const u32x2_a1 *)(r >= 0 ? p - window_back(nv) : (const int8_t *)&zero_piece);
            scale[d][u] = *(r >= 0 ? c.scale + r * c.ld_scale + (min(col, col + nv - 1) >> 5)
                                   : (const uint8_t *)&zero_piece);
        }
    }
    template <bool NARROW>
    __device__ __forceinline__ void store(int d, int nv, bool whole, char *lds)
    {
#pragma unroll
        for (int u = 0; u < B::U; ++u) {
            float f[8];
            ckpt_unpack(NARROW || whole ? q[d][u] : end_of_row(q[d][u], nv), scale[d][u], f);
            this->v[0][u] = pack8(f);
        }
        B::template store<true>(0, 0, true, lds);
    }
};

// A checkpoint by direct loads: the bytes of BK rows x N columns go to a ring of their own
// in LDS, 16 a lane with their scale; each lane restores what it copied itself into the
// tile that the fragments are read from.
template <int N, int NT, int BK>
struct CkptBytes {
    static constexpr int SLOTS = N / 16, U = BK * N / (NT * 16), BYTES = BK * N + U * NT * 4;
    static_assert(U * NT * 16 == BK * N, "whole pieces");
    __device__ static int krow(int u) { return ((u * (NT / 64) + wave_id()) * 64 + (threadIdx.x & 63)) / SLOTS; }
    __device__ static int col() { return ((int)threadIdx.x & (SLOTS - 1)) * 16; }
    // row: k row krow(u)'s index, negative for none; col: this thread's first column, < 0 past the last
    __device__ __forceinline__ static void copy(int u, const im_checkpoint &c, int64_t row, int col, char *lds)
    {
        const bool on = row >= 0 && col >= 0;
        const int at = u * (NT / 64) + wave_id();
        copy_to_lds(on ? (const void *)(c.q + row * c.ld_q + col) : (const void *)&zero_piece, lds + at * 1024);
        copy_byte_to_lds(on ? (const void *)(c.scale + row * c.ld_scale + (col >> 5)) : (const void *)&zero_piece,
                         lds + BK * N + at * 256);
    }
    __device__ __forceinline__ static void restore(const char *lds, char *tile)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = u * (NT / 64) + wave_id(), k = krow(u);
            const u32x4_r q = *(const u32x4_r *)(lds + at * 1024 + lane * 16);
            const int scale = *(const int *)(lds + BK * N + at * 256 + lane * 4);
            float f[16];
            ckpt_unpack(u32x2_r{q[0], q[1]}, scale, f);
            ckpt_unpack(u32x2_r{q[2], q[3]}, scale, f + 8);
            char *to = tile + k * (N * 2) + (((col() >> 3) ^ (AcrossTile<N, NT, BK, 1>::perm(k) << 2)) << 4);
            *(u32x4_r *)to = pack8(f);
            *(u32x4_r *)(to + 16) = pack8(f + 8);
        }
    }
};

// One K step's products from a stage in LDS.  The fragments of a substep are read before
// the one before it is multiplied, and the next steps' direct loads (copy(u), u < COPIES)
// are issued a few with each: with all loads first, every wavefront stands at its loads
// before its first product (the weight gradient 167 us for 157).  last(): work for the
// vector units beside the last substep's products.
template <typename P, typename Q, int TP, int TQ, int BK, int COPIES, typename F, typename G>
__device__ __forceinline__ void multiply_step(const char *ps, const char *qs, int wp, int wq, f32x16_t (&acc)[TP][TQ],
                                              F copy, G last)
{
    constexpr int S = BK / 16;
    bf16x8_t fp[2][TP], fq[2][TQ];
    auto read = [&](int s) {
#pragma unroll
        for (int i = 0; i < TP; ++i) fp[s & 1][i] = P::frag(ps, wp + 32 * i, s);
#pragma unroll
        for (int j = 0; j < TQ; ++j) fq[s & 1][j] = Q::frag(qs, wq + 32 * j, s);
    };
    read(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int c0 = COPIES * s / S, c1 = COPIES * (s + 1) / S;
        if (s + 1 < S) read(s + 1);
#pragma unroll
        for (int u = c0; u < c1; ++u) copy(u);
        if (s + 1 == S) last();
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
            for (int j = 0; j < TQ; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[s & 1][i], fq[s & 1][j], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Of eight values as four words, those that are positive (not zero, no sign, no NaN), in
// the sign bits of the words' halves: bf16, and a checkpoint's bytes.
__device__ __forceinline__ u32x4_r positive_bf16(u32x4_r h)
{
    typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
    u32x4_r r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        // 1 .. 0x7F80 becomes 0 .. 0x7F7F; 0x80 more sets the sign of what is above
        const u16x2_t t = __builtin_bit_cast(u16x2_t, (uint32_t)h[k]) - (u16x2_t){1, 1};
        const u16x2_t u = t + (u16x2_t){0x80, 0x80};
        r[k] = ~(__builtin_bit_cast(uint32_t, t) | __builtin_bit_cast(uint32_t, u)) & 0x80008000u;
    }
    return r;
}
__device__ __forceinline__ u32x4_r positive_bytes(u32x2_r q, int scale)
{
    u32x4_r r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t w = q[k], any = (w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu;
        const uint32_t m = scale == 255 ? 0 : any & ~w & 0x80808080u;
        r[2 * k] = __builtin_amdgcn_perm(m, m, 0x010C000Cu);       // bytes 0, 1 on top of the halves
        r[2 * k + 1] = __builtin_amdgcn_perm(m, m, 0x030C020Cu);   // bytes 2, 3
    }
    return r;
}
// All bits of each half where its sign is set.
__device__ __forceinline__ uint32_t half_signs(uint32_t w) { return __builtin_amdgcn_perm(w, w, 0x09090808u); }

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
//
// 65536 rows of 16 experts, unevenly drawn, 1024x1024: 179 us, 768 TFLOP/s.  Its parts alone:
// products 90 us, loads from the L2 into LDS 117 (1.6 GB), and 47 more where the outputs
// are stored.  Two blocks of 256 x 128 share a CU, so that one's loads and stores run beside
// the other's products; 256 x 256 tiles load less but leave one block (206 us).
// ---------------------------------------------------------------------------
template <int OP, int WP, int WQ, int TP, int TQ, int BK, int D>
struct RowsTile {
    static constexpr int NT = 64 * WP * WQ, BP = 32 * WP * TP, BQ = 32 * WQ * TQ;
    using P = std::conditional_t<OP == OP_FORWARD, AlongTile<BP, NT, BK, D>, AcrossTile<BP, NT, BK, D>>;
    using Q = AlongTile<BQ, NT, BK, D>;
    static constexpr int STAGE = P::BYTES + Q::BYTES;
    static constexpr int LDO = BP + 8;      // epilogue rows
};

// How operands come: by direct loads and NS stages, or through D register sets and two
// stages, and that for rows of at least 8 values or of fewer.
enum { BY_DIRECT, BY_REGISTERS, BY_VALUES };

template <int OP, int WP, int WQ, int TP, int TQ, int BK, int NS, int D, int BY>
struct RowsShape {
    static constexpr bool DIRECT = BY == BY_DIRECT, NARROW = BY == BY_VALUES;
    static_assert(DIRECT ? D == 1 : NS == 2, "stages");
    using T = RowsTile<OP, WP, WQ, TP, TQ, BK, D>;
    static constexpr int NT = T::NT;
    // LDS: the stages (the outputs at the end), the places' rows, the bias
    static constexpr int ROWS_AT = std::max(NS * T::STAGE, T::BQ * T::LDO * 2), BIAS_AT = ROWS_AT + T::BQ * 4;
    static constexpr int LDS = BIAS_AT + (OP == OP_FORWARD ? T::BP * 4 : 0);

    __device__ __forceinline__ static void run(const ExpertArgs &a, int p_tiles, int id, char *lds)
    {
        constexpr int BP = T::BP, BQ = T::BQ;
        int *row_of = (int *)(lds + ROWS_AT);
        float *bias = (float *)(lds + BIAS_AT);
        const Piece pc = find_piece(a.offsets, a.E, a.n, id / p_tiles, BQ);
        if (pc.e < 0) return;
        const int p0 = id % p_tiles * BP;
        const int NP = OP == OP_FORWARD ? a.out : a.in, K = OP == OP_FORWARD ? a.in : a.out;
        for (int i = threadIdx.x; i < BQ; i += NT) row_of[i] = i < pc.count ? row_at(a, pc.first + i) : -1;
        if constexpr (OP == OP_FORWARD)
            for (int i = threadIdx.x; i < BP; i += NT)
                bias[i] = a.bias && pc.e < a.E && p0 + i < NP ? a.bias[(int64_t)pc.e * a.out + p0 + i] : 0.0f;
        __syncthreads();

        const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
        const int wp = wave % WP * TP * 32, wq = wave / WP * TQ * 32;
        // the pieces of C that this thread stores: features f.. of the places i0, i0 + NT / (BP / 8), ..
        constexpr int PIECES = BQ * (BP / 8) / NT;
        constexpr bool MASKED = OP == OP_DX_X || OP == OP_DX_CKPT;
        const int i0 = tid / (BP / 8), f = tid % (BP / 8) * 8, nv = NP - p0 - f;
        const bool whole = NP - p0 >= BP;
        // Which inputs are positive: words of two, in their halves' sign bits, are shifted into one
        // register for four pieces, and read while the first steps load (at the end it would be
        // the whole latency of a row read at random).
        uint32_t positive[(PIECES + 3) / 4];
        auto read_positive = [&] {
            constexpr int B = PIECES < 4 ? PIECES : 4;
#pragma unroll
            for (int c0 = 0; c0 < PIECES; c0 += B) {
                u32x4_r h[B];
                u32x2_r q[B];
                int scale[B];
#pragma unroll
                for (int c = 0; c < B; ++c) {
                    const int64_t r = max(row_of[i0 + (c0 + c) * (NT / (BP / 8))], 0);
                    if constexpr (OP == OP_DX_X) {
                        h[c] = *(const u32x4_a2 *)(a.x + r * a.ld_x + p0 + f);
                    } else {
                        q[c] = *(const u32x2_a1 *)(a.c.q + r * a.c.ld_q + p0 + f);
                        scale[c] = a.c.scale[r * a.c.ld_scale + ((p0 + f) >> 5)];
                    }
                }
                uint32_t m = 0;
#pragma unroll
                for (int c = 0; c < B; ++c) {
                    if constexpr (OP == OP_DX_CKPT) h[c] = positive_bytes(q[c], scale[c]);
                    else h[c] = positive_bf16(h[c]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) m = m >> 1 | h[c][k];
                }
                positive[c0 / 4] = m;
            }
        };
        const bool has_expert = pc.e < a.E;      // else zeros are stored
        f32x16_t acc[TP][TQ];
        clear(acc);
        if (has_expert) {
            const uint16_t *q = OP == OP_FORWARD ? a.x : a.dy;
            const int64_t ldq = OP == OP_FORWARD ? a.ld_x : a.ld_dy;
            const uint16_t *w = a.w + (int64_t)pc.e * a.out * a.ld_w;
            typename T::P tp;
            typename T::Q tq;
            // rows past the tile's last read row 0: their sums are not stored
            tq.init([&](int i) { return q + (int64_t)max(row_of[i], 0) * ldq; });
            const uint16_t *wcol = nullptr;
            int nvp = 0;
            if constexpr (OP == OP_FORWARD) {
                tp.init([&](int i) { return w + (int64_t)min(p0 + i, NP - 1) * a.ld_w; });
            } else {
                nvp = NP - p0 - tp.col();
                wcol = w + p0 + tp.col();
            }
            constexpr int L = T::P::U + T::Q::U;      // direct loads of a step
            auto copy = [&](int u, int kt, char *st) {
                if (u >= T::P::U) tq.copy(u - T::P::U, kt, st + T::P::BYTES);
                else if constexpr (OP == OP_FORWARD) tp.copy(u, kt, st);
                else tp.copy(u, nvp > 0 ? wcol + (int64_t)(kt * BK + tp.krow(u)) * a.ld_w : nullptr, st);
            };
            auto load = [&](auto narrow, int d, int kt) {
                constexpr bool N = decltype(narrow)::value;
                if constexpr (OP == OP_FORWARD)
                    tp.template load<N>(d, kt, K);
                else
                    tp.template load<N>(d, [&](int u) -> const uint16_t * {
                        const int k = kt * BK + tp.krow(u);
                        return k < K ? wcol + (int64_t)k * a.ld_w : nullptr;
                    }, nvp);
                tq.template load<N>(d, kt, K);
            };
            auto store = [&](auto narrow, int d, int kt, char *st) {
                constexpr bool N = decltype(narrow)::value;
                if constexpr (OP == OP_FORWARD) tp.template store<N>(d, kt, K, st);
                else tp.template store<N>(d, nvp, NP - p0 >= BP, st);
                tq.template store<N>(d, kt, K, st + T::P::BYTES);
            };
            int now = 0;     // stage of step kt
            // a step's products, with `copies` direct loads of the step that comes NS - 1 later
            auto multiply = [&](auto copies, int kt) {
                const char *st = lds + now * T::STAGE;
                char *ahead = lds + (now == 0 ? NS - 1 : now - 1) * T::STAGE;
                multiply_step<typename T::P, typename T::Q, TP, TQ, BK, decltype(copies)::value>(
                    st, st + T::P::BYTES, wp, wq, acc, [&](int u) { copy(u, kt + NS - 1, ahead); }, [] {});
                now = now + 1 == NS ? 0 : now + 1;
            };
            using NoCopies = std::integral_constant<int, 0>;
            if constexpr (DIRECT) {
                const int nk = K / BK;
                // the last, shorter step comes first, through registers and the last stage
                const bool rest = K % BK != 0;
                const bool wide = K >= 8 && (OP == OP_FORWARD || NP >= 8);
                if (rest && wide) load(std::false_type(), 0, nk);
                for (int kt = 0; kt < NS - 1 && kt < nk; ++kt)
#pragma unroll
                    for (int u = 0; u < L; ++u) copy(u, kt, lds + kt * T::STAGE);
                if (MASKED && whole) read_positive();
                if (rest) {
                    now = NS - 1;
                    if (wide) {
                        store(std::false_type(), 0, nk, lds + now * T::STAGE);
                    } else {
                        load(std::true_type(), 0, nk);
                        store(std::true_type(), 0, nk, lds + now * T::STAGE);
                    }
                    meet();
                    multiply(NoCopies(), 0);
                }
                int kt = 0;
                for (; kt + NS - 1 < nk; ++kt) {
                    wait_loads<(NS - 2) * L>();
                    meet();
                    multiply(std::integral_constant<int, L>(), kt);
                }
                for (; kt < nk; ++kt) {
                    wait_for_step<L, NS - 2>(nk - 1 - kt);
                    meet();
                    multiply(NoCopies(), kt);
                }
            } else {
                const int nk = (K + BK - 1) / BK;
                const std::integral_constant<bool, NARROW> narrow;
                // the order of the direct loads: a last, shorter step first
                const bool rest = K % BK != 0;
                auto nth = [&](int i) { return rest && i < nk ? (i == 0 ? nk - 1 : i - 1) : i; };
#pragma unroll
                for (int d = 0; d < D; ++d) load(narrow, d, nth(d));
                if (MASKED && whole) read_positive();
                store(narrow, 0, nth(0), lds);
                load(narrow, 0, nth(D));
                for (int k0 = 0; k0 < nk; k0 += D) {
#pragma unroll
                    for (int d = 0; d < D; ++d) {
                        const int kt = k0 + d, next = (d + 1) % D;      // step, register set of the next one
                        if (kt >= nk) break;
                        meet();
                        store(narrow, next, nth(kt + 1), lds + (now ^ 1) * T::STAGE);
                        load(narrow, next, nth(kt + 1 + D));
                        multiply(NoCopies(), kt);
                    }
                }
            }
        }
        meet();

        // lane l: place wq + 32 j + l % 32, features wp + 32 i + 8 g + 4 (l / 32) + 0..3
        auto quad = [&](int i, int j, int g) {
            return f32x4_r{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        };
        // f: feature of the tile
        auto finish = [&](int f, f32x4_r v) {
            if constexpr (OP == OP_FORWARD) {
                v += *(const f32x4_r *)(bias + f);
                if (a.relu)
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = v[k] < 0.0f ? 0.0f : v[k];   // NaN stays
            }
            return v;
        };
        // fp32 rows leave from the registers, 32 bytes of 32 rows at a time: 65536 rows 1024x1024
        // 213 us for 179 in bf16, with 134 MB more to write
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
                        const f32x4_r v = finish(f - p0, quad(i, j, g));
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
        // bf16 rows meet in LDS and leave in 16-byte pieces
        uint16_t *out = (uint16_t *)lds;
#pragma unroll
        for (int j = 0; j < TQ; ++j)
#pragma unroll
            for (int i = 0; i < TP; ++i)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int f = wp + 32 * i + 8 * g + 4 * (lane >> 5);
                    const f32x4_r v = finish(f, quad(i, j, g));
                    const u32x2_r o = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                    *(u32x2_r *)(out + (wq + 32 * j + (lane & 31)) * T::LDO + f) = o;
                }
        __syncthreads();
        auto to = [&](int r) -> uint16_t * {
            return (OP == OP_FORWARD ? (uint16_t *)a.y + (int64_t)r * a.ld_y : a.dx + (int64_t)r * a.ld_dx) + p0 + f;
        };
        if (whole) {
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                const int i = i0 + c * (NT / (BP / 8)), r = row_of[i];
                u32x4_r o = *(const u32x4_r *)(out + i * T::LDO + f);
                if constexpr (MASKED) {
                    constexpr int B = PIECES < 4 ? PIECES : 4;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        o[k] &= half_signs(has_expert ? positive[c / 4] << (4 * B - 1 - (4 * (c % 4) + k)) : 0);
                }
                if (r >= 0) *(u32x4_a2 *)to(r) = o;
            }
        } else if (nv > 0) {
#pragma unroll 1
            for (int c = 0; c < PIECES; ++c) {
                const int i = i0 + c * (NT / (BP / 8)), r = row_of[i];
                if (r < 0) continue;
                u32x4_r o = *(const u32x4_r *)(out + i * T::LDO + f);
                if constexpr (MASKED) {
                    u32x4_r h;
                    const int64_t at = r;
                    if constexpr (OP == OP_DX_X)
                        h = positive_bf16(load8_bits(a.x + at * a.ld_x + p0 + f, nv));
                    else
                        h = positive_bytes(load8_bytes(a.c.q + at * a.c.ld_q + p0 + f, nv),
                                           a.c.scale[at * a.c.ld_scale + ((p0 + f) >> 5)]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[k] &= half_signs(h[k]);
                }
                store8_bits(to(r), nv, o);
            }
        }
    }
};

template <typename S>
__global__ __launch_bounds__(S::NT, 2) void expert_rows_kernel(ExpertArgs a, int p_tiles)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    S::run(a, p_tiles, xcd_order(blockIdx.x, gridDim.x), lds);
}

// ---------------------------------------------------------------------------
// Weight gradient.  The blocks are teams of one block for each tile (BQ outputs x BP
// inputs).  The places with an expert are counted in units of 64 of one expert, and each
// team takes an equal run of the units, whatever the experts' sizes; its blocks, which
// read the same rows, are neighbours in an L2.  Within its run a team forms one product for
// each expert.  An expert that lies in one run is written to dw; one that spans several
// leaves each team's part in the workspace, in slot 2 t + 1 if it begins in team t's run,
// else 2 t (a run has at most one of each), and expert_dw_sum_kernel adds the parts up in
// the teams' order.  The blocks of the first inputs also sum dy's columns for db, from the
// stages in LDS.  CK: x from its checkpoint, whose bytes each lane restores one step ahead.
//
// 65536 rows of 16 experts, 1024x512: 152 us with the sums of the parts (28 of them, and as
// much to write the parts, 94 MB), 450 TFLOP/s; bound by latency, a barrier and the
// restoring each 32 rows, as 256 x 256 tiles leave registers for two wavefronts a SIMD: the
// MFMA pipes are busy for 26% of the cycles, the LDS for 20, and wavefronts wait for 35% of
// theirs.  128 x 256 tiles on four wavefronts, two blocks a CU, were slower (both gradients 303
// us for 286), and addresses by 32-bit products brought nothing.
// With an even number of pieces a run each instead (64 x 64 partial tiles): 430 us.
// ---------------------------------------------------------------------------
constexpr int DW_UNIT = 64;

// Places and units of expert e.
struct Span {
    int first, count, units;
};
__device__ __forceinline__ Span span_of(const ExpertArgs &a, int e)
{
    const int f = min(max(a.offsets[e], 0), a.n), l = min(max(a.offsets[e + 1], f), a.n);
    return Span{f, l - f, (l - f + DW_UNIT - 1) / DW_UNIT};
}

// Sum over a wavefront, in every lane.
__device__ __forceinline__ int wave_sum(int x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}

// Units of the experts before `last` (all lanes).
__device__ __forceinline__ int units_before(const ExpertArgs &a, int last)
{
    int s = 0;
    for (int e = threadIdx.x & 63; e < last; e += 64) s += span_of(a, e).units;
    return wave_sum(s);
}

// Units of a team's run.
__device__ __forceinline__ int run_units(int all, int teams) { return max((all + teams - 1) / teams, 1); }

// Places whose row indices are held in LDS ahead of their use, a power of two.
constexpr int DW_ROWS = 512;

// teams 0: a team for each expert instead, which takes its rows alone and writes dw and db
// itself, zeros for none.
template <int WP, int WQ, int TP, int TQ, int BK, int NS, int D, int BY, bool CK>
struct DwShape {
    static constexpr bool DIRECT = BY == BY_DIRECT, NARROW = BY == BY_VALUES;
    static_assert(DIRECT ? D == 1 : NS == 2, "stages");
    static_assert(DW_ROWS / BK > NS + 1 && DW_ROWS / BK > D + 2, "row indices are there a step before they are used");
    static constexpr int NT = 64 * WP * WQ, BP = 32 * WP * TP, BQ = 32 * WQ * TQ;
    static constexpr bool BYTES = DIRECT && CK;      // x's bytes by direct loads
    using P = std::conditional_t<CK && !DIRECT, AcrossCkpt<BP, NT, BK, D>, AcrossTile<BP, NT, BK, D>>;
    using Q = AcrossTile<BQ, NT, BK, D>;
    using R = CkptBytes<BP, NT, BK>;
    // direct loads of a step
    static constexpr int LP = BYTES ? R::U : P::U, L = (BYTES ? 2 * R::U : P::U) + Q::U;
    // LDS: NS tiles of dy, of x (2 restored ones and NS of bytes), two sets of row indices
    static constexpr int PS = BYTES ? 2 : NS, P_AT = NS * Q::BYTES, R_AT = P_AT + PS * P::BYTES;
    static constexpr int ROWS_AT = R_AT + (BYTES ? NS * R::BYTES : 0), LDS = ROWS_AT + 2 * DW_ROWS * 4;

    __device__ __forceinline__ static void run(const ExpertArgs &a, int p_tiles, int q_tiles, int teams, int id,
                                               char *lds)
    {
        int *rows = (int *)(lds + ROWS_AT);
        const int team = id / (p_tiles * q_tiles);
        const int p0 = id % p_tiles * BP, q0 = id / p_tiles % q_tiles * BQ;
        const int lane = threadIdx.x & 63, wave = wave_id();
        const int wp = wave % WP * TP * 32, wq = wave / WP * TQ * 32;
        const bool with_db = a.db && p0 == 0;
        const int in4 = (a.in + 3) & ~3;

        P tp;
        Q tq;
        const int in = a.dw ? a.in : 0;      // db alone: x is not read
        const int pcol = p0 + tp.col(), qcol = q0 + tq.col(), rcol = p0 + R::col() < in ? p0 + R::col() : -1;
        const int nvp = in - pcol, nvq = a.out - qcol;
        f32x16_t acc[TP][TQ];
        float db[2];
        // db: a thread sums two columns of DB_ROWS rows of each step
        constexpr int PAIRS = BQ / 2, DB_ROWS = BK / (NT / PAIRS);

        // the product of K places from `first` on
        auto product = [&](int first, int K) {
            const int nk = (K + BK - 1) / BK;
            // row indices of places c DW_ROWS .. of the product: set c % 2
            constexpr int RU = DW_ROWS / NT;
            int held[RU];
            auto fetch = [&](int c) {
#pragma unroll
                for (int u = 0; u < RU; ++u) {
                    const int k = c * DW_ROWS + u * NT + (int)threadIdx.x;
                    held[u] = k < K ? row_at(a, first + k) : -1;
                }
            };
            auto keep = [&](int c) {
#pragma unroll
                for (int u = 0; u < RU; ++u) rows[(c & 1) * DW_ROWS + u * NT + threadIdx.x] = held[u];
            };
            auto row = [&](int kt, int k) { return rows[(kt * BK + k) & (2 * DW_ROWS - 1)]; };
            fetch(0);
            keep(0);
            fetch(1);
            keep(1);
            fetch(2);
            __syncthreads();

            auto x_at = [&](int kt, int u) -> const uint16_t * {
                const int r = row(kt, tp.krow(u));
                return r >= 0 && in > 0 ? a.x + (int64_t)r * a.ld_x + pcol : nullptr;
            };
            auto dy_at = [&](int kt, int u) -> const uint16_t * {
                const int r = row(kt, tq.krow(u));
                return r >= 0 ? a.dy + (int64_t)r * a.ld_dy + qcol : nullptr;
            };
            // direct loads: dy of step kt, x of step kt (its bytes of step kt + 1)
            auto copy = [&](int u, int kt) {
                char *q = lds + kt % NS * Q::BYTES;
                if (u >= LP) {
                    tq.copy(u - LP, nvq > 0 ? dy_at(kt, u - LP) : nullptr, q);
                } else if constexpr (BYTES) {
                    R::copy(u, a.c, row(kt + 1, R::krow(u)), rcol, lds + R_AT + (kt + 1) % NS * R::BYTES);
                } else {
                    tp.copy(u, nvp > 0 ? x_at(kt, u) : nullptr, lds + P_AT + kt % NS * P::BYTES);
                }
            };
            // through register set d
            auto load = [&](int d, int kt) {
                tq.template load<NARROW>(d, [&](int u) { return dy_at(kt, u); }, nvq);
                if constexpr (CK && !DIRECT)
                    tp.template load<NARROW>(d, a.c, [&](int u) { return in > 0 ? row(kt, tp.krow(u)) : -1; }, pcol,
                                             nvp);
                else
                    tp.template load<NARROW>(d, [&](int u) { return x_at(kt, u); }, nvp);
            };
            auto store = [&](int d, int stage) {
                tq.template store<NARROW>(d, nvq, a.out - q0 >= BQ, lds + stage * Q::BYTES);
                tp.template store<NARROW>(d, nvp, in - p0 >= BP, lds + P_AT + stage * P::BYTES);
            };
            auto restore = [&](int kt) {
                R::restore(lds + R_AT + kt % NS * R::BYTES, lds + P_AT + (kt & 1) * P::BYTES);
            };
            // a step after its loads: the next row indices now and then, db, the products
            auto step = [&](int kt, auto copies) {
                if (kt > 0 && kt * BK % DW_ROWS == 0) {
                    keep(kt * BK / DW_ROWS + 1);
                    fetch(kt * BK / DW_ROWS + 2);
                }
                const char *qs = lds + kt % NS * Q::BYTES, *ps = lds + P_AT + kt % PS * P::BYTES;
                if (with_db) {
                    const int pair = threadIdx.x % PAIRS, k0 = threadIdx.x / PAIRS * DB_ROWS;
#pragma unroll
                    for (int k = k0; k < k0 + DB_ROWS; ++k) {
                        const char *at = qs + k * Q::PITCH + ((pair >> 2) ^ (Q::perm(k) << 2)) * 16 + (pair & 3) * 4;
                        const uint32_t v = *(const uint32_t *)at;
                        db[0] += __uint_as_float(v << 16);
                        db[1] += __uint_as_float(v & 0xFFFF0000u);
                    }
                }
                multiply_step<P, Q, TP, TQ, BK, decltype(copies)::value>(
                    ps, qs, wp, wq, acc, [&](int u) { copy(u, kt + NS - 1); },
                    [&] { if constexpr (BYTES) restore(kt + 1); });
            };
            clear(acc);
            db[0] = db[1] = 0.0f;
            if constexpr (DIRECT) {
                // steps past the last have no rows: their loads bring zeros that nothing reads
                if constexpr (BYTES)
#pragma unroll
                    for (int u = 0; u < R::U; ++u) R::copy(u, a.c, row(0, R::krow(u)), rcol, lds + R_AT);
                for (int kt = 0; kt < NS - 1; ++kt)
#pragma unroll
                    for (int u = 0; u < LP + Q::U; ++u) copy(u, kt);
                if constexpr (BYTES) {
                    wait_loads<(NS - 1) * L>();
                    restore(0);
                }
                for (int kt = 0; kt < nk; ++kt) {
                    wait_loads<(NS - 2) * L>();
                    meet();
                    step(kt, std::integral_constant<int, LP + Q::U>());
                }
            } else {
#pragma unroll
                for (int d = 0; d < D; ++d) load(d, d);
                store(0, 0);
                load(0, D);
                for (int k0 = 0; k0 < nk; k0 += D) {
#pragma unroll
                    for (int d = 0; d < D; ++d) {
                        const int kt = k0 + d, next = (d + 1) % D;
                        if (kt >= nk) break;
                        meet();
                        store(next, (kt + 1) & 1);
                        load(next, kt + 1 + D);
                        step(kt, std::integral_constant<int, 0>());
                    }
                }
            }
            wait_loads<0>();
            meet();
        };

        // the product to dw and db of expert e (slot < 0), or to a slot of the workspace
        auto finish = [&](int e, int64_t slot) {
            float *c = slot < 0 ? a.dw + (int64_t)e * a.out * a.ld_dw : a.part + slot * a.out * in4;
            const int64_t ldc = slot < 0 ? a.ld_dw : in4;
            if (with_db) {
                float *red = (float *)lds;      // [NT / PAIRS][BQ]
                red[threadIdx.x / PAIRS * BQ + threadIdx.x % PAIRS * 2] = db[0];
                red[threadIdx.x / PAIRS * BQ + threadIdx.x % PAIRS * 2 + 1] = db[1];
                __syncthreads();
                float *d = slot < 0 ? a.db + (int64_t)e * a.out : a.part_db + slot * a.out;
                for (int i = threadIdx.x; i < BQ && q0 + i < a.out; i += NT) {
                    float t = 0.0f;
#pragma unroll
                    for (int r = 0; r < NT / PAIRS; ++r) t += red[r * BQ + i];
                    d[q0 + i] = t;
                }
                __syncthreads();
            }
            if (!a.dw) return;
#pragma unroll
            for (int j = 0; j < TQ; ++j) {
                const int o = q0 + wq + 32 * j + (lane & 31);
                if (o >= a.out) continue;
#pragma unroll
                for (int i = 0; i < TP; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int f = p0 + wp + 32 * i + 8 * g + 4 * (lane >> 5);
                        const f32x4_r v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                                           acc[i][j][4 * g + 3]};
                        if (f + 4 <= a.in) {
                            *(f32x4_a4 *)(c + o * ldc + f) = v;
                        } else {
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (f + k < a.in) c[o * ldc + f + k] = v[k];
                        }
                    }
            }
        };

        // the experts of the run [begin, end) of units; `u`: the units before expert e
        int begin = 0, end = 1, e = team, u = 0;
        if (teams > 0) {
            const int all = units_before(a, a.E), run = run_units(all, teams);
            begin = min(team * run, all);
            end = min(begin + run, all);
            // the first expert that ends past `begin`, 64 at a time
            e = a.E;
            int carry = 0;
            for (int e0 = 0; e0 < a.E; e0 += 64) {
                const int j = e0 + lane;
                const int k = j < a.E ? span_of(a, j).units : 0;
                int s = k;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int t = __shfl_up(s, d);
                    s += lane >= d ? t : 0;
                }
                const uint64_t hit = __ballot(carry + s > begin);
                if (hit) {
                    const int l = __builtin_ctzll(hit);
                    e = e0 + l;
                    u = carry + __builtin_amdgcn_readlane(s, l) - __builtin_amdgcn_readlane(k, l);
                    break;
                }
                carry += __builtin_amdgcn_readlane(s, 63);
            }
        }
        for (; u < end && e < a.E; ++e) {
            const Span sp = span_of(a, e);
            int k0 = 0, k1 = sp.count;
            int64_t slot = -1;
            if (teams > 0) {
                if (sp.units == 0) continue;
                k0 = (max(begin, u) - u) * DW_UNIT;
                k1 = min((min(end, u + sp.units) - u) * DW_UNIT, sp.count);
                if (u < begin || u + sp.units > end) slot = 2 * team + (u >= begin ? 1 : 0);
            }
            product(__builtin_amdgcn_readfirstlane(sp.first + k0), __builtin_amdgcn_readfirstlane(k1 - k0));
            finish(e, slot);
            if (teams == 0) break;
            u += sp.units;
        }
    }
};

template <typename S>
__global__ __launch_bounds__(S::NT, 2) void expert_dw_kernel(ExpertArgs a, int p_tiles, int q_tiles, int teams)
{
    __shared__ __attribute__((aligned(1024))) char lds[S::LDS];
    S::run(a, p_tiles, q_tiles, teams, xcd_order(blockIdx.x, gridDim.x), lds);
}

// Both gradients in one launch, the weights' blocks first: for few rows each of them is
// latency, which the other's blocks fill.
template <typename X, typename W>
__global__ __launch_bounds__(X::NT, 2) void expert_grad_kernel(ExpertArgs a, int x_tiles, int p_tiles, int q_tiles,
                                                               int teams, int w_blocks)
{
    static_assert(X::NT == W::NT, "one block size");
    __shared__ __attribute__((aligned(1024))) char lds[std::max(X::LDS, W::LDS)];
    const int b = blockIdx.x;
    if (b < w_blocks) W::run(a, p_tiles, q_tiles, teams, xcd_order(b, w_blocks), lds);
    else X::run(a, x_tiles, xcd_order(b - w_blocks, gridDim.x - w_blocks), lds);
}

// dw and db of the experts that no single team's run holds: the parts in the teams' order,
// zeros for an expert without rows.  blockIdx.y: the expert; x over [out][in4 / 4], then [out]
// of db.
__global__ __launch_bounds__(256) void expert_dw_sum_kernel(ExpertArgs a, int teams)
{
    const int e = blockIdx.y;
    const int mine = span_of(a, e).units;
    int t0 = 0, t1 = -1, u0 = 0, run = 1;
    if (mine > 0) {
        if (teams == 1) return;
        u0 = units_before(a, e);
        run = run_units(units_before(a, a.E), teams);
        t0 = u0 / run;
        t1 = (u0 + mine - 1) / run;
        if (t0 == t1) return;
    }
    // team t's part: its run began within the expert (slot 2 t), or goes on past it (2 t + 1)
    const int in4 = (a.in + 3) & ~3, q = in4 / 4;
    const int64_t size = (int64_t)a.out * q, t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < size) {
        if (!a.dw) return;
        const int o = (int)(t / q), f = (int)(t % q) * 4;
        f32x4_r s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int k = t0; k <= t1; ++k) {
            const int64_t slot = 2 * k + (u0 >= k * run ? 1 : 0);
            s += *(const f32x4_r *)(a.part + (slot * a.out + o) * in4 + f);
        }
        float *c = a.dw + ((int64_t)e * a.out + o) * a.ld_dw + f;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (f + k < a.in) c[k] = s[k];
    } else if (a.db && t - size < a.out) {
        const int o = (int)(t - size);
        float s = 0.0f;
        for (int k = t0; k <= t1; ++k) s += a.part_db[(2 * k + (u0 >= k * run ? 1 : 0)) * (int64_t)a.out + o];
        a.db[(int64_t)e * a.out + o] = s;
    }
}

// Tiles of a launch over rows, for any group sizes: whole tiles, and a shorter one for
// each expert and for the rest.
static int64_t row_tiles(const ExpertArgs &a, int rows) { return a.n / rows + std::min<int64_t>(a.E + 1, a.n); }

// Rows that direct loads can take: all at multiples of 16 bytes.
static bool rows_aligned(const void *p, int64_t ld, int64_t size = 2)
{
    return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0;
}

// Tiles (outputs x places) by the number of 256 x 128 ones that there would be: those from
// BIG_TILES on, 128 x 128 from MID_TILES, 128 x 64 from LOW_TILES, 64 x 64 below, each as long
// as the larger one leaves CUs without work.  us with the larger and the smaller one:
// 6000 rows 300x1000 of 10 experts (228) 16.7, 13.7 and with 128 x 64 16.9; 12000 rows 1024x256
// (104) 17.7, 15.5; 2000 rows 1024x1024 of 4 (80) 17.0, 13.8 and with 64 x 64 16.9; 6000 rows
// 1024x256 (57) 16.4, 10.5.  Rows of any alignment have the first (128 x 128) and the last.
// The largest runs on four wavefronts of 128 x 64 forward, on eight of 64 x 64 for dx (65536
// rows of 16 experts: 1024x1024 forward 181 us, on eight 200; dx of 1024x512 with its mask 124
// us, on four 133).
template <int OP>
using RowsBig = std::conditional_t<OP == OP_FORWARD, RowsShape<OP, 2, 2, 4, 2, 32, 3, 1, BY_DIRECT>,
                                   RowsShape<OP, 4, 2, 2, 2, 32, 3, 1, BY_DIRECT>>;
template <int OP>
using RowsMid = RowsShape<OP, 2, 2, 2, 2, 64, 2, 1, BY_DIRECT>;
template <int OP>
using RowsLow = RowsShape<OP, 2, 2, 2, 1, 64, 3, 1, BY_DIRECT>;
template <int OP, int BY>
using RowsSmall = RowsShape<OP, 2, 2, 1, 1, 64, BY == BY_DIRECT ? 3 : 2, BY == BY_REGISTERS ? 2 : 1, BY>;
template <int OP>
using RowsBigRegs = RowsShape<OP, 2, 2, 2, 2, 32, 2, 2, BY_REGISTERS>;
constexpr int64_t BIG_TILES = 256, MID_TILES = 150, LOW_TILES = 60;
// dx beside a weight gradient of 64 x 64 tiles shares its launch below this many: all blocks of
// the launch are of dx's smallest tiles then.  us of the whole gradient in one launch and in
// two, 8 experts: 500 rows 361x1024 (24 tiles) 18.2, 21.0; 4000 rows (80) 35.1, 42.5; 8000 rows
// (142) 75.1, 71.0; 4000 rows 1024x1024 (160) 74.5, 66.8; 8000 rows 1024x512 (284) 83.4, 71.7;
// 12000 rows (408) 113, 86; but 16000 rows 256x256 of 16 (142) 35.0, 40.6.  So the bound leaves
// up to 30% where wide layers have between 140 and 384 tiles, and gains 15% where narrow ones do.
constexpr int64_t GRAD_BIG_TILES = 384;

template <int OP>
static int64_t big_tiles(const ExpertArgs &a)
{
    return row_tiles(a, 128) * ceil_div(OP == OP_FORWARD ? a.out : a.in, 256);
}

template <typename S, int OP>
static void rows_go(const ExpertArgs &a, hipStream_t s)
{
    const int p_tiles = (int)ceil_div(OP == OP_FORWARD ? a.out : a.in, S::T::BP);
    expert_rows_kernel<S><<<dim3((unsigned)(row_tiles(a, S::T::BQ) * p_tiles)), dim3(S::NT), 0, s>>>(a, p_tiles);
}

template <int OP>
static void rows_launch(const ExpertArgs &a, bool direct, hipStream_t s)
{
    const int64_t tiles = big_tiles<OP>(a);
    if (direct) {
        if (tiles >= BIG_TILES) rows_go<RowsBig<OP>, OP>(a, s);
        else if (tiles >= MID_TILES) rows_go<RowsMid<OP>, OP>(a, s);
        else if (tiles >= LOW_TILES) rows_go<RowsLow<OP>, OP>(a, s);
        else rows_go<RowsSmall<OP, BY_DIRECT>, OP>(a, s);
    } else if (a.in < 8 || (OP != OP_FORWARD && a.out < 8)) {
        rows_go<RowsSmall<OP, BY_VALUES>, OP>(a, s);
    } else {
        if (tiles >= BIG_TILES) rows_go<RowsBigRegs<OP>, OP>(a, s);
        else rows_go<RowsSmall<OP, BY_REGISTERS>, OP>(a, s);
    }
}

hipError_t launch_expert_linear(const ExpertArgs &a, hipStream_t s)
{
    rows_launch<OP_FORWARD>(a, rows_aligned(a.x, a.ld_x) && rows_aligned(a.w, a.ld_w), s);
    return hipGetLastError();
}

template <int BY, bool CK>
using DwBig = DwShape<2, 4, 4, 2, 32, BY == BY_DIRECT ? 4 : 2, 1, BY, CK>;
// Few stages and register sets for the smallest tiles: more blocks a CU are worth more than
// steps loaded ahead (4095 rows 361x1024 of aligned rows 46.5 us with 4 stages, 37 with 2 and
// 3; 3000 rows 1000x500 through 3 register sets 48, 2 sets 41, 1 set 40 but 300 rows 12.1 for
// 11.7).
template <int BY, bool CK>
using DwSmall = DwShape<2, 2, 1, 1, 64, 2, BY == BY_REGISTERS ? 2 : 1, BY, CK>;

// The weight gradient's tile and teams: 256 x 256 tiles, a block on each CU, from
// DW_BIG_ROWS rows on where both widths exceed half of one; else 64 x 64 ones, a team for
// each expert up to DW_EXPERT_ROWS rows where that makes DW_EXPERT_BLOCKS blocks, or
// DW_SMALL_BLOCKS blocks whose teams have at least DW_RUN rows.  Both sides of each, us of dw and
// db with the sums of parts, replayed from a graph, even experts:
//   256 x 256 and 64 x 64 tiles: 361x1024 of 8 experts, 8000 rows 45.9, 43.8, 12000 rows 51.6,
//     53.8, 16384 rows 57.4, 64.7, 65536 rows 118, 198; 1024x1024 of 16, 8000 rows 81.5, 91.3.
//     Widths, 32768 rows: 100x1024 52.1, 45.9; 130x1024 53.7, 60.8.  Where both widths barely
//     exceed a tile it loses: 130x130 36.2, 23.9; 264x264 47.7, 37.8.
//   a team for each expert and runs: 361x1024, 1000 rows of 16 13.9, 30.1, 4000 rows 21.4, 35.9;
//     4000 rows of 4 23.2, 30.4, 8000 rows of 4 51.6, 39.5, of 16 33.8, 47.8, of 64 46.8, 77.0.  It
//     does not look at the experts' sizes, which the host does not know: one expert that holds
//     all rows is taken by one block a tile (2048 rows 55.4, 24.4; 4000 rows 103, 31.4).
//   by the blocks that a team for each expert makes: 4000 rows, 128x128 of 8 (32 blocks) 13.3,
//     15.6, 256x256 of 4 (64) 22.0, 16.4, 361x256 of 8 (192) 13.7, 18.7.  Below the bound few rows
//     would gain by it as well: 200 rows 64x64 of 64 experts 4.5, 165.
//   512, 1024 and 2048 blocks: 16000 rows 361x1024 of 8 95.8, 63.9, 69.4; 65536 rows 128x1024 of
//     16 117, 74.3, 84.4.
//   128, 256 and 512 rows at least: 128x256 of 8, 5000 rows 14.4, 16.7, 20.3, 16000 rows 21.8,
//     20.0, 22.0; 16000 rows 64x64 of 16 14.0, 15.4, 20.1.
constexpr int64_t DW_BIG_ROWS = 16384, DW_EXPERT_ROWS = 4096, DW_EXPERT_BLOCKS = 128, DW_SMALL_BLOCKS = 1024,
                  DW_RUN = 256;
struct DwPlan {
    int tile, teams;     // teams 0: the experts
};
static DwPlan dw_plan(int64_t n, int n_experts, int in, int out)
{
    const int64_t big = ceil_div(in, 256) * ceil_div(out, 256);
    if (n >= DW_BIG_ROWS && in > 128 && out > 128) return {256, (int)std::max<int64_t>(1, 256 / big)};
    const int64_t tiles = ceil_div(in, 64) * ceil_div(out, 64);
    if (n <= DW_EXPERT_ROWS && tiles * n_experts >= DW_EXPERT_BLOCKS) return {64, 0};
    return {64, (int)std::max<int64_t>(1, std::min<int64_t>(DW_SMALL_BLOCKS / tiles, n / DW_RUN))};
}

int expert_grad_teams(int64_t n, int n_experts, int in, int out) { return dw_plan(n, n_experts, in, out).teams; }

struct DwGrid {
    int p_tiles, q_tiles, blocks;
};
static DwGrid dw_grid(const ExpertArgs &a, const DwPlan &d)
{
    const int p = a.dw ? (int)ceil_div(a.in, d.tile) : 1, q = (int)ceil_div(a.out, d.tile);
    return {p, q, (d.teams > 0 ? d.teams : a.E) * p * q};
}

template <typename S>
static void dw_go(const ExpertArgs &a, const DwPlan &d, hipStream_t s)
{
    const DwGrid g = dw_grid(a, d);
    expert_dw_kernel<S><<<dim3((unsigned)g.blocks), dim3(S::NT), 0, s>>>(a, g.p_tiles, g.q_tiles, d.teams);
}

template <bool CK>
static void dw_launch(const ExpertArgs &a, const DwPlan &d, int by, hipStream_t s)
{
    if (d.tile == 256 && by == BY_DIRECT) dw_go<DwBig<BY_DIRECT, CK>>(a, d, s);
    else if (d.tile == 256) dw_go<DwBig<BY_REGISTERS, CK>>(a, d, s);
    else if (by == BY_DIRECT) dw_go<DwSmall<BY_DIRECT, CK>>(a, d, s);
    else if (by == BY_REGISTERS) dw_go<DwSmall<BY_REGISTERS, CK>>(a, d, s);
    else dw_go<DwSmall<BY_VALUES, CK>>(a, d, s);
}

template <int OP, int BY, bool CK>
static void grad_go(const ExpertArgs &a, const DwPlan &d, hipStream_t s)
{
    using X = RowsSmall<OP, BY>;
    using W = DwSmall<BY, CK>;
    const DwGrid g = dw_grid(a, d);
    const int x_tiles = (int)ceil_div(a.in, X::T::BP);
    expert_grad_kernel<X, W><<<dim3((unsigned)(g.blocks + row_tiles(a, X::T::BQ) * x_tiles)), dim3(X::NT), 0, s>>>(
        a, x_tiles, g.p_tiles, g.q_tiles, d.teams, g.blocks);
}

template <int BY>
static void grad_launch(const ExpertArgs &a, const DwPlan &d, bool ck, hipStream_t s)
{
    if (!a.relu) ck ? grad_go<OP_DX, BY, true>(a, d, s) : grad_go<OP_DX, BY, false>(a, d, s);
    // the mask reads x also where dw is not wanted
    else a.x ? grad_go<OP_DX_X, BY, false>(a, d, s) : grad_go<OP_DX_CKPT, BY, true>(a, d, s);
}

hipError_t launch_expert_grad(const ExpertArgs &a, hipStream_t s)
{
    const bool with_dx = a.dx && a.n > 0, with_dw = a.dw || a.db;
    const bool dy_ok = rows_aligned(a.dy, a.ld_dy), ck = a.dw && !a.x;
    const bool x_ok = !a.dw || (ck ? rows_aligned(a.c.q, a.c.ld_q, 1) : rows_aligned(a.x, a.ld_x));
    const bool dx_direct = dy_ok && rows_aligned(a.w, a.ld_w);
    const bool wide = a.out >= 8 && (a.in >= 8 || !a.dw);
    const int dw_by = dy_ok && x_ok ? BY_DIRECT : wide ? BY_REGISTERS : BY_VALUES;
    const DwPlan d = dw_plan(a.n, a.E, a.in, a.out);
    // one launch for both where both are small
    const bool both = with_dx && with_dw && a.n > 0 && d.tile == 64 && big_tiles<OP_DX>(a) < GRAD_BIG_TILES &&
                      a.in >= 8 && a.out >= 8;
    if (both) {
        if (dx_direct && dw_by == BY_DIRECT) grad_launch<BY_DIRECT>(a, d, ck, s);
        else grad_launch<BY_REGISTERS>(a, d, ck, s);
    } else if (with_dx) {
        if (!a.relu) rows_launch<OP_DX>(a, dx_direct, s);
        else if (a.x) rows_launch<OP_DX_X>(a, dx_direct, s);
        else rows_launch<OP_DX_CKPT>(a, dx_direct, s);
    }
    if (with_dw) {
        if (!both && (a.n > 0 || d.teams == 0)) {
            if (ck) dw_launch<true>(a, d, dw_by, s);
            else dw_launch<false>(a, d, dw_by, s);
        }
        if (d.teams > 0) {
            const int64_t work = (int64_t)a.out * ((a.in + 3) / 4) + a.out;
            expert_dw_sum_kernel<<<dim3((unsigned)ceil_div(work, 256), a.E), dim3(256), 0, s>>>(a, d.teams);
        }
    }
    return hipGetLastError();
}

}  // namespace im
