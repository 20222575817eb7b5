// scan_kernels.hip -- gated linear recurrence over the steps of a rollout, and its gradient.
//
// c_t = live_t (a_t c_(t-1) + (1 - a_t) x_t) is a map c -> P c + S of the state for any run of
// steps, and maps compose: with few envs the steps are cut into chunks, the first launch forms
// each chunk's map, the second composes them into the state before each chunk, and the third
// walks all chunks at once.  With many envs one launch walks all steps.  The gradient is the
// same recurrence backwards.  A thread holds V consecutive values of one env.  A map that an
// episode's end cuts has P = -1 (products of gates are never negative): what came before does
// not count, also where it is a NaN or an infinity.
#include <algorithm>
#include <type_traits>

#include "block8.h"
#include "recurrent.h"

namespace im {

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int KEEP = IM_SCAN_KEEP;
constexpr int64_t INFINITY_CACHE = 256 << 20;

// Values of a thread.  bf16 32 x 16384 x 256 forward with 8, 4, 2: 195, 212, 181 us; fp32 32 x 8192 x
// 256 with 4, 2: 208, 182 us; the gradients' registers hold 16 steps of 2 values.
constexpr int SCAN_V = 2;

// V values of a row as words, at any address of their element's alignment.  The last piece of a
// row whose width is no multiple of V takes the last V values of the row: `lo` of them belong
// to the piece before, which alone stores them.  Rows of fewer than V values: value by value.
// What a launch does: chunks' maps alone; chunks' steps; all steps; all steps of arrays that no cache holds
// (their loads and stores are marked as such: 32 x 16384 x 256 bf16 forward 181 us, 165 marked, the
// gradient 330 and 290; the chunks' second launch reads what the first one left in the caches, and
// takes 108 us for 95 if marked).
enum { MAP, CHUNKS, STEPS, STREAM };

template <typename E, int V, int MODE>
struct StepPiece {
    static constexpr int BYTES = sizeof(E) * V;
    typedef uint32_t word_t __attribute__((ext_vector_type(BYTES / 4)));
    typedef word_t at_t __attribute__((aligned(sizeof(E))));
    static_assert(BYTES % 4 == 0, "whole words");
    int at, lo, hi;      // first column; the values lo .. hi - 1 are this piece's own
    __device__ __forceinline__ void init(int64_t piece, int64_t d)
    {
        const int col = (int)piece * V;
        at = max(0, min(col, (int)d - V));
        lo = col - at;
        hi = min(V, (int)d);
    }
    // p: the address of column `at`
    __device__ __forceinline__ word_t load(const E *p) const
    {
        if (hi == V) return MODE == STREAM ? __builtin_nontemporal_load((const at_t *)p) : *(const at_t *)p;
        word_t r = {};
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < hi) {
                if constexpr (sizeof(E) == 2) r[k / 2] |= (uint32_t)p[k] << (16 * (k & 1));
                else r[k] = ((const uint32_t *)p)[k];
            }
        return r;
    }
    __device__ __forceinline__ static void unpack(word_t w, float (&v)[V])
    {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if constexpr (sizeof(E) == 4) v[k] = __uint_as_float(w[k]);
            else v[k] = __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
        }
    }
    __device__ __forceinline__ void store(E *p, const float (&v)[V]) const
    {
        word_t w;
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = __float_as_uint(v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < V / 2; ++k) w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
        }
        if (lo == 0 && hi == V) {
            if constexpr (MODE == STREAM) __builtin_nontemporal_store(w, (at_t *)p);
            else *(at_t *)p = w;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k >= lo && k < hi) {
                    if constexpr (sizeof(E) == 4) ((uint32_t *)p)[k] = w[k];
                    else p[k] = (E)(w[k / 2] >> (16 * (k & 1)));
                }
        }
    }
};

// An array's values of this thread: step t at base + t st, the same in all lanes, and a lane's
// own offset from its wavefront's first env, so that the steps' addresses take no vector
// registers (the gradient's five arrays of 16 steps would take them all).  O: the offset's type.
template <typename E, typename O>
struct Steps {
    E *base;
    int64_t st;
    O off;
    __device__ __forceinline__ void init(const void *p, int64_t st_, int64_t ld, int64_t env, int first, int at)
    {
        base = (E *)p + first * ld;
        st = st_;
        off = (O)(((env - first) * ld + at) * (int64_t)sizeof(E));
    }
    __device__ __forceinline__ E *operator[](int64_t t) const { return (E *)((char *)(base + t * st) + off); }
};

// a = 1 / (1 + exp(-g)) and b = 1 - a = 1 / (1 + exp(g)), neither by a difference.  exp2's
// argument in two parts: |g| log2 e rounds to 24 bits, which would leave exp with |g| / ln 2
// roundings.
__device__ __forceinline__ void gates(float g, float &a, float &b)
{
    const float L = 0x1.715476p+0f, L2 = 0x1.4ae0cp-26f;      // log2 e, and what its rounding left
    const float n = -fabsf(g), t = n * L;
    const float rest = fmaf(n, L2, fmaf(n, L, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = t > -150.0f ? fmaf(e * 0x1.62e43p-1f, rest, e) : e;      // infinities stay out of the products
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    const float s = e * r;
    a = g < 0.0f ? s : r;
    b = g < 0.0f ? r : s;
}

// Whether all of the wavefront's lanes are there and have the same env.
__device__ __forceinline__ bool one_env(int64_t env)
{
    return __ballot((int)env != __builtin_amdgcn_readfirstlane((int)env)) == 0 && __ballot(true) == ~0ull;
}

// Whether the env's episode ends with each of the U steps from t on, a bit a step (of the last ones
// some may not exist).  Where a wavefront has one env, its lanes take a byte each, the steps' first
// flags and their second ones.
template <int U>
__device__ __forceinline__ uint32_t load_ends(const ScanArgs &a, int64_t env, bool one, int64_t t, int64_t t1)
{
    const uint8_t *f1 = a.term ? a.term : a.trunc, *f2 = a.trunc ? a.trunc : a.term;
    if (!f1) return 0;
    if (one) {
        const int lane = threadIdx.x & 63;
        const int64_t q = min(t + (lane & (U - 1)), t1 - 1);
        const uint64_t m = __ballot(lane < 2 * U && (lane < U ? f1 : f2)[q * a.ld_flags + env] != 0);
        return (uint32_t)(m | m >> U) & ((1u << U) - 1);
    }
    uint32_t m[U], e = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t q = min(t + u, t1 - 1) * a.ld_flags + env;
        m[u] = f1[q] | f2[q];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) e |= m[u] ? 1u << u : 0;
    return e;
}

// ---------------------------------------------------------------------------
// A chunk's steps forward.  MAP: its map alone, from gate and x.  Bound by HBM: 32 x 16384 x 256
// bf16 155 us, 823 MB at 5.3 TB/s; few envs by the latency of the loads, 16 steps at a time (32 steps
// of one env 10.0 us).
// ---------------------------------------------------------------------------
template <typename E, int V, typename O, int MODE>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs a, int64_t pieces)
{
    typedef StepPiece<E, V, MODE> P;
    // steps whose loads are in flight together: with 16 all steps of 32 x 16384 x 256 bf16 take 155 us,
    // 165 with 8; chunks of 16383 x 2 x 361 floats, of which more wavefronts run beside each other, 70 and 60
    constexpr int U = MODE == MAP || MODE == CHUNKS ? KEEP / 2 : KEEP;
    const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= a.n * pieces) return;
    const int64_t env = id / pieces, chunk = blockIdx.y;
    P pc;
    pc.init(id - env * pieces, a.d);
    const int64_t t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.T);
    const int first = __builtin_amdgcn_readfirstlane((int)env);
    Steps<E, O> gate, x, h;
    gate.init(a.gate, a.st_gate, a.ld_gate, env, first, pc.at);
    x.init(a.x, a.st_x, a.ld_x, env, first, pc.at);
    h.init(a.h, a.st_h, a.ld_h, env, first, pc.at);
    const int64_t row = env * a.d;                 // of the states
    const bool one = one_env(env);

    float c[V], p[V];
#pragma unroll
    for (int k = 0; k < V; ++k) c[k] = 0.0f, p[k] = 1.0f;
    if constexpr (MODE != MAP) {
        const float *from = a.chunks > 1 ? a.maps + chunk * 2 * a.n * a.d : a.state;
        if (from)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < pc.hi) c[k] = from[row + pc.at + k];
    }
    typename P::word_t wg[2][U], wx[2][U];
    // steps past the last: the last once more
    auto fetch = [&](int s, int64_t t) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t q = min(t + u, t1 - 1);
            wg[s][u] = pc.load(gate[q]);
            wx[s][u] = pc.load(x[q]);
        }
    };
    auto walk = [&](int s, int64_t t, uint32_t end) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u >= t1) break;
            float g[V], v[V];
            P::unpack(wg[s][u], g);
            P::unpack(wx[s][u], v);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float ga, gb;
                gates(g[k], ga, gb);
                c[k] = fmaf(ga, c[k], gb * v[k]);
                if constexpr (MODE == MAP) p[k] = p[k] < 0.0f ? p[k] : p[k] * ga;
            }
            if constexpr (MODE != MAP) pc.store(h[t + u], c);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                c[k] = end >> u & 1 ? 0.0f : c[k];
                if constexpr (MODE == MAP) p[k] = end >> u & 1 ? -1.0f : p[k];
            }
        }
    };
    uint32_t next = 0;
    if (t0 < t1) {
        fetch(0, t0);
        next = load_ends<U>(a, env, one, t0, t1);
    }
    int64_t t = t0;
    auto turn = [&](auto set) __attribute__((always_inline)) {
        constexpr int s = decltype(set)::value;
        const uint32_t end = next;
        if (t + U < t1) {
            fetch(s ^ 1, t + U);
            next = load_ends<U>(a, env, one, t + U, t1);
        }
        if (MODE != MAP && a.keep && t % KEEP == 0)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k >= pc.lo && k < pc.hi) a.keep[t / KEEP * a.n * a.d + row + pc.at + k] = c[k];
        walk(s, t, end);
        t += U;
    };
    while (t < t1) {
        turn(std::integral_constant<int, 0>());
        if (t < t1) turn(std::integral_constant<int, 1>());
    }
    if constexpr (MODE == MAP) {
        float *m = a.maps + chunk * 2 * a.n * a.d + row;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= pc.lo && k < pc.hi) m[pc.at + k] = p[k], m[a.n * a.d + pc.at + k] = c[k];
    } else if (a.state_out && t1 == a.T) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= pc.lo && k < pc.hi) a.state_out[row + pc.at + k] = c[k];
    }
}

// ---------------------------------------------------------------------------
// Backwards: D, the gradient of the state that passes on from a step, starts from dstate;
// at each step G = dh + live D, D = a G.  The states within 16 steps are formed again from the
// kept one, and with them what G is multiplied by, which takes the place of gate and x in
// registers.  MAP: the chunk's map of D alone, from gate and dh.  32 x 16384 x 256 bf16 291 us, 1.41 GB
// at 4.8 TB/s, with three wavefronts a SIMD, which spill five registers (376 with the two that more registers
// leave, 639 with four, which spill many; of fp32 260 with two, 309 with three; of bf16 rows so far apart
// that their offsets take 64 bits 107 us of 32 x 24 x 65536 with two, 241 with three, which spill 77).
// 16383 x 2 x 361 floats 92 us: maps 25.7, their composition 7.7, steps 59, which read gate and dh again.
// ---------------------------------------------------------------------------
template <typename E, int V, typename O, int MODE>
__global__ __launch_bounds__(256, sizeof(E) == 2 && sizeof(O) == 4 ? 3 : 2) void scan_grad_kernel(ScanArgs a, int64_t pieces)
{
    typedef StepPiece<E, V, MODE> P;
    const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= a.n * pieces) return;
    const int64_t env = id / pieces, chunk = blockIdx.y;
    P pc;
    pc.init(id - env * pieces, a.d);
    const int64_t t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.T);
    const int first = __builtin_amdgcn_readfirstlane((int)env);
    Steps<E, O> gate, x, dh, dgate, dx;
    gate.init(a.gate, a.st_gate, a.ld_gate, env, first, pc.at);
    x.init(a.x, a.st_x, a.ld_x, env, first, pc.at);
    dh.init(a.dh, a.st_dh, a.ld_dh, env, first, pc.at);
    dgate.init(a.dgate, a.st_dgate, a.ld_dgate, env, first, pc.at);
    dx.init(a.dx, a.st_dx, a.ld_dx, env, first, pc.at);
    const int64_t row = env * a.d;
    const bool one = one_env(env);

    float D[V], p[V];
#pragma unroll
    for (int k = 0; k < V; ++k) D[k] = 0.0f, p[k] = 1.0f;
    if constexpr (MODE != MAP) {
        const float *from = a.chunks > 1 ? a.maps + chunk * 2 * a.n * a.d : a.state;
        if (from)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < pc.hi) D[k] = from[row + pc.at + k];
    }
    for (int64_t t = t0 + (t1 - 1 - t0) / KEEP * KEEP; t >= t0 && t < t1; t -= KEEP) {
        const int steps = (int)min((int64_t)KEEP, t1 - t);
        typename P::word_t wg[KEEP], wx[KEEP], wd[KEEP];
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            const int64_t q = t + min(u, steps - 1);
            wg[u] = pc.load(gate[q]);
            if constexpr (MODE != MAP) wx[u] = pc.load(x[q]);
        }
#pragma unroll
        for (int u = 0; u < KEEP; ++u) wd[u] = pc.load(dh[t + min(u, steps - 1)]);
        const uint32_t end = load_ends<KEEP>(a, env, one, t, t1);
        float ga[KEEP][V], gb[KEEP][V], diff[KEEP][V];
        float c[V];
#pragma unroll
        for (int k = 0; k < V; ++k)
            c[k] = MODE != MAP && k < pc.hi ? a.keep[t / KEEP * a.n * a.d + row + pc.at + k] : 0.0f;
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            float g[V], v[V];
            P::unpack(wg[u], g);
            if constexpr (MODE != MAP) P::unpack(wx[u], v);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                gates(g[k], ga[u][k], gb[u][k]);
                if constexpr (MODE != MAP) {
                    diff[u][k] = c[k] - v[k];
                    c[k] = end >> u & 1 ? 0.0f : fmaf(ga[u][k], c[k], gb[u][k] * v[k]);
                }
            }
        }
#pragma unroll
        for (int u = KEEP - 1; u >= 0; --u) {
            if (u >= steps) continue;
            float d[V], og[V], ox[V];
            P::unpack(wd[u], d);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float G = d[k] + (end >> u & 1 ? 0.0f : D[k]);
                D[k] = ga[u][k] * G;
                if constexpr (MODE == MAP) {
                    p[k] = end >> u & 1 || p[k] < 0.0f ? -1.0f : ga[u][k] * p[k];
                } else {
                    ox[k] = gb[u][k] * G;
                    og[k] = ga[u][k] * diff[u][k] * ox[k];
                }
            }
            if constexpr (MODE != MAP) {
                pc.store(dgate[t + u], og);
                pc.store(dx[t + u], ox);
            }
        }
    }
    if constexpr (MODE == MAP) {
        float *m = a.maps + chunk * 2 * a.n * a.d + row;
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= pc.lo && k < pc.hi) m[pc.at + k] = p[k], m[a.n * a.d + pc.at + k] = D[k];
    } else if (a.state_out && t0 == 0) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= pc.lo && k < pc.hi) a.state_out[row + pc.at + k] = D[k];
    }
}

// ---------------------------------------------------------------------------
// From the chunks' maps the state before each chunk (BACK: the gradient after it), left in the
// place of the maps' P.  A block has 16 values; each 16 lanes compose a 64th of the chunks, the
// maps of a wavefront's four parts meet by shuffles, those of the wavefronts in LDS, and each part
// then walks its own chunks.  512 chunks of 722 values: 64 values a block and a part for each
// wavefront took 11.5 us, 17.6 with a part's maps held in registers.
// ---------------------------------------------------------------------------
constexpr int COMPOSE_WAVES = 16, COMPOSE_VALUES = 16;
template <bool BACK>
__global__ __launch_bounds__(64 * COMPOSE_WAVES) void compose_kernel(ScanArgs a)
{
    __shared__ float lp[COMPOSE_WAVES][COMPOSE_VALUES], ls[COMPOSE_WAVES][COMPOSE_VALUES];
    const int at = threadIdx.x & 15, part = threadIdx.x >> 4, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t all = a.n * a.d, v = (int64_t)blockIdx.x * COMPOSE_VALUES + at;
    const int64_t per = (a.chunks + 4 * COMPOSE_WAVES - 1) / (4 * COMPOSE_WAVES);
    const int64_t first = min(part * per, a.chunks), last = min(first + per, a.chunks);
    const bool on = v < all;
    auto apply = [](float mp, float ms, float c) { return mp < 0.0f ? ms : fmaf(mp, c, ms); };
    auto map = [&](int64_t i) { return a.maps + (BACK ? a.chunks - 1 - i : i) * 2 * all + v; };
    float p = 1.0f, s = 0.0f;
    if (on)
#pragma unroll 8
        for (int64_t i = first; i < last; ++i) {
            const float *m = map(i);
            const float mp = m[0], ms = m[all];
            s = apply(mp, ms, s);
            p = mp < 0.0f || p < 0.0f ? -1.0f : p * mp;
        }
    // of this part and those before it in the wavefront
#pragma unroll
    for (int d = 16; d < 64; d *= 2) {
        const float bp = __shfl_up(p, d), bs = __shfl_up(s, d);
        if (lane >= d) {
            s = apply(p, s, bs);
            p = p < 0.0f || bp < 0.0f ? -1.0f : p * bp;
        }
    }
    if (lane >= 48) lp[w][at] = p, ls[w][at] = s;
    __syncthreads();
    float c = on && a.state ? a.state[v] : 0.0f;
    for (int k = 0; k < w; ++k) c = apply(lp[k][at], ls[k][at], c);
    // the parts before this one
    const float bp = __shfl_up(p, 16), bs = __shfl_up(s, 16);
    if (lane >= 16) c = apply(bp, bs, c);
    if (on)
#pragma unroll 8
        for (int64_t i = first; i < last; ++i) {
            float *m = map(i);
            const float mp = m[0], ms = m[all];
            m[0] = c;
            c = apply(mp, ms, c);
        }
}

// Steps of a chunk, by us of T x n x 512 bf16 forward (and backward), from a graph:
//             T 96 n 1     T 128 n 64    T 128 n 128   T 512 n 128    T 512 n 256    T 1024 n 1
//   one       26.5 (40.3)  34.8 (55.0)   37.4 (56.2)   134 (202)      140 (211)      261 (398)
//   chunks    21.8 (27.8)  36.9 (45.0)   53.6 (62.8)   100 (133)      189 (258)      22.3 (28.3)
// and 64 steps of one env 18.1 (28.0) in one launch, 22.0 (27.3) in three.  Chunks leave some
// 262144 threads; of 16383 x 2 x 361 floats with chunks of 16, 32, 64 and 128 steps 72, 64, 70, 91
// (97, 95, 95, 117).
int64_t scan_chunk(int64_t T, int64_t n, int64_t d)
{
    const int64_t lanes = n * ceil_div(d, SCAN_V);
    int64_t chunk = T;
    if (T > 64 && lanes <= std::min<int64_t>(64 * T, 32768))
        chunk = ceil_div(std::max<int64_t>(T * lanes / 262144, 32), KEEP) * KEEP;
    // a grid has 65535 chunks at most
    return std::max<int64_t>(chunk, ceil_div(ceil_div(T, 65535), KEEP) * KEEP);
}

// A call takes most maps neither at the largest T nor at the largest n: 1000 x 64 x 1024 is cut and
// 1000 x 65 x 1024 is not, and chunks grow with the lanes.  Chunks have 32 steps at least, and 32 of each 33
// that T lanes / 262144 comes to (it is rounded down before it is rounded up to 16): there are ceil(T / 32) or
// 262144 33 / 32 / lanes + 1 at most, of n d values each, which are 2 lanes at most and 65536 where
// lanes may be cut.
int64_t scan_workspace_bound(int64_t T, int64_t n, int64_t d)
{
    if (T <= 64) return 0;
    const int64_t values = std::min<int64_t>(n * d, 65536);
    return std::min(ceil_div(T, 32) * values, 540672 + values) * 2 * (int64_t)sizeof(float);
}

template <typename E, typename O, int MODE>
static void scan_launch(const ScanArgs &a, bool grad, dim3 g, dim3 b, int64_t pieces, hipStream_t s)
{
    if (grad) scan_grad_kernel<E, SCAN_V, O, MODE><<<g, b, 0, s>>>(a, pieces);
    else scan_kernel<E, SCAN_V, O, MODE><<<g, b, 0, s>>>(a, pieces);
}

template <typename E, typename O>
static void scan_by(const ScanArgs &a, bool grad, hipStream_t s)
{
    const int64_t pieces = ceil_div(a.d, SCAN_V);
    // chunks of few envs leave less of a small block idle
    const dim3 b(a.chunks > 1 ? 64 : 256), g((unsigned)ceil_div(a.n * pieces, b.x), (unsigned)a.chunks);
    if (a.chunks > 1) {
        const dim3 gc((unsigned)ceil_div(a.n * a.d, COMPOSE_VALUES)), bc(64 * COMPOSE_WAVES);
        scan_launch<E, O, MAP>(a, grad, g, b, pieces, s);
        if (grad) compose_kernel<true><<<gc, bc, 0, s>>>(a);
        else compose_kernel<false><<<gc, bc, 0, s>>>(a);
    }
    const int64_t bytes = a.T * a.n * a.d * (int64_t)sizeof(E) * (grad ? 5 : 3);
    if (a.chunks > 1) scan_launch<E, O, CHUNKS>(a, grad, g, b, pieces, s);
    else if (bytes > INFINITY_CACHE) scan_launch<E, O, STREAM>(a, grad, g, b, pieces, s);
    else scan_launch<E, O, STEPS>(a, grad, g, b, pieces, s);
}

hipError_t launch_scan(const ScanArgs &a, bool grad, bool f32, hipStream_t s)
{
    // a wavefront's envs, at most 64, from its first one on
    const int64_t ld = std::max({a.ld_gate, a.ld_x, a.ld_h, a.ld_dh, a.ld_dgate, a.ld_dx});
    const bool near = (63 * ld + a.d) * 4 < ((int64_t)1 << 32);
    if (f32) near ? scan_by<float, uint32_t>(a, grad, s) : scan_by<float, int64_t>(a, grad, s);
    else near ? scan_by<uint16_t, uint32_t>(a, grad, s) : scan_by<uint16_t, int64_t>(a, grad, s);
    return hipGetLastError();
}

}  // namespace im
