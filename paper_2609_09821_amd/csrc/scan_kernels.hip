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

// V values of a row as words, at any address of their element's alignment.  The last piece of a
// row whose width is no multiple of V takes the last V values of the row: `lo` of them belong
// to the piece before, which alone stores them.  Rows of fewer than V values: value by value.
template <typename E, int V>
struct StepPiece {
    static constexpr int BYTES = sizeof(E) * V;
    typedef uint32_t word_t __attribute__((ext_vector_type(BYTES >= 4 ? BYTES / 4 : 1)));
    typedef word_t at_t __attribute__((aligned(sizeof(E))));
    static_assert(BYTES >= 4 || V == 1, "whole words, or one value");
    int at, lo, hi;      // first column; the values lo .. hi - 1 are this piece's own
    __device__ __forceinline__ void init(int64_t piece, int64_t d)
    {
        const int col = (int)piece * V;
        at = max(0, min(col, (int)d - V));
        lo = col - at;
        hi = min(V, (int)d);
    }
    __device__ __forceinline__ word_t load(const E *row) const
    {
        if constexpr (V == 1) {
            word_t r;
            r[0] = sizeof(E) == 2 ? (uint32_t)((const uint16_t *)row)[at] : ((const uint32_t *)row)[at];
            return r;
        } else {
            if (hi == V) return *(const at_t *)(row + at);
            word_t r = {};
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < hi) {
                    if constexpr (sizeof(E) == 2) r[k / 2] |= (uint32_t)row[k] << (16 * (k & 1));
                    else r[k] = ((const uint32_t *)row)[k];
                }
            return r;
        }
    }
    __device__ __forceinline__ static void unpack(word_t w, float (&v)[V])
    {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if constexpr (sizeof(E) == 4) v[k] = __uint_as_float(w[k]);
            else v[k] = __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
        }
    }
    __device__ __forceinline__ void store(E *row, const float (&v)[V]) const
    {
        word_t w;
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int k = 0; k < V; ++k) w[k] = __float_as_uint(v[k]);
        } else if constexpr (V == 1) {
            w[0] = pack_bf16x2(v[0], 0.0f);
        } else {
#pragma unroll
            for (int k = 0; k < V / 2; ++k) w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
        }
        if (V > 1 && lo == 0 && hi == V) {
            *(at_t *)(row + at) = w;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k >= lo && k < hi) {
                    if constexpr (sizeof(E) == 4) ((uint32_t *)row)[at + k] = w[k];
                    else row[at + k] = (E)(w[k / 2] >> (16 * (k & 1)));
                }
        }
    }
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
    e = g == g && t > -150.0f ? fmaf(e * 0x1.62e43p-1f, rest, e) : e;      // infinities stay out of the products
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    const float s = e * r;
    a = g < 0.0f ? s : r;
    b = g < 0.0f ? r : s;
}

// ---------------------------------------------------------------------------
// A chunk's steps forward.  MAP: its map alone, from gate and x.
// ---------------------------------------------------------------------------
template <typename E, int V, bool MAP>
__global__ __launch_bounds__(256) void scan_kernel(ScanArgs a, int64_t pieces)
{
    typedef StepPiece<E, V> P;
    constexpr int U = KEEP / 2;      // steps whose loads are in flight together
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.n * pieces) return;
    const int64_t env = id / pieces, chunk = blockIdx.y;
    P pc;
    pc.init(id - env * pieces, a.d);
    const int64_t t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.T);
    const E *gate = (const E *)a.gate + env * a.ld_gate + t0 * a.st_gate;
    const E *x = (const E *)a.x + env * a.ld_x + t0 * a.st_x;
    E *h = MAP ? nullptr : (E *)a.h + env * a.ld_h + t0 * a.st_h;
    const int64_t row = env * a.d;                 // of the states
    const bool has_flags = a.term || a.trunc;
    const uint8_t *f1 = a.term ? a.term : a.trunc, *f2 = a.trunc ? a.trunc : a.term;

    float c[V], p[V];
#pragma unroll
    for (int k = 0; k < V; ++k) c[k] = 0.0f, p[k] = 1.0f;
    if constexpr (!MAP) {
        const float *from = a.chunks > 1 ? a.maps + chunk * 2 * a.n * a.d : a.state;
        if (from)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < pc.hi) c[k] = from[row + pc.at + k];
    }
    typename P::word_t wg[2][U], wx[2][U];
    uint32_t end[2];                               // of each step: the episode ends
    auto fetch = [&](int s, int64_t t) {
        uint32_t m[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t q = min(t + u, t1 - 1) - t0;      // steps past the last: the last once more
            wg[s][u] = pc.load(gate + q * a.st_gate);
            wx[s][u] = pc.load(x + q * a.st_x);
            m[u] = has_flags ? f1[(t0 + q) * a.ld_flags + env] | f2[(t0 + q) * a.ld_flags + env] : 0;
        }
        uint32_t e = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) e |= m[u] ? 1u << u : 0;
        end[s] = e;
    };
    auto walk = [&](int s, int64_t t) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u >= t1) break;
            if (!MAP && u == 0 && a.keep && t % KEEP == 0) {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (k >= pc.lo && k < pc.hi) a.keep[t / KEEP * a.n * a.d + row + pc.at + k] = c[k];
            }
            float g[V], v[V];
            P::unpack(wg[s][u], g);
            P::unpack(wx[s][u], v);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float ga, gb;
                gates(g[k], ga, gb);
                c[k] = fmaf(ga, c[k], gb * v[k]);
                if constexpr (MAP) p[k] = p[k] < 0.0f ? p[k] : p[k] * ga;
            }
            if constexpr (!MAP) pc.store(h + (t + u - t0) * a.st_h, c);
            if (end[s] >> u & 1)
#pragma unroll
                for (int k = 0; k < V; ++k) c[k] = 0.0f, p[k] = -1.0f;
        }
    };
    if (t0 < t1) fetch(0, t0);
    for (int64_t t = t0; t < t1; t += 2 * U) {
        if (t + U < t1) fetch(1, t + U);
        walk(0, t);
        if (t + U >= t1) break;
        if (t + 2 * U < t1) fetch(0, t + 2 * U);
        walk(1, t + U);
    }
    if constexpr (MAP) {
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
// kept one.  MAP: the chunk's map of D alone, from gate and dh.
// ---------------------------------------------------------------------------
template <typename E, int V, bool MAP>
__global__ __launch_bounds__(256) void scan_grad_kernel(ScanArgs a, int64_t pieces)
{
    typedef StepPiece<E, V> P;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= a.n * pieces) return;
    const int64_t env = id / pieces, chunk = blockIdx.y;
    P pc;
    pc.init(id - env * pieces, a.d);
    const int64_t t0 = chunk * a.chunk, t1 = min(t0 + a.chunk, a.T);
    const E *gate = (const E *)a.gate + env * a.ld_gate, *x = (const E *)a.x + env * a.ld_x;
    const E *dh = (const E *)a.dh + env * a.ld_dh;
    E *dgate = (E *)a.dgate + env * a.ld_dgate, *dx = (E *)a.dx + env * a.ld_dx;
    const int64_t row = env * a.d;
    const bool has_flags = a.term || a.trunc;
    const uint8_t *f1 = a.term ? a.term : a.trunc, *f2 = a.trunc ? a.trunc : a.term;

    float D[V], p[V];
#pragma unroll
    for (int k = 0; k < V; ++k) D[k] = 0.0f, p[k] = 1.0f;
    if constexpr (!MAP) {
        const float *from = a.chunks > 1 ? a.maps + chunk * 2 * a.n * a.d : a.state;
        if (from)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < pc.hi) D[k] = from[row + pc.at + k];
    }
    for (int64_t t = t0 + (t1 - 1 - t0) / KEEP * KEEP; t >= t0 && t < t1; t -= KEEP) {
        const int steps = (int)min((int64_t)KEEP, t1 - t);
        typename P::word_t wg[KEEP], wx[KEEP], wd[KEEP];
        uint32_t m[KEEP];
#pragma unroll
        for (int u = 0; u < KEEP; ++u) {
            const int64_t q = t + min(u, steps - 1);
            wg[u] = pc.load(gate + q * a.st_gate);
            if constexpr (!MAP) wx[u] = pc.load(x + q * a.st_x);
            wd[u] = pc.load(dh + q * a.st_dh);
            m[u] = has_flags ? f1[q * a.ld_flags + env] | f2[q * a.ld_flags + env] : 0;
        }
        float before[KEEP][V];
        if constexpr (!MAP) {
            float c[V];
#pragma unroll
            for (int k = 0; k < V; ++k) c[k] = k < pc.hi ? a.keep[t / KEEP * a.n * a.d + row + pc.at + k] : 0.0f;
#pragma unroll
            for (int u = 0; u < KEEP; ++u) {
                float g[V], v[V];
                P::unpack(wg[u], g);
                P::unpack(wx[u], v);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    before[u][k] = c[k];
                    float ga, gb;
                    gates(g[k], ga, gb);
                    c[k] = m[u] ? 0.0f : fmaf(ga, c[k], gb * v[k]);
                }
            }
        }
#pragma unroll
        for (int u = KEEP - 1; u >= 0; --u) {
            if (u >= steps) continue;
            float g[V], v[V], d[V], og[V], ox[V];
            P::unpack(wg[u], g);
            P::unpack(wd[u], d);
            if constexpr (!MAP) P::unpack(wx[u], v);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float ga, gb;
                gates(g[k], ga, gb);
                const float G = d[k] + (m[u] ? 0.0f : D[k]);
                D[k] = ga * G;
                if constexpr (MAP) {
                    p[k] = m[u] || p[k] < 0.0f ? -1.0f : ga * p[k];
                } else {
                    ox[k] = gb * G;
                    og[k] = ga * (before[u][k] - v[k]) * ox[k];
                }
            }
            if constexpr (!MAP) {
                pc.store(dgate + (t + u) * a.st_dgate, og);
                pc.store(dx + (t + u) * a.st_dx, ox);
            }
        }
    }
    if constexpr (MAP) {
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
// place of the maps' P: 64 values a block, wavefront w composes a sixteenth of the chunks, the
// wavefronts' maps meet in LDS, and each then walks its own chunks.
// ---------------------------------------------------------------------------
constexpr int COMPOSE_WAVES = 16;
template <bool BACK>
__global__ __launch_bounds__(64 * COMPOSE_WAVES) void compose_kernel(ScanArgs a)
{
    __shared__ float lp[COMPOSE_WAVES][64], ls[COMPOSE_WAVES][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t all = a.n * a.d, v = (int64_t)blockIdx.x * 64 + lane;
    const int64_t per = (a.chunks + COMPOSE_WAVES - 1) / COMPOSE_WAVES;
    const int64_t first = min(w * per, a.chunks), last = min(first + per, a.chunks);
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
    lp[w][lane] = p;
    ls[w][lane] = s;
    __syncthreads();
    float c = on && a.state ? a.state[v] : 0.0f;
    for (int k = 0; k < w; ++k) c = apply(lp[k][lane], ls[k][lane], c);
    if (on)
#pragma unroll 8
        for (int64_t i = first; i < last; ++i) {
            float *m = map(i);
            const float mp = m[0], ms = m[all];
            m[0] = c;
            c = apply(mp, ms, c);
        }
}

int64_t scan_chunk(int64_t T, int64_t n, int64_t d)
{
    // threads of a launch that walks all steps
    const int64_t lanes = n * ceil_div(d, 2);
    int64_t chunk = T;
    if (lanes < 65536 && T > 64) chunk = ceil_div(std::max<int64_t>(T * lanes / 262144, 32), KEEP) * KEEP;
    // a grid has 65535 chunks at most
    return std::max<int64_t>(chunk, ceil_div(ceil_div(T, 65535), KEEP) * KEEP);
}

template <typename E, int V>
static void scan_by(const ScanArgs &a, bool grad, hipStream_t s)
{
    const int64_t pieces = ceil_div(a.d, V);
    const dim3 g((unsigned)ceil_div(a.n * pieces, 256), (unsigned)a.chunks), b(256);
    const dim3 gc((unsigned)ceil_div(a.n * a.d, 64)), bc(64 * COMPOSE_WAVES);
    if (grad) {
        if (a.chunks > 1) {
            scan_grad_kernel<E, V, true><<<g, b, 0, s>>>(a, pieces);
            compose_kernel<true><<<gc, bc, 0, s>>>(a);
        }
        scan_grad_kernel<E, V, false><<<g, b, 0, s>>>(a, pieces);
    } else {
        if (a.chunks > 1) {
            scan_kernel<E, V, true><<<g, b, 0, s>>>(a, pieces);
            compose_kernel<false><<<gc, bc, 0, s>>>(a);
        }
        scan_kernel<E, V, false><<<g, b, 0, s>>>(a, pieces);
    }
}

hipError_t launch_scan(const ScanArgs &a, bool grad, bool f32, hipStream_t s)
{
    if (f32) scan_by<float, 2>(a, grad, s);
    else scan_by<uint16_t, 4>(a, grad, s);
    return hipGetLastError();
}

}  // namespace im
