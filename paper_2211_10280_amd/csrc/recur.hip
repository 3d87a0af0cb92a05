// A gated linear recurrence over packed sequences, its gradient, and its form for single tokens:
//   h[t] = a[t] h[t - 1] + (1 - a[t]) x[t],  a = 1 / (1 + exp(-gate))
//   l[t] = d_out[t] + a[t + 1] l[t + 1],  d_x = (1 - a) l,  d_gate[t] = l[t] (h[t - 1] - x[t]) a[t] (1 - a[t])
// States are fp32.  The forward pass leaves the state before every RECUR_TILE'th token, from which the gradient makes the states of a tile again: that is
// 1 / 256 of x in memory, and exact, where the outputs are rounded to their type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "layers.h"

namespace {

#define RECUR_TILE 256

struct RecurArgs {
    const void *x, *gate, *d;
    void *out, *dx, *dg;
    i64 x_stride, g_stride, d_stride, out_stride, dx_stride, dg_stride, n, n_seq;
    int C4;
    const int *offsets;
    const float *h0, *d_last;
    float *h_last, *dh0, *states;
    const float *kept;           // states, as the gradient reads them
    int *status;
};

// a = 1 / (1 + exp(-g)) and b = 1 - a without the difference
__device__ __forceinline__ void gate2(float g, float &a, float &b)
{
    const float e = __expf(-(g < -87.f ? -87.f : g)), d = 1.0f + e, r = __builtin_amdgcn_rcpf(d);
    a = fmaf(r, fmaf(-d, r, 1.0f), r);           // the reciprocal to half a unit: a is multiplied by itself for thousands of tokens
    b = e * a;
}
__device__ __forceinline__ void gate4(float4 g, float4 &a, float4 &b)
{
    gate2(g.x, a.x, b.x);
    gate2(g.y, a.y, b.y);
    gate2(g.z, a.z, b.z);
    gate2(g.w, a.w, b.w);
}
__device__ __forceinline__ float4 fma4(float4 a, float4 b, float4 c) { return make_float4(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w)); }

// ---- tiles.  The tokens are cut into tiles of RECUR_TILE whatever the sequences are: a sequence's first token resets the state, which is all that a tile has to know of
// them.  A workgroup has a tile's 4 * G channels; a thread has RECUR_RUN tokens that follow one another (a strand of G threads has their channels), in registers from load to
// store.  A run of tokens is a map h -> p h + q (with a reset in it: h -> q), and maps are put together: threads of a wave by shuffles, waves through LDS, tiles by the chain
// below.  What is put together with what, and in which order, hangs on the sizes and offsets alone.
#define RECUR_RUN 8
#define RECUR_STRANDS (RECUR_TILE / RECUR_RUN)
#define RECUR_GROUP 32           // tiles whose maps are put together by every tile of them; their last ones hand states on

struct Map {
    float4 p, q;
    int reset;                   // the state before does not matter; p is not used
};
__device__ __forceinline__ Map map_none() { return Map{make_float4(1.f, 1.f, 1.f, 1.f), make_float4(0.f, 0.f, 0.f, 0.f), 0}; }
// `first`, then `m`.  After a reset the state before is not multiplied by 0 but left out: it may be NaN, and another sequence's.
__device__ __forceinline__ Map then(const Map &first, Map m)
{
    if (!m.reset) {
        m.q = fma4(m.p, first.q, m.q);
        m.p = mul4(m.p, first.p);
        m.reset = first.reset;
    }
    return m;
}
__device__ __forceinline__ float4 apply(const Map &m, float4 h) { return m.reset ? m.q : fma4(m.p, h, m.q); }
template <bool DOWN>
__device__ __forceinline__ float lane_from(float x, int by) { return DOWN ? __shfl_down(x, by, WAVE) : __shfl_up(x, by, WAVE); }
template <bool DOWN>
__device__ __forceinline__ float4 lane_from(float4 x, int by)
{
    return make_float4(lane_from<DOWN>(x.x, by), lane_from<DOWN>(x.y, by), lane_from<DOWN>(x.z, by), lane_from<DOWN>(x.w, by));
}
template <bool DOWN>
__device__ __forceinline__ Map map_from(const Map &m, int by)
{
    return Map{lane_from<DOWN>(m.p, by), lane_from<DOWN>(m.q, by), DOWN ? __shfl_down(m.reset, by, WAVE) : __shfl_up(m.reset, by, WAVE)};
}

template <int G>
struct TileLds {
    static constexpr int WAVES = RECUR_STRANDS * G / WAVE;
    float4 p[WAVES][G], q[WAVES][G];
    int reset[WAVES][G];
    float4 carry[G];
    int head[RECUR_TILE], tail[RECUR_TILE];      // the sequence whose first / last token this is, or -1
    int tile;
};

// The map of all strands before a thread's own (REV: behind it, put together from behind), and of all strands.
template <int G, bool REV>
__device__ __forceinline__ Map strands_before(Map m, TileLds<G> &lds, Map &all)
{
    constexpr int PER = WAVE / G, WAVES = TileLds<G>::WAVES;
    const int lane = lane_id(), wave = uniform((int)threadIdx.x >> 6), l = lane % G, at = REV ? PER - 1 - lane / G : lane / G;
#pragma unroll
    for (int o = 1; o < PER; o *= 2) {
        const Map x = map_from<REV>(m, o * G);
        if (at >= o) m = then(x, m);
    }
    Map before = map_from<REV>(m, G);
    if (at == 0) before = map_none();
    __syncthreads();                             // what an earlier call left has been read
    if (at == PER - 1) {
        lds.p[wave][l] = m.p;
        lds.q[wave][l] = m.q;
        lds.reset[wave][l] = m.reset;
    }
    __syncthreads();
    Map run = map_none(), mine = map_none();
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
        const int w = REV ? WAVES - 1 - k : k;
        if (w == wave) mine = run;
        run = then(run, Map{lds.p[w][l], lds.q[w][l], lds.reset[w][l]});
    }
    all = run;
    return then(mine, before);
}

// ---- the chain of tiles: every tile publishes its map, the last of every RECUR_GROUP its state, each word with its value in it (0: not yet), so that no order of two
// stores matters.  A tile's state is the state handed on by the group before, then the maps of the group's tiles up to it.  Workgroups take tiles in order from a
// counter, so those that a tile waits for run already, and wait for none behind them.
struct Chain {
    u32 *ticket;
    u64 *maps, *states;          // [tiles][4 * C4], [groups][4 * C4]; zero at the start
    int tiles;
};
#define MAP_RESET 0xC0000000u
__device__ __forceinline__ void put_word(u64 *at, u32 hi, float v) { __hip_atomic_store(at, ((u64)hi << 32) | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ u64 wait_word(const u64 *at)
{
    u64 w;
    while ((w = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) == 0) __builtin_amdgcn_s_sleep(1);
    return w;
}
// p is a product of numbers in [0, 1], so its sign is free to say that the word is there
__device__ __forceinline__ u32 map_word(float p, int reset) { return reset ? MAP_RESET : (p == p ? __float_as_uint(p) : 0x7FC00000u) | 0x80000000u; }
__device__ __forceinline__ void put_state(u64 *at, float4 h)
{
    put_word(at, 1u, h.x);
    put_word(at + 1, 1u, h.y);
    put_word(at + 2, 1u, h.z);
    put_word(at + 3, 1u, h.w);
}
__device__ __forceinline__ float low_float(u64 w) { return __uint_as_float((u32)w); }

// The state that comes into the v'th tile (from the left, or, for the gradient, from the right), where it is `wanted`; `own`: the tile's map.
template <int G>
__device__ __forceinline__ float4 chain_state(const Chain &ch, int v, const Map &own, bool wanted, int col, int C4, TileLds<G> &lds)
{
    const int strand = (int)threadIdx.x / G, l = (int)threadIdx.x % G, D = 4 * C4, first = v / RECUR_GROUP * RECUR_GROUP;
    const bool last = v % RECUR_GROUP == RECUR_GROUP - 1, live = col < C4;
    wanted = wanted && v > 0;
    if (strand == 0 && live) {
        u64 *at = ch.maps + (size_t)v * D + 4 * col;
        put_word(at, map_word(own.p.x, own.reset), own.q.x);
        put_word(at + 1, map_word(own.p.y, own.reset), own.q.y);
        put_word(at + 2, map_word(own.p.z, own.reset), own.q.z);
        put_word(at + 3, map_word(own.p.w, own.reset), own.q.w);
        if (last && (own.reset || !wanted)) put_state(ch.states + (size_t)(v / RECUR_GROUP) * D + 4 * col, own.q);
    }
    if (!wanted) return make_float4(0.f, 0.f, 0.f, 0.f);
    Map m = map_none(), all;
    if (strand < v - first && live) {
        const u64 *at = ch.maps + (size_t)(first + strand) * D + 4 * col;
        const u64 a = wait_word(at), b = wait_word(at + 1), c = wait_word(at + 2), d = wait_word(at + 3);
        m.reset = (u32)(a >> 32) == MAP_RESET;
        m.p = make_float4(__uint_as_float((u32)(a >> 32) & 0x7FFFFFFFu), __uint_as_float((u32)(b >> 32) & 0x7FFFFFFFu), __uint_as_float((u32)(c >> 32) & 0x7FFFFFFFu),
                          __uint_as_float((u32)(d >> 32) & 0x7FFFFFFFu));
        m.q = make_float4(low_float(a), low_float(b), low_float(c), low_float(d));
    }
    strands_before<G, false>(m, lds, all);
    if (strand == 0 && live) {
        float4 h = make_float4(0.f, 0.f, 0.f, 0.f);
        if (first > 0 && !all.reset) {
            const u64 *at = ch.states + (size_t)(first / RECUR_GROUP - 1) * D + 4 * col;
            h = make_float4(low_float(wait_word(at)), low_float(wait_word(at + 1)), low_float(wait_word(at + 2)), low_float(wait_word(at + 3)));
        }
        h = apply(all, h);
        if (last && !own.reset) put_state(ch.states + (size_t)(v / RECUR_GROUP) * D + 4 * col, apply(own, h));
        lds.carry[l] = h;
    }
    __syncthreads();
    return lds.carry[l];
}

__global__ void __launch_bounds__(BLOCK) k_recur_clear(u64 *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * BLOCK + threadIdx.x; i < n; i += (size_t)gridDim.x * BLOCK) p[i] = 0;
}

// Which tokens of the tile begin and end sequences; the status bit of a share of the sequences, one workgroup of every tile looking at them.
template <int G>
__device__ __forceinline__ void mark_tile(const RecurArgs &a, i64 t0, int tile, int tiles, int side, TileLds<G> &lds)
{
    constexpr int THREADS = RECUR_STRANDS * G;
    const int t = (int)threadIdx.x;
    for (int i = t; i < RECUR_TILE; i += THREADS) lds.head[i] = lds.tail[i] = -1;
    if (side == 0 && a.status)
        for (i64 s = (i64)tile * THREADS + t; s < a.n_seq; s += (i64)tiles * THREADS) {
            const int lo = a.offsets[s], hi = a.offsets[s + 1];
            if (lo < 0 || hi < lo || hi > a.n) atomicOr(a.status, ST_BAD_ORDER);
        }
    // the first sequence that does not end before the tile, by as many probes at a time as there are threads
    i64 lo = 0, hi = a.n_seq;
    while (lo < hi) {
        const i64 step = (hi - lo + THREADS - 1) / THREADS, at = lo + (t + 1) * step - 1;
        const i64 m = __syncthreads_count(at < hi && a.offsets[at + 1] < t0);
        hi = std::min(hi, lo + (m + 1) * step - 1);
        lo += m * step;
    }
    __syncthreads();
    const bool end = tile == tiles - 1;
    for (i64 base = lo; base < a.n_seq; base += THREADS) {
        const i64 s = base + t;
        bool more = false;
        if (s < a.n_seq) {
            const i64 b = a.offsets[s], e = a.offsets[s + 1];
            more = b < t0 + RECUR_TILE;
            if (b < e) {
                if (b >= t0 && b < t0 + RECUR_TILE) lds.head[b - t0] = (int)s;
                if (e > t0 && e <= t0 + RECUR_TILE) lds.tail[e - 1 - t0] = (int)s;
            } else if (b >= t0 && (end || b < t0 + RECUR_TILE)) {            // no tokens: its state goes through
                float *to = a.dh0 ? a.dh0 : a.h_last;
                const float *from = a.dh0 ? a.d_last : a.h0;
                if (to)
                    for (int c = 0; c < G; ++c) {
                        const int col = side * G + c;
                        if (col < a.C4) st4(to + s * 4 * a.C4 + 4 * col, from ? ld4(from + s * 4 * a.C4 + 4 * col) : make_float4(0.f, 0.f, 0.f, 0.f));
                    }
            }
        }
        if (!end && !__syncthreads_or(more)) break;
    }
    __syncthreads();
}

template <typename T> __device__ __forceinline__ typename Raw4<T>::type raw_shut();      // gates that keep the state as it is
template <> __device__ __forceinline__ float4 raw_shut<float>() { const float inf = __uint_as_float(0x7F800000u); return make_float4(inf, inf, inf, inf); }
template <> __device__ __forceinline__ uint2 raw_shut<bf16_t>() { return make_uint2(0x7F807F80u, 0x7F807F80u); }

template <typename T, int G, bool CHAINED>
__global__ void __launch_bounds__(RECUR_STRANDS *G) k_recur(RecurArgs a, Chain ch)
{
    __shared__ TileLds<G> lds;
    const int strand = (int)threadIdx.x / G, l = (int)threadIdx.x % G, D = 4 * a.C4;
    int tile = 0, side = (int)blockIdx.x;
    if (CHAINED) {
        if (threadIdx.x == 0) lds.tile = (int)atomicAdd(ch.ticket, 1u);
        __syncthreads();
        const int sides = (a.C4 + G - 1) / G;
        tile = lds.tile / sides;
        side = lds.tile - tile * sides;
    }
    const int col = side * G + l;
    const i64 t0 = (i64)tile * RECUR_TILE, run = t0 + strand * RECUR_RUN;
    const i64 begin = std::max(0, a.offsets[0]), end = std::min<i64>(a.n, a.offsets[a.n_seq]);
    typename Raw4<T>::type x[RECUR_RUN], g[RECUR_RUN];
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        const i64 t = run + i;
        zero_raw(x[i]);
        g[i] = raw_shut<T>();
        if (t >= begin && t < end && col < a.C4) {
            x[i] = ldraw((const T *)a.x + t * a.x_stride + 4 * col);
            g[i] = ldraw((const T *)a.gate + t * a.g_stride + 4 * col);
        }
    }
    mark_tile<G>(a, t0, tile, ch.tiles, side, lds);
    float4 f[RECUR_RUN], q[RECUR_RUN];
    Map m = map_none();
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        float4 b;
        gate4(widen4(g[i]), f[i], b);
        q[i] = mul4(b, widen4(x[i]));
        const int s = lds.head[strand * RECUR_RUN + i];
        if (s >= 0) {
            if (a.h0 && col < a.C4) q[i] = fma4(f[i], ld4(a.h0 + (i64)s * D + 4 * col), q[i]);
            m.reset = 1;
            m.q = q[i];
        } else {
            m.q = fma4(f[i], m.q, q[i]);
            m.p = mul4(m.p, f[i]);
        }
    }
    Map all;
    const Map before = strands_before<G, false>(m, lds, all);
    float4 carry = make_float4(0.f, 0.f, 0.f, 0.f);
    if (CHAINED) {
        const bool wanted = t0 >= begin && t0 < end && lds.head[0] < 0;
        carry = chain_state<G>(ch, tile, all, wanted, col, a.C4, lds);
        if (a.states && wanted && strand == 0 && col < a.C4) st4(a.states + (i64)tile * D + 4 * col, carry);
    }
    float4 h = apply(before, carry);
    if (col >= a.C4) return;
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        const i64 t = run + i;
        if (t < begin || t >= end) continue;
        h = lds.head[strand * RECUR_RUN + i] >= 0 ? q[i] : fma4(f[i], h, q[i]);
        st4((T *)a.out + t * a.out_stride + 4 * col, h);
        const int s = lds.tail[strand * RECUR_RUN + i];
        if (a.h_last && s >= 0) st4(a.h_last + (i64)s * D + 4 * col, h);
    }
}

template <typename T, int G, bool CHAINED>
__global__ void __launch_bounds__(RECUR_STRANDS *G) k_recur_grad(RecurArgs a, Chain ch)
{
    __shared__ TileLds<G> lds;
    const int strand = (int)threadIdx.x / G, l = (int)threadIdx.x % G, D = 4 * a.C4;
    int v = 0, side = (int)blockIdx.x;                         // tiles are taken from behind
    if (CHAINED) {
        if (threadIdx.x == 0) lds.tile = (int)atomicAdd(ch.ticket, 1u);
        __syncthreads();
        const int sides = (a.C4 + G - 1) / G;
        v = lds.tile / sides;
        side = lds.tile - v * sides;
    }
    const int tile = ch.tiles - 1 - v, col = side * G + l;
    const i64 t0 = (i64)tile * RECUR_TILE, run = t0 + strand * RECUR_RUN;
    const i64 begin = std::max(0, a.offsets[0]), end = std::min<i64>(a.n, a.offsets[a.n_seq]);
    typename Raw4<T>::type x[RECUR_RUN], g[RECUR_RUN], d[RECUR_RUN];
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        const i64 t = run + i;
        zero_raw(x[i]);
        zero_raw(d[i]);
        g[i] = raw_shut<T>();
        if (t >= begin && t < end && col < a.C4) {
            x[i] = ldraw((const T *)a.x + t * a.x_stride + 4 * col);
            g[i] = ldraw((const T *)a.gate + t * a.g_stride + 4 * col);
            d[i] = ldraw((const T *)a.d + t * a.d_stride + 4 * col);
        }
    }
    mark_tile<G>(a, t0, tile, ch.tiles, side, lds);
    // the states again: from the one that the forward pass left before the tile
    float4 f[RECUR_RUN], b[RECUR_RUN], w[RECUR_RUN];
    Map m = map_none(), all;
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        gate4(widen4(g[i]), f[i], b[i]);
        float4 q = mul4(b[i], widen4(x[i]));
        const int s = lds.head[strand * RECUR_RUN + i];
        if (s >= 0) {
            if (a.h0 && col < a.C4) q = fma4(f[i], ld4(a.h0 + (i64)s * D + 4 * col), q);
            m.reset = 1;
            m.q = q;
        } else {
            m.q = fma4(f[i], m.q, q);
            m.p = mul4(m.p, f[i]);
        }
    }
    const Map before = strands_before<G, false>(m, lds, all);
    float4 h = make_float4(0.f, 0.f, 0.f, 0.f);
    if (CHAINED && t0 >= begin && t0 < end && lds.head[0] < 0 && col < a.C4) h = ld4(a.kept + (i64)tile * D + 4 * col);
    h = apply(before, h);
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {                      // w = (h[t - 1] - x) a
        const int s = lds.head[strand * RECUR_RUN + i];
        const float4 in = widen4(x[i]);
        if (s >= 0) h = a.h0 && col < a.C4 ? ld4(a.h0 + (i64)s * D + 4 * col) : make_float4(0.f, 0.f, 0.f, 0.f);
        w[i] = mul4(f[i], make_float4(h.x - in.x, h.y - in.y, h.z - in.z, h.w - in.w));
        h = fma4(f[i], h, mul4(b[i], in));
    }
    // c = a l, handed on to the token before
    m = map_none();
#pragma unroll
    for (int i = RECUR_RUN - 1; i >= 0; --i) {
        const int s = lds.tail[strand * RECUR_RUN + i];
        if (s >= 0) {
            m.reset = 1;
            m.q = a.d_last && col < a.C4 ? ld4(a.d_last + (i64)s * D + 4 * col) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        m.q = mul4(f[i], plus4(widen4(d[i]), m.q));
        m.p = mul4(m.p, f[i]);
    }
    const Map behind = strands_before<G, true>(m, lds, all);
    float4 c = make_float4(0.f, 0.f, 0.f, 0.f);
    if (CHAINED) {
        const i64 t1 = t0 + RECUR_TILE;
        c = chain_state<G>(ch, v, all, t1 > begin && t1 < end && lds.tail[RECUR_TILE - 1] < 0, col, a.C4, lds);
    }
    c = apply(behind, c);
    if (col >= a.C4) return;
#pragma unroll
    for (int i = RECUR_RUN - 1; i >= 0; --i) {
        const i64 t = run + i;
        if (t < begin || t >= end) continue;
        const int tail = lds.tail[strand * RECUR_RUN + i], head = lds.head[strand * RECUR_RUN + i];
        if (tail >= 0) c = a.d_last ? ld4(a.d_last + (i64)tail * D + 4 * col) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 lam = plus4(widen4(d[i]), c), dx = mul4(b[i], lam);
        st4((T *)a.dx + t * a.dx_stride + 4 * col, dx);
        st4((T *)a.dg + t * a.dg_stride + 4 * col, mul4(dx, w[i]));
        c = mul4(f[i], lam);
        if (a.dh0 && head >= 0) st4(a.dh0 + (i64)head * D + 4 * col, c);
    }
}

struct StepArgs {
    const void *x, *gate;
    void *out;
    i64 x_stride, g_stride, out_stride, state_stride, n, n_slots;
    int C4;
    const int *slots;
    float *state;
    int *status;
};

template <typename T>
__global__ void __launch_bounds__(BLOCK) k_recur_step(StepArgs a)
{
    const i64 id = (i64)blockIdx.x * BLOCK + threadIdx.x, i = id / a.C4;
    const int c = 4 * (int)(id - i * a.C4);
    if (i >= a.n) return;
    const i64 slot = a.slots ? a.slots[i] : i;
    if (slot < 0 || slot >= a.n_slots) {
        if (a.status && c == 0) atomicOr(a.status, ST_BAD_ID);
        if (a.out) st4((T *)a.out + i * a.out_stride + c, make_float4(0.f, 0.f, 0.f, 0.f));
        return;
    }
    if (a.slots)
        for (i64 j = 0; j < i; ++j)
            if (a.slots[j] == slot) return;                    // the slot's first row takes them all
    float4 h = ld4(a.state + slot * a.state_stride + c);
    for (i64 j = i; j < a.n; ++j) {
        if (j > i && (!a.slots || a.slots[j] != slot)) {
            if (!a.slots) break;
            continue;
        }
        float4 f, b;
        gate4(ld4((const T *)a.gate + j * a.g_stride + c), f, b);
        h = fma4(f, h, mul4(b, ld4((const T *)a.x + j * a.x_stride + c)));
        if (a.out) st4((T *)a.out + j * a.out_stride + c, h);
    }
    st4(a.state + slot * a.state_stride + c, h);
}

// bytes of the chain's words, or, with an address, the chain there and what of it has to be zero
size_t recur_carve(i64 n, int dim, char *ws, Chain *ch)
{
    const i64 tiles = std::max<i64>(1, (n + RECUR_TILE - 1) / RECUR_TILE), groups = (tiles + RECUR_GROUP - 1) / RECUR_GROUP;
    if (ch) {
        ch->ticket = (u32 *)ws;
        ch->maps = (u64 *)(ws + 256);
        ch->states = ch->maps + (size_t)tiles * dim;
        ch->tiles = (int)tiles;
    }
    return 256 + layer_up256(8 * (size_t)(tiles + groups) * (size_t)dim);
}

template <typename T, int G>
int launch_recur(const RecurArgs &a, void *workspace, hipStream_t st)
{
    Chain ch;
    const size_t bytes = recur_carve(a.n, 4 * a.C4, (char *)workspace, &ch);
    const int sides = (a.C4 + G - 1) / G;
    if ((i64)ch.tiles * sides > (i64)TN_MAX_BLOCKS * BLOCK / (RECUR_STRANDS * G)) return tn_fail(TENSAIR_EINVAL, "n * dim beyond what one launch covers");
    const dim3 blk(RECUR_STRANDS * G);
    const bool grad = a.dx != nullptr || a.kept != nullptr;
    if (ch.tiles == 1) {
        if (grad) hipLaunchKernelGGL((k_recur_grad<T, G, false>), dim3(sides), blk, 0, st, a, ch);
        else hipLaunchKernelGGL((k_recur<T, G, false>), dim3(sides), blk, 0, st, a, ch);
        return TENSAIR_OK;
    }
    hipLaunchKernelGGL(k_recur_clear, dim3((unsigned)std::min<size_t>(1024, (bytes / 8 + BLOCK - 1) / BLOCK)), dim3(BLOCK), 0, st, (u64 *)workspace, bytes / 8);
    const dim3 grid((unsigned)((i64)ch.tiles * sides));
    if (grad) hipLaunchKernelGGL((k_recur_grad<T, G, true>), grid, blk, 0, st, a, ch);
    else hipLaunchKernelGGL((k_recur<T, G, true>), grid, blk, 0, st, a, ch);
    return TENSAIR_OK;
}
int launch_recur(const RecurArgs &a, int32_t dtype, void *workspace, hipStream_t st)
{
    if (dtype == TENSAIR_F32) return a.C4 <= 8 ? launch_recur<float, 8>(a, workspace, st) : launch_recur<float, 16>(a, workspace, st);
    return a.C4 <= 8 ? launch_recur<bf16_t, 8>(a, workspace, st) : launch_recur<bf16_t, 16>(a, workspace, st);
}

int check_recur(const void *x, i64 x_stride, const void *gate, i64 gate_stride, int32_t dtype, i64 n, int32_t dim, const int32_t *offsets, i64 n_seq,
                const void *workspace, size_t workspace_bytes, const int32_t *status)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = layer_matrix(gate, n, gate_stride, dim, dtype, "gate"))) return rc;
    if (n_seq < 0 || n_seq > TENSAIR_MAX_ROWS) return tn_fail(TENSAIR_EINVAL, "n_seq must be in 0..TENSAIR_MAX_ROWS");
    if (!offsets || ((uintptr_t)offsets & 3)) return tn_fail(TENSAIR_EINVAL, "offsets must be 4-byte aligned and not NULL");
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    return layer_workspace(workspace, workspace_bytes, tensair_recur_workspace_bytes(n, dim), "tensair_recur_workspace_bytes");
}

}  // namespace

extern "C" {

int64_t tensair_recur_state_rows(int64_t n)
{
    if (layer_sizes(n, 4)) return TENSAIR_EINVAL;
    return std::max<i64>(1, (n + RECUR_TILE - 1) / RECUR_TILE);
}

size_t tensair_recur_workspace_bytes(int64_t n, int32_t dim)
{
    if (layer_sizes(n, dim)) return 0;
    return recur_carve(n, dim, nullptr, nullptr);
}

int tensair_recur(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *offsets,
                  int64_t n_seq, const float *h0, void *out, int64_t out_stride, float *h_last, float *states, void *workspace, size_t workspace_bytes,
                  int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_recur(x, x_stride, gate, gate_stride, dtype, n, dim, offsets, n_seq, workspace, workspace_bytes, status))) return rc;
    if ((rc = layer_matrix(out, n, out_stride, dim, dtype, "out"))) return rc;
    if ((rc = layer_floats(h0, "h0")) || (rc = layer_floats(h_last, "h_last")) || (rc = layer_floats(states, "states"))) return rc;
    if (n_seq == 0) return TENSAIR_OK;
    RecurArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x;
    a.gate = gate;
    a.out = out;
    a.x_stride = x_stride;
    a.g_stride = gate_stride;
    a.out_stride = out_stride;
    a.n = n;
    a.n_seq = n_seq;
    a.C4 = dim / 4;
    a.offsets = offsets;
    a.h0 = h0;
    a.h_last = h_last;
    a.states = states;
    a.status = status;
    hipStream_t st = (hipStream_t)stream;
    if ((rc = launch_recur(a, dtype, workspace, st))) return rc;
    return layer_launched("recur");
}

int tensair_recur_grad(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *offsets,
                       int64_t n_seq, const float *h0, const float *states, const void *d_out, int64_t d_stride, const float *d_last, void *d_x,
                       int64_t d_x_stride, void *d_gate, int64_t d_gate_stride, float *d_h0, void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_recur(x, x_stride, gate, gate_stride, dtype, n, dim, offsets, n_seq, workspace, workspace_bytes, status))) return rc;
    if ((rc = layer_matrix(d_out, n, d_stride, dim, dtype, "d_out")) || (rc = layer_matrix(d_x, n, d_x_stride, dim, dtype, "d_x")) ||
        (rc = layer_matrix(d_gate, n, d_gate_stride, dim, dtype, "d_gate")))
        return rc;
    if ((rc = layer_floats(h0, "h0")) || (rc = layer_floats(states, "states")) || (rc = layer_floats(d_last, "d_last")) || (rc = layer_floats(d_h0, "d_h0"))) return rc;
    if (!states) return tn_fail(TENSAIR_EINVAL, "states is NULL");
    if (n_seq == 0) return TENSAIR_OK;
    RecurArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x;
    a.gate = gate;
    a.d = d_out;
    a.dx = d_x;
    a.dg = d_gate;
    a.x_stride = x_stride;
    a.g_stride = gate_stride;
    a.d_stride = d_stride;
    a.dx_stride = d_x_stride;
    a.dg_stride = d_gate_stride;
    a.n = n;
    a.n_seq = n_seq;
    a.C4 = dim / 4;
    a.offsets = offsets;
    a.h0 = h0;
    a.d_last = d_last;
    a.dh0 = d_h0;
    a.kept = states;
    a.status = status;
    hipStream_t st = (hipStream_t)stream;
    if ((rc = launch_recur(a, dtype, workspace, st))) return rc;
    return layer_launched("recur_grad");
}

int tensair_recur_step(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *slots,
                       int64_t n_slots, float *state, int64_t state_stride, void *out, int64_t out_stride, int32_t *status, void *stream)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = layer_matrix(gate, n, gate_stride, dim, dtype, "gate"))) return rc;
    if (out && (rc = layer_matrix(out, n, out_stride, dim, dtype, "out"))) return rc;
    if ((rc = layer_matrix(state, n_slots, state_stride, dim, TENSAIR_F32, "state"))) return rc;
    if (n_slots < (n > 0) || n_slots > TENSAIR_MAX_ROWS) return tn_fail(TENSAIR_EINVAL, "n_slots must be in 1..TENSAIR_MAX_ROWS");
    if ((uintptr_t)slots & 3) return tn_fail(TENSAIR_EINVAL, "slots must be 4-byte aligned");
    if (slots ? n > TENSAIR_MAX_STEP_ROWS : n > n_slots) return tn_fail(TENSAIR_EINVAL, "n must be at most TENSAIR_MAX_STEP_ROWS with slots, n_slots without");
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    const StepArgs a = {x, gate, out, x_stride, gate_stride, out_stride, state_stride, n, n_slots, dim / 4, slots, state, status};
    const u64 blocks = ((u64)n * (u64)a.C4 + BLOCK - 1) / BLOCK;
    if (blocks > TN_MAX_BLOCKS) return tn_fail(TENSAIR_EINVAL, "n * dim beyond what one launch covers");
    const dim3 grid((unsigned)blocks), blk(BLOCK);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_recur_step<float>, grid, blk, 0, st, a);
    else hipLaunchKernelGGL(k_recur_step<bf16_t>, grid, blk, 0, st, a);
    return layer_launched("recur_step");
}

}  // extern "C"
