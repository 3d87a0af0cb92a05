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

// a = 1 / (1 + exp(-g)) and b = 1 - a as one number: the smaller of the two, e / (1 + e) with e = exp(-|g|), with g's sign, which says which of them it is.  The larger is
// 1 - that, within half a unit whatever the smaller one's last places are.
__device__ __forceinline__ float gate1(float g)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(g) * -1.44269504f);
    return copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), g);
}
__device__ __forceinline__ void open2(float s, float &a, float &b)
{
    const float small = fabsf(s), large = 1.0f - small;
    const bool low = __float_as_int(s) < 0;
    a = low ? small : large;
    b = low ? large : small;
}
__device__ __forceinline__ float4 gate4(float4 g) { return make_float4(gate1(g.x), gate1(g.y), gate1(g.z), gate1(g.w)); }
__device__ __forceinline__ void open4(float4 s, float4 &a, float4 &b)
{
    open2(s.x, a.x, b.x);
    open2(s.y, a.y, b.y);
    open2(s.z, a.z, b.z);
    open2(s.w, a.w, b.w);
}
__device__ __forceinline__ void gate4(float4 g, float4 &a, float4 &b) { open4(gate4(g), a, b); }
__device__ __forceinline__ float4 fma4(float4 a, float4 b, float4 c) { return make_float4(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w)); }

// ---- tiles.  The tokens are cut into tiles of RECUR_TILE whatever the sequences are: a sequence's first token resets the state, which is all that a tile has to know of
// them.  A workgroup has a tile's 4 * G channels; a thread has RECUR_RUN tokens that follow one another (a strand of G threads has their channels), in registers from load to
// store.  A run of tokens is a map h -> p h + q (with a reset in it: h -> q), and maps are put together: threads of a wave by shuffles, waves through LDS, tiles by the chain
// below.  What is put together with what, and in which order, hangs on the sizes and offsets alone.
#define RECUR_RUN 8
#define RECUR_STRANDS (RECUR_TILE / RECUR_RUN)

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
    float4 carry[G], own_p[G], own_q[G];
    int said[G];
    int head[RECUR_TILE], tail[RECUR_TILE];      // the sequence whose first / last token this is
    u32 heads[RECUR_STRANDS], tails[RECUR_STRANDS];   // the strands' tokens that are one, as bits; only there the above holds
    int tile;
};

// The map of all strands before a thread's own (REV: behind it, put together from behind); `all`: with its own, so the last strand's is that of the tile.
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
    Map run = map_none();
    for (int k = 0; k < (REV ? WAVES - 1 - wave : wave); ++k) {
        const int w = REV ? WAVES - 1 - k : k;
        run = then(run, Map{lds.p[w][l], lds.q[w][l], lds.reset[w][l]});
    }
    all = then(run, m);
    return then(run, before);
}

// ---- the chain of tiles: every tile publishes its map, the last of every group its state, each word with its value in it (0: not yet), so that no order of two
// stores matters.  A tile's state is the state handed on by the group before, then the maps of the group's tiles up to it.  Workgroups take tiles in order from a
// counter, so those that a tile waits for run already, and wait for none behind them.
struct Chain {
    u32 *ticket;
    u32 *lost;                   // set where a wait was given up
    u64 *maps, *states;          // [tiles][4 * C4], [groups][4 * C4]; zero at the start
    int tiles;
    int group;                   // tiles whose maps are put together by every tile of them; the last of a group hands the state on
};
#define MAP_RESET 0xC0000000u
__device__ __forceinline__ void put_word(u64 *at, u32 hi, float v) { __hip_atomic_store(at, ((u64)hi << 32) | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Every wait ends: the word comes, or, where another call uses the same workspace at the same time and has cleared it, the wait is given up after some seconds, and all others with
// it; what is made of it is NaN.
#define CHAIN_PATIENCE (1u << 22)
__device__ __forceinline__ u64 wait_word(const u64 *at, u32 *lost)
{
    u64 w;
    for (u32 n = 1; (w = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) == 0; ++n) {
        __builtin_amdgcn_s_sleep(1);
        if (n % 4096 == 0 && (n >= CHAIN_PATIENCE || __hip_atomic_load(lost, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))) {
            __hip_atomic_store(lost, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            return 0xC00000007FC00000ull;        // a reset to NaN
        }
    }
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

// The v'th tile's map, which its last strand has, to the others; its state too where nothing is waited for.
template <int G, bool REV>
__device__ __forceinline__ void chain_say(const Chain &ch, int v, const Map &own, bool wanted, int col, int C4, TileLds<G> &lds)
{
    const int strand = REV ? RECUR_STRANDS - 1 - (int)threadIdx.x / G : (int)threadIdx.x / G, l = (int)threadIdx.x % G, D = 4 * C4;
    if (strand < RECUR_STRANDS - 1 || col >= C4) return;
    u64 *at = ch.maps + (size_t)v * D + 4 * col;
    put_word(at, map_word(own.p.x, own.reset), own.q.x);
    put_word(at + 1, map_word(own.p.y, own.reset), own.q.y);
    put_word(at + 2, map_word(own.p.z, own.reset), own.q.z);
    put_word(at + 3, map_word(own.p.w, own.reset), own.q.w);
    if (v % ch.group < ch.group - 1) return;
    if (own.reset || !wanted || v == 0) {
        put_state(ch.states + (size_t)(v / ch.group) * D + 4 * col, own.q);
    } else {                                     // a thread's own words, for itself
        lds.own_p[l] = own.p;
        lds.own_q[l] = own.q;
    }
    lds.said[l] = own.reset || !wanted || v == 0;
}
// The state that comes into the v'th tile (from the left, or, for the gradient, from the right), where it is `wanted`.
template <int G, bool REV>
__device__ __forceinline__ float4 chain_state(const Chain &ch, int v, bool wanted, int col, int C4, TileLds<G> &lds)
{
    const int strand = REV ? RECUR_STRANDS - 1 - (int)threadIdx.x / G : (int)threadIdx.x / G, l = (int)threadIdx.x % G, D = 4 * C4, first = v / ch.group * ch.group;
    if (!wanted || v == 0) return make_float4(0.f, 0.f, 0.f, 0.f);
    Map m = map_none(), all;
    const int per = (ch.group + RECUR_STRANDS - 1) / RECUR_STRANDS;      // tiles that follow one another to a strand
    for (int tile = first + strand * per; tile < min(v, first + (strand + 1) * per) && col < C4; ++tile) {
        const u64 *at = ch.maps + (size_t)tile * D + 4 * col;
        const u64 a = wait_word(at, ch.lost), b = wait_word(at + 1, ch.lost), c = wait_word(at + 2, ch.lost), d = wait_word(at + 3, ch.lost);
        const Map x = {make_float4(__uint_as_float((u32)(a >> 32) & 0x7FFFFFFFu), __uint_as_float((u32)(b >> 32) & 0x7FFFFFFFu), __uint_as_float((u32)(c >> 32) & 0x7FFFFFFFu),
                                   __uint_as_float((u32)(d >> 32) & 0x7FFFFFFFu)),
                       make_float4(low_float(a), low_float(b), low_float(c), low_float(d)), (u32)(a >> 32) == MAP_RESET};
        m = then(m, x);
    }
    strands_before<G, REV>(m, lds, all);
    if (strand == RECUR_STRANDS - 1 && col < C4) {
        float4 h = make_float4(0.f, 0.f, 0.f, 0.f);
        if (first > 0 && !all.reset) {
            const u64 *at = ch.states + (size_t)(first / ch.group - 1) * D + 4 * col;
            h = make_float4(low_float(wait_word(at, ch.lost)), low_float(wait_word(at + 1, ch.lost)), low_float(wait_word(at + 2, ch.lost)), low_float(wait_word(at + 3, ch.lost)));
        }
        h = apply(all, h);
        if (v % ch.group == ch.group - 1 && !lds.said[l]) put_state(ch.states + (size_t)(v / ch.group) * D + 4 * col, fma4(lds.own_p[l], h, lds.own_q[l]));
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
    if (t < RECUR_STRANDS) lds.heads[t] = lds.tails[t] = 0;
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
                if (b >= t0 && b < t0 + RECUR_TILE) {
                    const int at = (int)(b - t0);
                    lds.head[at] = (int)s;
                    atomicOr(&lds.heads[at / RECUR_RUN], 1u << at % RECUR_RUN);
                }
                if (e > t0 && e <= t0 + RECUR_TILE) {
                    const int at = (int)(e - 1 - t0);
                    lds.tail[at] = (int)s;
                    atomicOr(&lds.tails[at / RECUR_RUN], 1u << at % RECUR_RUN);
                }
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

// Tokens of a tile in a matrix: an address that all threads share and, in 32 bits, places from there.
struct TileOf {
    char *p;
    u32 stride;                  // bytes from token to token
};
template <typename T>
__device__ __forceinline__ TileOf tile_of(const void *p, i64 stride, i64 t0) { return TileOf{(char *)p + t0 * stride * (i64)sizeof(T), (u32)stride * (u32)sizeof(T)}; }
// A thread's run of tokens, those of no sequence (first..last are of some) as the nearest that is of one: what they hold does not matter, since the sequences' first and last tokens reset what
// comes before or behind them.  The same for the columns, up to `col`.
template <typename T>
__device__ __forceinline__ void load_run(typename Raw4<T>::type (&r)[RECUR_RUN], const TileOf &m, int token, int col, int first, int last)
{
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) r[i] = ldraw((const T *)(m.p + (size_t)((u32)min(max(token + i, first), last) * m.stride + (u32)(4 * sizeof(T)) * (u32)col)));
}
template <typename T>
__device__ __forceinline__ void store_at(const TileOf &m, int token, int col, float4 v) { put4((T *)(m.p + (size_t)((u32)token * m.stride + (u32)(4 * sizeof(T)) * (u32)col)), v); }
// From here on the compiler takes the values for new ones: it widens and multiplies them again instead of keeping what it has made of them in registers.
__device__ __forceinline__ void forget(uint2 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y)); }
__device__ __forceinline__ void forget(float4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }
__device__ __forceinline__ float4 row_or_zero(const float *p, i64 row, int C4, int col)
{
    return p && col < C4 ? ld4(p + row * 4 * C4 + 4 * col) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// Forward.  262 144 tokens of 512 in 200 sequences, bfloat16: 270 us (805 MB, 3.0 TB/s), 131 072 of 128 in one 51, 4 096 of 128 in fp32 11.  Vector units are busy half of the time (37 instructions an
// element, of which 17 are the gate, the map and the state) and waves wait 54 % of theirs: without the wait for other tiles' maps it is 216 us, without putting maps together at all 198, while adding
// two matrices of these sizes takes 134.  Not kept: a grid as large as the card that takes tile after tile (its next ticket fetched ahead; 517 us, arguments read again and registers short), 16 tokens to a
// thread (274), 256 channels to a workgroup's row (337), the sides of a tile turned round from tile to tile (no difference).
template <typename T, int G, bool CHAINED>
__device__ __forceinline__ void k_recur_tile(const RecurArgs &a, const Chain &ch, int k, int sides, i64 begin, i64 end, TileLds<G> &lds)
{
    const int strand = (int)threadIdx.x / G, l = (int)threadIdx.x % G;
    const int tile = CHAINED ? k / sides : 0, side = k - tile * sides;
    const int col = side * G + l;
    const i64 t0 = (i64)tile * RECUR_TILE;
    const bool mine = col < a.C4;
    // the tile's tokens that sequences have; where there are none nothing comes through
    const int from = (int)std::min<i64>(RECUR_TILE, std::max<i64>(0, begin - t0)), to = (int)std::max<i64>(0, std::min<i64>(RECUR_TILE, end - t0));
    const int token = strand * RECUR_RUN, lo = from - token, hi = to - token, near = min(col, a.C4 - 1);
    typename Raw4<T>::type x[RECUR_RUN], g[RECUR_RUN];
    if (from < to) {
        load_run<T>(x, tile_of<T>(a.x, a.x_stride, t0), token, near, from, to - 1);
        load_run<T>(g, tile_of<T>(a.gate, a.g_stride, t0), token, near, from, to - 1);
    }
    mark_tile<G>(a, t0, tile, ch.tiles, side, lds);
    if (from >= to) {
        if (CHAINED) chain_say<G, false>(ch, tile, Map{make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f), 1}, false, col, a.C4, lds);
        return;
    }
    const u32 heads = lds.heads[strand], tails = lds.tails[strand];
    const bool ends = __any(heads | tails), full = mine && from == 0 && to == RECUR_TILE;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    float4 f[RECUR_RUN], q[RECUR_RUN];
    Map m = map_none(), all;
    m.q = zero;
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        float4 b;
        gate4(widen4(g[i]), f[i], b);
        q[i] = mul4(b, widen4(x[i]));
        if (ends && heads >> i & 1) {
            q[i] = fma4(f[i], row_or_zero(a.h0, lds.head[strand * RECUR_RUN + i], a.C4, col), q[i]);
            m.reset = 1;
            m.q = zero;
        }
        m.q = fma4(f[i], m.q, q[i]);
        m.p = mul4(m.p, f[i]);
    }
    const Map before = strands_before<G, false>(m, lds, all);
    float4 carry = make_float4(0.f, 0.f, 0.f, 0.f);
    if (CHAINED) {
        const bool wanted = from == 0 && !(lds.heads[0] & 1);
        chain_say<G, false>(ch, tile, all, wanted, col, a.C4, lds);
        carry = chain_state<G, false>(ch, tile, wanted, col, a.C4, lds);
        if (a.states && wanted && strand == 0 && mine) st4(a.states + ((i64)tile * a.C4 + col) * 4, carry);
    }
    float4 h = apply(before, carry);
    const TileOf out = tile_of<T>(a.out, a.out_stride, t0);
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        if (ends && heads >> i & 1) h = zero;
        h = fma4(f[i], h, q[i]);
        if (full || (mine && i >= lo && i < hi)) {
            store_at<T>(out, token + i, col, h);
            if (ends && a.h_last && tails >> i & 1) st4(a.h_last + ((i64)lds.tail[strand * RECUR_RUN + i] * a.C4 + col) * 4, h);
        }
    }
}

template <typename T, int G, bool CHAINED>
__global__ void __launch_bounds__(RECUR_STRANDS *G, 4) k_recur(RecurArgs a, Chain ch)
{
    __shared__ TileLds<G> lds;
    const i64 begin = std::max(0, a.offsets[0]), end = std::min<i64>(a.n, a.offsets[a.n_seq]);
    int k = (int)blockIdx.x;
    if (CHAINED) {
        if (threadIdx.x == 0) lds.tile = (int)atomicAdd(ch.ticket, 1u);
        __syncthreads();
        k = uniform(lds.tile);
        if ((u32)k >= (u32)(ch.tiles * ((a.C4 + G - 1) / G))) return;      // only where another call takes tickets from the same workspace
    }
    k_recur_tile<T, G, CHAINED>(a, ch, k, (a.C4 + G - 1) / G, begin, end, lds);
}

// Gradient: the states of the tile again, then from behind.  262 144 tokens of 512, bfloat16: 400 us, 131 072 of 128 in one sequence 72, 4 096 of 128 in fp32 14.5.  1.34 GB have to be moved (3.4 TB/s);
// 1.95 GB are, at the rate of a copy, since a workgroup takes half a line of a token and its other half is fetched again: memory bounds it.  In fp32, by whole lines, 511 us for 2.68 GB.  The vector units
// are busy 61 % of the time.  A gate's two sides held as one number, the gradients of the outputs in LDS, and what is made of them made again rather than held: 128 registers a thread, nothing in memory (595 us
// before, with 224; 525 with 128 and spills).
template <typename T, int G, bool CHAINED>
__device__ __forceinline__ void k_recur_grad_tile(const RecurArgs &a, const Chain &ch, int k, int sides, i64 begin, i64 end, TileLds<G> &lds, typename Raw4<T>::type (&kept_d)[RECUR_RUN][RECUR_STRANDS * G])
{
    const int strand = (int)threadIdx.x / G, l = (int)threadIdx.x % G;
    const int v = CHAINED ? k / sides : 0, side = k - v * sides;                         // tiles are taken from behind
    const int tile = ch.tiles - 1 - v, col = side * G + l;
    const i64 t0 = (i64)tile * RECUR_TILE;
    const bool mine = col < a.C4;
    // the tile's tokens that sequences have; where there are none nothing comes through
    const int from = (int)std::min<i64>(RECUR_TILE, std::max<i64>(0, begin - t0)), to = (int)std::max<i64>(0, std::min<i64>(RECUR_TILE, end - t0));
    const int token = strand * RECUR_RUN, lo = from - token, hi = to - token, near = min(col, a.C4 - 1);
    typename Raw4<T>::type x[RECUR_RUN], g[RECUR_RUN], d[RECUR_RUN];
    if (from < to) {
        load_run<T>(x, tile_of<T>(a.x, a.x_stride, t0), token, near, from, to - 1);
        load_run<T>(g, tile_of<T>(a.gate, a.g_stride, t0), token, near, from, to - 1);
        load_run<T>(d, tile_of<T>(a.d, a.d_stride, t0), token, near, from, to - 1);
    }
    mark_tile<G>(a, t0, tile, ch.tiles, side, lds);
    if (from >= to) {
        if (CHAINED) chain_say<G, true>(ch, v, Map{make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f), 1}, false, col, a.C4, lds);
        return;
    }
    const u32 heads = lds.heads[strand], tails = lds.tails[strand];
    const bool ends = __any(heads | tails), full = mine && from == 0 && to == RECUR_TILE;
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) kept_d[i][threadIdx.x] = d[i];
    // two maps of the run: of the state, from the left, and of c = a l, which a token hands on to the one before, from the right
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    float4 s[RECUR_RUN], w[RECUR_RUN], f, b;
    Map m = map_none(), n = map_none(), all;
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        s[i] = gate4(widen4(g[i]));
        open4(s[i], f, b);
        if (ends && heads >> i & 1) {
            m.reset = 1;
            m.q = row_or_zero(a.h0, lds.head[strand * RECUR_RUN + i], a.C4, col);
        }
        m.q = fma4(f, m.q, mul4(b, widen4(x[i])));
        m.p = mul4(m.p, f);
    }
#pragma unroll
    for (int i = RECUR_RUN - 1; i >= 0; --i) {
        forget(s[i]);
        open4(s[i], f, b);
        if (ends && tails >> i & 1) {
            n.reset = 1;
            n.q = row_or_zero(a.d_last, lds.tail[strand * RECUR_RUN + i], a.C4, col);
        }
        n.q = mul4(f, plus4(widen4(kept_d[i][threadIdx.x]), n.q));
    }
    n.p = m.p;
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {
        forget(s[i]);
        forget(x[i]);
    }
    float4 h = zero, c = zero;
    if (CHAINED && from == 0 && !(lds.heads[0] & 1) && mine) h = ld4(a.kept + ((i64)tile * a.C4 + col) * 4);
    h = apply(strands_before<G, false>(m, lds, all), h);
    const Map behind = strands_before<G, true>(n, lds, all);
    const bool wanted = to == RECUR_TILE && t0 + RECUR_TILE < end && !(lds.tails[RECUR_STRANDS - 1] >> (RECUR_RUN - 1));
    if (CHAINED) chain_say<G, true>(ch, v, all, wanted, col, a.C4, lds);
#pragma unroll
    for (int i = 0; i < RECUR_RUN; ++i) {                      // w = (h[t - 1] - x) a
        const float4 in = widen4(x[i]);
        if (ends && heads >> i & 1) h = row_or_zero(a.h0, lds.head[strand * RECUR_RUN + i], a.C4, col);
        open4(s[i], f, b);
        w[i] = mul4(f, make_float4(h.x - in.x, h.y - in.y, h.z - in.z, h.w - in.w));
        h = fma4(f, h, mul4(b, in));
        forget(s[i]);
        forget(w[i]);
    }
    if (CHAINED) c = chain_state<G, true>(ch, v, wanted, col, a.C4, lds);
    c = apply(behind, c);
    const TileOf dx = tile_of<T>(a.dx, a.dx_stride, t0), dg = tile_of<T>(a.dg, a.dg_stride, t0);
#pragma unroll
    for (int i = RECUR_RUN - 1; i >= 0; --i) {
        if (ends && tails >> i & 1) c = row_or_zero(a.d_last, lds.tail[strand * RECUR_RUN + i], a.C4, col);
        open4(s[i], f, b);
        const float4 lam = plus4(widen4(kept_d[i][threadIdx.x]), c), o = mul4(b, lam);
        c = mul4(f, lam);
        if (full || (mine && i >= lo && i < hi)) {
            store_at<T>(dx, token + i, col, o);
            store_at<T>(dg, token + i, col, mul4(o, w[i]));
            if (ends && a.dh0 && heads >> i & 1) st4(a.dh0 + ((i64)lds.head[strand * RECUR_RUN + i] * a.C4 + col) * 4, c);
        }
    }
}

template <typename T, int G, bool CHAINED>
__global__ void __launch_bounds__(RECUR_STRANDS *G, sizeof(T) == 2 ? 4 : 3) k_recur_grad(RecurArgs a, Chain ch)
{
    __shared__ TileLds<G> lds;
    __shared__ typename Raw4<T>::type kept_d[RECUR_RUN][RECUR_STRANDS * G];   // a thread's own, out of its registers' way until they are used again
    const i64 begin = std::max(0, a.offsets[0]), end = std::min<i64>(a.n, a.offsets[a.n_seq]);
    int k = (int)blockIdx.x;
    if (CHAINED) {
        if (threadIdx.x == 0) lds.tile = (int)atomicAdd(ch.ticket, 1u);
        __syncthreads();
        k = uniform(lds.tile);
        if ((u32)k >= (u32)(ch.tiles * ((a.C4 + G - 1) / G))) return;      // only where another call takes tickets from the same workspace
    }
    k_recur_grad_tile<T, G, CHAINED>(a, ch, k, (a.C4 + G - 1) / G, begin, end, lds, kept_d);
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

// A workgroup to ROWS rows: 64 rows of 256 3.7 us, a launch and three loads that wait for each other.  Whether another row has the slot of one of them is seen by comparing all slots with theirs, a slot to a thread at a time, while the rows and
// states are on their way.  A slot's first row takes those that follow, in order; the others leave it.
template <typename T, int ROWS>
__global__ void __launch_bounds__(BLOCK) k_recur_step(StepArgs a)
{
    __shared__ u32 lds[2];
    const int t = (int)threadIdx.x, total = ROWS * a.C4;
    const i64 row0 = (i64)blockIdx.x * ROWS;
    if (a.slots) {
        int mine[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) mine[r] = row0 + r < a.n ? a.slots[row0 + r] : 0;
        if (t < 2) lds[t] = 0;
        __syncthreads();
        u32 earlier = 0, later = 0;
#pragma unroll 8
        for (int j = t; j < (int)a.n; j += BLOCK) {
            const int s = a.slots[j];
            u32 same = 0;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) same |= s == mine[r] ? 1u << r : 0u;
            const i64 at = j - row0;                           // rows before this one of the workgroup's come after it, and the other way round
            const u32 before = at <= 0 ? 0u : at >= ROWS ? ~0u : (1u << at) - 1u, after = at >= ROWS - 1 ? 0u : at < 0 ? ~0u : ~0u << (at + 1);
            later |= same & before;
            earlier |= same & after;
        }
        earlier = wave_or(earlier);
        later = wave_or(later);
        if (lane_id() == 0 && (earlier | later)) {
            atomicOr(&lds[0], earlier);
            atomicOr(&lds[1], later);
        }
        __syncthreads();
    }
    for (int k = t; k < total; k += BLOCK) {
        const int r = k / a.C4, c = 4 * (k - r * a.C4);
        const i64 i = row0 + r;
        if (i >= a.n) break;
        const i64 slot = a.slots ? a.slots[i] : i;
        if (slot < 0 || slot >= a.n_slots) {
            if (a.status && c == 0) atomicOr(a.status, ST_BAD_ID);
            if (a.out) st4((T *)a.out + i * a.out_stride + c, make_float4(0.f, 0.f, 0.f, 0.f));
            continue;
        }
        if (a.slots && lds[0] >> r & 1) continue;
        const bool more = a.slots && lds[1] >> r & 1;
        float4 h = ld4(a.state + slot * a.state_stride + c);
        for (i64 j = i; j < a.n; ++j) {
            if (j > i && a.slots[j] != slot) continue;
            float4 f, b;
            gate4(ld4((const T *)a.gate + j * a.g_stride + c), f, b);
            h = fma4(f, h, mul4(b, ld4((const T *)a.x + j * a.x_stride + c)));
            if (a.out) put4((T *)a.out + j * a.out_stride + c, h);
            if (!more) break;
        }
        st4(a.state + slot * a.state_stride + c, h);
    }
}

#define RECUR_LEAST_GROUP 32
// bytes of the chain's words, or, with an address, the chain there and what of it has to be zero
size_t recur_carve(i64 n, int dim, char *ws, Chain *ch)
{
    const i64 tiles = std::max<i64>(1, (n + RECUR_TILE - 1) / RECUR_TILE), groups = (tiles + RECUR_LEAST_GROUP - 1) / RECUR_LEAST_GROUP;
    if (ch) {
        ch->ticket = (u32 *)ws;
        ch->lost = ch->ticket + 1;
        ch->maps = (u64 *)(ws + 256);
        ch->states = ch->maps + (size_t)tiles * dim;
        ch->tiles = (int)tiles;
        ch->group = RECUR_LEAST_GROUP;
    }
    return 256 + layer_up256(8 * (size_t)(tiles + groups) * (size_t)dim);
}

template <typename T, int G, bool GRAD>
int launch_recur(const RecurArgs &a, void *workspace, hipStream_t st)
{
    Chain ch;
    const size_t bytes = recur_carve(a.n, 4 * a.C4, (char *)workspace, &ch);
    const int sides = (a.C4 + G - 1) / G;
    // Larger groups hand the state on less often, and read more maps to every tile of them: 131 072 tokens in one sequence, forward, groups of 16 / 32 / 64: 32 channels 53 / 36 / 28 us,
    // 64 61 / 44 / 36, 128 65 / 55 / 54, 256 82 / 80 / 82; 262 144 tokens of 512 257 / 259 / 266.
    if (sides <= 2) ch.group = 2 * RECUR_LEAST_GROUP;
    if ((i64)ch.tiles * sides > (i64)TN_MAX_BLOCKS * BLOCK / (RECUR_STRANDS * G)) return tn_fail(TENSAIR_EINVAL, "n * dim beyond what one launch covers");
    const dim3 blk(RECUR_STRANDS * G);
    if (ch.tiles == 1) {
        if constexpr (GRAD) hipLaunchKernelGGL((k_recur_grad<T, G, false>), dim3(sides), blk, 0, st, a, ch);
        else hipLaunchKernelGGL((k_recur<T, G, false>), dim3(sides), blk, 0, st, a, ch);
        return TENSAIR_OK;
    }
    hipLaunchKernelGGL(k_recur_clear, dim3((unsigned)std::min<size_t>(1024, (bytes / 8 + BLOCK - 1) / BLOCK)), dim3(BLOCK), 0, st, (u64 *)workspace, bytes / 8);
    const dim3 grid((unsigned)(ch.tiles * sides));
    if constexpr (GRAD) hipLaunchKernelGGL((k_recur_grad<T, G, true>), grid, blk, 0, st, a, ch);
    else hipLaunchKernelGGL((k_recur<T, G, true>), grid, blk, 0, st, a, ch);
    return TENSAIR_OK;
}
// Lanes to a token: a line of memory for fp32, and for bfloat16 forward; half a line for the gradient in bfloat16, which keeps more than a workgroup of 512 threads has registers for
// (262 144 tokens of 512: forward with a line 270 us, with half of one 290; gradient 460 and 413; the halves' workgroups on one die, by their order: no difference).
int launch_recur(const RecurArgs &a, int32_t dtype, bool grad, void *workspace, hipStream_t st)
{
    if (dtype == TENSAIR_F32) return grad ? launch_recur<float, 8, true>(a, workspace, st) : launch_recur<float, 8, false>(a, workspace, st);
    if (grad) return launch_recur<bf16_t, 8, true>(a, workspace, st);
    return a.C4 <= 8 ? launch_recur<bf16_t, 8, false>(a, workspace, st) : launch_recur<bf16_t, 16, false>(a, workspace, st);
}

// a tile's places are kept in 32 bits
int recur_matrix(const void *p, i64 rows, i64 stride, int32_t dim, int32_t dtype, const char *what)
{
    if (stride > TENSAIR_MAX_RECUR_STRIDE) return tn_fail(TENSAIR_EINVAL, "%s: the row stride must be at most TENSAIR_MAX_RECUR_STRIDE", what);
    return layer_matrix(p, rows, stride, dim, dtype, what);
}

int check_recur(const void *x, i64 x_stride, const void *gate, i64 gate_stride, int32_t dtype, i64 n, int32_t dim, const int32_t *offsets, i64 n_seq,
                const void *workspace, size_t workspace_bytes, const int32_t *status)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = recur_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = recur_matrix(gate, n, gate_stride, dim, dtype, "gate"))) return rc;
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
    if ((rc = recur_matrix(out, n, out_stride, dim, dtype, "out"))) return rc;
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
    if ((rc = launch_recur(a, dtype, false, workspace, st))) return rc;
    return layer_launched("recur");
}

int tensair_recur_grad(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *offsets,
                       int64_t n_seq, const float *h0, const float *states, const void *d_out, int64_t d_stride, const float *d_last, void *d_x,
                       int64_t d_x_stride, void *d_gate, int64_t d_gate_stride, float *d_h0, void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_recur(x, x_stride, gate, gate_stride, dtype, n, dim, offsets, n_seq, workspace, workspace_bytes, status))) return rc;
    if ((rc = recur_matrix(d_out, n, d_stride, dim, dtype, "d_out")) || (rc = recur_matrix(d_x, n, d_x_stride, dim, dtype, "d_x")) ||
        (rc = recur_matrix(d_gate, n, d_gate_stride, dim, dtype, "d_gate")))
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
    if ((rc = launch_recur(a, dtype, true, workspace, st))) return rc;
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
    // few rows to a workgroup where there are few rows, so that each has one chunk of them to a thread; more of them share the look through the slots, which is all that counts where rows are
    // many (4 096 rows of 32 8 us with slots and 7 without, 16 384 of 256 36 and 8, 65 536 of 32 412 and 8)
    const int rows = n <= 4096 ? 4 : 16;
    const u64 blocks = ((u64)n + rows - 1) / rows;
    if (blocks > TN_MAX_BLOCKS) return tn_fail(TENSAIR_EINVAL, "n beyond what one launch covers");
    const dim3 grid((unsigned)blocks), blk(BLOCK);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == TENSAIR_F32 && rows == 4) hipLaunchKernelGGL((k_recur_step<float, 4>), grid, blk, 0, st, a);
    else if (dtype == TENSAIR_F32) hipLaunchKernelGGL((k_recur_step<float, 16>), grid, blk, 0, st, a);
    else if (rows == 4) hipLaunchKernelGGL((k_recur_step<bf16_t, 4>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_recur_step<bf16_t, 16>), grid, blk, 0, st, a);
    return layer_launched("recur_step");
}

}  // extern "C"
