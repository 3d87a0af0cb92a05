// A table as the input layer of a model: rows looked up and scaled, and the gradient of that by sorted tokens.
//   out[i] = scale * table[ids[i]]                        tensair_embed
//   G[r]   = scale * sum over i with ids[i] = r of d[i]   tensair_embed_grad (rows of a sparse gradient), _dense (a table)
// The sums are taken in fp32 in an order that is a function of the ids alone, without atomics on values.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "../../include/tensair.h"
#include "dev_common.h"
#include "kernels.h"
#include "prep_dev.h"

namespace {

// ---------------------------------------------------------------- lookup
struct EmbedArgs {
    const void *table;
    const int *ids;
    void *out;
    i64 n, V, stride, out_stride;
    int C4;            // chunks of 4 elements of a row
    u32 magic;         // x / C4 = (x * magic) >> 32 for x < C4 + 1024; 0 where C4 = 1
    float scale;
    int *status;
};

#define EMBED_CHUNKS 4
// The outputs are taken as one list of chunks of 4 elements, so that rows of any length fill the waves; a thread takes one
// chunk of every 256 of its workgroup's 1024, the ids and then the rows of all of them in flight at once.  The way to memory bounds it:
// 16 384 words of 512 from bfloat16 to fp32 8 us (50 MB, 6 TB/s), 64 words the time of a launch.
template <typename T, typename TO>
__global__ void __launch_bounds__(BLOCK) k_embed(EmbedArgs a)
{
    const u64 base = (u64)blockIdx.x * (BLOCK * EMBED_CHUNKS);
    const u64 row0 = base / (u32)a.C4;
    const u32 first = (u32)(base - row0 * (u32)a.C4);
    int id[EMBED_CHUNKS];
    u32 col[EMBED_CHUNKS];
    i64 row[EMBED_CHUNKS];
#pragma unroll
    for (int j = 0; j < EMBED_CHUNKS; ++j) {
        const u32 x = first + (u32)j * BLOCK + threadIdx.x;
        const u32 q = a.magic ? (u32)(((u64)x * a.magic) >> 32) : x;
        col[j] = x - q * (u32)a.C4;
        row[j] = (i64)(row0 + q);
        id[j] = row[j] < a.n ? a.ids[row[j]] : -1;
    }
    typename Raw4<T>::type v[EMBED_CHUNKS];
#pragma unroll
    for (int j = 0; j < EMBED_CHUNKS; ++j) {
        zero_raw(v[j]);
        if ((u32)id[j] < (u64)a.V) v[j] = ldraw((const T *)a.table + (i64)id[j] * a.stride + 4 * col[j]);
    }
#pragma unroll
    for (int j = 0; j < EMBED_CHUNKS; ++j) {
        if (row[j] >= a.n) continue;
        if ((u32)id[j] >= (u64)a.V && col[j] == 0 && a.status) atomicOr(a.status, ST_BAD_ID);
        float4 w = widen4(v[j]);
        w.x *= a.scale;
        w.y *= a.scale;
        w.z *= a.scale;
        w.w *= a.scale;
        st4((TO *)a.out + row[j] * a.out_stride + 4 * col[j], w);
    }
}

// ---------------------------------------------------------------- gradient
// Where a row's sum goes.
struct RowsOut {
    void *rows;
    i64 stride;
    int by_id;         // a row of a table (at its id) or of a sparse gradient (at its place among the touched ones)
    int dtype, add;
    float scale;
};

struct EmbedGradArgs {
    const int *ids;
    const void *d;     // [n][d_stride]
    i64 d_stride, V;
    int n, C4;
    RowsOut out;
    int *row_ids, *n_rows;       // of the sparse gradient (a table: row_ids in the workspace, n_rows NULL)
    int *status;
    // in the workspace
    u32 *first;                  // few tokens: the id where a token is its word's first, else ~0
    u32 *keys, *vals;            // sorted
    int *seg_of, *seg_start;
    int *valid;                  // [1] tokens whose ids are in range: they come first in the sorted order
    float *part;                 // [tiles][2][4 * C4]
    int *long_n, *long_list;     // rows that cross a border of tiles, by the tile that they begin in
    int tile;                    // tokens to a tile, a power of two
    float *blocks;               // [tiles / EMBED_BLOCK][4 * C4] shares of a row that has all of a block's tiles (NULL: few tiles)
};

__device__ __forceinline__ void add4(float4 &a, float4 b)
{
    a.x += b.x;
    a.y += b.y;
    a.z += b.z;
    a.w += b.w;
}
// `old`: what is there, where the row is added to it and that was read before
__device__ __forceinline__ void put_row_chunk(const RowsOut &o, i64 at, int chunk, float4 v, const float4 *old = nullptr)
{
    v.x *= o.scale;
    v.y *= o.scale;
    v.z *= o.scale;
    v.w *= o.scale;
    at = at * o.stride + 4 * chunk;
    if (old) add4(v, *old);
    if (o.dtype == TENSAIR_F32) {
        if (o.add && !old) add4(v, ld4((const float *)o.rows + at));
        st4((float *)o.rows + at, v);
    } else {
        if (o.add && !old) add4(v, ld4((const bf16_t *)o.rows + at));
        st4((bf16_t *)o.rows + at, v);
    }
}

// ---- few tokens: no sort.  Every token looks through all ids; the first of its word sums the word's tokens.  Two launches
// that wait for memory a few times each are what it takes: 1 024 tokens of 128 10 us.  (Rows of 300: 2 048 tokens 24 us, by the seven
// launches of the sort 33; 4 096 tokens 44 and 42, the gaps between the launches not counted.)
#define EMBED_FEW 4096
// marks the tokens that are their words' first, so that the next launch can count the words below a word
__global__ void __launch_bounds__(BLOCK) k_embed_first(EmbedGradArgs a)
{
    const int lane = lane_id();
    const int i = (int)blockIdx.x * WAVES_PER_BLOCK + uniform((int)(threadIdx.x >> 6));
    if (i >= a.n) return;
    const int id = a.ids[i];
    bool ok = (u32)id < (u64)a.V;
    if (!ok && lane == 0 && a.status) atomicOr(a.status, ST_BAD_ID);
    bool seen = false;
    for (int j = lane; j < i; j += WAVE) seen |= a.ids[j] == id;
    if (__ballot(seen)) ok = false;
    if (lane == 0) a.first[i] = ok ? (u32)id : ~0u;
}

// A workgroup per token: G lanes to a row, BLOCK / G shares of the word's tokens, each in order, added up in order.
template <typename T, int G, int ITERS>
__global__ void __launch_bounds__(BLOCK) k_embed_few(EmbedGradArgs a)
{
    constexpr int SHARES = BLOCK / G;
    __shared__ unsigned short list[EMBED_FEW];
    __shared__ int counts[3][WAVES_PER_BLOCK];
    __shared__ float4 sums[SHARES > 1 ? (SHARES - 1) * G * ITERS : 1];
    const int i = (int)blockIdx.x, t = (int)threadIdx.x, lane = lane_id(), wave = t >> 6;
    const int id = a.ids[i];
    const bool sparse = a.n_rows != nullptr;
    if ((u32)id >= (u64)a.V && !sparse && t == 0 && a.status) atomicOr(a.status, ST_BAD_ID);
    if (sparse ? a.first[i] == ~0u && i > 0 : (u32)id >= (u64)a.V) return;      // the first workgroup counts the rows
    // the word's tokens, in order; the words below it; all words
    int below = 0, all = 0, found = 0;
    for (int base = 0; base < a.n; base += BLOCK) {
        const int j = base + t;
        const bool in = j < a.n, same = in && a.ids[j] == id;
        if (sparse) {
            const u32 f = in ? a.first[j] : ~0u;
            below += f < (u32)id ? 1 : 0;
            all += f != ~0u ? 1 : 0;
        } else if (same && j < i) {
            below = 1;                                                          // another token is the first
        }
        const u64 b = __ballot(same);
        __syncthreads();
        if (lane == 0) counts[0][wave] = (int)__popcll(b);
        __syncthreads();
        int at = found;
#pragma unroll
        for (int w = 0; w < WAVES_PER_BLOCK; ++w) {
            if (w < wave) at += counts[0][w];
            found += counts[0][w];
        }
        if (same) list[at + (int)__popcll(b & ((1ull << lane) - 1ull))] = (unsigned short)j;
    }
    below = (int)wave_sum((float)below);                                        // at most EMBED_FEW: exact
    all = (int)wave_sum((float)all);
    if (lane == 0) {
        counts[1][wave] = below;
        counts[2][wave] = all;
    }
    __syncthreads();
    below = all = 0;
#pragma unroll
    for (int w = 0; w < WAVES_PER_BLOCK; ++w) {
        below += counts[1][w];
        all += counts[2][w];
    }
    if (sparse) {
        if (i == 0 && t == 0) *a.n_rows = all;
        if (a.first[i] == ~0u) return;
        if (t == 0) a.row_ids[below] = id;
    } else if (below) {
        return;
    }
    const int share = t / G, l = t % G;
    const int per = (found + SHARES - 1) / SHARES, lo = share * per, hi = min(found, lo + per);
    float4 acc[ITERS];
    zero_row<ITERS>(acc);
    for (int e = lo; e < hi; e += 4) {
        typename Raw4<T>::type r[4][ITERS];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            zero_row_raw<ITERS>(r[k]);
            if (e + k < hi) {
                const T *row = (const T *)a.d + (i64)list[e + k] * a.d_stride;
#pragma unroll
                for (int it = 0; it < ITERS; ++it)
                    if (l + G * it < a.C4) r[k][it] = ldraw(row + 4 * (l + G * it));
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (e + k < hi) add_row_raw<ITERS>(acc, r[k]);
    }
    if (share > 0)
#pragma unroll
        for (int it = 0; it < ITERS; ++it) sums[((share - 1) * ITERS + it) * G + l] = acc[it];
    __syncthreads();
    if (share > 0) return;
    const int used = per > 0 ? (found + per - 1) / per : 0;
    for (int s = 1; s < used; ++s)
#pragma unroll
        for (int it = 0; it < ITERS; ++it) add4(acc[it], sums[((s - 1) * ITERS + it) * G + l]);
    const i64 at = a.out.by_id ? (i64)id : (i64)below;
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
        if (l + G * it < a.C4) put_row_chunk(a.out, at, l + G * it, acc[it]);
}

// ---- many tokens: sorted by id (the passes of the mini-batch's sort), tiles of the sorted tokens summed, rows that cross tiles
// put together.  The launches up to the sums are short and wait for one another (32 767 tokens of a million words: keys 7 us, three
// passes of the sort 8 each, rows 6; 262 143 tokens of 10 000: 8, two of 12, 7.5).
struct EmbedKeys {
    const int *ids;
    u32 *keys;
    u32 *hist;          // [passes][2^bits], zero before (NULL: counted passes)
    i64 V;
    int n, passes, bits;
    int *status;
};
#define EMBED_KEYS_TILE 2048
// Keys: the ids, an id out of range as V, which sorts behind all others.
__global__ void __launch_bounds__(BLOCK) k_embed_keys(EmbedKeys a)
{
    __shared__ u32 lds[TN_RADIX_MAX_PASSES_ND + TN_RADIX_MAX_ND];
    const int nd = 1 << a.bits;
    if (a.hist)
        for (int i = threadIdx.x; i < a.passes * nd; i += BLOCK) lds[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EMBED_KEYS_TILE / BLOCK; ++j) {
        const i64 i = (i64)blockIdx.x * EMBED_KEYS_TILE + j * BLOCK + threadIdx.x;
        if (i >= a.n) break;
        u32 k = (u32)a.ids[i];
        if ((u64)k >= (u64)a.V) {
            k = (u32)a.V;
            if (a.status) atomicOr(a.status, ST_BAD_ID);
        }
        a.keys[i] = k;
        if (a.hist)
            for (int p = 0; p < a.passes; ++p) atomicAdd(&lds[p * nd + ((k >> (p * a.bits)) & (u32)(nd - 1))], 1u);
    }
    if (!a.hist) return;
    __syncthreads();
    for (int i = threadIdx.x; i < a.passes * nd; i += BLOCK)
        if (lds[i]) atomicAdd(&a.hist[i], lds[i]);
}

// Rows of the sorted keys: the row of every token, the first token of every row, the rows' ids and number.  Chained: by the
// published scan; else k_embed_segments<.., true> counts per tile in a launch of its own.
template <bool CHAINED, bool HEADS>
__global__ void __launch_bounds__(BLOCK) k_embed_segments(EmbedGradArgs a, u64 *state, u32 *ticket)
{
    constexpr int IPT = TN_SCAN_TILE / BLOCK;
    __shared__ u32 word, sm[WAVES_PER_BLOCK], lower;
    const int lane = lane_id(), wave = uniform((int)(threadIdx.x >> 6));
    const int tile = CHAINED ? take_ticket(ticket, &word) : (int)blockIdx.x;
    if (tile == 0 && threadIdx.x == 0 && !HEADS) *a.long_n = 0;
    const i64 wbase = (i64)tile * TN_SCAN_TILE + wave * (IPT * WAVE);
    const u32 V = (u32)a.V;
    u32 key[IPT];
    u64 head[IPT];
#pragma unroll
    for (int it = 0; it < IPT; ++it) {
        const i64 i = wbase + it * WAVE + lane;
        key[it] = i < a.n ? a.keys[i] : V;
    }
    u32 last = (wbase > 0 && wbase <= a.n) ? a.keys[wbase - 1] : ~0u, heads = 0;
#pragma unroll
    for (int it = 0; it < IPT; ++it) {
        const u32 up = (u32)__shfl_up((int)key[it], 1, WAVE);
        head[it] = __ballot(key[it] < V && key[it] != (lane == 0 ? last : up));
        last = (u32)rd_lane((int)key[it], WAVE - 1);
        heads += (u32)__popcll(head[it]);
    }
    if (lane == 0) sm[wave] = heads;
    __syncthreads();
    u32 mine = 0, before = 0;
#pragma unroll
    for (int w = 0; w < WAVES_PER_BLOCK; ++w) {
        if (w < wave) before += sm[w];
        mine += sm[w];
    }
    if constexpr (HEADS) {
        if (threadIdx.x == 0) state[tile] = mine;
        return;
    }
    if (wave == 0) {
        u64 below = 0;
        if (CHAINED) {
            if (tile > 0) {
                if (lane == 0) post(state + tile, PREP_SEG_OWN | (u64)mine);
                below = prep_below(state, tile, lane);
            }
            if (lane == 0) post(state + tile, PREP_SEG_INCL | (below + mine));
        } else {
#pragma unroll 8
            for (int t = lane; t < tile; t += WAVE) below += state[t];
            below = wave_sum64(below);
        }
        if (lane == 0) lower = (u32)below;
    }
    __syncthreads();
    u32 rows = lower + before;
    const u64 upto = (lane == 63) ? ~0ull : ((2ull << lane) - 1ull);
#pragma unroll
    for (int it = 0; it < IPT; ++it) {
        const i64 i = wbase + it * WAVE + lane;
        const int seg = (int)(rows + (u32)__popcll(head[it] & upto)) - 1;
        if (i < a.n) {
            const bool ok = key[it] < V;
            if (ok) a.seg_of[i] = seg;
            if ((head[it] >> lane) & 1ull) {
                a.seg_start[seg] = (int)i;
                a.row_ids[seg] = (int)key[it];
            }
            // the last token in range ends the last row
            const bool end = i == a.n - 1 || a.keys[i + 1] >= V;
            if (ok && end) {
                a.seg_start[seg + 1] = (int)i + 1;
                *a.valid = (int)i + 1;
                if (a.n_rows) *a.n_rows = seg + 1;
            }
            if (!ok && i == 0) {
                *a.valid = 0;
                if (a.n_rows) *a.n_rows = 0;
            }
        }
        rows += (u32)__popcll(head[it]);
    }
}

#define EMBED_MAX_TILE 64
// G lanes sum a tile of sorted tokens, row by row; a row that neither begins before the tile nor goes on behind it
// is written, of another the tile's share is kept: slot 0 where the row began before, else slot 1.  ADD: what a row of the table holds is
// read beside the tokens' rows, not when its sum is done.
// What bounds it is the way to rows in random order: 262 143 rows of 256 in bfloat16 27.5 us (4.9 TB/s), 32 767 rows of 300 in fp32 added
// to a table 18 us (39 MB read, 9 840 rows read and written).
template <typename T, int G, int ITERS, bool ADD>
__global__ void __launch_bounds__(BLOCK) k_embed_reduce(EmbedGradArgs a)
{
    constexpr int FLIGHT = ITERS > (ADD ? 1 : 2) ? 4 : 8, SIDE = WAVE / G;
    // the places and rows of a wave's tokens, which follow one another, and where the rows go
    __shared__ int2 entries[WAVES_PER_BLOCK][SIDE * EMBED_MAX_TILE];
    __shared__ int targets[WAVES_PER_BLOCK][SIDE * EMBED_MAX_TILE];
    const int l = (int)threadIdx.x % G, valid = *a.valid, wave = (int)threadIdx.x / WAVE;
    const i64 tile = ((i64)blockIdx.x * BLOCK + threadIdx.x) / G, wave0 = (tile - lane_id() / G) * a.tile;
    const int here = (int)min((i64)SIDE * a.tile, valid - wave0);
    for (int x = lane_id(); x < here; x += WAVE) {
        const int seg = a.seg_of[wave0 + x];
        entries[wave][x] = make_int2((int)a.vals[wave0 + x], seg);
        targets[wave][x] = a.out.by_id ? (int)a.keys[wave0 + x] : seg;
    }
    __syncthreads();
    if (tile * a.tile >= valid) return;
    const int base = (int)(tile * a.tile), end = min(valid, base + a.tile);
    const int2 *mine = entries[wave] + (base - wave0);
    const int *to = targets[wave] + (base - wave0);
    const int first = mine[0].y, next = end < valid ? a.seg_of[end] : -1;
    bool before = base > 0 && a.seg_of[base - 1] == first, open = false;
    const bool began = before;
    float4 acc[ITERS];
    zero_row<ITERS>(acc);
    for (int e = base; e < end; e += FLIGHT) {
        bool ends[FLIGHT];                                        // tokens that are their rows' last
        typename Raw4<T>::type r[FLIGHT][ITERS];
        float4 old[ADD ? FLIGHT : 1][ITERS];
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            zero_row_raw<ITERS>(r[k]);
            ends[k] = false;
            if (e + k < end) {
                const int2 x = mine[e + k - base];
                ends[k] = (e + k + 1 < end ? mine[e + k + 1 - base].y : next) != x.y;
                const T *row = (const T *)a.d + (i64)(u32)x.x * a.d_stride;
#pragma unroll
                for (int it = 0; it < ITERS; ++it)
                    if (l + G * it < a.C4) r[k][it] = ldraw(row + 4 * (l + G * it));
                if (ADD && ends[k] && !(began && x.y == first)) {
                    const i64 at = to[e + k - base] * a.out.stride + 4 * l;
#pragma unroll
                    for (int it = 0; it < ITERS; ++it)
                        if (l + G * it < a.C4)
                            old[k][it] = a.out.dtype == TENSAIR_F32 ? ld4((const float *)a.out.rows + at + 4 * G * it) : ld4((const bf16_t *)a.out.rows + at + 4 * G * it);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            add_row_raw<ITERS>(acc, r[k]);                        // zero behind the tile's end
            open |= e + k < end;
            if (ends[k]) {
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int c = l + G * it;
                    if (c < a.C4) {
                        if (before) st4(a.part + ((2 * tile) * a.C4 + c) * 4, acc[it]);
                        else put_row_chunk(a.out, to[e + k - base], c, acc[it], ADD ? &old[k][it] : nullptr);
                    }
                }
                zero_row<ITERS>(acc);
                before = open = false;
            }
        }
    }
    if (!open) return;                                            // the last row goes on behind the tile
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int c = l + G * it;
        if (c < a.C4) st4(a.part + ((2 * tile + (before ? 0 : 1)) * a.C4 + c) * 4, acc[it]);
    }
    if (!before && l == 0) a.long_list[atomicAdd(a.long_n, 1)] = (int)tile;
}

#define EMBED_BLOCK 32            // of tiles (32 767 tokens added to a table of 300: k_embed_join 9.3 us, 14 with 64)
#define EMBED_BLOCK_MIN 1024      // tiles from which on adding up whole blocks of them is worth a launch
// adds up what at() gives for every share, in THREADS / G parts of shares that follow one another (the same for every thread of the
// workgroup); true for the threads that have the sum
template <int G, int ITERS, int THREADS, typename F>
__device__ __forceinline__ bool sum_shares(float4 (&acc)[ITERS], int shares, int C4, float4 *sums, F at)
{
    constexpr int PARTS = THREADS / G, FLIGHT = ITERS > 2 ? 4 : 8;
    const int l = (int)threadIdx.x % G, part = (int)threadIdx.x / G;
    const int per = (shares + PARTS - 1) / PARTS, lo = part * per, hi = min(shares, lo + per);
    zero_row<ITERS>(acc);
    for (int e = lo; e < hi; e += FLIGHT) {
        float4 r[FLIGHT][ITERS];
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k)
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int c = l + G * it;
                r[k][it] = e + k < hi && c < C4 ? ld4(at(e + k) + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k)
            if (e + k < hi) add_row<ITERS>(acc, r[k]);
    }
    if (part > 0)
#pragma unroll
        for (int it = 0; it < ITERS; ++it) sums[((part - 1) * ITERS + it) * G + l] = acc[it];
    __syncthreads();
    if (part == 0) {
        const int used = (shares + per - 1) / per;
        for (int s = 1; s < used; ++s)
#pragma unroll
            for (int it = 0; it < ITERS; ++it) add4(acc[it], sums[((s - 1) * ITERS + it) * G + l]);
    }
    __syncthreads();
    return part == 0;
}
// A block of EMBED_BLOCK tiles that one row has all of, having begun before: their shares summed.  (A word that is a third of
// 262 143 tokens: 2 700 shares, by one workgroup of k_embed_join alone 35 us.)
template <int G, int ITERS>
__global__ void __launch_bounds__(BLOCK) k_embed_blocks(EmbedGradArgs a)
{
    __shared__ float4 sums[(BLOCK / G > 1 ? BLOCK / G - 1 : 1) * G * ITERS];
    const i64 tile = (i64)blockIdx.x * EMBED_BLOCK;
    const int valid = *a.valid;
    if ((tile + EMBED_BLOCK) * a.tile > valid) return;
    const int seg = a.seg_of[tile * a.tile];
    if (a.seg_start[seg] >= tile * a.tile || a.seg_start[seg + 1] < (tile + EMBED_BLOCK) * a.tile) return;
    float4 acc[ITERS];
    if (!sum_shares<G, ITERS, BLOCK>(acc, EMBED_BLOCK, a.C4, sums, [&](int e) -> const float * { return a.part + 2 * (tile + e) * a.C4 * 4; })) return;
    const int l = (int)threadIdx.x % G;
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
        if (l + G * it < a.C4) st4(a.blocks + ((i64)blockIdx.x * a.C4 + l + G * it) * 4, acc[it]);
}
// A row that crosses tiles: its shares are those of the tiles up to a border of blocks, whole blocks, the tiles behind them.
struct LongRow {
    i64 tile, first_block, end_block;
    int seg, head, blocks, tail;
    __device__ __forceinline__ LongRow(const EmbedGradArgs &a, int x)
    {
        tile = a.long_list[x];
        seg = a.seg_of[tile * a.tile + a.tile - 1];                             // its first tile's last token's: it goes on behind it
        const i64 end = (i64)a.seg_start[seg + 1], last = (end - 1) / a.tile;
        first_block = tile / EMBED_BLOCK + 1;
        end_block = end / ((i64)a.tile * EMBED_BLOCK);
        blocks = a.blocks && end_block > first_block ? (int)(end_block - first_block) : 0;
        head = blocks ? (int)(first_block * EMBED_BLOCK - tile) : (int)(last - tile) + 1;
        tail = blocks ? (int)(last + 1 - end_block * EMBED_BLOCK) : 0;
    }
    __device__ __forceinline__ int shares() const { return head + blocks + tail; }
    __device__ __forceinline__ const float *at(const EmbedGradArgs &a, int e) const
    {
        if (e < head) return a.part + (2 * (tile + e) + (e == 0 ? 1 : 0)) * a.C4 * 4;
        if (e < head + blocks) return a.blocks + (first_block + e - head) * a.C4 * 4;
        return a.part + 2 * (end_block * EMBED_BLOCK + e - head - blocks) * a.C4 * 4;
    }
    template <int G, int ITERS>
    __device__ __forceinline__ void put(const EmbedGradArgs &a, const float4 (&acc)[ITERS], int l) const
    {
        const i64 to = a.out.by_id ? (i64)a.row_ids[seg] : (i64)seg;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (l + G * it < a.C4) put_row_chunk(a.out, to, l + G * it, acc[it]);
    }
};
// A workgroup per row that crosses tiles (9 us both for 32 767 tokens of 300, a word an eighth of them, and for 262 143 of 256).
template <int G, int ITERS>
__global__ void __launch_bounds__(BLOCK) k_embed_join(EmbedGradArgs a)
{
    __shared__ float4 sums[(BLOCK / G > 1 ? BLOCK / G - 1 : 1) * G * ITERS];
    const int rows = *a.long_n;
    for (int x = (int)blockIdx.x; x < rows; x += (int)gridDim.x) {
        const LongRow row(a, x);
        float4 acc[ITERS];
        if (sum_shares<G, ITERS, BLOCK>(acc, row.shares(), a.C4, sums, [&](int e) { return row.at(a, e); }))
            row.template put<G, ITERS>(a, acc, (int)threadIdx.x % G);
    }
}

// zero in a table, its padding left alone
template <typename T>
__global__ void __launch_bounds__(BLOCK) k_embed_zero(T *rows, i64 V, i64 stride, int C4)
{
    const i64 all = V * C4, step = (i64)gridDim.x * BLOCK;
    for (i64 c = (i64)blockIdx.x * BLOCK + threadIdx.x; c < all; c += step) {
        const i64 r = c / C4;
        st4(rows + r * stride + 4 * (c - r * C4), make_float4(0.f, 0.f, 0.f, 0.f));
    }
}

// ---------------------------------------------------------------- host
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct EmbedSizes {
    bool few, chained;
    int passes, bits, tiles, seg_tiles, sum_tiles, tile;
    size_t nd, pub, clear, tile0, per_pass, seg_state, hist, none;     // words of the published area
};
// Most tokens that are summed in tiles of so many: few to a tile where there are few, so that enough waves are there to hide the way to
// memory, but more tiles have more shares to write and to read again.  Whole calls, rows of 300 added to a table / of 64 in fp32 / of 256 in
// bfloat16, us: 12 000 tokens by tiles of 4 58 / 42 / 44, of 8 57 / 40 / 42, of 16 58 / 38 / 47; 24 000 of 8 64 / 44 / 45, of 16 64 / 43 / 45, of 32
// 70 / 43 / 53; 65 536 of 16 82 / 51 / 53, of 32 83 / 51 / 55; 100 000 94 / 59 / 60, 94 / 56 / 60; 131 072 108 / 65 / 65, 104 / 60 / 62; 400 000 of 32
// 240 / 97 / 100, of 64 238 / 88 / 100; 200 000 133 / 69 / 74, 142 / 71 / 76.
i64 most_in_tiles(int tile) { return (i64)(tile < 16 ? 2048 : tile < 32 ? 6144 : 16384) * tile + tile - 1; }
EmbedSizes embed_sizes(i64 V, i64 n)
{
    EmbedSizes s;
    memset(&s, 0, sizeof(s));
    s.few = n <= EMBED_FEW;
    int key_bits = 1;
    while (key_bits < 31 && (V >> key_bits) > 0) ++key_bits;     // keys 0..V
    tn_radix_shape(key_bits, &s.passes, &s.bits);
    s.nd = (size_t)1 << s.bits;
    s.tiles = tn_prep_tiles(n);
    s.seg_tiles = tn_prep_seg_tiles(n);
    s.tile = 4;
    while (s.tile < EMBED_MAX_TILE && n > most_in_tiles(s.tile)) s.tile *= 2;
    s.sum_tiles = (int)((n + s.tile - 1) / s.tile);
    s.chained = s.tiles <= TN_PREP_CHAIN_OWN;
    // tickets (a word per pass and one of the segments), the segments' words, digit counts, the tiles' words of each pass
    s.seg_state = 8;
    s.hist = s.seg_state + 2 * (size_t)s.seg_tiles;
    s.tile0 = s.hist + s.passes * s.nd * (s.chained ? 1 : (size_t)tn_prep_groups(s.tiles) + 1);
    s.per_pass = s.chained ? s.tiles * s.nd : 0;
    s.none = s.tile0 + (s.chained ? s.passes : 1) * s.tiles * s.nd;     // the digit counts of the second list, which is empty
    s.pub = s.none + s.nd;
    s.clear = s.chained ? s.pub : s.tile0;
    return s;
}
// carves the workspace; returns its size
size_t embed_carve(const EmbedSizes &s, i64 V, i64 n, int dim, char *base, EmbedGradArgs *a, u32 **keys, u32 **vals, u32 **pub)
{
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = base ? base + at : nullptr;
        at += up256(bytes);
        return p;
    };
    const size_t rows = (size_t)std::min<i64>(V, n) + 2;
    char *ids = take(4 * rows);
    char *first = take(4 * (size_t)(s.few ? n : 0));
    if (a) {
        a->row_ids = (int *)ids;
        a->first = (u32 *)first;
    }
    if (s.few) return at;
    const size_t N = (size_t)n;
    for (int k = 0; k < 2; ++k) {
        char *p = take(4 * N), *q = take(4 * N);
        if (keys) keys[k] = (u32 *)p;
        if (vals) vals[k] = (u32 *)q;
    }
    char *seg_of = take(4 * N), *seg_start = take(4 * rows), *flags = take(256), *list = take(4 * (size_t)s.sum_tiles);
    char *part = take((size_t)s.sum_tiles * 2 * dim * 4), *words = take(4 * s.pub);
    const bool many = s.sum_tiles > EMBED_BLOCK_MIN;
    char *blocks = take(many ? ((size_t)s.sum_tiles / EMBED_BLOCK + 1) * dim * 4 : 0);
    if (a) {
        a->seg_of = (int *)seg_of;
        a->seg_start = (int *)seg_start;
        a->valid = (int *)flags;
        a->long_n = (int *)flags + 1;
        a->long_list = (int *)list;
        a->part = (float *)part;
        a->tile = s.tile;
        a->blocks = many ? (float *)blocks : nullptr;
    }
    if (pub) *pub = (u32 *)words;
    return at;
}

template <typename T, int G, int ITERS>
void launch_sums(const EmbedGradArgs &a, const EmbedSizes &s, hipStream_t st)
{
    if (s.few) {
        hipLaunchKernelGGL((k_embed_few<T, G, ITERS>), dim3(a.n), dim3(BLOCK), 0, st, a);
        return;
    }
    const i64 blocks = ((i64)s.sum_tiles * G + BLOCK - 1) / BLOCK;
    if (a.out.add) hipLaunchKernelGGL((k_embed_reduce<T, G, ITERS, true>), dim3((unsigned)blocks), dim3(BLOCK), 0, st, a);
    else hipLaunchKernelGGL((k_embed_reduce<T, G, ITERS, false>), dim3((unsigned)blocks), dim3(BLOCK), 0, st, a);
    if (a.blocks && s.sum_tiles / EMBED_BLOCK > 0)
        hipLaunchKernelGGL((k_embed_blocks<G, ITERS>), dim3((unsigned)(s.sum_tiles / EMBED_BLOCK)), dim3(BLOCK), 0, st, a);
    if (s.sum_tiles > 1)
        hipLaunchKernelGGL((k_embed_join<G, ITERS>), dim3((unsigned)std::min(s.sum_tiles, 4096)), dim3(BLOCK), 0, st, a);
}
// G lanes to a row: the fewest of 8, 16, 32, 64 that hold it in one chunk a lane; then several chunks a lane
template <typename T>
void launch_sums_t(const EmbedGradArgs &a, const EmbedSizes &s, hipStream_t st)
{
    if (a.C4 <= 8) launch_sums<T, 8, 1>(a, s, st);
    else if (a.C4 <= 16) launch_sums<T, 16, 1>(a, s, st);
    else if (a.C4 <= 32) launch_sums<T, 32, 1>(a, s, st);
    else if (a.C4 <= 64) launch_sums<T, 64, 1>(a, s, st);
    else if (a.C4 <= 128) launch_sums<T, 64, 2>(a, s, st);
    else launch_sums<T, 64, 4>(a, s, st);
}

int check_ids(const int32_t *ids, i64 n, i64 vocab, int32_t dim)
{
    if (n < 0 || n > 0x7FFFFFFFLL - 4096) return tn_fail(TENSAIR_EINVAL, "n out of range");
    if (vocab < 1 || vocab > TENSAIR_MAX_VOCAB) return tn_fail(TENSAIR_EINVAL, "vocab outside 1..TENSAIR_MAX_VOCAB");
    if (dim < 4 || dim > TENSAIR_MAX_DIM || dim % 4) return tn_fail(TENSAIR_EINVAL, "dim must be a multiple of 4 in 4..1024");
    if (n > 0 && !ids) return tn_fail(TENSAIR_EINVAL, "ids is NULL");
    if ((uintptr_t)ids & 3) return tn_fail(TENSAIR_EINVAL, "ids must be 4-byte aligned");
    return TENSAIR_OK;
}
int check_matrix(const void *p, i64 rows, i64 stride, int32_t dim, int32_t dtype, const char *what)
{
    if (dtype != TENSAIR_F32 && dtype != TENSAIR_BF16) return tn_fail(TENSAIR_EINVAL, "%s: unknown dtype", what);
    if (rows > 0 && !p) return tn_fail(TENSAIR_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p & 15) return tn_fail(TENSAIR_EINVAL, "%s must be 16-byte aligned", what);
    if (stride < dim || stride % 4) return tn_fail(TENSAIR_EINVAL, "%s: the row stride must be >= dim and a multiple of 4", what);
    return TENSAIR_OK;
}
int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TENSAIR_OK : tn_fail(TENSAIR_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// of the gradient of n > 0 tokens; before anything is launched
int check_workspace(i64 vocab, i64 n, int dim, const void *workspace, size_t workspace_bytes)
{
    if (workspace_bytes < embed_carve(embed_sizes(vocab, n), vocab, n, dim, nullptr, nullptr, nullptr, nullptr, nullptr))
        return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see tensair_embed_workspace_bytes");
    if (!workspace) return tn_fail(TENSAIR_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace & 255) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    return TENSAIR_OK;
}
// the gradient's sums, where a.out and the sparse gradient's buffers are set
int embed_grad(EmbedGradArgs &a, int32_t d_dtype, int dim, void *workspace, hipStream_t st)
{
    const EmbedSizes s = embed_sizes(a.V, a.n);
    int *row_ids = a.row_ids;
    u32 *keys[2] = {}, *vals[2] = {}, *pub = nullptr;
    embed_carve(s, a.V, a.n, dim, (char *)workspace, &a, keys, vals, &pub);
    if (row_ids) a.row_ids = row_ids;
    if (s.few) {
        if (a.n_rows) hipLaunchKernelGGL(k_embed_first, dim3((a.n + WAVES_PER_BLOCK - 1) / WAVES_PER_BLOCK), dim3(BLOCK), 0, st, a);
    } else {
        tn_launch_prep_clear(pub, (int)s.clear, st);
        EmbedKeys k = {a.ids, keys[0], s.chained ? pub + s.hist : nullptr, a.V, a.n, s.passes, s.bits, a.status};
        hipLaunchKernelGGL(k_embed_keys, dim3((unsigned)(((i64)a.n + EMBED_KEYS_TILE - 1) / EMBED_KEYS_TILE)), dim3(BLOCK), 0, st, k);
        for (int i = 0; i < s.passes; ++i) {
            PrepPhase x;
            memset(&x, 0, sizeof(x));
            x.blocks = s.tiles;
            PrepPass &p = x.pass;
            p.ticket = pub + i;
            p.shift = i * s.bits;
            p.bits = s.bits;
            p.first = i == 0;
            p.scanned = !s.chained && tn_prep_groups(s.tiles) > TN_PREP_GROUPS_OWN;
            PrepPassList &q = p.p[0];
            q.kin = keys[i & 1];
            q.kout = keys[(i & 1) ^ 1];
            q.vin = vals[i & 1];
            q.vout = vals[(i & 1) ^ 1];
            q.n = a.n;
            q.tiles = s.tiles;
            q.state = pub + s.tile0 + i * s.per_pass;
            q.hist = pub + s.hist + i * s.nd * (s.chained ? 1 : (size_t)tn_prep_groups(s.tiles) + 1);
            p.p[1].hist = pub + s.none;
            if (!s.chained) {
                x.kind = PREP_COUNT;
                tn_launch_prep(x, st);
            }
            x.kind = s.chained ? PREP_PASS : PREP_PASS_COUNTED;
            tn_launch_prep(x, st);
        }
        a.keys = keys[s.passes & 1];
        a.vals = vals[s.passes & 1];
        u64 *state = (u64 *)(pub + s.seg_state);
        u32 *ticket = pub + s.passes;
        if (s.chained) {
            hipLaunchKernelGGL((k_embed_segments<true, false>), dim3(s.seg_tiles), dim3(BLOCK), 0, st, a, state, ticket);
        } else {
            hipLaunchKernelGGL((k_embed_segments<false, true>), dim3(s.seg_tiles), dim3(BLOCK), 0, st, a, state, ticket);
            hipLaunchKernelGGL((k_embed_segments<false, false>), dim3(s.seg_tiles), dim3(BLOCK), 0, st, a, state, ticket);
        }
    }
    if (d_dtype == TENSAIR_F32) launch_sums_t<float>(a, s, st);
    else launch_sums_t<bf16_t>(a, s, st);
    return launched("embed_grad");
}

}  // namespace

extern "C" {

int tensair_embed(const void *table, int32_t dtype, int64_t vocab, int32_t dim, int64_t row_stride, const int32_t *ids, int64_t n,
                  float scale, void *out, int32_t out_dtype, int64_t out_stride, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_ids(ids, n, vocab, dim))) return rc;
    if ((rc = check_matrix(table, vocab, row_stride, dim, dtype, "table"))) return rc;
    if ((rc = check_matrix(out, n, out_stride, dim, out_dtype, "out"))) return rc;
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    EmbedArgs a;
    a.table = table;
    a.ids = ids;
    a.out = out;
    a.n = n;
    a.V = vocab;
    a.stride = row_stride;
    a.out_stride = out_stride;
    a.C4 = dim / 4;
    a.magic = a.C4 == 1 ? 0u : (u32)(((1ull << 32) + (u32)a.C4 - 1) / (u32)a.C4);
    a.scale = scale;
    a.status = status;
    const u64 blocks = ((u64)n * a.C4 + BLOCK * EMBED_CHUNKS - 1) / (BLOCK * EMBED_CHUNKS);
    if (blocks > TN_MAX_BLOCKS) return tn_fail(TENSAIR_EINVAL, "n * dim beyond what one launch covers");
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)blocks), blk(BLOCK);
    if (dtype == TENSAIR_F32 && out_dtype == TENSAIR_F32) hipLaunchKernelGGL((k_embed<float, float>), grid, blk, 0, st, a);
    else if (dtype == TENSAIR_F32) hipLaunchKernelGGL((k_embed<float, bf16_t>), grid, blk, 0, st, a);
    else if (out_dtype == TENSAIR_F32) hipLaunchKernelGGL((k_embed<bf16_t, float>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_embed<bf16_t, bf16_t>), grid, blk, 0, st, a);
    return launched("embed");
}

size_t tensair_embed_workspace_bytes(int64_t vocab, int32_t dim, int64_t n)
{
    if (check_ids((const int32_t *)4, n, vocab, dim)) return 0;
    // the most of all numbers of tokens up to n: it grows with them but for where tiles become longer and the sort is another
    size_t most = 0;
    auto take = [&](i64 k) {
        if (k <= n) most = std::max(most, embed_carve(embed_sizes(vocab, k), vocab, k, dim, nullptr, nullptr, nullptr, nullptr, nullptr));
    };
    take(n);
    for (int tile = 4; tile < EMBED_MAX_TILE; tile *= 2) take(most_in_tiles(tile));
    take(EMBED_FEW);
    take((i64)TN_PREP_CHAIN_OWN * TN_RADIX_TILE);
    return most;
}

int tensair_embed_grad(const int32_t *ids, int64_t n, const void *d_out, int32_t d_dtype, int64_t d_stride, int64_t vocab, int32_t dim,
                       float scale, const tensair_sparse_rows *grad, void *workspace, size_t workspace_bytes, int32_t *status,
                       void *stream)
{
    int rc;
    if ((rc = check_ids(ids, n, vocab, dim))) return rc;
    if ((rc = check_matrix(d_out, n, d_stride, dim, d_dtype, "d_out"))) return rc;
    if (!grad || !grad->n_rows) return tn_fail(TENSAIR_EINVAL, "grad is NULL");
    if (n > 0 && (!grad->row_ids || !grad->row_grads)) return tn_fail(TENSAIR_EINVAL, "grad: NULL pointer");
    if (((uintptr_t)grad->row_grads & 15) || ((uintptr_t)grad->row_ids & 3) || ((uintptr_t)grad->n_rows & 3))
        return tn_fail(TENSAIR_EINVAL, "grad: rows must be 16-byte aligned, ids and counts 4-byte aligned");
    if (grad->capacity < std::min(vocab, n)) return tn_fail(TENSAIR_ECAPACITY, "grad: capacity below min(vocab, n)");
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    if (n == 0) {
        tn_launch_prep_clear((u32 *)grad->n_rows, 1, st);
        return launched("embed_grad");
    }
    if ((rc = check_workspace(vocab, n, dim, workspace, workspace_bytes))) return rc;
    EmbedGradArgs a;
    memset(&a, 0, sizeof(a));
    a.ids = ids;
    a.d = d_out;
    a.d_stride = d_stride;
    a.V = vocab;
    a.n = (int)n;
    a.C4 = dim / 4;
    a.out.rows = grad->row_grads;
    a.out.stride = dim;
    a.out.dtype = TENSAIR_F32;
    a.out.scale = scale;
    a.row_ids = grad->row_ids;
    a.n_rows = grad->n_rows;
    a.status = status;
    return embed_grad(a, d_dtype, dim, workspace, st);
}

int tensair_embed_grad_dense(const int32_t *ids, int64_t n, const void *d_out, int32_t d_dtype, int64_t d_stride, int64_t vocab,
                             int32_t dim, float scale, void *grad, int32_t grad_dtype, int64_t grad_stride, int32_t accumulate,
                             void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_ids(ids, n, vocab, dim))) return rc;
    if ((rc = check_matrix(d_out, n, d_stride, dim, d_dtype, "d_out"))) return rc;
    if ((rc = check_matrix(grad, vocab, grad_stride, dim, grad_dtype, "grad"))) return rc;
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    if (n > 0 && (rc = check_workspace(vocab, n, dim, workspace, workspace_bytes))) return rc;
    hipStream_t st = (hipStream_t)stream;
    if (n == 0 && accumulate) return TENSAIR_OK;
    if (!accumulate) {
        const i64 want = (vocab * (dim / 4) + BLOCK - 1) / BLOCK;
        const dim3 grid((unsigned)std::min<i64>(want, 16384)), blk(BLOCK);
        if (grad_dtype == TENSAIR_F32) hipLaunchKernelGGL(k_embed_zero<float>, grid, blk, 0, st, (float *)grad, vocab, grad_stride, dim / 4);
        else hipLaunchKernelGGL(k_embed_zero<bf16_t>, grid, blk, 0, st, (bf16_t *)grad, vocab, grad_stride, dim / 4);
    }
    if (n == 0) return launched("embed_grad_dense");
    EmbedGradArgs a;
    memset(&a, 0, sizeof(a));
    a.ids = ids;
    a.d = d_out;
    a.d_stride = d_stride;
    a.V = vocab;
    a.n = (int)n;
    a.C4 = dim / 4;
    a.out.rows = grad;
    a.out.stride = grad_stride;
    a.out.by_id = 1;
    a.out.dtype = grad_dtype;
    a.out.add = accumulate != 0;
    a.out.scale = scale;
    a.status = status;
    return embed_grad(a, d_dtype, dim, workspace, st);
}

}  // extern "C"
