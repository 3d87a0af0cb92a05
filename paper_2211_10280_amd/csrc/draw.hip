// One word for every row of logits: temperature, top-k, top-p, min-p and the draw by a given random number.  With w[v] = exp((z[v] - max z) / T) in 64 bits, what the
// filters leave is a head of the words in the order of falling logits (equal ones by their numbers), so a row comes down to one border in that order.  The border's place and the
// draw are decided by sums of weights: they are taken in 64 bits, or, so that they hang on no order, as whole numbers of 2^-78 (in 32 bits they would move the border by whole words; so would 2^-50, since
// a tail of 2^24 words can decide it with weights of 2^-48).
//   k_draw_top      the largest logit of every part of a row
//   k_draw_bins     words and weights by their distance from the row's largest logit, in bins
//   k_draw_border   the bin that the border falls into
//   (both again, for vocabularies of more than a million words: where that bin has more words than a list, its 4 096th parts)
//   k_draw_gather   the words that may be in (those of the border's bin and, where they are few, all of the bins above) as a list, else the parts' weights above it
//   k_draw          the border among the list, the part that the draw falls into, the word in it
// A row without top-k and top-p needs no bins, a row of few words only the last of these, which then takes the row itself for the list; so it does where a list is too short
// (thousands of words within a 256th of each other's logits at the border, or of one logit, or more than a list of masked words, which all lie in the last bin, where fewer are left than top-k keeps).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "layers.h"

namespace {

#define DRAW_THREADS 512         // of k_draw; with 1 024 its registers go to memory and back
#define BORDER_THREADS 1024      // of k_draw_border
#define PART_THREADS 512         // of the other kernels: a workgroup to a part of a row
#define DRAW_SOLO 8192           // words of a row that k_draw alone takes
#define DRAW_PART 4096           // fewest words of a part
#define DRAW_PARTS 512           // most parts of a row
#define DRAW_WORKGROUPS 4096     // parts of all rows that are aimed at
#define DRAW_BINS 4096           // 256 to a doubling of (distance + 1)
#define DRAW_COARSE 1048576      // most words for which a bin is taken as it is: the launches that cut it again are 5 us; without them 16.8 million words of spread logits with top-p 0.9 take 44.8 ms, with them 206 us
#define DRAW_DIGITS 2048         // of places
#define DRAW_LIST 16384          // most words of a row's list
#define DRAW_STAGED 2048         // of a part's words that go to it, most that are put together in LDS before
#define DRAW_SHORT 512           // most words of a list that need not hold those above the border's bin
#define DRAW_FEW 128             // words of a list that are compared each with each
#define DRAW_PAIRS 128           // words of the border's bin that are
#define DRAW_ROWS 256            // rows at a time, so that the lists take 67 MB at most

struct DrawArgs {
    const void *z;
    i64 stride;
    int n, V;
    const float *temperature, *top_p, *min_p, *u;
    const int *top_k;
    int *words, *status;
    float *prob;
    int part, parts;             // words of a part, parts of a row; 0 parts: k_draw alone
    int counted;                 // parts that k_draw_bins takes at a time where words are only counted
    bool fine;                   // bins are cut again where they have more words than a list
    // in the workspace
    u32 *tops;                   // [n][parts]
    u32 *counts;                 // [n][DRAW_BINS]
    u64 *hi, *lo;                // [n][DRAW_BINS] weights as whole numbers (Fixed)
    struct Border *borders;      // [n]
    u32 *listed;                 // [n]
    ulong2 *list;                // [n][DRAW_LIST] places in the order (~key, word) and weights, as the bits of a double: min_p and the probability look at the weight itself
    double *mass;                // [n][parts]
};

// fp32 numbers in their order as unsigned ones; NaN as minus infinity
#define KEY_LOWEST 0x007FFFFFu       // of minus infinity
__device__ __forceinline__ u32 key_of(float f)
{
    if (f != f) return KEY_LOWEST;
    const u32 u = __float_as_uint(f + 0.0f);                   // minus zero is zero
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(u32 k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

// 2^t: whole part by the exponent, the rest, at most 1/2, by the series of exp up to the 11th power (the 12th term is below 7e-15 of the sum)
__device__ __forceinline__ double exp2_of(double t)
{
    const double n = rint(t), f = t - n;
    double p = 4.4455382718708101e-10;           // ln(2)^k / k!, k = 11 .. 0
    p = fma(p, f, 7.0549116208011209e-09);
    p = fma(p, f, 1.0178086009239696e-07);
    p = fma(p, f, 1.3215486790144305e-06);
    p = fma(p, f, 1.5252733804059838e-05);
    p = fma(p, f, 1.5403530393381606e-04);
    p = fma(p, f, 1.3333558146428441e-03);
    p = fma(p, f, 9.6181291076284769e-03);
    p = fma(p, f, 5.5504108664821576e-02);
    p = fma(p, f, 2.4022650695910069e-01);
    p = fma(p, f, 6.9314718055994529e-01);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}
// weight of a logit beside the largest; slope: log2(e) / T
__device__ __forceinline__ double weight_of(u32 key, u32 top, double slope)
{
    const double t = ((double)of_key(key) - (double)of_key(top)) * slope;
    const double w = t > -1075.0 ? exp2_of(t) : 0.0;             // NaN (minus infinity beside an endless temperature): none
    return key == top ? 1.0 : key == KEY_LOWEST ? 0.0 : w;
}

// what a row asks for
struct Row {
    double slope, p, least;
    int k;                       // 0: all
    bool first;                  // the first word in the order
};
__device__ __forceinline__ Row row_of(const DrawArgs &a, int i)
{
    Row r;
    const double T = a.temperature ? (double)a.temperature[i] : 1.0;
    r.p = a.top_p ? (double)a.top_p[i] : 1.0;
    r.least = a.min_p && a.min_p[i] == a.min_p[i] ? fmin((double)a.min_p[i], 1.0) : 0.0;
    r.k = a.top_k ? a.top_k[i] : 0;
    if (r.k < 1 || r.k >= a.V) r.k = 0;
    r.first = !(T > 0.0) || !(r.p > 0.0) || r.k == 1;
    r.slope = 1.4426950408889634 / (T > 0.0 ? T : 1.0);
    return r;
}
// The bin of a word: its distance below the largest logit, plus 1, with 8 bits behind the leading one.  Falls with the logit.
#define BIN_SHIFT 15
#define FINE_SHIFT 3             // a bin's 4 096th parts
__device__ __forceinline__ int bin_of(u32 key, u32 top, int shift = BIN_SHIFT)
{
    if (key == top) return 0;
    const float d = of_key(top) - of_key(key);
    const u32 b = (__float_as_uint(d + 1.0f) - 0x3F800000u) >> shift;
    return (int)(shift == BIN_SHIFT ? min((u32)(DRAW_BINS - 1), b) : b);
}
__device__ __forceinline__ u64 place_of(u32 key, u32 word) { return ((u64)~key << 32) | word; }
__device__ __forceinline__ ulong2 item_of(u64 place, double w) { return make_ulong2(place, (u64)__double_as_longlong(w)); }
__device__ __forceinline__ double weight_in_item(ulong2 x) { return __longlong_as_double((long long)x.y); }
// A weight, at most 1, as a whole number of 2^-78 in two words, at least 1 where there is one: hi in 2^-39, to nearest, and what is left, signed, in 2^-78.  A row's 2^24 words fit into each, and
// what they are off by together is at most 2^-54 of the largest weight, less than a sum in 64 bits.
struct Fixed {
    u64 hi, lo;
};
__device__ __forceinline__ Fixed fixed_of(double w)
{
    // a sum with 1.5 * 2^52 has the whole part of the number in its last bits
    const double x = w * 0x1p39, big = x + 0x1.8p52, rest = (x - (big - 0x1.8p52)) * 0x1p39 + 0x1.8p52;
    const u64 zero = (u64)__double_as_longlong(0x1.8p52);
    Fixed f = {(u64)__double_as_longlong(big) - zero, (u64)__double_as_longlong(rest) - zero};
    if (w > 0.0 && (f.hi | f.lo) == 0) f.lo = 1;
    return f;
}
__device__ __forceinline__ double mass_of(u64 hi, u64 lo) { return (double)hi * 0x1p-39 + (double)(i64)lo * 0x1p-78; }

// f(word, logit) for the words lo..hi of a row, 16 bytes at a time where they are aligned
template <int THREADS, typename F>
__device__ __forceinline__ void each_word(const float *z, int lo, int hi, F f)
{
    const int t = (int)threadIdx.x;
    const int head = min(hi - lo, (int)(-((uintptr_t)(z + lo) >> 2) & 3));
    if (t < head) f(lo + t, z[lo + t]);
    lo += head;
    const int chunks = (hi - lo) / 4;
    for (int c = t; c < chunks; c += 4 * THREADS) {
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k * THREADS < chunks) v[k] = ld4(z + lo + 4 * (c + k * THREADS));
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k * THREADS < chunks) {
                const int at = lo + 4 * (c + k * THREADS);
                f(at, v[k].x);
                f(at + 1, v[k].y);
                f(at + 2, v[k].z);
                f(at + 3, v[k].w);
            }
    }
    if (t < (hi - lo) % 4) f(lo + 4 * chunks + t, z[lo + 4 * chunks + t]);
}
template <int THREADS, typename F>
__device__ __forceinline__ void each_word(const bf16_t *z, int lo, int hi, F f)
{
    const int t = (int)threadIdx.x;
    const int head = min(hi - lo, (int)(-((uintptr_t)(z + lo) >> 1) & 7));
    if (t < head) f(lo + t, bf16_to_f32(z[lo + t]));
    lo += head;
    const int chunks = (hi - lo) / 8;
    for (int c = t; c < chunks; c += 2 * THREADS) {
        uint4 v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (c + k * THREADS < chunks) v[k] = *reinterpret_cast<const uint4 *>(z + lo + 8 * (c + k * THREADS));
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (c + k * THREADS < chunks) {
                const int at = lo + 8 * (c + k * THREADS);
                const u32 w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f(at + 2 * q, __uint_as_float(w[q] << 16));
                    f(at + 2 * q + 1, __uint_as_float(w[q] & 0xFFFF0000u));
                }
            }
    }
    if (t < (hi - lo) % 8) f(lo + 8 * chunks + t, bf16_to_f32(z[lo + 8 * chunks + t]));
}

__device__ __forceinline__ u32 shfl_add(u32 x, int o) { return x + (u32)__shfl_xor((int)x, o, WAVE); }
__device__ __forceinline__ u64 shfl_add(u64 x, int o) { return x + (u64)__shfl_xor((unsigned long long)x, o, WAVE); }
__device__ __forceinline__ double shfl_add(double x, int o) { return x + __shfl_xor(x, o, WAVE); }
template <int THREADS, typename S>
__device__ __forceinline__ S block_sum(S x, S *lds)
{
    for (int o = 32; o > 0; o >>= 1) x = shfl_add(x, o);
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int k = 1; k < THREADS / WAVE; ++k) x += lds[k];
    return x;
}
template <int THREADS>
__device__ __forceinline__ u32 block_max(u32 x, u32 *lds)
{
    for (int o = 32; o > 0; o >>= 1) x = max(x, (u32)__shfl_xor((int)x, o, WAVE));
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = lds[0];
    for (int k = 1; k < THREADS / WAVE; ++k) x = max(x, lds[k]);
    return x;
}
// sum of what the threads before have.
template <int THREADS, typename S>
__device__ __forceinline__ S block_before(S x, S *lds, S &all)
{
    S run = x;
    for (int o = 1; o < WAVE; o *= 2) {
        const S y = __shfl_up(run, o, WAVE);
        if (lane_id() >= o) run += y;
    }
    S before = __shfl_up(run, 1, WAVE);
    if (lane_id() == 0) before = 0;
    __syncthreads();
    if (lane_id() == WAVE - 1) lds[threadIdx.x >> 6] = run;
    __syncthreads();
    S base = 0;
    all = 0;
    for (int k = 0; k < THREADS / WAVE; ++k) {
        if (k == (int)(threadIdx.x >> 6)) base = all;
        all += lds[k];
    }
    return base + before;
}
struct Three {
    u64 n, hi, lo;
};
template <int THREADS>
__device__ __forceinline__ Three block_before(Three x, Three *lds, Three &all)
{
    Three run = x;
    for (int o = 1; o < WAVE; o *= 2) {
        const u64 a = __shfl_up(run.n, o, WAVE), b = __shfl_up(run.hi, o, WAVE), c = __shfl_up(run.lo, o, WAVE);
        if (lane_id() >= o) {
            run.n += a;
            run.hi += b;
            run.lo += c;
        }
    }
    __syncthreads();
    if (lane_id() == WAVE - 1) lds[threadIdx.x >> 6] = run;
    __syncthreads();
    Three base = {0, 0, 0};
    all = base;
    for (int k = 0; k < THREADS / WAVE; ++k) {
        if (k == (int)(threadIdx.x >> 6)) base = all;
        all.n += lds[k].n;
        all.hi += lds[k].hi;
        all.lo += lds[k].lo;
    }
    return Three{base.n + run.n - x.n, base.hi + run.hi - x.hi, base.lo + run.lo - x.lo};
}
__device__ __forceinline__ double wave_sum64(double x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, WAVE);
    return x;
}
__device__ __forceinline__ double rd_lane(double x, int l) { return __longlong_as_double((long long)rd_lane64((u64)__double_as_longlong(x), l)); }
__device__ __forceinline__ unsigned long long *atom(u64 *p) { return (unsigned long long *)p; }

// Where a row's border lies, as far as the bins tell.
struct Border {
    int bin;                     // the bin that it falls into; all bins above it are in
    int shift;                   // what bins these are
    u32 above, in;               // words of the bins above, of this bin
    int how;
    double above_mass, whole;    // weight of the bins above and of the row, where that is needed
};
enum { BORDER_NONE, BORDER_ALL_LISTED, BORDER_BIN_LISTED, BORDER_ROW };
// whether a row's bin is to be cut once more: top-p beside top-k looks at what top-k left, and the last bin has no end
__device__ __forceinline__ bool cut_again(const Row &r, const Border &o) { return o.how == BORDER_ROW && !(r.k && r.p < 1.0) && o.bin < DRAW_BINS - 1; }
template <int THREADS>
__device__ __forceinline__ u32 row_top(const DrawArgs &a, int i, u32 *lds)
{
    u32 top = 0;
    for (int c = (int)threadIdx.x; c < a.parts; c += THREADS) top = max(top, a.tops[(i64)i * a.parts + c]);
    return block_max<THREADS>(top, lds);
}

// The row is read: 256 rows of 100 003 in fp32 19 us (102 MB, 5.4 TB/s; the following kernels find most of them in the last cache), one of a million in bfloat16 4.
template <typename T>
__global__ void __launch_bounds__(PART_THREADS) k_draw_top(DrawArgs a)
{
    __shared__ u32 lds[PART_THREADS / WAVE];
    const int i = (int)blockIdx.x / a.parts, c = (int)blockIdx.x - i * a.parts, t = (int)threadIdx.x;
    for (int b = c * PART_THREADS + t; b < DRAW_BINS; b += a.parts * PART_THREADS) {
        a.counts[(i64)i * DRAW_BINS + b] = 0;
        a.hi[(i64)i * DRAW_BINS + b] = a.lo[(i64)i * DRAW_BINS + b] = 0;
    }
    if (c == 0 && t == 0) a.listed[i] = 0;
    u32 top = 0;
    each_word<PART_THREADS>((const T *)a.z + (i64)i * a.stride, c * a.part, min(a.V, (c + 1) * a.part), [&](int, float z) { top = max(top, key_of(z)); });
    top = block_max<PART_THREADS>(top, lds);
    if (t == 0) a.tops[(i64)i * a.parts + c] = top;
}

// A weight in 64 bits for every word of a row with top-p alone, and three additions in LDS: 256 rows, a quarter of them such, 32 us (sums of 2^-50 and less in one word, which three workgroups to a compute unit have room for, 31); one of a million 17 (the workgroups add to the same few hundred
// bins in memory).  Rows with top-k only count.
template <typename T, bool FINE>
__global__ void __launch_bounds__(PART_THREADS) k_draw_bins(DrawArgs a)
{
    // two workgroups of 80 KB to a compute unit: the largest logits of waves lie where counts do afterwards
    __shared__ u32 counts[DRAW_BINS];
    __shared__ u64 hi[DRAW_BINS], lo[DRAW_BINS];
    // the same part of all rows, then the next one, a row further on: a row's workgroups come neither at the same time, to add to the same bins, nor to the same die
    const int c = (int)blockIdx.x / a.n, i = ((int)blockIdx.x - c * a.n + c) % a.n, t = (int)threadIdx.x;
    const Row r = row_of(a, i);
    if (r.first || (r.k == 0 && r.p >= 1.0)) return;
    const bool weigh = r.k == 0;                 // else top-p looks at what top-k left, which is listed
    const int many = weigh ? 1 : a.counted;      // parts to a workgroup
    if (c % many) return;
    int bin = 0;
    if (FINE) {
        const Border o = a.borders[i];
        if (!cut_again(r, o)) return;
        bin = o.bin;
    }
    const u32 top = row_top<PART_THREADS>(a, i, counts);
    __syncthreads();
    for (int b = t; b < DRAW_BINS; b += PART_THREADS) {
        counts[b] = 0;
        if (weigh) hi[b] = lo[b] = 0;
    }
    __syncthreads();
    each_word<PART_THREADS>((const T *)a.z + (i64)i * a.stride, c * a.part, min(a.V, (c + many) * a.part), [&](int, float z) {
        const u32 key = key_of(z);
        int b = bin_of(key, top);
        if (FINE) {
            if (b != bin) return;
            b = bin_of(key, top, FINE_SHIFT) & (DRAW_BINS - 1);
        }
        atomicAdd(&counts[b], 1u);
        if (!weigh) return;
        const Fixed w = fixed_of(weight_of(key, top, r.slope));
        atomicAdd(atom(&hi[b]), w.hi);
        atomicAdd(atom(&lo[b]), w.lo);
    });
    __syncthreads();
    for (int b = t; b < DRAW_BINS; b += PART_THREADS) {
        if (!counts[b]) continue;
        const i64 at = (i64)i * DRAW_BINS + b;
        atomicAdd(&a.counts[at], counts[b]);
        if (!weigh) continue;
        atomicAdd(atom(&a.hi[at]), hi[b]);
        atomicAdd(atom(&a.lo[at]), lo[b]);
    }
}

// One workgroup to a row, a launch of its own (8 to 10 us, loads and a running sum that wait for each other): made by every workgroup of the next kernel instead it cost more there.
template <bool FINE>
__global__ void __launch_bounds__(BORDER_THREADS) k_draw_border(DrawArgs a)
{
    constexpr int PER = DRAW_BINS / BORDER_THREADS;
    static_assert(PER == 4, "a thread loads its bins at once");
    __shared__ Three lds[BORDER_THREADS / WAVE];
    __shared__ int pick;
    const int t = (int)threadIdx.x, i = (int)blockIdx.x;
    const Row r = row_of(a, i);
    const i64 at = (i64)i * DRAW_BINS + t * PER;
    const uint4 n = *reinterpret_cast<const uint4 *>(a.counts + at);
    const ulong2 h0 = *reinterpret_cast<const ulong2 *>(a.hi + at), h1 = *reinterpret_cast<const ulong2 *>(a.hi + at + 2);
    const ulong2 l0 = *reinterpret_cast<const ulong2 *>(a.lo + at), l1 = *reinterpret_cast<const ulong2 *>(a.lo + at + 2);
    if (r.first || (r.k == 0 && r.p >= 1.0)) return;
    Border up = {0, BIN_SHIFT, 0, 0, BORDER_ROW, 0.0, 0.0};     // what lies above the bins looked at
    if (FINE) {
        up = a.borders[i];
        if (!cut_again(r, up)) return;
    }
    // sums up to each of the four bins; weights are 0 where top-k decides
    const Three s0 = {n.x, h0.x, l0.x}, s1 = {s0.n + n.y, s0.hi + h0.y, s0.lo + l0.y}, s2 = {s1.n + n.z, s1.hi + h1.x, s1.lo + l1.x}, s3 = {s2.n + n.w, s2.hi + h1.y, s2.lo + l1.y};
    if (t == 0) pick = DRAW_BINS;
    Three all;
    const Three run = block_before<BORDER_THREADS>(s3, lds, all);
    const double whole = FINE ? up.whole : mass_of(all.hi, all.lo), want = r.p * whole;
    Border o = {DRAW_BINS, FINE ? FINE_SHIFT : BIN_SHIFT, 0, 0, BORDER_ROW, 0.0, whole};
    auto look = [&](int j, const Three &before, const Three &to) {
        if (o.bin < DRAW_BINS || to.n == before.n) return;
        if (r.k ? up.above + run.n + to.n >= (u64)r.k : up.above_mass + mass_of(run.hi + to.hi, run.lo + to.lo) >= want) {
            o.bin = t * PER + j;
            o.above = up.above + (u32)(run.n + before.n);
            o.in = (u32)(to.n - before.n);
            o.above_mass = up.above_mass + mass_of(run.hi + before.hi, run.lo + before.lo);
        }
    };
    look(0, Three{0, 0, 0}, s0);
    look(1, s0, s1);
    look(2, s1, s2);
    look(3, s2, s3);
    if (o.bin < DRAW_BINS) atomicMin(&pick, o.bin);
    __syncthreads();
    if (!FINE && a.fine) {                       // for the same kernels again
        *reinterpret_cast<uint4 *>(a.counts + at) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<ulong2 *>(a.hi + at) = *reinterpret_cast<ulong2 *>(a.hi + at + 2) = make_ulong2(0, 0);
        *reinterpret_cast<ulong2 *>(a.lo + at) = *reinterpret_cast<ulong2 *>(a.lo + at + 2) = make_ulong2(0, 0);
    }
    if (o.bin == DRAW_BINS || o.bin != pick) return;             // all words' number and weight are enough: there is one (or, FINE, the row itself is looked at)
    if (FINE) o.bin |= up.bin * DRAW_BINS;
    // top-p looks at what top-k left; else the words above the border's bin need not be listed, and are not where they are many
    const bool both = r.k && r.p < 1.0;
    if (o.above + o.in <= (both ? DRAW_LIST : DRAW_SHORT)) o.how = BORDER_ALL_LISTED;
    else if (o.in <= DRAW_LIST && !both) o.how = BORDER_BIN_LISTED;
    a.borders[i] = o;
}
__device__ __forceinline__ Border border_of(const DrawArgs &a, const Row &r, int i)
{
    if (r.k == 0 && r.p >= 1.0) return Border{DRAW_BINS, BIN_SHIFT, 0, 0, BORDER_NONE, 0.0, 0.0};
    return a.borders[i];
}

// The row again: 256 rows 30 us, one of a million 7.  Weights in 64 bits for what is not listed (a row without filters: all of it).
template <typename T>
__global__ void __launch_bounds__(PART_THREADS) k_draw_gather(DrawArgs a)
{
    __shared__ u32 tops[PART_THREADS / WAVE];
    __shared__ double sums[PART_THREADS / WAVE];
    __shared__ u64 staged[DRAW_STAGED];
    __shared__ u32 some, base;
    const int i = (int)blockIdx.x / a.parts, c = (int)blockIdx.x - i * a.parts, t = (int)threadIdx.x;
    const Row r = row_of(a, i);
    if (r.first) return;
    const Border o = border_of(a, r, i);
    if (o.how == BORDER_ROW) return;
    if (t == 0) some = 0;
    const u32 top = row_top<PART_THREADS>(a, i, tops);           // waits for all threads
    if (top <= KEY_LOWEST) return;
    const bool weigh = o.how != BORDER_ALL_LISTED;
    ulong2 *list = a.list + (i64)i * DRAW_LIST;
    double m = 0.0;
    each_word<PART_THREADS>((const T *)a.z + (i64)i * a.stride, c * a.part, min(a.V, (c + 1) * a.part), [&](int v, float z) {
        const u32 key = key_of(z);
        const int b = o.how == BORDER_NONE ? 0 : bin_of(key, top, o.shift);
        if (b > o.bin) return;
        if (o.how != BORDER_NONE && (b == o.bin || !weigh)) {
            const u32 at = atomicAdd(&some, 1u);
            if (at < DRAW_STAGED) {
                staged[at] = place_of(key, (u32)v);
            } else {                             // more than are put together: one by one
                const u32 to = atomicAdd(&a.listed[i], 1u);
                if (to < DRAW_LIST) list[to] = item_of(place_of(key, (u32)v), weight_of(key, top, r.slope));
            }
        } else {
            const double w = weight_of(key, top, r.slope);
            if (w >= r.least) m += w;
        }
    });
    __syncthreads();
    const u32 n = min(some, (u32)DRAW_STAGED);
    if (n) {
        if (t == 0) base = atomicAdd(&a.listed[i], n);
        __syncthreads();
        for (u32 q = t; q < n; q += PART_THREADS) {
            const u64 x = staged[q];
            if (base + q < DRAW_LIST) list[base + q] = item_of(x, weight_of(~(u32)(x >> 32), top, r.slope));
        }
    }
    if (!weigh) return;
    m = block_sum<PART_THREADS>(m, sums);
    if (t == 0) a.mass[(i64)i * a.parts + c] = m;
}

struct DrawLds {
    u32 counts[DRAW_DIGITS], tops[DRAW_THREADS / WAVE];
    alignas(16) u64 hi[DRAW_DIGITS];             // by digits, then by parts
    u64 lo[DRAW_DIGITS];
    Three three[DRAW_THREADS / WAVE];
    u64 sums[DRAW_THREADS / WAVE];
    double mass[DRAW_THREADS / WAVE];
    u64 found[4];
    int pick;
};
// The place in the order of the word with which the items, of those for which `among` holds, reach a number (or, BY_MASS, a weight): digits of 11 bits of the
// distance from the first place, until one word is left.  each(f): calls f(place, weight) for the items, every thread for its own, the weight as a function.
template <bool BY_MASS, typename Each, typename Among>
__device__ __forceinline__ u64 place_at(Each each, Among among, u64 number, double mass, DrawLds &lds)
{
    constexpr int PER = DRAW_DIGITS / DRAW_THREADS;
    const int t = (int)threadIdx.x;
    u64 first = ~0ull, last = 0;
    __syncthreads();
    if (t == 0) {
        lds.found[0] = ~0ull;
        lds.found[1] = 0;
    }
    each([&](u64 x, auto) {
        if (!among(x)) return;
        first = x < first ? x : first;
        last = x > last ? x : last;
    });
    for (int o = 32; o > 0; o >>= 1) {
        const u64 x = (u64)__shfl_xor((unsigned long long)first, o, WAVE), y = (u64)__shfl_xor((unsigned long long)last, o, WAVE);
        first = x < first ? x : first;
        last = y > last ? y : last;
    }
    __syncthreads();
    if (lane_id() == 0) {
        atomicMin(atom(&lds.found[0]), first);
        atomicMax(atom(&lds.found[1]), last);
    }
    __syncthreads();
    first = lds.found[0];
    last = lds.found[1];
    double before = 0.0;                         // weight of what is in for sure
    while (first < last) {
        const int bits = 64 - __clzll((long long)(last - first)), shift = bits > 11 ? bits - 11 : 0;
        __syncthreads();
        for (int b = t; b < DRAW_DIGITS; b += DRAW_THREADS) {
            lds.counts[b] = 0;
            if (BY_MASS) lds.hi[b] = lds.lo[b] = 0;
        }
        if (t == 0) lds.pick = DRAW_DIGITS;
        __syncthreads();
        each([&](u64 x, auto weight) {
            if (x < first || x > last) return;
            const int b = (int)((x - first) >> shift);
            atomicAdd(&lds.counts[b], 1u);
            if (BY_MASS) {
                const Fixed w = fixed_of(weight());
                atomicAdd(atom(&lds.hi[b]), w.hi);
                atomicAdd(atom(&lds.lo[b]), w.lo);
            }
        });
        __syncthreads();
        Three x[PER], sum = {0, 0, 0}, all;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            x[j] = Three{lds.counts[t * PER + j], 0, 0};
            if (BY_MASS) {
                x[j].hi = lds.hi[t * PER + j];
                x[j].lo = lds.lo[t * PER + j];
            }
            sum = Three{sum.n + x[j].n, sum.hi + x[j].hi, sum.lo + x[j].lo};
        }
        Three run = block_before<DRAW_THREADS>(sum, lds.three, all);
        int mine = DRAW_DIGITS, filled = -1;
        Three at = run;
        u32 there = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const Three to = {run.n + x[j].n, run.hi + x[j].hi, run.lo + x[j].lo};
            if (x[j].n) {
                if (mine == DRAW_DIGITS) {
                    at = run;                    // in the end that of the digit that is taken, or of the last one
                    there = (u32)x[j].n;
                    filled = t * PER + j;
                    if (BY_MASS ? before + mass_of(to.hi, to.lo) >= mass : to.n >= number) mine = t * PER + j;
                }
            }
            run = to;
        }
        if (mine < DRAW_DIGITS) atomicMin(&lds.pick, mine);
        __syncthreads();
        int b = lds.pick;
        if (b == DRAW_DIGITS) {                  // a weight that rounding put out of reach: the last word
            __syncthreads();
            if (t == 0) lds.pick = -1;
            __syncthreads();
            if (filled >= 0) atomicMax(&lds.pick, filled);
            __syncthreads();
            b = lds.pick;
            if (b < 0) return first;             // no word at all: only where another call has changed the list meanwhile
        }
        if (b == filled) {
            lds.found[0] = at.n;
            lds.found[1] = at.hi;
            lds.found[2] = at.lo;
            lds.found[3] = there;
        }
        __syncthreads();
        if (!BY_MASS) number -= lds.found[0];
        if (BY_MASS) before += mass_of(lds.found[1], lds.found[2]);
        const bool one = lds.found[3] == 1;
        const u64 low = first + ((u64)b << shift), high = low + (((u64)1 << shift) - 1);
        first = low;
        last = high < last ? high : last;
        if (one && shift) {                      // one word: its place
            __syncthreads();
            each([&](u64 x, auto) {
                if (x >= first && x <= last) lds.found[0] = x;
            });
            __syncthreads();
            first = last = lds.found[0];
        }
    }
    __syncthreads();
    return first;
}

// The same where at most DRAW_PAIRS items are in question (else ~0): each is compared with each, an item to a thread.  One word after the other is in while those
// before it do not reach the number or the weight.
template <bool BY_MASS, typename Each, typename Among>
__device__ __forceinline__ u64 place_among_few(Each each, Among among, u64 number, double mass, DrawLds &lds)
{
    ulong2 *items = (ulong2 *)lds.hi;
    const int t = (int)threadIdx.x;
    __syncthreads();
    if (t == 0) {
        lds.pick = 0;
        lds.found[0] = 0;
    }
    __syncthreads();
    each([&](u64 x, auto weight) {
        if (!among(x)) return;
        const int at = atomicAdd(&lds.pick, 1);
        if (at >= DRAW_PAIRS) return;
        const Fixed w = fixed_of(BY_MASS ? weight() : 0.0);
        items[at] = make_ulong2(x, w.hi);
        lds.lo[at] = w.lo;
    });
    __syncthreads();
    const int n = lds.pick;
    if (n > DRAW_PAIRS) return ~0ull;
    if (t < n) {
        const u64 x = items[t].x;
        u64 rank = 0, hi = 0, lo = 0;
#pragma unroll 4
        for (int q = 0; q < n; ++q) {
            const ulong2 y = items[q];
            if (y.x < x) {
                ++rank;
                hi += y.y;
                lo += lds.lo[q];
            }
        }
        if (rank == 0 || (BY_MASS ? mass_of(hi, lo) < mass : rank < number)) atomicMax(atom(&lds.found[0]), x);
    }
    __syncthreads();
    return lds.found[0];
}

// A list of at most DRAW_FEW words: each compared with each, a word to a thread, which puts them in order.  Their weights are added up in that order, so the list's own does not matter.
__device__ __forceinline__ void draw_few(const DrawArgs &a, const Row &r, int i, double whole, int items, bool here, DrawLds &lds)
{
    const int t = (int)threadIdx.x;
    ulong2 *list = (ulong2 *)lds.hi;             // DRAW_FEW of them
    double *sorted = (double *)lds.lo;           // their weights in the order of the logits, then, of those that are in, in the order of the words
    ulong2 x = make_ulong2(~0ull, 0);
    if (t < items) {
        x = here ? list[t] : a.list[(i64)i * DRAW_LIST + t];     // here: in LDS already
        list[t] = x;
    }
    const double w = weight_in_item(x);
    __syncthreads();
    int rank = 0;
    if (t < items) {
        for (int q = 0; q < items; ++q) rank += list[q].x < x.x;
        sorted[rank] = w;
    }
    __syncthreads();
    bool in = t < items && (r.k == 0 || rank < r.k);
    if (in && r.p < 1.0) {
        if (r.k) {
            whole = 0.0;
            for (int q = 0; q < min(r.k, items); ++q) whole += sorted[q];
        }
        double before = 0.0;
        for (int q = 0; q < rank; ++q) before += sorted[q];
        in = rank == 0 || before < r.p * whole;
    }
    in = in && w > 0.0 && w >= r.least;
    __syncthreads();
    if (t < items) list[t].x = in ? (u32)x.x : ~0ull;            // by words now
    if (t == 0) lds.found[0] = ~0ull;
    __syncthreads();
    rank = 0;
    int left = 0;                                // words that are
    if (t < items)
        for (int q = 0; q < items; ++q) {
            rank += list[q].x < (u32)x.x;
            left += list[q].x != ~0ull;
        }
    if (in) sorted[rank] = w;
    __syncthreads();
    double to = 0.0, total = 0.0;
    if (in)
        for (int q = 0; q < left; ++q) {
            total += sorted[q];
            if (q == rank) to = total;
        }
    double u = a.u[i];
    u = u > 0.0 ? fmin(u, 1.0) : 0.0;
    if (in && to > u * total) atomicMin(atom(&lds.found[0]), (u64)(u32)x.x);
    __syncthreads();
    if (lds.found[0] == ~0ull) {                 // u is 1: the last word
        __syncthreads();
        if (t == 0) lds.found[0] = 0;
        __syncthreads();
        if (in) atomicMax(atom(&lds.found[0]), (u64)(u32)x.x);
        __syncthreads();
    }
    if (in && (u32)x.x == (u32)lds.found[0]) {
        a.words[i] = (int)(u32)x.x;
        if (a.prob) a.prob[i] = (float)(w / total);
    }
}

// One workgroup to a row: 10 us where a list is short (64 rows, top-k 50), 22 for one of a million with top-p (3 400 words listed), 33 for 256 rows of all kinds: a chain of loads, sums and barriers,
// vector units busy 6 %.
template <typename T>
__global__ void __launch_bounds__(DRAW_THREADS) k_draw(DrawArgs a)
{
    __shared__ DrawLds lds;
    const int i = (int)blockIdx.x, t = (int)threadIdx.x, V = a.V;
    const T *z = (const T *)a.z + (i64)i * a.stride;
    const Row r = row_of(a, i);
    const bool solo = a.parts == 0;
    const int part = solo ? V : a.part, parts = solo ? 1 : a.parts;
    u32 top = 0;
    if (solo) {
        each_word<DRAW_THREADS>(z, 0, V, [&](int, float x) { top = max(top, key_of(x)); });
        top = block_max<DRAW_THREADS>(top, lds.tops);
    } else {
        top = row_top<DRAW_THREADS>(a, i, lds.tops);
    }
    if (top <= KEY_LOWEST) {
        if (t == 0) {
            a.words[i] = -1;
            if (a.prob) a.prob[i] = 0.f;
            if (a.status) atomicOr(a.status, ST_BAD_ID);
        }
        return;
    }
    double u = a.u[i];
    u = u > 0.0 ? fmin(u, 1.0) : 0.0;
    u64 limit = ~0ull;                           // the last place that is in
    double total = 0.0, before = 0.0, want = 0.0;
    int c = 0;                                   // the part that the word is in
    bool end = !r.first && u >= 1.0;             // the last word of it that is in; not left to sums, whose last places differ with what is added up first
    auto weigh = [&](u64 x) { return weight_of(~(u32)(x >> 32), top, r.slope); };
    auto weight_in = [&](u64 x) {
        if (x > limit) return 0.0;
        const double w = weigh(x);
        return w >= r.least ? w : 0.0;
    };
    if (r.first) {
        // the first part that has the largest logit
        if (t == 0) lds.pick = parts;
        __syncthreads();
        if (!solo)
            for (int q = t; q < parts; q += DRAW_THREADS)
                if (a.tops[(i64)i * parts + q] == top) atomicMin(&lds.pick, q);
        __syncthreads();
        c = solo ? 0 : lds.pick;
        limit = place_of(top, 0xFFFFFFFFu);      // the first word of that logit: nothing is drawn
    } else {
        if (solo && r.k && r.k <= DRAW_FEW) {
            // few words are left of few: the bins (two and two) and the list here, so that the words are compared each with each (256 rows of 8 000, top-k 50, top-p 0.9: 15 us, as all rows 48)
            constexpr int PER = DRAW_DIGITS / DRAW_THREADS;
            __syncthreads();
            for (int b = t; b < DRAW_DIGITS; b += DRAW_THREADS) lds.counts[b] = 0;
            if (t == 0) lds.pick = DRAW_DIGITS;
            __syncthreads();
            each_word<DRAW_THREADS>(z, 0, V, [&](int, float x) { atomicAdd(&lds.counts[bin_of(key_of(x), top) >> 1], 1u); });
            __syncthreads();
            u64 mine = 0, all;
            for (int j = 0; j < PER; ++j) mine += lds.counts[t * PER + j];
            u64 run = block_before<DRAW_THREADS>(mine, lds.sums, all);
            for (int j = 0; j < PER; ++j) {
                const u64 next = run + lds.counts[t * PER + j];
                if (run < (u64)r.k && next >= (u64)r.k) {
                    lds.pick = t * PER + j;
                    lds.found[0] = next;
                }
                run = next;
            }
            __syncthreads();
            const int bin = lds.pick, items = (int)lds.found[0];
            if (items <= DRAW_FEW) {
                __syncthreads();
                if (t == 0) lds.pick = 0;
                __syncthreads();
                ulong2 *list = (ulong2 *)lds.hi;
                each_word<DRAW_THREADS>(z, 0, V, [&](int v, float x) {
                    const u32 key = key_of(x);
                    if (bin_of(key, top) >> 1 <= bin) list[atomicAdd(&lds.pick, 1)] = item_of(place_of(key, (u32)v), weight_of(key, top, r.slope));
                });
                __syncthreads();
                draw_few(a, r, i, 0.0, items, true, lds);
                return;
            }
        }
        Border o = {DRAW_BINS, BIN_SHIFT, 0, 0, r.k == 0 && r.p >= 1.0 ? BORDER_NONE : BORDER_ROW, 0.0, 0.0};
        if (!solo) o = border_of(a, r, i);
        const bool listed = o.how == BORDER_ALL_LISTED || o.how == BORDER_BIN_LISTED;
        const int items = listed ? (int)min(a.listed[i], (u32)DRAW_LIST) : 0;
        if (o.how == BORDER_ALL_LISTED && items <= DRAW_FEW) {
            draw_few(a, r, i, o.whole, items, false, lds);
            return;
        }
        auto each = [&](auto f) {
            if (listed) {
                const ulong2 *list = a.list + (i64)i * DRAW_LIST;
                for (int q = t; q < items; q += 4 * DRAW_THREADS) {          // four in flight at a time
                    ulong2 x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (q + k * DRAW_THREADS < items) x[k] = list[q + k * DRAW_THREADS];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (q + k * DRAW_THREADS < items) f((u64)x[k].x, [&] { return weight_in_item(x[k]); });
                }
            } else {
                each_word<DRAW_THREADS>(z, 0, V, [&](int v, float x) {
                    const u32 key = key_of(x);
                    f(place_of(key, (u32)v), [&] { return weight_of(key, top, r.slope); });
                });
            }
        };
        // the border is among the words of its bin; where top-p looks at what top-k left, among those
        bool binned = listed;
        auto among = [&](u64 x) { return x <= limit && (!binned || bin_of(~(u32)(x >> 32), top, o.shift) == o.bin); };
        auto mass_within = [&] {
            u64 h = 0, l = 0;
            each([&](u64 x, auto weight) {
                if (x > limit) return;
                const Fixed w = fixed_of(weight());
                h += w.hi;
                l += w.lo;
            });
            h = block_sum<DRAW_THREADS>(h, lds.sums);
            l = block_sum<DRAW_THREADS>(l, lds.sums);
            return mass_of(h, l);
        };
        if (r.k) {
            const u64 number = (u64)r.k - (listed ? o.above : 0);
            if (listed) limit = place_among_few<false>(each, among, number, 0.0, lds);
            if (limit == ~0ull) limit = place_at<false>(each, among, number, 0.0, lds);
        }
        if (r.p < 1.0) {
            binned = listed && !r.k;
            const double want = binned ? r.p * o.whole - o.above_mass : r.p * mass_within();
            const u64 found = listed || (r.k && r.k <= DRAW_PAIRS) ? place_among_few<true>(each, among, 0, want, lds) : ~0ull;
            limit = found == ~0ull ? place_at<true>(each, among, 0, want, lds) : found;
        }
        // weights of the parts
        __syncthreads();
        // the likely words of a vocabulary lie side by side, so that most of a list may be of one part: neighbouring lanes add to copies of their own
        int copies = 0;
        while ((parts << (copies + 1)) <= DRAW_DIGITS && copies < 5) ++copies;
        for (int q = t; q < parts << copies; q += DRAW_THREADS) lds.hi[q] = lds.lo[q] = 0;
        __syncthreads();
        if (solo || o.how == BORDER_ROW) {
            // one part after the other; a part's words in 64 bits, in the threads' order
            for (int q = 0; q < parts; ++q) {
                u64 h = 0, l = 0;
                each_word<DRAW_THREADS>(z, q * part, min(V, (q + 1) * part), [&](int v, float x) {
                    const Fixed w = fixed_of(weight_in(place_of(key_of(x), (u32)v)));
                    h += w.hi;
                    l += w.lo;
                });
                h = block_sum<DRAW_THREADS>(h, lds.sums);
                l = block_sum<DRAW_THREADS>(l, lds.sums);
                if (t == 0) {
                    lds.hi[q << copies] = h;
                    lds.lo[q << copies] = l;
                }
            }
        } else if (listed) {
            each([&](u64 x, auto weight) {
                const double w = weight();
                if (x > limit || !(w > 0.0) || w < r.least) return;
                const Fixed f = fixed_of(w);
                const int q = min((int)((u32)x / (u32)part), parts - 1) << copies | (t & ((1 << copies) - 1));
                atomicAdd(atom(&lds.hi[q]), f.hi);
                atomicAdd(atom(&lds.lo[q]), f.lo);
            });
        }
        __syncthreads();
        double m = 0.0;
        if (t < parts) {
            u64 h = 0, l = 0;
            for (int q = t << copies; q < (t + 1) << copies; ++q) {
                h += lds.hi[q];
                l += lds.lo[q];
            }
            m = mass_of(h, l);
            if (!solo && (o.how == BORDER_NONE || o.how == BORDER_BIN_LISTED)) m += a.mass[(i64)i * parts + t];
        }
        const double run = block_before<DRAW_THREADS>(m, lds.mass, total);
        want = u * total;
        if (t == 0) lds.pick = parts;
        __syncthreads();
        if (!end && m > 0.0 && run + m > want) atomicMin(&lds.pick, t);
        __syncthreads();
        c = lds.pick;
        if (c == parts) {                        // u is 1, or next to it: the last word
            end = true;
            __syncthreads();
            if (t == 0) lds.pick = 0;
            __syncthreads();
            if (m > 0.0) atomicMax(&lds.pick, t);
            __syncthreads();
            c = lds.pick;
        }
        if (t == c) lds.mass[0] = run;
        __syncthreads();
        before = lds.mass[0];
        __syncthreads();
        // Below 2^-24, between 0 and the least number of a generator of 24 bits, what is before the word may be far below the whole numbers' unit: the parts' weights in 64 bits, one part
        // after the other.
        if (u > 0.0 && u < 0x1p-24 && parts > 1) {
            for (c = 0, before = 0.0; c < parts - 1; ++c) {
                double m = 0.0;
                each_word<DRAW_THREADS>(z, c * part, min(V, (c + 1) * part), [&](int v, float x) { m += weight_in(place_of(key_of(x), (u32)v)); });
                m = block_sum<DRAW_THREADS>(m, lds.mass);
                if (before + m > want) break;
                before += m;
            }
        }
    }
    // the word in part c: an eighth of it to a wave, then an eighth of the one that has it, then 64 words at a time
    constexpr int WAVES = DRAW_THREADS / WAVE;
    const int lane = lane_id(), wave = t / WAVE;
    auto weight_at = [&](int v, int to) {
        if (v >= to) return 0.0;
        const u32 key = key_of(widen1(z[v]));
        return r.first ? (key == top ? 1.0 : 0.0) : weight_in(place_of(key, (u32)v));
    };
    int from = c * part, len = (min(V - from, part) + WAVES * WAVES * WAVE - 1) / (WAVES * WAVES * WAVE) * (WAVES * WAVES * WAVE);
    const int stop = min(V, from + part);
#pragma unroll 1
    for (int level = 0; level < 2; ++level) {
        len /= WAVES;
        const int lo = from + wave * len;
        double m = 0.0;
#pragma unroll 4
        for (int v = lo; v < lo + len; v += WAVE) m += weight_at(v + lane, stop);
        m = wave_sum64(m);
        __syncthreads();
        if (lane == 0) lds.mass[wave] = m;
        __syncthreads();
        // the first that the draw falls into; the last one that is not empty where u is 1 or sums differ in their last places
        int got = -1, filled = 0;
        double run = before, at = before;
        for (int w = 0; w < WAVES; ++w) {
            const double x = lds.mass[w];
            if (x > 0.0 && got < 0) {
                filled = w;
                at = run;
                if (!end && run + x > want) got = w;
            }
            run += x;
        }
        end = end || got < 0;
        from += filled * len;
        before = at;
    }
    if (wave > 0) return;
    for (int v = from; v < from + len; v += WAVE) {
        const double w = weight_at(v + lane, stop);
        double run = w;
#pragma unroll
        for (int o = 1; o < WAVE; o *= 2) {
            const double x = __shfl_up(run, o, WAVE);
            if (lane >= o) run += x;
        }
        const u64 in = __ballot(w > 0.0), above = end ? 0 : __ballot(w > 0.0 && before + run > want);
        u64 later = 0;                           // whether a word further on is left
        if (!above && in)
            for (int x = v + WAVE; x < from + len && !later; x += WAVE) later = __ballot(weight_at(x + lane, stop) > 0.0);
        before += rd_lane(run, WAVE - 1);
        if (!above && (!in || later)) continue;
        const int got = above ? __ffsll((long long)above) - 1 : 63 - __clzll((long long)in);
        if (lane == got) {
            a.words[i] = v + lane;
            if (a.prob) a.prob[i] = r.first ? 1.f : (float)(w / total);
        }
        return;
    }
    if (lane == 0) {                             // no word at all: only where another call has changed the workspace meanwhile
        a.words[i] = -1;
        if (a.prob) a.prob[i] = 0.f;
    }
}

// the parts of a row, and where what lies in the workspace
void draw_plan(i64 n, i64 V, int *part, int *parts)
{
    *part = *parts = 0;
    if (V <= DRAW_SOLO) return;
    // the smallest parts only where larger ones would leave compute units without: one row of a million, parts of 4 096 / 8 192 59 / 62 us, 64 rows of 50 000 45 / 40; more than 2 048
    // workgroups to 256 rows of 100 003 140 -> 127
    i64 p = n * ((V + 2 * DRAW_PART - 1) / (2 * DRAW_PART)) >= 256 ? 2 * DRAW_PART : DRAW_PART;
    while ((V + p - 1) / p > DRAW_PARTS || (n * ((V + p - 1) / p) > DRAW_WORKGROUPS && p < V)) p *= 2;
    *part = (int)p;
    *parts = (int)((V + p - 1) / p);
}
size_t draw_carve(i64 n, i64 V, char *ws, DrawArgs *a)
{
    int part, parts;
    draw_plan(n, V, &part, &parts);
    if (a) {
        a->part = part;
        a->parts = parts;
        a->fine = V > DRAW_COARSE;
        a->counted = part <= 2 * DRAW_PART && n * parts >= 2048 ? 4 : 1;      // 256 rows of 100 003 with top-k alone: 1 / 4 102 / 94 us
    }
    if (!parts) return 256;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = ws ? ws + at : nullptr;
        at += layer_up256(bytes);
        return p;
    };
    const size_t N = (size_t)n;
    char *tops = take(4 * N * parts), *counts = take(4 * N * DRAW_BINS), *hi = take(8 * N * DRAW_BINS), *lo = take(8 * N * DRAW_BINS), *listed = take(4 * N),
         *borders = take(sizeof(Border) * N), *list = take(16 * N * DRAW_LIST), *mass = take(8 * N * parts);
    if (a) {
        a->tops = (u32 *)tops;
        a->counts = (u32 *)counts;
        a->hi = (u64 *)hi;
        a->lo = (u64 *)lo;
        a->listed = (u32 *)listed;
        a->borders = (Border *)borders;
        a->list = (ulong2 *)list;
        a->mass = (double *)mass;
    }
    return at;
}

template <typename T>
void launch_draw(const DrawArgs &a, hipStream_t st)
{
    if (a.parts) {
        const dim3 grid((unsigned)(a.n * a.parts)), blk(PART_THREADS);
        hipLaunchKernelGGL(k_draw_top<T>, grid, blk, 0, st, a);
        const dim3 rows((unsigned)a.n);
        if (a.top_k || a.top_p) {
            hipLaunchKernelGGL((k_draw_bins<T, false>), grid, blk, 0, st, a);
            hipLaunchKernelGGL(k_draw_border<false>, rows, dim3(BORDER_THREADS), 0, st, a);
            if (a.fine) {
                hipLaunchKernelGGL((k_draw_bins<T, true>), grid, blk, 0, st, a);
                hipLaunchKernelGGL(k_draw_border<true>, rows, dim3(BORDER_THREADS), 0, st, a);
            }
        }
        hipLaunchKernelGGL(k_draw_gather<T>, grid, blk, 0, st, a);
    }
    hipLaunchKernelGGL(k_draw<T>, dim3((unsigned)a.n), dim3(DRAW_THREADS), 0, st, a);
}

}  // namespace

extern "C" {

size_t tensair_sample_workspace_bytes(int64_t n, int64_t vocab)
{
    if (n < 0 || n > TENSAIR_MAX_SAMPLE_ROWS || vocab < 1 || vocab > TENSAIR_MAX_SAMPLE_VOCAB) {
        tn_fail(TENSAIR_EINVAL, "n must be in 0..TENSAIR_MAX_SAMPLE_ROWS, vocab in 1..TENSAIR_MAX_SAMPLE_VOCAB");
        return 0;
    }
    // the most of all rows up to n and all vocabularies up to vocab: fewer rows have more parts
    if (vocab <= DRAW_SOLO) return 256;
    n = std::min<int64_t>(n, DRAW_ROWS);
    return std::max<size_t>(256, layer_up256((size_t)n * 16 * DRAW_LIST) + layer_up256((size_t)n * sizeof(Border)) + 2 * layer_up256((size_t)n * 8 * DRAW_BINS) + layer_up256((size_t)n * 4 * DRAW_BINS) +
                                     layer_up256((size_t)n * 4) + layer_up256((size_t)n * 4 * DRAW_PARTS) + layer_up256((size_t)n * 8 * DRAW_PARTS));
}

int tensair_sample(const void *logits, int32_t dtype, int64_t stride, int64_t n, int64_t vocab, const float *temperature, const int32_t *top_k,
                   const float *top_p, const float *min_p, const float *u, int32_t *words, float *prob, void *workspace, size_t workspace_bytes,
                   int32_t *status, void *stream)
{
    const size_t need = tensair_sample_workspace_bytes(n, vocab);
    if (!need) return TENSAIR_EINVAL;
    if (dtype != TENSAIR_F32 && dtype != TENSAIR_BF16) return tn_fail(TENSAIR_EINVAL, "logits: unknown dtype");
    if (n > 0 && (!logits || !u || !words)) return tn_fail(TENSAIR_EINVAL, "NULL pointer argument");
    if ((uintptr_t)logits & (dtype == TENSAIR_F32 ? 3 : 1)) return tn_fail(TENSAIR_EINVAL, "logits must have the alignment of an element");
    if (stride < vocab) return tn_fail(TENSAIR_EINVAL, "logits: the row stride must be >= vocab");
    if (((uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)u | (uintptr_t)words | (uintptr_t)prob | (uintptr_t)status) & 3)
        return tn_fail(TENSAIR_EINVAL, "vectors must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    if (int rc = layer_workspace(workspace, workspace_bytes, need, "tensair_sample_workspace_bytes")) return rc;
    hipStream_t st = (hipStream_t)stream;
    for (int64_t i = 0; i < n; i += DRAW_ROWS) {
        DrawArgs a;
        memset(&a, 0, sizeof(a));
        a.z = (const char *)logits + i * stride * (dtype == TENSAIR_F32 ? 4 : 2);
        a.stride = stride;
        a.n = (int)std::min<int64_t>(DRAW_ROWS, n - i);
        a.V = (int)vocab;
        a.temperature = temperature ? temperature + i : nullptr;
        a.top_k = top_k ? top_k + i : nullptr;
        a.top_p = top_p ? top_p + i : nullptr;
        a.min_p = min_p ? min_p + i : nullptr;
        a.u = u + i;
        a.words = words + i;
        a.status = status;
        a.prob = prob ? prob + i : nullptr;
        draw_carve(a.n, vocab, (char *)workspace, &a);
        if (dtype == TENSAIR_F32) launch_draw<float>(a, st);
        else launch_draw<bf16_t>(a, st);
    }
    return layer_launched("sample");
}

}  // extern "C"
