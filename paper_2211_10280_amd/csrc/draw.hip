// One word for every row of logits: temperature, top-k, top-p, min-p and the draw by a given random number.  With w[v] = exp((z[v] - max z) / T) in 64 bits, what the
// filters leave is a head of the words in the order of falling logits (equal ones by their numbers), so a row comes down to one border: a logit and how many of
// the words equal to it are in.  The border's place and the draw are decided by sums of weights, which are taken in 64 bits and in an order that is a function of
// the sizes alone: a sum in 32 bits would move the border by whole words.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "layers.h"

namespace {

#define DRAW_THREADS 1024

struct DrawArgs {
    const void *z;
    i64 stride;
    int n, V;
    const float *temperature, *top_p, *min_p, *u;
    const int *top_k;
    int *words, *status;
    float *prob;
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

// weight of a logit beside the largest
__device__ __forceinline__ double weight_of(u32 key, u32 top, double T)
{
    if (key == KEY_LOWEST) return 0.0;
    if (key == top) return 1.0;
    const double w = exp(((double)of_key(key) - (double)of_key(top)) / T);
    return w == w ? w : 0.0;
}

template <typename S>
__device__ __forceinline__ S block_sum(S x, S *lds)
{
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, WAVE);
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0;
    for (int k = 0; k < DRAW_THREADS / WAVE; ++k) x += lds[k];
    return x;
}

// A workgroup to a row, and a pass over the row for every bit of the borders.
template <typename T>
__global__ void __launch_bounds__(DRAW_THREADS) k_draw(DrawArgs a)
{
    __shared__ double sums[DRAW_THREADS / WAVE];
    __shared__ u64 counts[DRAW_THREADS / WAVE];
    __shared__ int answer;
    const int i = (int)blockIdx.x, t = (int)threadIdx.x;
    const T *z = (const T *)a.z + (i64)i * a.stride;
    const int V = a.V;
    auto key = [&](int v) { return key_of(widen1(z[v])); };
    u32 top = 0;
    for (int v = t; v < V; v += DRAW_THREADS) top = max(top, key(v));
    for (int o = 32; o > 0; o >>= 1) top = max(top, (u32)__shfl_xor((int)top, o, WAVE));
    if (lane_id() == 0) counts[t >> 6] = top;
    __syncthreads();
    for (int k = 0; k < DRAW_THREADS / WAVE; ++k) top = max(top, (u32)counts[k]);
    __syncthreads();
    if (top <= KEY_LOWEST) {
        if (t == 0) {
            a.words[i] = -1;
            if (a.prob) a.prob[i] = 0.f;
            if (a.status) atomicOr(a.status, ST_BAD_ID);
        }
        return;
    }
    const double T0 = a.temperature ? (double)a.temperature[i] : 1.0, p = a.top_p ? (double)a.top_p[i] : 1.0;
    const bool greedy = !(T0 > 0.0), first = !(p > 0.0);
    const double Tq = greedy ? 1.0 : T0;
    int k = a.top_k ? a.top_k[i] : 0;
    if (k < 1 || k > V) k = V;
    if (greedy || first) k = 1;
    // the border: words above key `low` are in, of those equal to it the first `ties`
    u32 low = 0;
    int ties = V;
    double above = 0.0;                                        // weight above the border
    auto weight = [&](u32 x) { return weight_of(x, top, Tq); };
    auto at_least = [&](u64 b, double &m, u64 &c) {            // weight and number of the words of keys >= b, as far as top-k left them
        m = 0.0;
        c = 0;
        for (int v = t; v < V; v += DRAW_THREADS) {
            const u32 x = key(v);
            if ((u64)x >= b) {
                m += weight(x);
                ++c;
            }
        }
        m = block_sum<double>(m, sums);
        c = block_sum<u64>(c, counts);
    };
    double m;
    u64 c;
    if (k < V) {
        for (int bit = 31; bit >= 0; --bit) {                  // the largest key that k words reach
            at_least((u64)low | (1ull << bit), m, c);
            if (c >= (u64)k) low |= 1u << bit;
        }
        at_least((u64)low + 1, above, c);
        ties = k - (int)c;
    }
    if (p < 1.0 && !first) {
        at_least(0, m, c);
        const double whole = k < V ? above + ties * weight(low) : m;
        const double want = p * whole;
        u32 b = 0;
        for (int bit = 31; bit >= 0; --bit) {                  // the largest key whose words and those above have `want`
            const u32 next = b | (1u << bit);
            if (k < V && next <= low) {
                b = next;
                continue;
            }
            at_least((u64)next, m, c);
            if (m >= want) b = next;
        }
        at_least((u64)b + 1, m, c);
        const double w = weight(b);
        const double more = w > 0.0 ? ceil((want - m) / w) : 1.0;
        const int some = more > 1.0 ? (more < (double)V ? (int)more : V) : 1;
        ties = k < V && b == low ? std::min(ties, some) : some;
        low = b;
    }
    const double floor_ = a.min_p && a.min_p[i] == a.min_p[i] ? std::min((double)a.min_p[i], 1.0) : 0.0;
    // a run of words to a thread, so that running sums go by the words' numbers
    const int per = (V + DRAW_THREADS - 1) / DRAW_THREADS, lo = std::min(V, t * per), hi = std::min(V, lo + per);
    int equal = 0;
    for (int v = lo; v < hi; ++v) equal += key(v) == low;
    __shared__ int before[DRAW_THREADS];
    __shared__ double mass[DRAW_THREADS];
    before[t] = equal;
    __syncthreads();
    int rank = 0;
    for (int q = 0; q < t; ++q) rank += before[q];
    const int rank0 = rank;
    auto kept = [&](u32 x) {
        if (x < low || (x == low && rank++ >= ties)) return 0.0;
        const double w = weight(x);
        return w >= floor_ ? w : 0.0;
    };
    m = 0.0;
    for (int v = lo; v < hi; ++v) m += kept(key(v));
    mass[t] = m;
    if (t == 0) answer = V;
    __syncthreads();
    double run = 0.0, total = 0.0;
    for (int q = 0; q < DRAW_THREADS; ++q) {
        if (q == t) run = total;
        total += mass[q];
    }
    double u = a.u[i];
    u = u > 0.0 ? std::min(u, 1.0) : 0.0;
    const double want = u * total;
    rank = rank0;
    int mine = V, last = -1;
    double w_mine = 0.0, w_last = 0.0;
    for (int v = lo; v < hi; ++v) {
        const double w = kept(key(v));
        if (w > 0.0) {
            last = v;
            w_last = w;
        }
        run += w;
        if (w > 0.0 && run > want && mine == V) {
            mine = v;
            w_mine = w;
        }
    }
    if (mine < V) atomicMin(&answer, mine);
    __syncthreads();
    int got = answer;
    __syncthreads();
    if (got == V) {                                            // u times the sum is the sum: the last word that is left
        if (t == 0) answer = -1;
        __syncthreads();
        if (last >= 0) atomicMax(&answer, last);
        __syncthreads();
        got = answer;
        mine = last;
        w_mine = w_last;
    }
    if (mine == got) {
        a.words[i] = got;
        if (a.prob) a.prob[i] = (float)(w_mine / total);
    }
}

}  // namespace

extern "C" {

size_t tensair_sample_workspace_bytes(int64_t n, int64_t vocab)
{
    if (n < 0 || n > TENSAIR_MAX_SAMPLE_ROWS || vocab < 1 || vocab > TENSAIR_MAX_SAMPLE_VOCAB) {
        tn_fail(TENSAIR_EINVAL, "n must be in 0..TENSAIR_MAX_SAMPLE_ROWS, vocab in 1..TENSAIR_MAX_SAMPLE_VOCAB");
        return 0;
    }
    return 256;
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
    const DrawArgs a = {logits, stride, (int)n, (int)vocab, temperature, top_p, min_p, u, top_k, words, status, prob};
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)n), blk(DRAW_THREADS);
    if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_draw<float>, grid, blk, 0, st, a);
    else hipLaunchKernelGGL(k_draw<bf16_t>, grid, blk, 0, st, a);
    return layer_launched("sample");
}

}  // extern "C"
