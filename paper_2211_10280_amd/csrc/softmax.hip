// Softmax cross entropy against every row of a table, and its gradient.  With z = scale * hidden table^T (tokens by words),
//   lse_i = log sum_v exp z_iv,   loss_i = lse_i - z_i,label,   dz_iv = d_i (exp(z_iv - lse_i) - [v = label_i]),
//   d_hidden = scale * dz table,   d_table = scale * dz^T hidden.
// The logits are never kept: the loss makes a pass over the words with a running maximum and sum per token; the gradient makes
// the logits once more, a range of words at a time, and keeps dz of that range for the two products, in the inputs' type: a bfloat16
// or three of them.
// dz in one bfloat16: a second part would double what is written and read of it and the products.  Most of its elements are near nothing,
// and their roundings are lost in the sums; a label's is near d_i, and its rounding would be as large in a gradient as that of the output (0.00165 of
// its size).  So what the tokens have in common of d_i is taken out of dz, but for a power of two (the sums are no larger for it): a label's
// element is then that of p - 1, which is nearly exact for the many tokens with a small p.  And d_hidden, which has a token's elements in one row, gets what the rounding cut off in its last step.
// (26 tokens, 2 439 words of 148: d_hidden and d_table off from 64 bits by 0.00168 and 0.00171 of their size, without either 0.0034; 16 384
// tokens, 10 000 words of 512 0.00167 both; a call of 4 096 tokens and a million words of 300 0.5 % longer.)
// All products are tiles of matrix instructions in bfloat16 with fp32 sums.  fp32 inputs are three bfloat16 parts each (24 bits
// together), and of the nine products of parts the six that matter at 2^-24 are summed, the smallest first.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "../../include/tensair.h"
#include "dev_common.h"
#include "kernels.h"

namespace {

typedef short bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 hw_bf16x8 __attribute__((ext_vector_type(8)));
typedef short bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef u32 v4u __attribute__((ext_vector_type(4)));

#define SM_BM 256              // words of a tile of logits
#define LOG2E 1.44269504088896340736f
#define LN2 0.69314718055994530942f

// A matrix of bfloat16 parts in memory, in blocks of 32 columns: a block is its rows one after the other, 64 bytes each.  So the
// tile of a step is whole lines of memory whichever of its indices is summed, and so is what a wave writes of dz (rows of 64 bytes
// a row's pitch apart were fetched at half the rate).
#define BK 32                  // columns of a block, and of the summed index per step
struct Operand {
    const bf16_t *p;
    i64 rows, plane;           // rows of a block, elements from part to part
    __device__ __forceinline__ const bf16_t *at(int part, i64 r, i64 c) const { return p + part * plane + (c / BK) * (rows * BK) + r * BK + (c & (BK - 1)); }
    // the bytes from there to the part's end (none beyond it)
    __device__ __forceinline__ i64 left(i64 r, i64 c) const { return (plane - ((c / BK) * (rows * BK) + r * BK + (c & (BK - 1)))) * 2; }
};
// Where the next step's tile of an operand begins: kept from step to step, since working it out anew takes the scalar unit longer than
// the step has to spare (loss of 4 096 tokens, a million words, rows of 300: 2.6 ms, so 2.4).
struct Cursor {
    const char *p;
    i64 left;
    __device__ __forceinline__ void move(i64 bytes)
    {
        p += bytes;
        left -= bytes;
    }
};
// which parts of either operand are multiplied, in this order: of three parts (0 the largest) six pairs, the smallest products first
template <int PARTS> struct Pairs;
template <> struct Pairs<1> {
    static constexpr int N = 1, A[1] = {0}, B[1] = {0};
};
template <> struct Pairs<3> {
    static constexpr int N = 6, A[6] = {2, 0, 1, 1, 0, 0}, B[6] = {0, 2, 1, 0, 1, 0};
};

// The tile of one operand of one step, ROWS of the kept index by BK of the summed one, from memory straight into LDS, 16 bytes
// a lane.  LDS holds it in the order of the lanes, so what keeps the 32 lanes of a fragment off each other's banks is which chunk
// of 16 bytes a lane fetches.
// By rows of the kept index (T = false): a row is BK elements, its chunks change places by the row's number.
// By rows of the summed index (T = true): as in memory, a row's chunks turned round by its number, so that the four rows that
// the transposing load takes lie in four groups of banks.  What lies outside the matrix comes as zero.
template <int ROWS, int THREADS, bool T>
struct Tile {
    static constexpr int CHUNKS = ROWS * BK / 8, PER = (CHUNKS + THREADS - 1) / THREADS;
    static constexpr int CPR = T ? ROWS / 8 : BK / 8;         // chunks of a row
    static constexpr int LDS = ROWS * BK;                     // elements
    static_assert(CHUNKS % WAVE == 0, "whole waves");                   // where the chunks do not go round, some are fetched twice
    int offset[PER];           // of the lane's chunks from the tile's first element, in bytes

    static __device__ __forceinline__ int turn(int row)       // chunks that a row is turned by, or its mask of the places
    {
        if (!T) return (row >> 2) & 3;
        return CPR % 16 == 0 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
    }
    __device__ __forceinline__ void place(const Operand &o)
    {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int q = ((int)threadIdx.x + j * THREADS) % CHUNKS, row = q / CPR, at = q % CPR;
            int c = T ? at - turn(row) : at ^ turn(row);
            if (c < 0) c += CPR;
            offset[j] = (int)(((u32)(8 * c / BK) * (u32)o.rows + (u32)row) * BK + (8 * c & (BK - 1))) * 2;
        }
    }
    typedef __amdgpu_buffer_rsrc_t Source;
    static __device__ __forceinline__ Cursor begin(const Operand &o, i64 row0, i64 k0)
    {
        const i64 r0 = T ? k0 : row0, c0 = T ? row0 : k0;
        return Cursor{(const char *)o.at(0, r0, c0), o.left(r0, c0)};
    }
    // bytes from a step's tile to the next one's
    static __device__ __forceinline__ i64 stride(const Operand &o) { return T ? BK * BK * 2 : o.rows * (BK * 2); }
    static __device__ __forceinline__ Source source(const Cursor &c, i64 part_bytes)
    {
        const i64 n = c.left < 0 ? 0 : c.left > 0x7FFFFFF0 ? 0x7FFFFFF0 : c.left;
        return __builtin_amdgcn_make_buffer_rsrc((void *)(c.p + part_bytes), 0, (int)n, 0x00027000);
    }
    __device__ __forceinline__ void fetch(Source from, int j, bf16_t *__restrict lds, int wave) const
    {
#ifdef __HIP_DEVICE_COMPILE__      // the host's pass does not know the 16-byte form and would leave the kernels' handles out
        typedef __attribute__((address_space(3))) void lds_void;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)(lds + (j * THREADS + wave * WAVE) % CHUNKS * 8), 16, offset[j], 0, 0, 0);
#endif
    }
    __device__ __forceinline__ void fetch_all(Source from, bf16_t *__restrict lds, int wave) const
    {
#pragma unroll
        for (int j = 0; j < PER; ++j) fetch(from, j, lds, wave);
    }
    // the fragment of 32 rows from `row` on, 16 of the summed index from 16 * kk on: lane l holds row l % 32, 8 * (l / 32) and on
    static __device__ __forceinline__ hw_bf16x8 fragment(const bf16_t *__restrict lds, int row, int kk)
    {
        const int lane = lane_id();
        if constexpr (!T) {
            const int m = row + (lane & 31), c = 2 * kk + (lane >> 5);
            return *(const hw_bf16x8 *)(lds + m * BK + 8 * (c ^ turn(m)));
        } else {
            typedef __attribute__((address_space(3))) bf16x4 lds4;
            const int g = lane >> 4, i = lane & 15, k = 16 * kk + 8 * (g >> 1) + (i >> 2);
            int c = row / 8 + 2 * (g & 1) + ((i & 3) >> 1) + turn(k);          // the same for k + 4
            if (c >= CPR) c -= CPR;
            const bf16_t *at = lds + k * ROWS + 8 * c + 4 * (i & 1);
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)at);
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 4 * ROWS));
            const bf16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(hw_bf16x8, v);
        }
    }
};

// Waits for all but the last N of this wave's fetches, which come back in order, and for its reads of LDS, then for the other waves.
template <int N>
__device__ __forceinline__ void meet()
{
    static_assert(N < 64, "the counter's bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((N >> 4) << 14));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A workgroup's tile of a product: BM of A's rows by BN of B's, WM by WN waves of TM by TN fragments of 32 by 32.  Lane l of a
// fragment holds the column (B's row) l % 32 and the rows (A's) 8 (r / 4) + 4 (l / 32) + r % 4 in its 16 registers r.
template <int TM, int TN, int WM, int WN, int STAGES, int PARTS, bool AT, bool BT>
struct Product {
    static constexpr int THREADS = 64 * WM * WN, BM = 32 * TM * WM, BN = 32 * TN * WN;
    typedef Tile<BM, THREADS, AT> A;
    typedef Tile<BN, THREADS, BT> B;
    static constexpr int LDS = PARTS * (A::LDS + B::LDS);     // elements of a stage: A's parts, B's parts
    f32x16 acc[TM][TN];
    A a;
    B b;

    static __device__ __forceinline__ void fragments(const bf16_t *__restrict lds, int wm, int wn, int kk, hw_bf16x8 (&fa)[PARTS][TM], hw_bf16x8 (&fb)[PARTS][TN])
    {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[part][i] = A::fragment(lds + part * A::LDS, (wm * TM + i) * 32, kk);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[part][j] = B::fragment(lds + PARTS * A::LDS + part * B::LDS, (wn * TN + j) * 32, kk);
        }
    }
    __device__ __forceinline__ void fetch(const Cursor &x, i64 plane_x, const Cursor &y, i64 plane_y, bf16_t *__restrict lds, int wave) const
    {
#pragma unroll
        for (int part = 0; part < PARTS; ++part) a.fetch_all(A::source(x, part * plane_x), lds + part * A::LDS, wave);
#pragma unroll
        for (int part = 0; part < PARTS; ++part) b.fetch_all(B::source(y, part * plane_y), lds + PARTS * A::LDS + part * B::LDS, wave);
    }
    // One step with STAGES tiles in LDS, that of the step itself in `cur`, of a sum that begins here (FIRST) or goes on: the tiles of the
    // step STAGES - 1 later set out into `next`; fragments of 16 of the summed index are read while those before are multiplied; in
    // the end the next step's tiles are there, and every wave is done with these.
    template <bool FIRST>
    __device__ __forceinline__ void step(const Cursor &x, i64 plane_x, const Cursor &y, i64 plane_y, bf16_t *__restrict next,
                                         const bf16_t *__restrict cur, int wave, int wm, int wn)
    {
        constexpr int KK = BK / 16;
        fetch(x, plane_x, y, plane_y, next, wave);
        __builtin_amdgcn_sched_barrier(0);
        hw_bf16x8 fa[2][PARTS][TM], fb[2][PARTS][TN];
        f32x16 zero;
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r] = 0.f;
        fragments(cur, wm, wn, 0, fa[0], fb[0]);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            if (kk + 1 < KK) fragments(cur, wm, wn, kk + 1, fa[(kk + 1) & 1], fb[(kk + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < Pairs<PARTS>::N; ++q)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[kk & 1][Pairs<PARTS>::A[q]][i], fb[kk & 1][Pairs<PARTS>::B[q]][j],
                                                                            FIRST && kk == 0 && q == 0 ? zero : acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        meet<(STAGES - 2) * PARTS * (A::PER + B::PER)>();
    }
};

// Workgroups that follow one another go to the eight dies in turn: work w of n such that a die's workgroups take neighbouring work.
__device__ __forceinline__ int die_order(int b, int n)
{
    const int die = b % 8, i = b / 8, share = n / 8, more = n % 8;
    return die * share + min(die, more) + i;
}

// the caller's labels: the word of token i, -1 where it has no loss
struct Labels {
    const int *p;
    int ignore;
    i64 V;
    __device__ __forceinline__ int at(i64 i) const
    {
        const int l = p[i];
        return (u64)(u32)l < (u64)V && l != ignore ? l : -1;
    }
    __device__ __forceinline__ bool bad(i64 i) const { return p[i] != ignore && (u64)(u32)p[i] >= (u64)V; }
};

// ---------------------------------------------------------------- logits
struct LogitsArgs {
    Operand w, h;              // words' and tokens' rows
    int K;
    i64 word0, V;              // first word of this launch's range; words in all
    int tiles, per, strips;    // tiles of words (of the kernel's size) of the range, of a strip; strips
    int token_tiles;
    i64 Np;
    float c;                   // |scale| * log2(e): the scale's sign went into the tokens' rows
    const int *label;          // [Np], -1: none
    // loss
    float2 *part;              // [strips * WM][Np] maximum, sum (of powers of two)
    float *picked;             // [Np] the label's logit, in units of log 2
    // inputs of three parts: the numbers themselves
    const float *table, *hidden;
    i64 table_stride, hidden_stride, n;
    int D;
    float sign;
    // gradient
    const float *lse2, *d;     // [Np]
    const float *unit;         // of dz (NULL: 1)
    float *rest;               // [Np] what the rounding of the label's element cut off
    bf16_t *dz;                // an Operand: rows are tokens, columns words
    i64 dz_plane;
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
// two floats rounded to nearest even, in one instruction
__device__ __forceinline__ u32 pack2(float a, float b) { return __builtin_bit_cast(u32, __builtin_convertvector(f32x2{a, b}, bf16x2)); }

// the four registers of a group of 4 rows from this lane and its partner 32 lanes on: 8 rows that follow one another (lanes below
// 32: of group x, the others: of group y), as bfloat16
__device__ __forceinline__ v4u join_halves(u32 x0, u32 x1, u32 y0, u32 y1)
{
    // the upper half of x for the lower half of y
    const auto p = __builtin_amdgcn_permlane32_swap(x0, y0, false, false);
    const auto q = __builtin_amdgcn_permlane32_swap(x1, y1, false, false);
    return v4u{(u32)p[0], (u32)q[0], (u32)p[1], (u32)q[1]};
}

// A token's running sum over many words, of powers of two relative to `top`, with what its roundings have cut off so far: the words may
// be the whole vocabulary, and added to the plain sum its many small ones would be lost one by one beside a large one.  `top` is the
// largest logit so far or the whole number above it, so that a sum is brought to another one without a rounding.
struct Running {
    float top, sum, low;
    __device__ __forceinline__ float ref() const { return top == -INFINITY ? 0.f : top; }
    __device__ __forceinline__ void raise(float logit)
    {
        const float was = top;
        top = fmaxf(ceilf(logit), was);
        const float f = __builtin_amdgcn_exp2f(was - ref());
        sum *= f;
        low *= f;
    }
    __device__ __forceinline__ void add(float x)
    {
        const float more = x - low, was = sum;
        sum = was + more;
        low = (sum - was) - more;
    }
};
// a maximum and a sum of powers of two relative to it, joined by another pair
__device__ __forceinline__ void join_sums(float &top, float &sum, float t, float s)
{
    const float now = fmaxf(top, t), ref = now == -INFINITY ? 0.f : now;
    sum = sum * __builtin_amdgcn_exp2f(top - ref) + s * __builtin_amdgcn_exp2f(t - ref);
    top = now;
}
// What is done with a wave's tile of logits, acc: TM by TN fragments of words from w0 on by tokens from tok on.
// words that are none: no share in any sum
template <int TM, int TN>
__device__ __forceinline__ void no_words(f32x16 (&acc)[TM][TN], i64 w0, i64 V)
{
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (w0 + 32 * i + 8 * (r / 4) + 4 * (lane_id() >> 5) + r % 4 >= V)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j][r] = -INFINITY;
}
// Products of parts that are NaN or infinite where the product of the numbers need not be: those that overflow beside one of the other
// sign (a word masked by the lowest number, times several hundred), an infinity times a number below the smallest bfloat16.  Such logits
// are made once more, from the numbers in 64 bits, a lane each; minus infinity is right as it is.  (4 096 tokens, 100 000 words of 300, a
// hundredth of the words masked by the lowest number times several hundred: the loss 3.4 ms instead of 1.5, half of them 36.)
template <int TM, int TN>
__device__ __forceinline__ void mend_logits(f32x16 (&acc)[TM][TN], const LogitsArgs &a, i64 w0, i64 tok)
{
    const int lane = lane_id();
    float all = 0.f;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) all += acc[i][j][r];
    if (!__ballot(!(all < INFINITY))) return;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const i64 token = tok + 32 * j + (lane & 31), word0 = w0 + 32 * i + 4 * (lane >> 5);
            u32 bad = 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) bad |= !(acc[i][j][r] < INFINITY) && token < a.n && word0 + 8 * (r / 4) + r % 4 < a.V ? 1u << r : 0u;
            for (; bad; bad &= bad - 1) {
                const int at = __ffs((int)bad) - 1;
                const float *w = a.table + (word0 + 8 * (at / 4) + at % 4) * a.table_stride, *h = a.hidden + token * a.hidden_stride;
                double z = 0.0;
                for (int k = 0; k < a.D && z == z; k += 4) {
                    const float4 x = ld4(w + k), y = ld4(h + k);
                    z = fma((double)x.x, (double)y.x, fma((double)x.y, (double)y.y, fma((double)x.z, (double)y.z, fma((double)x.w, (double)y.w, z))));
                }
                const float v = (float)z * a.sign;
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = r == at ? v : acc[i][j][r];
            }
        }
}
// into the running sums; the label's logit kept
template <int TM, int TN>
__device__ __forceinline__ void add_words(f32x16 (&acc)[TM][TN], const LogitsArgs &a, i64 w0, i64 tok, const int (&label)[TN], Running (&run)[TN])
{
    const int lane = lane_id();
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        float best = -INFINITY;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const i64 lw = (i64)label[j] - (w0 + 32 * i);      // the label's row in this fragment
            if (__ballot(lw >= 0 && lw < 32)) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (lw == 8 * (r / 4) + 4 * (lane >> 5) + r % 4) a.picked[tok + 32 * j + (lane & 31)] = acc[i][j][r] * a.c;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) best = fmaxf(best, acc[i][j][r]);
        }
        Running &x = run[j];
        x.raise(best * a.c);
        const float ref = x.ref();
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], a.c, -ref));
        x.add(s);
    }
}
// dz, to the blocks of columns from `block` on
template <int TM, int TN, int PARTS>
__device__ __forceinline__ void put_dz(f32x16 (&acc)[TM][TN], const LogitsArgs &a, i64 w0, i64 block, i64 tok, const int (&label)[TN], const float (&l2)[TN],
                                       const float (&d)[TN])
{
    const int lane = lane_id();
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        bf16_t *row = a.dz + (tok + 32 * j + (lane & 31)) * BK + 8 * (lane >> 5);
        const u32 keep = label[j] >= 0 ? ~0u : 0u;             // a token without a loss: zero even where a word's row makes its logit NaN
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int lw = label[j] - (int)(w0 + 32 * i);
            float g[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) g[r] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], a.c, -l2[j]));
            if (__ballot((u32)lw < 32u)) {
                const int at = lw - 4 * (lane >> 5);
                float own = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool is = at == 8 * (r / 4) + r % 4;
                    g[r] -= is ? 1.0f : 0.0f;
                    own = is ? g[r] : own;
                }
                if (PARTS == 1 && (u32)lw < 32u && (lw >> 2 & 1) == lane >> 5) {       // the lane that has it
                    own *= d[j];
                    a.rest[tok + 32 * j + (lane & 31)] = own - __uint_as_float(pack2(own, 0.f) << 16);
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) g[r] *= d[j];
#pragma unroll
            for (int part = 0; part < PARTS; ++part) {
                u32 q[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) q[r] = pack2(g[2 * r], g[2 * r + 1]) & keep;
                bf16_t *to = row + part * a.dz_plane + (block + i) * (a.Np * BK);
                *(v4u *)to = join_halves(q[0], q[1], q[2], q[3]);
                *(v4u *)(to + 16) = join_halves(q[4], q[5], q[6], q[7]);
                if (part + 1 < PARTS)
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        g[2 * r] -= __uint_as_float(q[r] << 16);
                        g[2 * r + 1] -= __uint_as_float(q[r] & 0xFFFF0000u);
                    }
            }
        }
    }
}
// a wave's maxima and sums, of the two halves of its rows together
template <int TN>
__device__ __forceinline__ void put_sums(const LogitsArgs &a, int slot, i64 tok, const Running (&run)[TN])
{
    const int lane = lane_id();
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        float t = run[j].top, s = run[j].sum;
        join_sums(t, s, __shfl_xor(t, 32, WAVE), __shfl_xor(s, 32, WAVE));
        if (lane < 32) a.part[(i64)slot * a.Np + tok + 32 * j + lane] = make_float2(t, s);
    }
}

// GRAD false: the running maximum and sum of every token over a strip of words; true: dz of the strip, in PARTS bfloat16 parts.
// A strip's tiles follow one another without a pause: the next tile's first step is in flight while this one's logits are used.
// What bounds it is what comes to LDS (a tile's products are 85 operations a byte of its operands, of either form): 10 000 words, 16 384
// tokens, rows of 512 in bfloat16 155 to 190 us, 0.9 to 1.1 PFLOP/s; fp32, 50 000 words, 1 024 tokens, rows of 128 77 to 91 us, 0.86 to 1.0
// PFLOP/s of its bfloat16 products.
template <int TM, int TN, int WM, int WN, int STAGES, bool GRAD, int PARTS>
__global__ void __launch_bounds__(64 * WM * WN, PARTS == 1 ? 2 : 1) k_logits(LogitsArgs a)
{
    typedef Product<TM, TN, WM, WN, STAGES, PARTS, false, false> P;
    __shared__ __attribute__((aligned(16))) bf16_t lds[P::LDS * STAGES];
    const int work = die_order((int)blockIdx.x, (int)gridDim.x);
    const int strip = work / a.token_tiles, tt = work % a.token_tiles;
    const int wave = uniform((int)(threadIdx.x >> 6)), wm = wave / WN, wn = wave % WN, lane = lane_id();
    const i64 tok0 = (i64)tt * P::BN;
    const int t0 = strip * a.per, t1 = min(a.tiles, t0 + a.per), steps = a.K / BK;
    P p;
    Running run[TN];
    float l2[TN], d[TN];
    int label[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const i64 tok = tok0 + (wn * TN + j) * 32 + (lane & 31);
        label[j] = a.label[tok];
        run[j] = Running{-INFINITY, 0.f, 0.f};
        if (GRAD) {
            l2[j] = a.lse2[tok];
            d[j] = a.unit ? a.d[tok] / *a.unit : a.d[tok];
        }
    }
    i64 word = a.word0 + (i64)t0 * P::BM;
    p.a.place(a.w);
    p.b.place(a.h);
    // the step to be fetched next: its number within its tile of words; behind the strip's last nobody uses it (a wave's end waits for it)
    Cursor from_w = P::A::begin(a.w, (i64)t0 * P::BM, 0), from_h = P::B::begin(a.h, tok0, 0);
    const i64 stride_w = P::A::stride(a.w), stride_h = P::B::stride(a.h), plane_w = a.w.plane * 2, plane_h = a.h.plane * 2;
    int k = 0, cur = 0;
    auto advance = [&] {
        from_w.move(stride_w);
        from_h.move(stride_h);
        if (++k == steps) {
            k = 0;
            from_w.move(P::BM * BK * 2 - steps * stride_w);
            from_h.move(-steps * stride_h);
        }
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        p.fetch(from_w, plane_w, from_h, plane_h, lds + s * P::LDS, wave);
        advance();
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t, word += P::BM) {
        auto step = [&](auto first) {
            p.template step<first()>(from_w, plane_w, from_h, plane_h, lds + (cur == 0 ? STAGES - 1 : cur - 1) * P::LDS, lds + cur * P::LDS, wave, wm, wn);
            advance();
            cur = cur == STAGES - 1 ? 0 : cur + 1;
        };
        step(std::true_type{});
        for (int s = 1; s < steps; ++s) step(std::false_type{});
        const i64 w0 = word + wm * TM * 32;
        if constexpr (PARTS > 1) mend_logits<TM, TN>(p.acc, a, w0, tok0 + wn * TN * 32);
        if (word + P::BM > a.V) no_words<TM, TN>(p.acc, w0, a.V);
        if constexpr (GRAD) put_dz<TM, TN, PARTS>(p.acc, a, w0, t * (P::BM / BK) + wm * TM, tok0 + wn * TN * 32, label, l2, d);
        else add_words<TM, TN>(p.acc, a, w0, tok0 + wn * TN * 32, label, run);
    }
    if constexpr (!GRAD) put_sums<TN>(a, strip * WM + wm, tok0 + wn * TN * 32, run);
}

// The same for rows of up to 32 KB elements: a wave holds 64 tokens' whole rows in registers, as fragments, and the words' rows alone come
// through LDS, 32 words to a tile, for the 256 tokens of a workgroup: a third of what the other form fetches, which is what bounds
// that one.  Two workgroups to a compute unit: one's exponentials run beside the other's products.
// 4 096 tokens, rows of 300 in bfloat16: the loss against a million words 1.9 to 2.1 ms (the other form 2.5), 1.2 to 1.3 PFLOP/s, the matrix units
// busy 79 % of it; dz of 125 000 words 385 to 400 us (514).  129 to 256 tokens: 172 us (195 to 203), dz 241 (282 to 288).
// Short rows are bound by the exponentials: rows of 128, 50 000 words, 65 us.
#define HELD_WORDS 32
#define HELD_STAGES 4
template <int KB, bool GRAD>
__global__ void __launch_bounds__(256, 2) k_logits_held(LogitsArgs a)
{
    typedef Tile<HELD_WORDS, 256, false> Words;               // of a block of columns
    constexpr int TN = 2, KK = 2 * KB, GROUP = 4, PER = KB / 2, LDS = Words::LDS * KB;
    constexpr int STORES = GRAD ? 2 * TN : 0;                 // of a tile, by a lane
    static_assert(KB % 2 == 0, "a fetch of all threads is two blocks of columns");
    __shared__ __attribute__((aligned(16))) bf16_t lds[LDS * HELD_STAGES];
    const int work = die_order((int)blockIdx.x, (int)gridDim.x);
    const int strip = work / a.token_tiles, tt = work % a.token_tiles;
    const int wave = uniform((int)(threadIdx.x >> 6)), lane = lane_id();
    const i64 tok0 = (i64)tt * 256 + wave * (32 * TN);
    const int t0 = strip * a.per, t1 = min(a.tiles, t0 + a.per);
    hw_bf16x8 h[TN][KK];
    Running run[TN];
    float l2[TN], d[TN];
    int label[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const i64 tok = tok0 + 32 * j + (lane & 31);
        label[j] = a.label[tok];
        run[j] = Running{-INFINITY, 0.f, 0.f};
        if (GRAD) {
            l2[j] = a.lse2[tok];
            d[j] = a.unit ? a.d[tok] / *a.unit : a.d[tok];
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) h[j][kk] = *(const hw_bf16x8 *)a.h.at(0, tok, 16 * kk + 8 * (lane >> 5));
    }
    // a thread's chunk of a tile's first two blocks; of the next ones and of other tiles it is as far off for all threads
    const int row = ((int)threadIdx.x & 127) / 4, chunk = ((int)threadIdx.x & 3) ^ Words::turn(row);
    [[maybe_unused]] const u32 own = ((u32)(threadIdx.x / 128) * (u32)a.w.rows + (u32)row) * (BK * 2) + 16u * chunk;
    [[maybe_unused]] const auto from = __builtin_amdgcn_make_buffer_rsrc((void *)a.w.p, 0, (int)(a.w.plane * 2), 0x00027000);
    auto fetch = [&](int t, int stage) {
        [[maybe_unused]] const u32 at = (u32)min(t, t1 - 1) * (HELD_WORDS * BK * 2);   // behind the last tile: once more that
#pragma unroll
        for (int j = 0; j < PER; ++j) {
#ifdef __HIP_DEVICE_COMPILE__
            typedef __attribute__((address_space(3))) void lds_void;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void *)(lds + stage * LDS + (j * 256 + wave * WAVE) * 8), 16, (int)own,
                                                     (int)(at + (u32)j * 2 * (u32)a.w.rows * (BK * 2)), 0, 0);
#endif
        }
    };
#pragma unroll
    for (int x = 0; x < HELD_STAGES - 1; ++x) fetch(t0 + x, x);
    __syncthreads();
    int cur = 0;
    for (int t = t0; t < t1; ++t) {
        fetch(t + HELD_STAGES - 1, (cur + HELD_STAGES - 1) % HELD_STAGES);
        __builtin_amdgcn_sched_barrier(0);
        const bf16_t *__restrict tile = lds + cur * LDS;
        hw_bf16x8 w[2][GROUP];
        f32x16 acc[1][TN];
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[0][j][r] = 0.f;
        auto read = [&](int group) {
#pragma unroll
            for (int k = 0; k < GROUP; ++k) {
                const int kk = group * GROUP + k;
                w[group & 1][k] = Words::fragment(tile + kk / 2 * Words::LDS, 0, kk & 1);
            }
        };
        read(0);
#pragma unroll
        for (int group = 0; group < KK / GROUP; ++group) {
            if (group + 1 < KK / GROUP) read(group + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < GROUP; ++k)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[0][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[group & 1][k], h[j][group * GROUP + k], acc[0][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        const i64 w0 = a.word0 + (i64)t * HELD_WORDS;
        if (w0 + HELD_WORDS > a.V) no_words<1, TN>(acc, w0, a.V);
        if constexpr (GRAD) put_dz<1, TN, 1>(acc, a, w0, t, tok0, label, l2, d);
        else add_words<1, TN>(acc, a, w0, tok0, label, run);
        // of the fetches and writes, which come back in order, those behind the next tile's may be under way
        meet<(HELD_STAGES - 2) * PER + (HELD_STAGES - 1) * STORES>();
        cur = (cur + 1) % HELD_STAGES;
    }
    if constexpr (!GRAD) put_sums<TN>(a, strip, tok0, run);
}

// maxima and sums of the strips put together: a workgroup takes 64 tokens, its waves the strips in turn (4.8 us, which is the way to
// memory and back a few times)
struct LossArgs {
    const float2 *part;
    int slots;
    i64 Np, n;
    const float *picked;
    Labels labels;
    float *loss, *lse;
};
__device__ __forceinline__ void put_loss(const LossArgs &a, i64 i, float top, float sum)
{
    const float lse = top + log2f(sum);
    a.lse[i] = lse * LN2;
    a.loss[i] = a.labels.at(i) >= 0 ? (lse - a.picked[i]) * LN2 : 0.f;
}
__global__ void __launch_bounds__(1024) k_loss(LossArgs a)
{
    __shared__ float2 other[16][WAVE];
    const int lane = lane_id(), wave = (int)(threadIdx.x >> 6);
    const i64 i = (i64)blockIdx.x * WAVE + lane;
    Running run = {-INFINITY, 0.f, 0.f};
    for (int s = wave; s < a.slots; s += 16 * 8) {
        float2 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s + 16 * k < a.slots ? a.part[(i64)(s + 16 * k) * a.Np + i] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            run.raise(v[k].x);
            run.add(v[k].y * __builtin_amdgcn_exp2f(v[k].x - run.ref()));
        }
    }
    float top = run.top, sum = run.sum;
    other[wave][lane] = make_float2(top, sum);
    __syncthreads();
    if (wave > 0 || i >= a.n) return;
    for (int w = 1; w < 16; ++w) {
        join_sums(top, sum, other[w][lane].x, other[w][lane].y);
    }
    put_loss(a, i, top, sum);
}

// ---------------------------------------------------------------- few tokens
// At most FEW_TOKENS tokens: nothing is laid out and no matrix instruction used; the words' rows are read once, where they are, and
// both gradients are made while a row is held.  Memory bounds it: one token, a million rows of 300 bfloat16, 97 us, 6.2 TB/s.
// (8 tokens: the loss 245 us, by tiles 424; the gradient, which the vector units bound, 833 and 845.)
// G lanes hold a word's row, ITERS chunks of 4 elements each, ROWS rows at a time; the tokens' rows lie in LDS, fp32.
#define FEW_TOKENS 8
#define FEW_BLOCKS 1024
struct FewArgs {
    const void *hidden, *table;
    i64 hidden_stride, table_stride, V;
    int n, C4;
    float c, sign;             // |scale| log2(e); the scale's sign goes into the tokens' rows
    Labels labels;
    int *status;
    // loss
    float2 *part;              // [n][workgroups]
    float *picked;
    // gradient
    const float *lse, *d_loss;
    float *slots;              // [workgroups][n][4 * C4]
    void *d_table;             // NULL: not wanted
    i64 d_stride;
    float scale;               // of d_table
};
template <int G>
__device__ __forceinline__ float group_sum(float x)
{
    x += dpp_get<0xB1, 0xF>(x);
    x += dpp_get<0x4E, 0xF>(x);
    x += dpp_get<0x141, 0xF>(x);
    x += dpp_get<0x140, 0xF>(x);
    if (G >= 32) x += __shfl_xor(x, 16, WAVE);
    if (G >= 64) x += __shfl_xor(x, 32, WAVE);
    return x;
}
template <typename T, int G, int ITERS, int NT, bool GRAD>
__global__ void __launch_bounds__(BLOCK) k_few(FewArgs a)
{
    constexpr int ROWS = GRAD ? 2 : 4, SIDE = WAVE / G, C = G * ITERS;
    __shared__ float4 h[NT][C];
    __shared__ float2 stats[WAVES_PER_BLOCK][NT];
    const int lane = lane_id(), l = lane % G, side = lane / G, wave = uniform((int)(threadIdx.x >> 6));
    for (int x = threadIdx.x; x < NT * C; x += BLOCK) {
        const int t = x / C, c = x % C;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (t < a.n && c < a.C4 && (!GRAD || a.labels.at(t) >= 0)) v = ld4((const T *)a.hidden + t * a.hidden_stride + 4 * c);
        h[t][c] = make_float4(v.x * a.sign, v.y * a.sign, v.z * a.sign, v.w * a.sign);
    }
    int label[NT];
    float l2[NT], d[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        label[t] = t < a.n ? a.labels.at(t) : -1;
        l2[t] = GRAD && label[t] >= 0 ? a.lse[t] * LOG2E : 0.f;
        d[t] = GRAD && label[t] >= 0 ? a.d_loss[t] : 0.f;
    }
    if (blockIdx.x == 0 && (int)threadIdx.x < a.n && a.status && a.labels.bad(threadIdx.x)) atomicOr(a.status, ST_BAD_ID);
    Running run = {-INFINITY, 0.f, 0.f};                      // of the token of this lane's number
    float4 dh[GRAD ? NT : 1][ITERS];
#pragma unroll
    for (int t = 0; t < (GRAD ? NT : 1); ++t) zero_row<ITERS>(dh[t]);
    __syncthreads();
    const i64 step = (i64)gridDim.x * WAVES_PER_BLOCK * (SIDE * ROWS);
    for (i64 base = ((i64)blockIdx.x * WAVES_PER_BLOCK + wave) * (SIDE * ROWS); base < a.V; base += step) {
        typename Raw4<T>::type w[ROWS][ITERS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const i64 row = base + r * SIDE + side;
            zero_row_raw<ITERS>(w[r]);
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
                if (row < a.V && l + G * it < a.C4) w[r][it] = ldraw_s((const T *)a.table + row * a.table_stride + 4 * (l + G * it));
        }
        float z[ROWS][NT];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) z[r][t] = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float4 x = h[t][l + G * it];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float4 y = widen4(w[r][it]);
                    z[r][t] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, z[r][t]))));
                }
            }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int t = 0; t < NT; ++t) z[r][t] = group_sum<G>(z[r][t]);
        if constexpr (!GRAD) {
            float mine[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const i64 row = base + r * SIDE + side;
                mine[r] = z[r][0];
#pragma unroll
                for (int t = 1; t < NT; ++t)
                    if (l == t) mine[r] = z[r][t];
                mine[r] = row < a.V ? mine[r] * a.c : -INFINITY;
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    if (l == t && row == label[t]) a.picked[t] = mine[r];
            }
            float best = mine[0];
#pragma unroll
            for (int r = 1; r < ROWS; ++r) best = fmaxf(best, mine[r]);
            run.raise(best);
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) s += __builtin_amdgcn_exp2f(mine[r] - run.ref());
            run.add(s);
        } else {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const i64 row = base + r * SIDE + side;
                float g[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float p = __builtin_amdgcn_exp2f(fmaf(z[r][t], a.c, -l2[t]));
                    if (row == label[t]) p -= 1.0f;
                    g[t] = label[t] >= 0 && row < a.V ? d[t] * p : 0.f;
                }
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const float4 y = widen4(w[r][it]);
                    float4 dw = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const float4 x = h[t][l + G * it];
                        dw = make_float4(fmaf(g[t], x.x, dw.x), fmaf(g[t], x.y, dw.y), fmaf(g[t], x.z, dw.z), fmaf(g[t], x.w, dw.w));
                        float4 &e = dh[t][it];
                        e = make_float4(fmaf(g[t], y.x, e.x), fmaf(g[t], y.y, e.y), fmaf(g[t], y.z, e.z), fmaf(g[t], y.w, e.w));
                    }
                    if (a.d_table && row < a.V && l + G * it < a.C4) {
                        dw = make_float4(dw.x * a.scale, dw.y * a.scale, dw.z * a.scale, dw.w * a.scale);
                        st4s((T *)a.d_table + row * a.d_stride + 4 * (l + G * it), dw);
                    }
                }
            }
        }
    }
    if constexpr (!GRAD) {
        float top = run.top, sum = run.sum;
        // the lanes of a token: one of every group
#pragma unroll
        for (int o = G; o < WAVE; o <<= 1) join_sums(top, sum, __shfl_xor(top, o, WAVE), __shfl_xor(sum, o, WAVE));
        if (lane < NT) stats[wave][lane] = make_float2(top, sum);
        __syncthreads();
        if (threadIdx.x < NT && (int)threadIdx.x < a.n) {
            for (int w = 1; w < WAVES_PER_BLOCK; ++w) join_sums(top, sum, stats[w][lane].x, stats[w][lane].y);
            a.part[(i64)threadIdx.x * gridDim.x + blockIdx.x] = make_float2(top, sum);
        }
    } else {
        // the groups of a wave, then the waves in turn (the tokens' rows have served: their place is taken)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                float4 &e = dh[t][it];
#pragma unroll
                for (int o = G; o < WAVE; o <<= 1) {
                    e.x += __shfl_xor(e.x, o, WAVE);
                    e.y += __shfl_xor(e.y, o, WAVE);
                    e.z += __shfl_xor(e.z, o, WAVE);
                    e.w += __shfl_xor(e.w, o, WAVE);
                }
            }
        __syncthreads();
        for (int w = 0; w < WAVES_PER_BLOCK; ++w) {
            if (wave == w && side == 0)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int it = 0; it < ITERS; ++it) {
                        float4 e = dh[t][it];
                        if (w > 0) {
                            const float4 o = h[t][l + G * it];
                            e = make_float4(o.x + e.x, o.y + e.y, o.z + e.z, o.w + e.w);
                        }
                        h[t][l + G * it] = e;
                    }
            __syncthreads();
        }
        for (int x = threadIdx.x; x < a.n * a.C4; x += BLOCK)
            st4(a.slots + ((i64)blockIdx.x * a.n * a.C4 + x) * 4, h[x / a.C4][x % a.C4]);
    }
}
// the workgroups' maxima and sums of a token put together, by a workgroup
__global__ void __launch_bounds__(BLOCK) k_loss_few(LossArgs a)
{
    __shared__ float2 other[WAVES_PER_BLOCK];
    const int i = (int)blockIdx.x;
    const float2 *part = a.part + (i64)i * a.slots;
    float top = -INFINITY, sum = 0.f;
    float2 v[FEW_BLOCKS / BLOCK];
#pragma unroll
    for (int k = 0; k < FEW_BLOCKS / BLOCK; ++k) {
        const int s = k * BLOCK + (int)threadIdx.x;
        v[k] = s < a.slots ? part[s] : make_float2(-INFINITY, 0.f);
    }
#pragma unroll
    for (int k = 0; k < FEW_BLOCKS / BLOCK; ++k) join_sums(top, sum, v[k].x, v[k].y);
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) join_sums(top, sum, __shfl_xor(top, o, WAVE), __shfl_xor(sum, o, WAVE));
    if (lane_id() == 0) other[threadIdx.x / WAVE] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x > 0) return;
    for (int w = 1; w < WAVES_PER_BLOCK; ++w) join_sums(top, sum, other[w].x, other[w].y);
    put_loss(a, i, top, sum);
}

// ---------------------------------------------------------------- products with dz
// d_hidden = dz table (the summed index: words, split so that every compute unit has work, the splits' sums kept apart) and
// d_table = dz^T hidden (tokens).  A tile is as wide as short rows are, so that dz is read once.  4 096 tokens, 125 000 words, rows of
// 300 in bfloat16 (dz: 1 GB): 357 and 330 us, 0.9 PFLOP/s, the matrix units busy 44 % of it, the waves waiting for tiles as long (256
// tokens to a tile, 8 waves, 3 stages: 336 and 335); fp32, 1 024 tokens, 50 000 words of 128: 92 and 96 us.
struct ProductArgs {
    Operand a, b;              // C[n][m] = sum_k a(m, k) b(n, k)
    i64 M, N, K;
    int m_tiles, n_tiles, splits;
    i64 k_per;                 // of a split, a multiple of BK
    float *slots;              // [splits][N][M] sums (NULL: written as the output)
    int add;                   // the sums begin with what the slots hold
    void *out;
    i64 out_stride;
    int dtype;
    float scale;
    const float *unit;         // of dz (NULL: 1), for what is written as the output
};
template <int TM, int TN, int WM, int WN, int STAGES, int PARTS, bool BT>
__global__ void __launch_bounds__(64 * WM * WN, PARTS == 1 ? 2 : 1) k_product(ProductArgs a)
{
    typedef Product<TM, TN, WM, WN, STAGES, PARTS, true, BT> P;
    __shared__ __attribute__((aligned(16))) bf16_t lds[P::LDS * STAGES];
    int work = die_order((int)blockIdx.x, (int)gridDim.x);
    const int mt = work % a.m_tiles;
    work /= a.m_tiles;
    const int nt = work % a.n_tiles, split = work / a.n_tiles;
    const int wave = uniform((int)(threadIdx.x >> 6)), wm = wave / WN, wn = wave % WN, lane = lane_id();
    const i64 m0 = (i64)mt * P::BM, n0 = (i64)nt * P::BN;
    const i64 k0 = split * a.k_per, k1 = min(a.K, k0 + a.k_per);
    P p;
    p.a.place(a.a);
    p.b.place(a.b);
    const int steps = (int)((k1 - k0) / BK);
    Cursor from_a = P::A::begin(a.a, m0, k0), from_b = P::B::begin(a.b, n0, k0);      // behind the last step tiles are fetched that nobody uses
    const i64 stride_a = P::A::stride(a.a), stride_b = P::B::stride(a.b), plane_a = a.a.plane * 2, plane_b = a.b.plane * 2;
    int cur = 0;
    // (read behind the products instead, a chunk at a time, what the slots hold cost 12 % of the launch)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const i64 n = n0 + (wn * TN + j) * 32 + (lane & 31);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const i64 m = m0 + (wm * TM + i) * 32 + 8 * (r / 4) + 4 * (lane >> 5);
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (a.add && n < a.N && m < a.M) v = ld4(a.slots + ((i64)split * a.N + n) * a.M + m);
                p.acc[i][j][r] = v.x;
                p.acc[i][j][r + 1] = v.y;
                p.acc[i][j][r + 2] = v.z;
                p.acc[i][j][r + 3] = v.w;
            }
    }
    auto advance = [&] {
        from_a.move(stride_a);
        from_b.move(stride_b);
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        p.fetch(from_a, plane_a, from_b, plane_b, lds + s * P::LDS, wave);
        advance();
    }
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        p.template step<false>(from_a, plane_a, from_b, plane_b, lds + (cur == 0 ? STAGES - 1 : cur - 1) * P::LDS, lds + cur * P::LDS, wave, wm, wn);
        advance();
        cur = cur == STAGES - 1 ? 0 : cur + 1;
    }
    const float scale = a.unit ? a.scale * *a.unit : a.scale;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const i64 n = n0 + (wn * TN + j) * 32 + (lane & 31);
        if (n >= a.N) continue;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const i64 m = m0 + (wm * TM + i) * 32 + 8 * (r / 4) + 4 * (lane >> 5);
                if (m >= a.M) continue;
                float4 v = make_float4(p.acc[i][j][r], p.acc[i][j][r + 1], p.acc[i][j][r + 2], p.acc[i][j][r + 3]);
                if (a.slots) {
                    st4(a.slots + ((i64)split * a.N + n) * a.M + m, v);
                } else {
                    v = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
                    if (a.dtype == TENSAIR_F32) st4((float *)a.out + n * a.out_stride + m, v);
                    else st4((bf16_t *)a.out + n * a.out_stride + m, v);
                }
            }
        }
    }
}

// sums of the splits put together in order; a row without a label (labels given) is zero
struct JoinArgs {
    const float *slots;
    int n_slots;
    i64 n, stride;             // rows; of the output
    int C4;
    Labels labels;             // (none: no row is)
    void *out;
    int dtype;
    float scale;
    const float *unit;         // of dz (NULL: 1)
    const float *rest;         // what was cut off the labels' elements (NULL: nothing), to be multiplied by the words' rows
    const bf16_t *table;
    i64 table_stride;
};
__device__ __forceinline__ void put_joined(const JoinArgs &a, i64 c, float4 v)
{
    const i64 row = c / a.C4, col = 4 * (c - row * a.C4), at = row * a.stride + col;
    const int label = a.labels.p ? a.labels.at(row) : 0;
    if (a.rest && label >= 0) {
        const float x = a.rest[row];
        const float4 w = ld4(a.table + label * a.table_stride + col);
        v = make_float4(fmaf(x, w.x, v.x), fmaf(x, w.y, v.y), fmaf(x, w.z, v.z), fmaf(x, w.w, v.w));
    }
    const float scale = a.unit ? a.scale * *a.unit : a.scale;
    v = make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale);
    if (label < 0) v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.dtype == TENSAIR_F32) st4((float *)a.out + at, v);
    else st4((bf16_t *)a.out + at, v);
}
// a thread takes a chunk of 4 elements of all slots
__global__ void __launch_bounds__(BLOCK) k_join_flat(JoinArgs a)
{
    const i64 all = a.n * a.C4;
    for (i64 c = (i64)blockIdx.x * BLOCK + threadIdx.x; c < all; c += (i64)gridDim.x * BLOCK) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < a.n_slots; ++s) {
            const float4 x = ld4(a.slots + ((i64)s * all + c) * 4);
            v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
        }
        put_joined(a, c, v);
    }
}
// a workgroup takes 64 chunks of 4 elements, its 16 waves parts of the slots that follow one another
__global__ void __launch_bounds__(1024) k_join(JoinArgs a)
{
    __shared__ float4 sums[15][WAVE];
    const i64 all = a.n * a.C4;
    const int lane = lane_id(), wave = uniform((int)(threadIdx.x >> 6));
    const int per = (a.n_slots + 15) / 16, lo = wave * per, hi = min(a.n_slots, lo + per);
    for (i64 base = (i64)blockIdx.x * WAVE; base < all; base += (i64)gridDim.x * WAVE) {
        const i64 c = base + lane;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < all)
#pragma unroll 4
            for (int s = lo; s < hi; ++s) {
                const float4 x = ld4(a.slots + ((i64)s * all + c) * 4);
                v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
            }
        if (wave > 0) sums[wave - 1][lane] = v;
        __syncthreads();
        if (wave == 0 && c < all) {
            for (int w = 1; w < 16 && w * per < a.n_slots; ++w) {
                const float4 x = sums[w - 1][lane];
                v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
            }
            put_joined(a, c, v);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- inputs laid out for the products
// One pass over the inputs, which memory bounds: 125 000 words of 300 in bfloat16 57 us where they come from memory.
struct PackArgs {
    const void *src;
    i64 stride, rows;          // of the source
    int D, blocks;             // columns; blocks of columns of the copy (zero from D on)
    i64 out_rows, plane;       // rows of the copy (zero from `rows` on), elements from part to part
    bf16_t *out;
    Labels labels;             // rows without a label are zero (none: no row is)
    float sign;                // 1 or -1
};
// what the kernels need of every token, padded ones among them
struct TokenArgs {
    Labels labels;
    const float *lse, *d_loss; // NULL: for the loss
    i64 n, Np;
    int *label, *status;
    float *lse2, *d, *unit;    // unit: NULL where dz is in units of 1
};
__device__ __forceinline__ void tokens(const TokenArgs &a, i64 i)
{
    if (i >= a.Np) return;
    const int y = i < a.n ? a.labels.at(i) : -1;
    if (i < a.n && a.status && a.labels.bad(i)) atomicOr(a.status, ST_BAD_ID);
    a.label[i] = y;
    if (a.lse) {
        a.lse2[i] = y >= 0 ? a.lse[i] * LOG2E : 0.f;
        a.d[i] = y >= 0 ? a.d_loss[i] : 0.f;
    }
}
// The unit of dz, by a workgroup: the significant digits, as a number from 1 to 2, of the first token's d_i that has one, as a rule the same for all
// of them; 1 where it is none or not among the first of a great many tokens.
#define SM_UNIT_TOKENS 16384
__device__ __forceinline__ void find_unit(const TokenArgs &a)
{
    __shared__ int first;
    if (threadIdx.x == 0) first = SM_UNIT_TOKENS;
    __syncthreads();
    for (int base = 0; base < SM_UNIT_TOKENS && base < a.n; base += BLOCK) {
        const int i = base + (int)threadIdx.x;
        if (i < a.n && a.labels.at(i) >= 0 && a.d_loss[i] != 0.f) atomicMin(&first, i);
        __syncthreads();
        const bool found = first < SM_UNIT_TOKENS;
        __syncthreads();
        if (found) break;
    }
    if (threadIdx.x > 0) return;
    const float d = first < SM_UNIT_TOKENS ? fabsf(a.d_loss[first]) : 1.f;
    *a.unit = d >= 0x1p-126f && d < INFINITY ? __uint_as_float((__float_as_uint(d) & 0x007FFFFFu) | 0x3F800000u) : 1.f;
}
// workgroup `first` of `blocks`: a thread takes 8 elements, a wave 16 rows of a block of columns
template <typename T>
__device__ __forceinline__ void parts(const PackArgs &a, int first, int blocks)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    const i64 groups = a.out_rows / 16 * a.blocks, step = (i64)blocks * WAVES_PER_BLOCK;
    const int lane = lane_id();
    for (i64 g = (i64)first * WAVES_PER_BLOCK + uniform((int)(threadIdx.x >> 6)); g < groups; g += step) {
        const i64 row = g / a.blocks * 16 + lane / 4;
        const int block = (int)(g % a.blocks), col = block * BK + lane % 4 * 8;
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (row < a.rows && (!a.labels.p || a.labels.at(row) >= 0)) {
#pragma unroll
            for (int k = 0; k < 8; k += 4)
                if (col + k < a.D) {
                    const float4 v = ld4((const T *)a.src + row * a.stride + col + k);
                    x[k] = v.x * a.sign;
                    x[k + 1] = v.y * a.sign;
                    x[k + 2] = v.z * a.sign;
                    x[k + 3] = v.w * a.sign;
                }
        }
        bf16_t *to = a.out + (i64)block * a.out_rows * BK + row * BK + lane % 4 * 8;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            u32 h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                h[k] = f32_to_bf16(x[k]);
                if (PARTS > 1) {
                    // Infinity is the last part, which is multiplied by the other number's first one alone: that is zero where the number is.
                    const bool infinite = fabsf(x[k]) == INFINITY;
                    if (infinite && part + 1 < PARTS) h[k] = 0;
                    // beyond the largest bfloat16: cut, so that the rest is finite
                    if ((h[k] & 0x7FFFu) == 0x7F80u && !infinite) h[k] = (h[k] & 0x8000u) | 0x7F7Fu;
                    if (!infinite) x[k] = (h[k] & 0x7F80u) == 0x7F80u ? 0.f : x[k] - __uint_as_float(h[k] << 16);
                }
            }
            *(v4u *)(to + part * a.plane) = v4u{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
        }
    }
}
// All of it that a call begins with in one launch: the tokens, their rows, the words' rows (of the first range).
struct LayOutArgs {
    TokenArgs tokens;
    PackArgs h, w;
    int token_blocks, h_blocks, w_blocks;
    int unit_block;            // 1: a workgroup for the unit of dz
};
template <typename T>
__global__ void __launch_bounds__(BLOCK) k_lay_out(LayOutArgs a)
{
    const int b = (int)blockIdx.x;
    if (b < a.token_blocks) tokens(a.tokens, (i64)b * BLOCK + threadIdx.x);
    else if (b < a.token_blocks + a.unit_block) find_unit(a.tokens);
    else if (b < a.token_blocks + a.unit_block + a.h_blocks) parts<T>(a.h, b - a.token_blocks - a.unit_block, a.h_blocks);
    else parts<T>(a.w, b - a.token_blocks - a.unit_block - a.h_blocks, a.w_blocks);
}
__global__ void __launch_bounds__(BLOCK) k_zero_rows(void *out, int dtype, i64 rows, i64 stride, int C4)
{
    for (i64 c = (i64)blockIdx.x * BLOCK + threadIdx.x; c < rows * C4; c += (i64)gridDim.x * BLOCK) {
        const i64 row = c / C4, at = row * stride + 4 * (c - row * C4);
        if (dtype == TENSAIR_F32) st4((float *)out + at, make_float4(0.f, 0.f, 0.f, 0.f));
        else st4((bf16_t *)out + at, make_float4(0.f, 0.f, 0.f, 0.f));
    }
}

// ---------------------------------------------------------------- host
size_t up256(size_t x) { return (x + 255) / 256 * 256; }
i64 cdiv(i64 a, i64 b) { return (a + b - 1) / b; }
int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TENSAIR_OK : tn_fail(TENSAIR_EHIP, "%s: %s", what, hipGetErrorString(e));
}
// workgroups for so many items, a thread each or, of very many, several
unsigned blocks_for(i64 items) { return (unsigned)std::min<i64>(cdiv(items, BLOCK), 1 << 20); }

// Tiles of logits where tokens are not held in registers: 256 words by 128 tokens, a wave's 128 by 64, two workgroups to a compute
// unit, so that one's exponentials run beside the other's products; three stages, as much as LDS holds twice.  Of three parts 64 words
// by 128 tokens, for the same reason (50 000 words, 1 024 tokens, rows of 300: 228 us and with dz 272; with 256 words, one workgroup,
// 244 and 299).
#define SM_BN 128              // tokens of a tile
#define SM_BN_HELD 256         // ... of tokens held in registers
#define SM_HELD_DIM 320        // rows that are: longer ones want more registers than a wave of two to a SIMD has
#define SM_BN_FEW 64           // ... where there are at most so many
#define SM_WAVES_M 2           // rows of waves of a tile, each with a maximum and a sum of its own
#define SM_RANGE_TILES 4096    // tiles of a range, at most: a fetch is off its tile's first element by up to 10 blocks of columns, which fits 31 bits
                               // (of words here, of tokens by TENSAIR_MAX_TOKENS)
#define SM_BLOCKS 512          // workgroups that fill the chip, two to a compute unit
#define SM_DZ_BYTES ((i64)1 << 30)   // dz of a range, about: with half as much the products took 3 to 8 % longer
#define SM_DZ_TILES 8          // ... but never fewer tiles, since each range reads and writes d_hidden's sums

struct SoftmaxPlan {
    bool few;                  // at most FEW_TOKENS tokens
    int few_blocks;
    int parts, Dp, bn, token_tiles, wm;
    bool held;                 // tokens held in registers
    i64 Np, tiles;             // tokens, padded; tiles of words
    i64 range_tiles, ranges;   // tiles of words that are laid out, and whose dz is kept, at a time
    int unit, per, strips;     // tiles of the logits' kernel to SM_BM words; of those to a strip; strips of a range
    int tm, m_tiles, pn;       // of the products: fragments of a wave along the row length, tiles; rows of a tile
    int h_splits, t_splits;    // of d_hidden's sum over a range's words, of d_table's over the tokens
    int t_most;                // ... of as many tokens as fill the last SM_CLASS of them, at most
    i64 h_k, t_k;
};

SoftmaxPlan plan_of(i64 n, i64 V, int D, int dtype, bool grad)
{
    SoftmaxPlan s;
    memset(&s, 0, sizeof(s));
    s.few = n <= FEW_TOKENS;
    s.few_blocks = (int)std::max<i64>(1, std::min<i64>(cdiv(V, 64), grad ? FEW_BLOCKS / 2 : FEW_BLOCKS));
    s.parts = dtype == TENSAIR_F32 ? 3 : 1;
    const bool few = n <= SM_BN_FEW;
    // Two tiles of 256 tokens that are half empty make dz slower than three of 128 (gradient, 300 tokens, 125 000 words of 300: 207 us, by the
    // latter 193, of 200: 130, 121; 385 tokens 221, 229; 640, three tiles of which one is half empty: 285, 281), but not the loss (73, 71).
    s.held = s.parts == 1 && D <= SM_HELD_DIM && n > SM_BN && !(grad && n > SM_BN_HELD && n <= SM_BN_HELD + SM_BN);
    s.Dp = (int)cdiv(D, s.held ? 2 * BK : BK) * (s.held ? 2 * BK : BK);
    s.bn = s.held ? SM_BN_HELD : few ? SM_BN_FEW : SM_BN;
    s.wm = s.held ? 1 : few ? 4 : SM_WAVES_M;
    s.Np = cdiv(n, s.bn) * s.bn;
    s.token_tiles = (int)(s.Np / s.bn);
    s.tiles = cdiv(V, SM_BM);
    s.range_tiles = std::min<i64>(s.tiles, SM_RANGE_TILES);
    if (grad) s.range_tiles = std::min(s.range_tiles, std::max<i64>(SM_DZ_TILES, SM_DZ_BYTES / (s.Np * SM_BM * 2 * s.parts)));
    s.ranges = cdiv(s.tiles, s.range_tiles);
    s.range_tiles = cdiv(s.tiles, s.ranges);
    s.ranges = cdiv(s.tiles, s.range_tiles);
    // strips of such a length that the workgroups fill the chip a whole number of times, each with two tiles' time to begin (fp32, 50 000
    // words, 1 024 tokens, rows of 128: 85 us, as 784 workgroups for 512 places 103)
    s.unit = s.held ? SM_BM / HELD_WORDS : s.parts == 3 && !few ? 4 : 1;
    const i64 units = s.range_tiles * s.unit, room = s.held && s.Dp <= 64 ? 2 * SM_BLOCKS : s.held && s.Dp <= 128 ? SM_BLOCKS / 2 * 3 : SM_BLOCKS;
    i64 shortest = -1;
    for (int k = 1; k <= 4; ++k) {
        const i64 per = cdiv(units, std::max<i64>(1, k * room / s.token_tiles)), time = cdiv(cdiv(units, per) * s.token_tiles, room) * (per + 2);
        if (shortest < 0 || time < shortest) {
            shortest = time;
            s.per = (int)per;
        }
    }
    s.strips = (int)cdiv(units, s.per);
    // fragments of a wave along the row length, two waves to a tile: few columns beyond the row, but a wider tile fetches less.  Of three
    // parts one: six products a fetch are enough, and two workgroups find room on a compute unit (50 000 words, 1 024 tokens, rows of
    // 300: the two products 188 and 182 us, with three fragments 241 and 281).
    i64 least = -1;
    for (int tm = 1; tm <= (s.parts == 1 ? 5 : 1); ++tm) {
        const i64 cost = cdiv(D, 64 * tm) * 64 * (2 * tm + 1); // columns times 1 + 1 / (2 tm)
        if (least < 0 || cost <= least) {
            least = cost;
            s.tm = tm;
        }
    }
    s.m_tiles = (int)cdiv(D, 64 * s.tm);
    s.pn = s.parts == 1 && s.tm <= 2 ? 256 : 128;             // short rows: what is fetched for a product would be more than the memory pipe gives
    const i64 range_words = s.range_tiles * SM_BM;
    const i64 h_tiles = s.m_tiles * cdiv(n, s.pn), t_tiles = s.m_tiles * cdiv(range_words, s.pn);
    i64 splits = std::max<i64>(1, std::min<i64>(SM_BLOCKS / h_tiles, range_words / 512));
    s.h_k = cdiv(cdiv(range_words, splits), BK) * BK;
    s.h_splits = (int)cdiv(range_words, s.h_k);
    splits = std::max<i64>(1, std::min<i64>(SM_BLOCKS / t_tiles, n / 512));
    s.t_most = (int)splits;
    s.t_k = cdiv(cdiv(n, splits), BK) * BK;
    s.t_splits = (int)cdiv(n, s.t_k);
    return s;
}

struct SoftmaxBuffers {
    int *label;
    float *lse2, *d, *unit, *rest, *picked, *h_slots, *t_slots;
    bf16_t *h, *w, *dz;
    float2 *part;
};
// Of more than FEW_TOKENS tokens the size is the same for all n that are the same number of SM_CLASS, which every border in plan_of is a
// multiple of, the last one rounded up.
#define SM_CLASS 64
size_t softmax_carve(const SoftmaxPlan &s, i64 n, int D, bool grad, char *base, SoftmaxBuffers *b)
{
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = base ? base + at : nullptr;
        at += up256(bytes);
        return p;
    };
    SoftmaxBuffers x;
    memset(&x, 0, sizeof(x));
    x.label = (int *)take(4 * (size_t)s.Np);
    if (s.few) {
        x.picked = (float *)take(4 * (size_t)s.Np);
        x.part = (float2 *)take(8 * (size_t)s.few_blocks * n);
        if (grad) x.h_slots = (float *)take(4 * (size_t)s.few_blocks * n * D);
        if (b) *b = x;
        return at;
    }
    x.h = (bf16_t *)take(2 * (size_t)s.Np * s.Dp * s.parts);
    x.w = (bf16_t *)take(2 * (size_t)s.range_tiles * SM_BM * s.Dp * s.parts);
    if (!grad) {
        x.picked = (float *)take(4 * (size_t)s.Np);
        x.part = (float2 *)take(8 * (size_t)s.ranges * s.strips * s.wm * s.Np);
    } else {
        x.lse2 = (float *)take(4 * (size_t)s.Np);
        x.d = (float *)take(4 * (size_t)s.Np);
        if (s.parts == 1) {
            x.unit = (float *)take(4);
            x.rest = (float *)take(4 * (size_t)s.Np);
        }
        x.dz = (bf16_t *)take(2 * (size_t)s.Np * s.range_tiles * SM_BM * s.parts);
        x.h_slots = (float *)take(4 * (size_t)s.h_splits * (cdiv(n, SM_CLASS) * SM_CLASS) * D);
        if (s.t_most > 1) x.t_slots = (float *)take(4 * (size_t)s.t_most * s.range_tiles * SM_BM * D);
    }
    if (b) *b = x;
    return at;
}

int check_softmax(i64 n, i64 vocab, int32_t dim, int32_t dtype)
{
    if (n < 0 || n > TENSAIR_MAX_TOKENS) return tn_fail(TENSAIR_EINVAL, "n outside 0..TENSAIR_MAX_TOKENS");
    if (vocab < 1 || vocab > TENSAIR_MAX_VOCAB) return tn_fail(TENSAIR_EINVAL, "vocab outside 1..TENSAIR_MAX_VOCAB");
    if (dim < 4 || dim > TENSAIR_MAX_DIM || dim % 4) return tn_fail(TENSAIR_EINVAL, "dim must be a multiple of 4 in 4..1024");
    if (dtype != TENSAIR_F32 && dtype != TENSAIR_BF16) return tn_fail(TENSAIR_EINVAL, "unknown dtype");
    return TENSAIR_OK;
}
int check_scale(float scale)
{
    if (!(fabsf(scale) > 0.f) || !(fabsf(scale) < INFINITY)) return tn_fail(TENSAIR_EINVAL, "scale must be finite and not zero");
    return TENSAIR_OK;
}
int check_rows(const void *p, i64 rows, i64 stride, int32_t dim, const char *what)
{
    if (rows > 0 && !p) return tn_fail(TENSAIR_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p & 15) return tn_fail(TENSAIR_EINVAL, "%s must be 16-byte aligned", what);
    if (stride < dim || stride % 4) return tn_fail(TENSAIR_EINVAL, "%s: the row stride must be >= dim and a multiple of 4", what);
    return TENSAIR_OK;
}

// rows [0, rows) of a matrix laid out for the products, out_rows (a multiple of 16) with what is zero; its workgroups
PackArgs lay_out(const SoftmaxPlan &s, const void *src, i64 stride, i64 rows, i64 out_rows, int D, Labels labels, float sign, bf16_t *out, int *blocks)
{
    *blocks = (int)blocks_for(out_rows / 16 * (s.Dp / BK) * WAVE);
    return PackArgs{src, stride, rows, D, s.Dp / BK, out_rows, out_rows * s.Dp, out, labels, sign};
}
// one range of words: its rows laid out, and what its logits' launch needs
struct Range {
    i64 word0, words, tiles, rows;
};
Range range_of(const SoftmaxPlan &s, i64 range, i64 V)
{
    Range r;
    const i64 tile0 = range * s.range_tiles;
    r.tiles = std::min(s.range_tiles, s.tiles - tile0);
    r.word0 = tile0 * SM_BM;
    r.words = std::min(r.tiles * SM_BM, V - r.word0);
    r.rows = r.tiles * SM_BM;
    return r;
}
// `x`: what else is laid out with the first range
LogitsArgs lay_out_range(const SoftmaxPlan &s, const SoftmaxBuffers &b, const Range &r, LayOutArgs &x, const void *table, i64 table_stride, int dtype, int D,
                         i64 V, float scale, hipStream_t st)
{
    const char *src = (const char *)table + (size_t)r.word0 * table_stride * (dtype == TENSAIR_F32 ? 4 : 2);
    x.w = lay_out(s, src, table_stride, r.words, r.rows, D, Labels{}, 1.f, b.w, &x.w_blocks);
    const dim3 grid((unsigned)(x.token_blocks + x.unit_block + x.h_blocks + x.w_blocks)), blk(BLOCK);
    if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_lay_out<float>, grid, blk, 0, st, x);
    else hipLaunchKernelGGL(k_lay_out<bf16_t>, grid, blk, 0, st, x);
    x.token_blocks = x.h_blocks = x.unit_block = 0;
    LogitsArgs a;
    memset(&a, 0, sizeof(a));
    a.w = Operand{b.w, r.rows, r.rows * s.Dp};
    a.h = Operand{b.h, s.Np, s.Np * s.Dp};
    a.K = s.Dp;
    a.word0 = r.word0;
    a.V = V;
    a.tiles = (int)r.tiles * s.unit;
    a.per = s.per;
    a.strips = (int)cdiv(a.tiles, s.per);
    a.token_tiles = s.token_tiles;
    a.Np = s.Np;
    a.c = fabsf(scale) * LOG2E;
    a.table = (const float *)table;
    a.table_stride = table_stride;
    a.hidden = (const float *)x.h.src;
    a.hidden_stride = x.h.stride;
    a.n = x.h.rows;
    a.D = D;
    a.sign = x.h.sign;
    a.label = b.label;
    a.part = b.part;
    a.picked = b.picked;
    a.lse2 = b.lse2;
    a.d = b.d;
    a.unit = b.unit;
    a.rest = b.rest;
    a.dz = b.dz;
    a.dz_plane = s.Np * s.range_tiles * SM_BM;
    return a;
}
template <typename T, int NT, bool GRAD>
void launch_few_n(const FewArgs &a, int blocks, hipStream_t st)
{
    const dim3 grid((unsigned)blocks), blk(BLOCK);
    if (a.C4 <= 32) hipLaunchKernelGGL((k_few<T, 16, 2, NT, GRAD>), grid, blk, 0, st, a);
    else if (a.C4 <= 96) hipLaunchKernelGGL((k_few<T, 32, 3, NT, GRAD>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_few<T, 64, 4, NT, GRAD>), grid, blk, 0, st, a);
}
template <typename T, bool GRAD>
void launch_few_t(const FewArgs &a, int blocks, hipStream_t st)
{
    if (a.n == 1) launch_few_n<T, 1, GRAD>(a, blocks, st);
    else if (a.n <= 4) launch_few_n<T, 4, GRAD>(a, blocks, st);
    else launch_few_n<T, FEW_TOKENS, GRAD>(a, blocks, st);
}
FewArgs few_args(const SoftmaxPlan &s, const SoftmaxBuffers &b, const void *hidden, i64 hidden_stride, const void *table, i64 table_stride, i64 n,
                 int D, float scale, Labels labels, int *status)
{
    FewArgs a;
    memset(&a, 0, sizeof(a));
    a.hidden = hidden;
    a.table = table;
    a.hidden_stride = hidden_stride;
    a.table_stride = table_stride;
    a.V = labels.V;
    a.n = (int)n;
    a.C4 = D / 4;
    a.c = fabsf(scale) * LOG2E;
    a.sign = scale < 0.f ? -1.f : 1.f;
    a.labels = labels;
    a.status = status;
    a.part = b.part;
    a.picked = b.picked;
    a.slots = b.h_slots;
    a.scale = fabsf(scale);
    return a;
}
template <bool GRAD, int PARTS>
void launch_logits(const SoftmaxPlan &s, const LogitsArgs &a, hipStream_t st)
{
    constexpr int STAGES = PARTS == 1 ? 3 : 2;
    const dim3 grid((unsigned)(a.strips * a.token_tiles)), blk(256);
    if constexpr (PARTS == 1)
        if (s.held) {
            if (s.Dp <= 64) hipLaunchKernelGGL((k_logits_held<2, GRAD>), grid, blk, 0, st, a);
            else if (s.Dp <= 128) hipLaunchKernelGGL((k_logits_held<4, GRAD>), grid, blk, 0, st, a);
            else if (s.Dp <= 192) hipLaunchKernelGGL((k_logits_held<6, GRAD>), grid, blk, 0, st, a);
            else if (s.Dp <= 256) hipLaunchKernelGGL((k_logits_held<8, GRAD>), grid, blk, 0, st, a);
            else hipLaunchKernelGGL((k_logits_held<10, GRAD>), grid, blk, 0, st, a);
            return;
        }
    if (s.bn == SM_BN_FEW) hipLaunchKernelGGL((k_logits<2, 2, 4, 1, STAGES, GRAD, PARTS>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_logits<PARTS == 1 ? 4 : 1, 2, 2, 2, STAGES, GRAD, PARTS>), grid, blk, 0, st, a);
}
template <bool BT>
void launch_product(const SoftmaxPlan &s, const ProductArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)(a.m_tiles * a.n_tiles * a.splits)), blk(256);
    if (s.parts == 3) hipLaunchKernelGGL((k_product<1, 2, 2, 2, 2, 3, BT>), grid, blk, 0, st, a);
    else if (s.tm == 1) hipLaunchKernelGGL((k_product<1, 4, 2, 2, 2, 1, BT>), grid, blk, 0, st, a);
    else if (s.tm == 2) hipLaunchKernelGGL((k_product<2, 4, 2, 2, 2, 1, BT>), grid, blk, 0, st, a);
    else if (s.tm == 3) hipLaunchKernelGGL((k_product<3, 2, 2, 2, 2, 1, BT>), grid, blk, 0, st, a);
    else if (s.tm == 4) hipLaunchKernelGGL((k_product<4, 2, 2, 2, 2, 1, BT>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_product<5, 2, 2, 2, 2, 1, BT>), grid, blk, 0, st, a);
}
void launch_join(const float *slots, int n_slots, i64 rows, i64 stride, int D, Labels labels, void *out, int dtype, float scale, const float *unit,
                 const float *rest, const void *table, i64 table_stride, hipStream_t st)
{
    JoinArgs j = {slots, n_slots, rows, stride, D / 4, labels, out, dtype, scale, unit, rest, (const bf16_t *)table, table_stride};
    // many slots of a small matrix (one token against a million words: 512) want the parallel form, others fill the chip without
    const i64 chunks = rows * (D / 4);
    if (n_slots <= 16 || chunks >= 65536) {
        hipLaunchKernelGGL(k_join_flat, dim3(blocks_for(chunks)), dim3(BLOCK), 0, st, j);
        return;
    }
    hipLaunchKernelGGL(k_join, dim3((unsigned)std::min<i64>(cdiv(rows * (D / 4), WAVE), 1 << 18)), dim3(1024), 0, st, j);
}

}  // namespace

extern "C" {

size_t tensair_softmax_workspace_bytes(int64_t n, int64_t vocab, int32_t dim, int32_t dtype, int32_t with_grad)
{
    if (check_softmax(n, vocab, dim, dtype)) return 0;
    if (n == 0) return 256;
    // The loss has a plan of its own, with more words to a range where dz need not be kept; and fewer tokens may want more than more of
    // them do, since a range then holds more words: the most of all numbers of tokens up to n.
    size_t most = 0;
    auto take = [&](i64 k) {
        most = std::max(most, softmax_carve(plan_of(k, vocab, dim, dtype, false), k, dim, false, nullptr, nullptr));
        if (with_grad) most = std::max(most, softmax_carve(plan_of(k, vocab, dim, dtype, true), k, dim, true, nullptr, nullptr));
    };
    take(std::min<i64>(n, FEW_TOKENS));
    if (n > FEW_TOKENS)
        for (i64 k = SM_CLASS; k < n + SM_CLASS; k += SM_CLASS) take(k);
    return most;
}

int tensair_softmax_loss(const void *hidden, int64_t hidden_stride, const void *table, int64_t table_stride, int32_t dtype, int64_t n,
                         int64_t vocab, int32_t dim, const int32_t *labels, int32_t ignore_label, float scale, float *loss, float *lse,
                         void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_softmax(n, vocab, dim, dtype))) return rc;
    if ((rc = check_scale(scale))) return rc;
    if ((rc = check_rows(hidden, n, hidden_stride, dim, "hidden"))) return rc;
    if ((rc = check_rows(table, vocab, table_stride, dim, "table"))) return rc;
    if (n > 0 && (!labels || !loss || !lse)) return tn_fail(TENSAIR_EINVAL, "NULL pointer argument");
    if (((uintptr_t)labels | (uintptr_t)loss | (uintptr_t)lse | (uintptr_t)status) & 3)
        return tn_fail(TENSAIR_EINVAL, "labels, loss, lse and status must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    const SoftmaxPlan s = plan_of(n, vocab, dim, dtype, false);
    if (workspace_bytes < softmax_carve(s, n, dim, false, nullptr, nullptr))
        return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see tensair_softmax_workspace_bytes");
    if (!workspace || ((uintptr_t)workspace & 255)) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    SoftmaxBuffers b;
    softmax_carve(s, n, dim, false, (char *)workspace, &b);
    hipStream_t st = (hipStream_t)stream;
    const Labels lab = {labels, ignore_label, vocab};
    int slots = 0;
    if (s.few) {
        const FewArgs f = few_args(s, b, hidden, hidden_stride, table, table_stride, n, dim, scale, lab, status);
        if (dtype == TENSAIR_F32) launch_few_t<float, false>(f, s.few_blocks, st);
        else launch_few_t<bf16_t, false>(f, s.few_blocks, st);
        slots = s.few_blocks;
    } else {
        LayOutArgs x;
        memset(&x, 0, sizeof(x));
        x.tokens = TokenArgs{lab, nullptr, nullptr, n, s.Np, b.label, status, nullptr, nullptr, nullptr};
        x.token_blocks = (int)cdiv(s.Np, BLOCK);
        x.h = lay_out(s, hidden, hidden_stride, n, s.Np, dim, Labels{}, scale < 0.f ? -1.f : 1.f, b.h, &x.h_blocks);
        for (i64 range = 0; range < s.ranges; ++range) {
            LogitsArgs a = lay_out_range(s, b, range_of(s, range, vocab), x, table, table_stride, dtype, dim, vocab, scale, st);
            a.part += (i64)slots * s.Np;
            if (s.parts == 1) launch_logits<false, 1>(s, a, st);
            else launch_logits<false, 3>(s, a, st);
            slots += a.strips * s.wm;
        }
    }
    LossArgs l = {b.part, slots, s.Np, n, b.picked, lab, loss, lse};
    if (s.few) hipLaunchKernelGGL(k_loss_few, dim3((unsigned)n), dim3(BLOCK), 0, st, l);
    else hipLaunchKernelGGL(k_loss, dim3((unsigned)(s.Np / WAVE)), dim3(1024), 0, st, l);
    return launched("softmax_loss");
}

int tensair_softmax_grad(const void *hidden, int64_t hidden_stride, const void *table, int64_t table_stride, int32_t dtype, int64_t n,
                         int64_t vocab, int32_t dim, const int32_t *labels, int32_t ignore_label, float scale, const float *lse,
                         const float *d_loss, void *d_hidden, int64_t d_hidden_stride, void *d_table, int64_t d_table_stride,
                         void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_softmax(n, vocab, dim, dtype))) return rc;
    if ((rc = check_scale(scale))) return rc;
    if ((rc = check_rows(hidden, n, hidden_stride, dim, "hidden"))) return rc;
    if ((rc = check_rows(table, vocab, table_stride, dim, "table"))) return rc;
    if (d_hidden && (rc = check_rows(d_hidden, n, d_hidden_stride, dim, "d_hidden"))) return rc;
    if (d_table && (rc = check_rows(d_table, vocab, d_table_stride, dim, "d_table"))) return rc;
    if (n > 0 && (!labels || !lse || !d_loss)) return tn_fail(TENSAIR_EINVAL, "NULL pointer argument");
    if (((uintptr_t)labels | (uintptr_t)lse | (uintptr_t)d_loss | (uintptr_t)status) & 3)
        return tn_fail(TENSAIR_EINVAL, "labels, lse, d_loss and status must be 4-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    if (!d_hidden && !d_table) return TENSAIR_OK;
    if (n == 0) {                                             // a sum over nothing
        if (d_table)
            hipLaunchKernelGGL(k_zero_rows, dim3(blocks_for(vocab * (dim / 4))), dim3(BLOCK), 0, st, d_table, (int)dtype, vocab, d_table_stride, dim / 4);
        return launched("softmax_grad");
    }
    const SoftmaxPlan s = plan_of(n, vocab, dim, dtype, true);
    if (workspace_bytes < softmax_carve(s, n, dim, true, nullptr, nullptr))
        return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see tensair_softmax_workspace_bytes");
    if (!workspace || ((uintptr_t)workspace & 255)) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    SoftmaxBuffers b;
    softmax_carve(s, n, dim, true, (char *)workspace, &b);
    const Labels lab = {labels, ignore_label, vocab};
    if (s.few) {
        FewArgs f = few_args(s, b, hidden, hidden_stride, table, table_stride, n, dim, scale, lab, status);
        f.lse = lse;
        f.d_loss = d_loss;
        f.d_table = d_table;
        f.d_stride = d_table_stride;
        if (dtype == TENSAIR_F32) launch_few_t<float, true>(f, s.few_blocks, st);
        else launch_few_t<bf16_t, true>(f, s.few_blocks, st);
        if (d_hidden) launch_join(b.h_slots, s.few_blocks, n, d_hidden_stride, dim, lab, d_hidden, dtype, scale, nullptr, nullptr, nullptr, 0, st);
        return launched("softmax_grad");
    }
    LayOutArgs x;
    memset(&x, 0, sizeof(x));
    x.tokens = TokenArgs{lab, lse, d_loss, n, s.Np, b.label, status, b.lse2, b.d, b.unit};
    x.unit_block = b.unit ? 1 : 0;
    x.token_blocks = (int)cdiv(s.Np, BLOCK);
    x.h = lay_out(s, hidden, hidden_stride, n, s.Np, dim, lab, scale < 0.f ? -1.f : 1.f, b.h, &x.h_blocks);   // what a token without a loss holds must reach no sum
    for (i64 range = 0; range < s.ranges; ++range) {
        const Range r = range_of(s, range, vocab);
        const LogitsArgs a = lay_out_range(s, b, r, x, table, table_stride, dtype, dim, vocab, scale, st);
        if (s.parts == 1) launch_logits<true, 1>(s, a, st);
        else launch_logits<true, 3>(s, a, st);
        const Operand dz = {b.dz, s.Np, a.dz_plane};
        ProductArgs p;
        memset(&p, 0, sizeof(p));
        p.m_tiles = s.m_tiles;
        p.M = dim;
        p.dtype = dtype;
        p.scale = scale;
        p.unit = b.unit;
        if (d_hidden) {
            p.a = a.w;
            p.b = dz;
            p.N = n;
            p.K = cdiv(r.words, BK) * BK;
            p.n_tiles = (int)cdiv(n, s.pn);
            p.k_per = s.h_k;
            p.splits = (int)cdiv(p.K, p.k_per);
            p.slots = b.h_slots;                              // the first range has all splits, the last may have fewer
            p.add = range > 0;
            launch_product<false>(s, p, st);
            p.add = 0;
        }
        if (d_table) {
            p.scale = fabsf(scale);                           // the tokens' rows have its sign
            p.a = a.h;
            p.b = dz;
            p.N = r.words;
            p.K = cdiv(n, BK) * BK;
            p.n_tiles = (int)cdiv(r.words, s.pn);
            p.k_per = s.t_k;
            p.splits = s.t_splits;
            p.slots = s.t_splits > 1 ? b.t_slots : nullptr;
            char *out = (char *)d_table + (size_t)r.word0 * d_table_stride * (dtype == TENSAIR_F32 ? 4 : 2);
            p.out = out;
            p.out_stride = d_table_stride;
            launch_product<true>(s, p, st);
            if (s.t_splits > 1) launch_join(b.t_slots, s.t_splits, r.words, d_table_stride, dim, Labels{}, out, dtype, fabsf(scale), b.unit, nullptr, nullptr, 0, st);
        }
    }
    if (d_hidden) {
        const int slots = (int)cdiv(cdiv(range_of(s, 0, vocab).words, BK) * BK, s.h_k);
        launch_join(b.h_slots, slots, n, d_hidden_stride, dim, lab, d_hidden, dtype, scale, b.unit, b.rest, table, table_stride, st);
    }
    return launched("softmax_grad");
}

}  // extern "C"
