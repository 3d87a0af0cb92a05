// Softmax cross entropy against every row of a table, and its gradient.  With z = scale * hidden table^T (tokens by words),
//   lse_i = log sum_v exp z_iv,   loss_i = lse_i - z_i,label,   dz_iv = d_i (exp(z_iv - lse_i) - [v = label_i]),
//   d_hidden = scale * dz table,   d_table = scale * dz^T hidden.
// The logits are never kept: the loss makes a pass over the words with a running maximum and sum per token; the gradient makes
// the logits once more, a range of words at a time, and keeps dz of that range in bfloat16 for the two products.
// All products are tiles of matrix instructions in bfloat16 with fp32 sums.  fp32 inputs are three bfloat16 parts each (24 bits
// together), and of the nine products of parts the six that matter at 2^-24 are summed, the smallest first.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "../../include/tensair.h"
#include "dev_common.h"
#include "kernels.h"

namespace {

typedef short bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 hw_bf16x8 __attribute__((ext_vector_type(8)));
typedef short bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef u32 v4u __attribute__((ext_vector_type(4)));

#define LOG2E 1.44269504088896340736f
#define LN2 0.69314718055994530942f
#define BK 64                  // elements of the summed index per step
#define T_PAD 32               // elements behind a row of a tile kept by rows of the summed index: four rows, four groups of banks

// A matrix of bfloat16 parts in memory.
struct Operand {
    const bf16_t *p;
    i64 pitch, plane;          // elements from row to row, from part to part
    i64 rows, cols;
};
// which parts of either operand a product's segment takes, two bits each: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
#define PARTS_A 0x052u         // 2 0 1 1 0 0
#define PARTS_B 0x118u         // 0 2 1 0 1 0
__device__ __forceinline__ int part_a(int seg, int nseg) { return nseg == 1 ? 0 : (int)(PARTS_A >> (2 * seg)) & 3; }
__device__ __forceinline__ int part_b(int seg, int nseg) { return nseg == 1 ? 0 : (int)(PARTS_B >> (2 * seg)) & 3; }

// the bytes of a buffer that begins at row r, column c
__device__ __forceinline__ u32 bytes_left(const Operand &o, i64 r, i64 c)
{
    const i64 n = r < o.rows ? ((o.rows - 1 - r) * o.pitch + o.cols - c) * 2 : 0;
    return (u32)(n < 0 ? 0 : n > 0x7FFFFFF0 ? 0x7FFFFFF0 : n);
}

// The tile of one operand of one step, ROWS of the kept index by BK of the summed one, from memory into registers and from there
// into LDS.  By rows of the kept index (T = false): rows of 128 bytes whose chunks of 16 change places by the row's number, so
// that the 32 lanes of a fragment spread over the banks.  By rows of the summed index (T = true): as in memory, padded;
// fragments are read with the transposing load.  What lies outside the matrix comes as zero.
template <int ROWS, int THREADS, bool T>
struct Tile {
    static constexpr int CHUNKS = ROWS * BK / 8, PER = CHUNKS / THREADS;
    static constexpr int PITCH = T ? ROWS + T_PAD : BK;       // elements
    static constexpr int LDS = (T ? BK : ROWS) * PITCH;       // elements
    static_assert(CHUNKS % THREADS == 0, "");
    v4u r[PER];

    __device__ __forceinline__ void load(const Operand &o, int part, i64 row0, i64 k0)
    {
        const i64 r0 = T ? k0 : row0, c0 = T ? row0 : k0;
        const bf16_t *base = o.p + part * o.plane + r0 * o.pitch + c0;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)bytes_left(o, r0, c0), 0x00027000);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int q = (int)threadIdx.x + j * THREADS;
            const int row = T ? q / (ROWS / 8) : q / 8, c = T ? q % (ROWS / 8) : q % 8;
            r[j] = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)((u32)row * (u32)o.pitch + 8u * c) * 2, 0, 0);
        }
    }
    __device__ __forceinline__ void store(bf16_t *lds) const
    {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int q = (int)threadIdx.x + j * THREADS;
            const int row = T ? q / (ROWS / 8) : q / 8, c = T ? q % (ROWS / 8) : q % 8;
            const int at = T ? row * PITCH + 8 * c : row * PITCH + 8 * (c ^ (row & 7));
            *(v4u *)(lds + at) = r[j];
        }
    }
    // the fragment of 32 rows from `row` on, 16 of the summed index from 16 * kk on: lane l holds row l % 32, 8 * (l / 32) and on
    static __device__ __forceinline__ hw_bf16x8 fragment(const bf16_t *lds, int row, int kk)
    {
        const int lane = lane_id();
        if constexpr (!T) {
            const int m = row + (lane & 31), c = 2 * kk + (lane >> 5);
            return *(const hw_bf16x8 *)(lds + m * PITCH + 8 * (c ^ (m & 7)));
        } else {
            typedef __attribute__((address_space(3))) bf16x4 lds4;
            const int g = lane >> 4, i = lane & 15;
            const bf16_t *at = lds + (16 * kk + 8 * (g >> 1) + (i >> 2)) * PITCH + row + 16 * (g & 1) + 4 * (i & 3);
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)at);
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(at + 4 * PITCH));
            const bf16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(hw_bf16x8, v);
        }
    }
};

// A workgroup's tile of a product: BM of A's rows by BN of B's, WM by WN waves of TM by TN fragments of 32 by 32.  Lane l of a
// fragment holds the column (B's row) l % 32 and the rows (A's) 8 (r / 4) + 4 (l / 32) + r % 4 in its 16 registers r.
template <int TM, int TN, int WM, int WN, bool AT, bool BT>
struct Product {
    static constexpr int THREADS = 64 * WM * WN, BM = 32 * TM * WM, BN = 32 * TN * WN;
    typedef Tile<BM, THREADS, AT> A;
    typedef Tile<BN, THREADS, BT> B;
    static constexpr int LDS = A::LDS + B::LDS;               // elements
    f32x16 acc[TM][TN];
    A a;
    B b;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }
    // the registers' tiles into LDS, once every wave is done with what is there
    __device__ __forceinline__ void stage(bf16_t *lds)
    {
        __syncthreads();
        a.store(lds);
        b.store(lds + A::LDS);
        __syncthreads();
    }
    __device__ __forceinline__ void multiply(const bf16_t *lds, int wm, int wn)
    {
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            hw_bf16x8 fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = A::fragment(lds, (wm * TM + i) * 32, kk);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = B::fragment(lds + A::LDS, (wn * TN + j) * 32, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
        }
    }
};

// Workgroups that follow one another go to the eight dies in turn: work w of n such that a die's workgroups take neighbouring work.
__device__ __forceinline__ int die_order(int b, int n)
{
    const int die = b % 8, i = b / 8, share = n / 8, more = n % 8;
    return die * share + min(die, more) + i;
}

// ---------------------------------------------------------------- logits
struct LogitsArgs {
    Operand w, h;              // words' and tokens' rows
    int nseg, ksteps;
    i64 word0, V;              // first word of this launch's range; words in all
    int tiles, per, strips;    // tiles of words of the range, of a strip; strips
    int token_tiles;
    i64 Np;
    float c;                   // scale * log2(e)
    const int *label;          // [Np], -1: none
    // loss
    float2 *part;              // [strips * WM][Np] maximum, sum (of powers of two)
    float *picked;             // [Np] the label's logit, in units of log 2
    // gradient
    const float *lse2, *d;     // [Np]
    bf16_t *dz;                // [parts][Np][pitch]
    i64 dz_pitch, dz_plane;
};

__device__ __forceinline__ u32 pack2(float a, float b) { return (u32)f32_to_bf16(a) | ((u32)f32_to_bf16(b) << 16); }

// the four registers of a group of 4 rows from this lane and its partner 32 lanes on: 8 rows that follow one another (lanes below
// 32: of group x, the others: of group y), as bfloat16
__device__ __forceinline__ v4u join_halves(u32 x0, u32 x1, u32 y0, u32 y1)
{
    // the upper half of x for the lower half of y
    const auto p = __builtin_amdgcn_permlane32_swap(x0, y0, false, false);
    const auto q = __builtin_amdgcn_permlane32_swap(x1, y1, false, false);
    return v4u{(u32)p[0], (u32)q[0], (u32)p[1], (u32)q[1]};
}

// GRAD false: the running maximum and sum of every token over a strip of words; true: dz of the strip, in PARTS bfloat16 parts.
// A strip's tiles follow one another without a pause: the next tile's first step is in flight while this one's logits are used.
template <int TM, int TN, int WM, int WN, bool GRAD, int PARTS>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_logits(LogitsArgs a)
{
    typedef Product<TM, TN, WM, WN, false, false> P;
    __shared__ __attribute__((aligned(16))) bf16_t lds[P::LDS];
    const int work = die_order((int)blockIdx.x, (int)gridDim.x);
    const int strip = work / a.token_tiles, tt = work % a.token_tiles;
    const int wave = uniform((int)(threadIdx.x >> 6)), wm = wave / WN, wn = wave % WN, lane = lane_id();
    const i64 tok0 = (i64)tt * P::BN;
    const int t0 = strip * a.per, t1 = min(a.tiles, t0 + a.per), steps = a.ksteps * a.nseg;
    P p;
    float top[TN], sum[TN], l2[TN], d[TN];
    int label[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const i64 tok = tok0 + (wn * TN + j) * 32 + (lane & 31);
        label[j] = a.label[tok];
        top[j] = -INFINITY;
        sum[j] = 0.f;
        if (GRAD) {
            l2[j] = a.lse2[tok];
            d[j] = a.d[tok];
        }
    }
    i64 word = a.word0 + (i64)t0 * P::BM;
    p.a.load(a.w, part_a(0, a.nseg), word, 0);
    p.b.load(a.h, part_b(0, a.nseg), tok0, 0);
    for (int t = t0; t < t1; ++t, word += P::BM) {
        p.clear();
        int k = 0, seg = 0;
        for (int s = 0; s < steps; ++s) {
            p.stage(lds);
            i64 next = word;
            if (++k == a.ksteps) {
                k = 0;
                if (++seg == a.nseg) {
                    seg = 0;
                    next += P::BM;                            // behind the strip's last a tile is loaded that nobody uses
                }
            }
            p.a.load(a.w, part_a(seg, a.nseg), next, (i64)k * BK);
            p.b.load(a.h, part_b(seg, a.nseg), tok0, (i64)k * BK);
            p.multiply(lds, wm, wn);
        }
        const i64 w0 = word + wm * TM * 32;
        const bool whole = word + P::BM <= a.V;
        if constexpr (!GRAD) {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                float best = -INFINITY;
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const i64 lw = (i64)label[j] - (w0 + 32 * i);              // the label's row in this fragment
                    if (__ballot(lw >= 0 && lw < 32)) {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (lw == 8 * (r / 4) + 4 * (lane >> 5) + r % 4)
                                a.picked[tok0 + (wn * TN + j) * 32 + (lane & 31)] = p.acc[i][j][r] * a.c;
                    }
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        float z = p.acc[i][j][r] * a.c;
                        if (!whole && w0 + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4 >= a.V) z = -INFINITY;
                        p.acc[i][j][r] = z;
                        best = fmaxf(best, z);
                    }
                }
                const float now = fmaxf(best, top[j]), ref = now == -INFINITY ? 0.f : now;
                float s = sum[j] * __builtin_amdgcn_exp2f(top[j] - ref);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s += __builtin_amdgcn_exp2f(p.acc[i][j][r] - ref);
                top[j] = now;
                sum[j] = s;
            }
        } else {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                bf16_t *row = a.dz + (tok0 + (wn * TN + j) * 32 + (lane & 31)) * a.dz_pitch + (w0 - a.word0) + 8 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const i64 lw = (i64)label[j] - (w0 + 32 * i);
                    const bool any = __ballot(lw >= 0 && lw < 32) != 0;
                    float g[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) g[r] = d[j] * __builtin_amdgcn_exp2f(fmaf(p.acc[i][j][r], a.c, -l2[j]));
                    if (any) {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (lw == 8 * (r / 4) + 4 * (lane >> 5) + r % 4)
                                g[r] = d[j] * (__builtin_amdgcn_exp2f(fmaf(p.acc[i][j][r], a.c, -l2[j])) - 1.0f);
                    }
                    if (!whole) {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (w0 + 32 * i + 8 * (r / 4) + 4 * (lane >> 5) + r % 4 >= a.V) g[r] = 0.f;
                    }
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        u32 q[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) q[r] = pack2(g[2 * r], g[2 * r + 1]);
                        bf16_t *to = row + part * a.dz_plane + 32 * i;
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
    }
    if constexpr (!GRAD) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const float ot = __shfl_xor(top[j], 32, WAVE), os = __shfl_xor(sum[j], 32, WAVE);
            const float now = fmaxf(top[j], ot), ref = now == -INFINITY ? 0.f : now;
            const float s = sum[j] * __builtin_amdgcn_exp2f(top[j] - ref) + os * __builtin_amdgcn_exp2f(ot - ref);
            if (lane < 32) a.part[(i64)(strip * WM + wm) * a.Np + tok0 + (wn * TN + j) * 32 + lane] = make_float2(now, s);
        }
    }
}

// maxima and sums of the strips put together: a workgroup takes 64 tokens, its waves the strips in turn
struct LossArgs {
    const float2 *part;
    int slots;
    i64 Np, n;
    const float *picked;
    const int *label;
    float *loss, *lse;
};
__global__ void __launch_bounds__(1024) k_loss(LossArgs a)
{
    __shared__ float2 other[16][WAVE];
    const int lane = lane_id(), wave = (int)(threadIdx.x >> 6);
    const i64 i = (i64)blockIdx.x * WAVE + lane;
    float top = -INFINITY, sum = 0.f;
    for (int s = wave; s < a.slots; s += 16) {
        const float2 v = a.part[(i64)s * a.Np + i];
        const float now = fmaxf(top, v.x), ref = now == -INFINITY ? 0.f : now;
        sum = sum * __builtin_amdgcn_exp2f(top - ref) + v.y * __builtin_amdgcn_exp2f(v.x - ref);
        top = now;
    }
    other[wave][lane] = make_float2(top, sum);
    __syncthreads();
    if (wave > 0 || i >= a.n) return;
    for (int w = 1; w < 16; ++w) {
        const float2 v = other[w][lane];
        const float now = fmaxf(top, v.x), ref = now == -INFINITY ? 0.f : now;
        sum = sum * __builtin_amdgcn_exp2f(top - ref) + v.y * __builtin_amdgcn_exp2f(v.x - ref);
        top = now;
    }
    const float lse = top + log2f(sum);
    a.lse[i] = lse * LN2;
    a.loss[i] = a.label[i] >= 0 ? (lse - a.picked[i]) * LN2 : 0.f;
}

// ---------------------------------------------------------------- products with dz
struct ProductArgs {
    Operand a, b;              // C[n][m] = sum_k a(m, k) b(n, k)
    int nseg;
    i64 M, N, K;
    int m_tiles, n_tiles, splits;
    i64 k_per;                 // of a split, a multiple of BK
    float *slots;              // [splits][N][M] sums (NULL: written as the output)
    void *out;
    i64 out_stride;
    int dtype;
    float scale;
};
template <int TM, int TN, int WM, int WN, bool BT>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_product(ProductArgs a)
{
    typedef Product<TM, TN, WM, WN, true, BT> P;
    __shared__ __attribute__((aligned(16))) bf16_t lds[P::LDS];
    int work = die_order((int)blockIdx.x, (int)gridDim.x);
    const int mt = work % a.m_tiles;
    work /= a.m_tiles;
    const int nt = work % a.n_tiles, split = work / a.n_tiles;
    const int wave = uniform((int)(threadIdx.x >> 6)), wm = wave / WN, wn = wave % WN, lane = lane_id();
    const i64 m0 = (i64)mt * P::BM, n0 = (i64)nt * P::BN;
    const i64 k0 = split * a.k_per, k1 = min(a.K, k0 + a.k_per);
    P p;
    p.clear();
    p.a.load(a.a, part_a(0, a.nseg), m0, k0);
    p.b.load(a.b, part_b(0, a.nseg), n0, k0);
    const int steps = (int)((k1 - k0) / BK) * a.nseg;
    int seg = 0;
    i64 k = k0;
    for (int s = 0; s < steps; ++s) {
        p.stage(lds);
        k += BK;
        if (k >= k1) {
            k = k0;
            seg = min(seg + 1, a.nseg - 1);                   // behind the last step a tile is loaded that nobody uses
        }
        p.a.load(a.a, part_a(seg, a.nseg), m0, k);
        p.b.load(a.b, part_b(seg, a.nseg), n0, k);
        p.multiply(lds, wm, wn);
    }
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
                    v = make_float4(v.x * a.scale, v.y * a.scale, v.z * a.scale, v.w * a.scale);
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
    const int *label;
    void *out;
    int dtype;
    float scale;
};
__global__ void __launch_bounds__(BLOCK) k_join(JoinArgs a)
{
    const i64 all = a.n * a.C4;
    for (i64 c = (i64)blockIdx.x * BLOCK + threadIdx.x; c < all; c += (i64)gridDim.x * BLOCK) {
        const i64 row = c / a.C4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!a.label || a.label[row] >= 0) {
            for (int s = 0; s < a.n_slots; ++s) {
                const float4 x = ld4(a.slots + ((i64)s * all + c) * 4);
                v.x += x.x;
                v.y += x.y;
                v.z += x.z;
                v.w += x.w;
            }
            v = make_float4(v.x * a.scale, v.y * a.scale, v.z * a.scale, v.w * a.scale);
        }
        const i64 at = row * a.stride + 4 * (c - row * a.C4);
        if (a.dtype == TENSAIR_F32) st4((float *)a.out + at, v);
        else st4((bf16_t *)a.out + at, v);
    }
}

// ---------------------------------------------------------------- inputs laid out for the products
struct PackArgs {
    const void *src;
    i64 stride, rows;          // of the source
    int D, Dp;                 // columns, of the copy (zero from D on)
    i64 out_rows, plane;       // rows of the copy (zero from `rows` on), elements from part to part
    bf16_t *out;
    const int *label;          // rows without a label are zero (NULL: none are)
};
template <typename T>
__global__ void __launch_bounds__(BLOCK) k_parts(PackArgs a)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    const int C4 = a.Dp / 4;
    const i64 all = a.out_rows * C4;
    for (i64 c = (i64)blockIdx.x * BLOCK + threadIdx.x; c < all; c += (i64)gridDim.x * BLOCK) {
        const i64 row = c / C4;
        const int col = 4 * (int)(c - row * C4);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < a.rows && col < a.D && (!a.label || a.label[row] >= 0)) v = ld4((const T *)a.src + row * a.stride + col);
        float x[4] = {v.x, v.y, v.z, v.w};
        bf16_t *to = a.out + row * a.Dp + col;
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            bf16_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[k] = f32_to_bf16(x[k]);
                if (PARTS > 1) {
                    // beyond the largest bfloat16: cut, so that the rest is finite
                    if ((h[k] & 0x7FFFu) == 0x7F80u && fabsf(x[k]) < INFINITY) h[k] = (bf16_t)((h[k] & 0x8000u) | 0x7F7Fu);
                    x[k] = (h[k] & 0x7F80u) == 0x7F80u ? 0.f : x[k] - bf16_to_f32(h[k]);
                }
            }
            *(uint2 *)(to + part * a.plane) = make_uint2((u32)h[0] | ((u32)h[1] << 16), (u32)h[2] | ((u32)h[3] << 16));
        }
    }
}

// what the kernels need of every token, padded ones among them
struct TokenArgs {
    const int *labels;
    const float *lse, *d_loss; // NULL: for the loss
    i64 n, Np, V;
    int ignore;
    int *label, *status;
    float *lse2, *d;
};
__global__ void __launch_bounds__(BLOCK) k_tokens(TokenArgs a)
{
    const i64 i = (i64)blockIdx.x * BLOCK + threadIdx.x;
    if (i >= a.Np) return;
    int y = -1;
    if (i < a.n) {
        const int l = a.labels[i];
        if ((u64)(u32)l < (u64)a.V && l != a.ignore) y = l;
        else if (l != a.ignore && a.status) atomicOr(a.status, ST_BAD_ID);
    }
    a.label[i] = y;
    if (a.lse) {
        a.lse2[i] = y >= 0 ? a.lse[i] * LOG2E : 0.f;
        a.d[i] = y >= 0 ? a.d_loss[i] : 0.f;
    }
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

#define SM_BM 256              // words of a tile of logits
#define SM_BN 128              // tokens of one
#define SM_BN_FEW 64           // ... where there are at most so many
#define SM_WAVES_M 2           // rows of waves of a tile, each with a maximum and a sum of its own
#define SM_BLOCKS 512          // workgroups that fill the chip, two to a compute unit
#define SM_DZ_BYTES ((i64)512 << 20)

struct SoftmaxPlan {
    int parts, nseg, Dp, ksteps, bn, token_tiles, wm;
    bool pack;                 // the table is copied (padded, or in parts)
    i64 Np, tiles;             // tokens, padded; tiles of words
    int per, strips;           // loss: tiles to a strip
    // gradient
    i64 range_tiles, ranges;   // tiles of words whose dz is kept at a time
    int dz_per, dz_strips;
    int tm, m_tiles;           // of the products: fragments of a wave along the row length, tiles
    int h_splits, t_splits;    // of d_hidden's sum over a range's words, of d_table's over the tokens
    i64 h_k, t_k;
};

SoftmaxPlan plan_of(i64 n, i64 V, int D, int dtype, i64 table_stride, const void *table)
{
    SoftmaxPlan s;
    memset(&s, 0, sizeof(s));
    s.parts = dtype == TENSAIR_F32 ? 3 : 1;
    s.nseg = dtype == TENSAIR_F32 ? 6 : 1;
    s.Dp = (int)cdiv(D, BK) * BK;
    s.ksteps = s.Dp / BK;
    s.pack = dtype == TENSAIR_F32 || D % BK || table_stride % 8 || ((uintptr_t)table & 15);
    const bool few = n <= SM_BN_FEW;
    s.bn = few ? SM_BN_FEW : SM_BN;
    s.wm = few ? 4 : SM_WAVES_M;
    s.Np = cdiv(n, s.bn) * s.bn;
    s.token_tiles = (int)(s.Np / s.bn);
    s.tiles = cdiv(V, SM_BM);
    const i64 want = std::max<i64>(1, std::min<i64>(s.tiles, cdiv(SM_BLOCKS * 2, s.token_tiles)));
    s.per = (int)cdiv(s.tiles, want);
    s.strips = (int)cdiv(s.tiles, s.per);
    s.range_tiles = std::max<i64>(1, std::min(s.tiles, SM_DZ_BYTES / (s.Np * SM_BM * 2 * s.parts)));
    s.ranges = cdiv(s.tiles, s.range_tiles);
    s.range_tiles = cdiv(s.tiles, s.ranges);
    s.ranges = cdiv(s.tiles, s.range_tiles);
    const i64 dz_want = std::max<i64>(1, std::min<i64>(s.range_tiles, cdiv(SM_BLOCKS * 2, s.token_tiles)));
    s.dz_per = (int)cdiv(s.range_tiles, dz_want);
    s.dz_strips = (int)cdiv(s.range_tiles, s.dz_per);
    // fragments of a wave (two to a tile along the row length): the fewest columns beyond the row, then the largest tile
    i64 least = -1;
    for (int tm = 1; tm <= 5; ++tm) {
        const i64 cols = cdiv(s.Dp, 64 * tm) * 64 * tm;
        if (least < 0 || cols <= least) {
            least = cols;
            s.tm = tm;
        }
    }
    s.m_tiles = (int)cdiv(s.Dp, 64 * s.tm);
    const i64 range_words = s.range_tiles * SM_BM;
    const i64 h_tiles = s.m_tiles * cdiv(s.Np, 128), t_tiles = s.m_tiles * cdiv(range_words, 128);
    i64 splits = std::max<i64>(1, std::min<i64>(cdiv(SM_BLOCKS, h_tiles), range_words / 512));
    s.h_k = cdiv(cdiv(range_words, splits), BK) * BK;
    s.h_splits = (int)cdiv(range_words, s.h_k);
    splits = std::max<i64>(1, std::min<i64>(SM_BLOCKS / t_tiles, s.Np / 512));
    s.t_k = cdiv(cdiv(s.Np, splits), BK) * BK;
    s.t_splits = (int)cdiv(s.Np, s.t_k);
    return s;
}

struct SoftmaxBuffers {
    int *label;
    float *lse2, *d, *picked, *h_slots, *t_slots;
    bf16_t *h, *w, *dz;
    float2 *part;
};
size_t softmax_carve(const SoftmaxPlan &s, i64 n, i64 V, int D, bool grad, char *base, SoftmaxBuffers *b)
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
    x.h = (bf16_t *)take(2 * (size_t)s.Np * s.Dp * s.parts);
    if (s.pack) x.w = (bf16_t *)take(2 * (size_t)V * s.Dp * s.parts);
    const size_t head = at;
    x.picked = (float *)take(4 * (size_t)s.Np);
    x.part = (float2 *)take(8 * (size_t)s.strips * s.wm * s.Np);
    const size_t loss_end = at;
    at = head;
    if (grad) {
        x.lse2 = (float *)take(4 * (size_t)s.Np);
        x.d = (float *)take(4 * (size_t)s.Np);
        x.dz = (bf16_t *)take(2 * (size_t)s.Np * s.range_tiles * SM_BM * s.parts);
        x.h_slots = (float *)take(4 * (size_t)s.ranges * s.h_splits * n * D);
        if (s.t_splits > 1) x.t_slots = (float *)take(4 * (size_t)s.t_splits * s.range_tiles * SM_BM * D);
    }
    if (b) *b = x;
    return std::max(at, loss_end);
}

int check_softmax(i64 n, i64 vocab, int32_t dim, int32_t dtype)
{
    if (n < 0 || n > TENSAIR_MAX_TOKENS) return tn_fail(TENSAIR_EINVAL, "n outside 0..TENSAIR_MAX_TOKENS");
    if (vocab < 1 || vocab > TENSAIR_MAX_VOCAB) return tn_fail(TENSAIR_EINVAL, "vocab outside 1..TENSAIR_MAX_VOCAB");
    if (dim < 4 || dim > TENSAIR_MAX_DIM || dim % 4) return tn_fail(TENSAIR_EINVAL, "dim must be a multiple of 4 in 4..1024");
    if (dtype != TENSAIR_F32 && dtype != TENSAIR_BF16) return tn_fail(TENSAIR_EINVAL, "unknown dtype");
    return TENSAIR_OK;
}
int check_rows(const void *p, i64 rows, i64 stride, int32_t dim, const char *what)
{
    if (rows > 0 && !p) return tn_fail(TENSAIR_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p & 15) return tn_fail(TENSAIR_EINVAL, "%s must be 16-byte aligned", what);
    if (stride < dim || stride % 4) return tn_fail(TENSAIR_EINVAL, "%s: the row stride must be >= dim and a multiple of 4", what);
    return TENSAIR_OK;
}

// tokens, hidden and, where it is copied, the table
void lay_out(const SoftmaxPlan &s, const SoftmaxBuffers &b, const void *hidden, i64 hidden_stride, const void *table, i64 table_stride,
             int dtype, i64 n, i64 V, int D, bool grad, hipStream_t st)
{
    PackArgs p;
    memset(&p, 0, sizeof(p));
    p.D = D;
    p.Dp = s.Dp;
    for (int side = 0; side < (s.pack ? 2 : 1); ++side) {
        p.src = side ? table : hidden;
        p.stride = side ? table_stride : hidden_stride;
        p.rows = side ? V : n;
        p.out_rows = side ? V : s.Np;
        p.plane = p.out_rows * s.Dp;
        p.out = side ? b.w : b.h;
        p.label = !side && grad ? b.label : nullptr;      // what a token without a loss holds must reach no sum
        const dim3 grid(blocks_for(p.out_rows * (s.Dp / 4))), blk(BLOCK);
        if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_parts<float>, grid, blk, 0, st, p);
        else hipLaunchKernelGGL(k_parts<bf16_t>, grid, blk, 0, st, p);
    }
}
LogitsArgs logits_args(const SoftmaxPlan &s, const SoftmaxBuffers &b, const void *table, i64 table_stride, i64 V, float scale)
{
    LogitsArgs a;
    memset(&a, 0, sizeof(a));
    a.w = s.pack ? Operand{b.w, s.Dp, V * s.Dp, V, s.Dp} : Operand{(const bf16_t *)table, table_stride, 0, V, s.Dp};
    a.h = Operand{b.h, s.Dp, s.Np * s.Dp, s.Np, s.Dp};
    a.nseg = s.nseg;
    a.ksteps = s.ksteps;
    a.V = V;
    a.token_tiles = s.token_tiles;
    a.Np = s.Np;
    a.c = scale * LOG2E;
    a.label = b.label;
    a.part = b.part;
    a.picked = b.picked;
    a.lse2 = b.lse2;
    a.d = b.d;
    a.dz = b.dz;
    a.dz_pitch = s.range_tiles * SM_BM;
    a.dz_plane = s.Np * a.dz_pitch;
    return a;
}
template <bool GRAD, int PARTS>
void launch_logits(const SoftmaxPlan &s, const LogitsArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)(a.strips * a.token_tiles)), blk(256);
    if (s.bn == SM_BN_FEW) hipLaunchKernelGGL((k_logits<2, 2, 4, 1, GRAD, PARTS>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_logits<4, 2, 2, 2, GRAD, PARTS>), grid, blk, 0, st, a);
}
template <bool BT>
void launch_product(int tm, const ProductArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)(a.m_tiles * a.n_tiles * a.splits)), blk(256);
    switch (tm) {
    case 1: hipLaunchKernelGGL((k_product<1, 2, 2, 2, BT>), grid, blk, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_product<2, 2, 2, 2, BT>), grid, blk, 0, st, a); break;
    case 3: hipLaunchKernelGGL((k_product<3, 2, 2, 2, BT>), grid, blk, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_product<4, 2, 2, 2, BT>), grid, blk, 0, st, a); break;
    default: hipLaunchKernelGGL((k_product<5, 2, 2, 2, BT>), grid, blk, 0, st, a); break;
    }
}
void launch_join(const float *slots, int n_slots, i64 rows, i64 stride, int D, const int *label, void *out, int dtype, float scale, hipStream_t st)
{
    JoinArgs j = {slots, n_slots, rows, stride, D / 4, label, out, dtype, scale};
    hipLaunchKernelGGL(k_join, dim3(blocks_for(rows * (D / 4))), dim3(BLOCK), 0, st, j);
}

}  // namespace

extern "C" {

size_t tensair_softmax_workspace_bytes(int64_t n, int64_t vocab, int32_t dim, int32_t dtype, int32_t with_grad)
{
    if (check_softmax(n, vocab, dim, dtype)) return 0;
    if (n == 0) return 256;
    // as if the table had to be copied: whether it has depends on its stride
    return softmax_carve(plan_of(n, vocab, dim, dtype, 4, nullptr), n, vocab, dim, with_grad != 0, nullptr, nullptr);
}

int tensair_softmax_loss(const void *hidden, int64_t hidden_stride, const void *table, int64_t table_stride, int32_t dtype, int64_t n,
                         int64_t vocab, int32_t dim, const int32_t *labels, int32_t ignore_label, float scale, float *loss, float *lse,
                         void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_softmax(n, vocab, dim, dtype))) return rc;
    if ((rc = check_rows(hidden, n, hidden_stride, dim, "hidden"))) return rc;
    if ((rc = check_rows(table, vocab, table_stride, dim, "table"))) return rc;
    if (n > 0 && (!labels || !loss || !lse)) return tn_fail(TENSAIR_EINVAL, "NULL pointer argument");
    if (((uintptr_t)labels | (uintptr_t)loss | (uintptr_t)lse | (uintptr_t)status) & 3)
        return tn_fail(TENSAIR_EINVAL, "labels, loss, lse and status must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    const SoftmaxPlan s = plan_of(n, vocab, dim, dtype, table_stride, table);
    if (workspace_bytes < softmax_carve(s, n, vocab, dim, false, nullptr, nullptr))
        return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see tensair_softmax_workspace_bytes");
    if (!workspace || ((uintptr_t)workspace & 255)) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    SoftmaxBuffers b;
    softmax_carve(s, n, vocab, dim, false, (char *)workspace, &b);
    hipStream_t st = (hipStream_t)stream;
    TokenArgs t = {labels, nullptr, nullptr, n, s.Np, vocab, ignore_label, b.label, status, nullptr, nullptr};
    hipLaunchKernelGGL(k_tokens, dim3((unsigned)cdiv(s.Np, BLOCK)), dim3(BLOCK), 0, st, t);
    lay_out(s, b, hidden, hidden_stride, table, table_stride, dtype, n, vocab, dim, false, st);
    LogitsArgs a = logits_args(s, b, table, table_stride, vocab, scale);
    a.tiles = (int)s.tiles;
    a.per = s.per;
    a.strips = s.strips;
    launch_logits<false, 1>(s, a, st);
    LossArgs l = {b.part, s.strips * s.wm, s.Np, n, b.picked, b.label, loss, lse};
    hipLaunchKernelGGL(k_loss, dim3((unsigned)(s.Np / WAVE)), dim3(1024), 0, st, l);
    return launched("softmax_loss");
}

int tensair_softmax_grad(const void *hidden, int64_t hidden_stride, const void *table, int64_t table_stride, int32_t dtype, int64_t n,
                         int64_t vocab, int32_t dim, const int32_t *labels, int32_t ignore_label, float scale, const float *lse,
                         const float *d_loss, void *d_hidden, int64_t d_hidden_stride, void *d_table, int64_t d_table_stride,
                         void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_softmax(n, vocab, dim, dtype))) return rc;
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
    const SoftmaxPlan s = plan_of(n, vocab, dim, dtype, table_stride, table);
    if (workspace_bytes < softmax_carve(s, n, vocab, dim, true, nullptr, nullptr))
        return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see tensair_softmax_workspace_bytes");
    if (!workspace || ((uintptr_t)workspace & 255)) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    SoftmaxBuffers b;
    softmax_carve(s, n, vocab, dim, true, (char *)workspace, &b);
    TokenArgs t = {labels, lse, d_loss, n, s.Np, vocab, ignore_label, b.label, status, b.lse2, b.d};
    hipLaunchKernelGGL(k_tokens, dim3((unsigned)cdiv(s.Np, BLOCK)), dim3(BLOCK), 0, st, t);
    lay_out(s, b, hidden, hidden_stride, table, table_stride, dtype, n, vocab, dim, true, st);
    for (i64 range = 0; range < s.ranges; ++range) {
        const i64 tile0 = range * s.range_tiles, tiles = std::min(s.range_tiles, s.tiles - tile0);
        const i64 word0 = tile0 * SM_BM, words = std::min(tiles * SM_BM, vocab - word0);
        LogitsArgs a = logits_args(s, b, table, table_stride, vocab, scale);
        a.word0 = word0;
        a.tiles = (int)tiles;
        a.per = s.dz_per;
        a.strips = (int)cdiv(tiles, s.dz_per);
        if (s.parts == 1) launch_logits<true, 1>(s, a, st);
        else launch_logits<true, 3>(s, a, st);
        const Operand dz = {b.dz, a.dz_pitch, a.dz_plane, s.Np, a.dz_pitch};
        ProductArgs p;
        memset(&p, 0, sizeof(p));
        p.nseg = s.nseg;
        p.m_tiles = s.m_tiles;
        p.M = dim;
        p.dtype = dtype;
        p.scale = scale;
        if (d_hidden) {
            p.a = a.w;
            p.a.p += word0 * a.w.pitch;
            p.a.rows = vocab - word0;
            p.b = dz;
            p.N = n;
            p.K = cdiv(words, BK) * BK;
            p.n_tiles = (int)cdiv(s.Np, 128);
            p.k_per = s.h_k;
            p.splits = (int)cdiv(p.K, p.k_per);
            p.slots = b.h_slots + range * s.h_splits * n * dim;
            launch_product<false>(s.tm, p, st);
        }
        if (d_table) {
            p.a = a.h;
            p.b = dz;
            p.N = words;
            p.K = s.Np;
            p.n_tiles = (int)cdiv(words, 128);
            p.k_per = s.t_k;
            p.splits = s.t_splits;
            p.slots = s.t_splits > 1 ? b.t_slots : nullptr;
            char *out = (char *)d_table + (size_t)word0 * d_table_stride * (dtype == TENSAIR_F32 ? 4 : 2);
            p.out = out;
            p.out_stride = d_table_stride;
            launch_product<true>(s.tm, p, st);
            if (s.t_splits > 1) launch_join(b.t_slots, s.t_splits, words, d_table_stride, dim, nullptr, out, dtype, scale, st);
        }
    }
    if (d_hidden) {
        // the last range may have fewer splits than the others
        const i64 last = std::min(s.range_tiles, s.tiles - (s.ranges - 1) * s.range_tiles) * SM_BM;
        const i64 words = std::min(last, vocab - (s.ranges - 1) * s.range_tiles * SM_BM);
        const int slots = (int)((s.ranges - 1) * s.h_splits + cdiv(cdiv(words, BK) * BK, s.h_k));
        launch_join(b.h_slots, slots, n, d_hidden_stride, dim, b.label, d_hidden, dtype, scale, st);
    }
    return launched("softmax_grad");
}

}  // extern "C"
