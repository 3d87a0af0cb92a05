// Layer norm and its gradient.  With m and r a row's mean and 1 / sqrt(variance + eps), y = (x - m) r:
//   out = y w + b                                                              tensair_norm
//   d_x = d_add + r (g - mean g - y mean(g y)), g = d_out w;  d_w = sum over the rows of d_out y, d_b = sum of d_out    tensair_norm_grad
// A row lies in the registers of G lanes of a wave from its load to its store, so that mean and variance are two sums over the same registers
// (no difference of large squares) and memory is read once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "layers.h"

namespace {

struct NormArgs {
    const void *x;
    void *out;
    i64 x_stride, out_stride, n;
    int C4;                      // chunks of 4 elements of a row
    float inv, eps;              // 1 / dim
    const float *w, *b;
    float *mean, *rstd;
};

// A row to a group of G lanes.  Memory bounds it: 262 143 rows of 300, fp32 to bfloat16, 97 us (472 MB, 4.9 TB/s); two rows to a group, their loads side by side, 101, four 116.
template <typename T, typename TO, int G, int ITERS>
__global__ void __launch_bounds__(BLOCK) k_norm(NormArgs a)
{
    const int l = (int)threadIdx.x % G;
    for (i64 row = (i64)blockIdx.x * (BLOCK / G) + (int)threadIdx.x / G; row < a.n; row += (i64)gridDim.x * (BLOCK / G)) {
        const T *src = (const T *)a.x + row * a.x_stride;
        float4 v[ITERS];
        float sum = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c = l + G * it;
            v[it] = c < a.C4 ? ld4(src + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
            sum += hsum4(v[it]);
        }
        const float mean = lanes_sum<G>(sum) * a.inv;
        sum = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
            if (l + G * it < a.C4) {
                v[it] = make_float4(v[it].x - mean, v[it].y - mean, v[it].z - mean, v[it].w - mean);
                sum += hsum4(mul4(v[it], v[it]));
            }
        const float rstd = 1.0f / sqrtf(lanes_sum<G>(sum) * a.inv + a.eps);
        if (l == 0 && a.mean) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
        TO *dst = (TO *)a.out + row * a.out_stride;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c = l + G * it;
            if (c >= a.C4) continue;
            float4 y = make_float4(v[it].x * rstd, v[it].y * rstd, v[it].z * rstd, v[it].w * rstd);
            if (a.w) y = mul4(y, ld4(a.w + 4 * c));
            if (a.b) y = plus4(y, ld4(a.b + 4 * c));
            put4(dst + 4 * c, y);
        }
    }
}

struct NormGradArgs {
    const void *d, *x, *add;
    void *dx;
    i64 d_stride, x_stride, add_stride, dx_stride, n;
    int C4;
    float inv;
    const float *w, *mean, *rstd;
    float *dw, *db;              // NULL: not wanted
    float *part;                 // [blocks][2][4 * C4] shares of d_w and d_b
    int per;                     // rows of a group of lanes
    int blocks;
};
#define NORM_MOST_ROWS 256       // that one lane adds up in fp32; so are the sums of a workgroup's 4 to 32 groups of lanes, and the workgroups' shares in 64 bits
// Workgroups that few rows are spread over: twice what the card holds at the registers of rows of 300 (262 143 of them, fp32, with a residual's gradient: 1 536 workgroups 244 us,
// 1 024 295, 2 048 257; 16 384 rows of 512 in bfloat16 14 each, but more shares to put together).
#define NORM_BLOCKS 1536

// A group of G lanes takes `per` rows of a run that its workgroup has to itself, and holds its columns' sums of d_w and d_b meanwhile.  Memory bounds it: 262 143 rows of 300,
// fp32 with bfloat16 gradients and a residual's, 244 us (1.1 GB, 4.5 TB/s).
template <typename T, typename TD, int G, int ITERS>
__global__ void __launch_bounds__(BLOCK) k_norm_grad(NormGradArgs a)
{
    constexpr int GROUPS = BLOCK / G;
    __shared__ float4 lds[2][GROUPS > 1 ? (GROUPS - 1) * G * ITERS : 1];
    const int l = (int)threadIdx.x % G, group = (int)threadIdx.x / G;
    float4 w[ITERS], dw[ITERS], db[ITERS];
    zero_row<ITERS>(dw);
    zero_row<ITERS>(db);
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int c = l + G * it;
        w[it] = c >= a.C4 ? make_float4(0.f, 0.f, 0.f, 0.f) : a.w ? ld4(a.w + 4 * c) : make_float4(1.f, 1.f, 1.f, 1.f);
    }
    const i64 first = (i64)blockIdx.x * GROUPS * a.per + group;
    for (int k = 0; k < a.per; ++k) {
        const i64 row = first + (i64)k * GROUPS;
        if (row >= a.n) break;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float4 d[ITERS], y[ITERS];
        typename Raw4<T>::type add[ITERS];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c = l + G * it;
            d[it] = y[it] = make_float4(0.f, 0.f, 0.f, 0.f);
            zero_raw(add[it]);
            if (c >= a.C4) continue;
            if (a.add) add[it] = ldraw((const T *)a.add + row * a.add_stride + 4 * c);
            d[it] = ld4((const TD *)a.d + row * a.d_stride + 4 * c);
            y[it] = ld4((const T *)a.x + row * a.x_stride + 4 * c);
        }
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            if (l + G * it >= a.C4) continue;
            y[it] = make_float4((y[it].x - mean) * rstd, (y[it].y - mean) * rstd, (y[it].z - mean) * rstd, (y[it].w - mean) * rstd);
            db[it] = plus4(db[it], d[it]);
            dw[it] = plus4(dw[it], mul4(d[it], y[it]));
            d[it] = mul4(d[it], w[it]);
            s1 += hsum4(d[it]);
            s2 += hsum4(mul4(d[it], y[it]));
        }
        s1 = lanes_sum<G>(s1) * a.inv;
        s2 = lanes_sum<G>(s2) * a.inv;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int c = l + G * it;
            if (c >= a.C4) continue;
            float4 o = make_float4(rstd * (d[it].x - s1 - y[it].x * s2), rstd * (d[it].y - s1 - y[it].y * s2), rstd * (d[it].z - s1 - y[it].z * s2),
                                   rstd * (d[it].w - s1 - y[it].w * s2));
            o = plus4(widen4(add[it]), o);
            put4((T *)a.dx + row * a.dx_stride + 4 * c, o);
        }
    }
    if (!a.part) return;
    if (group > 0)
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            lds[0][((group - 1) * ITERS + it) * G + l] = dw[it];
            lds[1][((group - 1) * ITERS + it) * G + l] = db[it];
        }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int c = l + G * it;
        for (int g = 1; g < GROUPS; ++g) {
            dw[it] = plus4(dw[it], lds[0][((g - 1) * ITERS + it) * G + l]);
            db[it] = plus4(db[it], lds[1][((g - 1) * ITERS + it) * G + l]);
        }
        if (c >= a.C4) continue;
        st4(a.part + ((i64)blockIdx.x * 2 + 0) * 4 * a.C4 + 4 * c, dw[it]);
        st4(a.part + ((i64)blockIdx.x * 2 + 1) * 4 * a.C4 + 4 * c, db[it]);
    }
}

#define JOIN_THREADS 1024
// The workgroups' shares put together: 8 chunks of columns and 128 runs of shares to a workgroup, in 64 bits, in an order that hangs on their number alone.
__global__ void __launch_bounds__(JOIN_THREADS) k_norm_join(const float *part, int blocks, int C4, float *dw, float *db)
{
    __shared__ double lds[JOIN_THREADS / WAVE][8][4];
    const int l = (int)threadIdx.x & 7, run = (int)threadIdx.x >> 3, c = (int)blockIdx.x * 8 + l;    // of 2 * C4 chunks
    double s[4] = {0, 0, 0, 0};
    if (c < 2 * C4) {
        const float *p = part + 4 * c;
#pragma unroll 8
        for (int b = run; b < blocks; b += JOIN_THREADS / 8) {
            const float4 v = ld4(p + (i64)b * 8 * C4);
            s[0] += v.x;
            s[1] += v.y;
            s[2] += v.z;
            s[3] += v.w;
        }
    }
    for (int k = 0; k < 4; ++k) {
        for (int o = 8; o < WAVE; o *= 2) s[k] += __shfl_xor(s[k], o, WAVE);
        if (lane_id() < 8) lds[threadIdx.x >> 6][l][k] = s[k];
    }
    __syncthreads();
    if (run > 0 || c >= 2 * C4) return;
    for (int r = 1; r < JOIN_THREADS / WAVE; ++r)
        for (int k = 0; k < 4; ++k) s[k] += lds[r][l][k];
    float *to = c < C4 ? dw : db;
    if (to) st4(to + 4 * (c < C4 ? c : c - C4), make_float4((float)s[0], (float)s[1], (float)s[2], (float)s[3]));
}

// Lanes to a row, the fewest whose loads stay below 6 a lane: rows of 300 in 16 lanes of 5 chunks leave 6 % of them idle (in 64 of 2: 41 %), and four rows share a wave's sums.
int norm_lanes(int C4) { return C4 <= 8 ? 8 : C4 <= 80 ? 16 : C4 <= 160 ? 32 : 64; }
void norm_blocks(i64 n, int dim, int *per, i64 *blocks)
{
    const i64 groups = BLOCK / norm_lanes(dim / 4);
    const i64 rows = std::min<i64>(NORM_MOST_ROWS, std::max<i64>(1, (n + groups * NORM_BLOCKS - 1) / (groups * NORM_BLOCKS)));
    *per = (int)rows;
    *blocks = (n + groups * rows - 1) / (groups * rows);
}

// f(lanes, loads of a lane) as constants
template <int N> struct Int {
    static constexpr int value = N;
};
template <typename F>
void norm_shape(int C4, F f)
{
    const int G = norm_lanes(C4), iters = (C4 + G - 1) / G;
    if (G == 8) f(Int<8>(), Int<1>());
    else if (G == 16 && iters == 1) f(Int<16>(), Int<1>());
    else if (G == 16 && iters == 2) f(Int<16>(), Int<2>());
    else if (G == 16 && iters == 3) f(Int<16>(), Int<3>());
    else if (G == 16 && iters == 4) f(Int<16>(), Int<4>());
    else if (G == 16) f(Int<16>(), Int<5>());
    else if (G == 32 && iters == 3) f(Int<32>(), Int<3>());
    else if (G == 32 && iters == 4) f(Int<32>(), Int<4>());
    else if (G == 32) f(Int<32>(), Int<5>());
    else if (iters == 3) f(Int<64>(), Int<3>());
    else f(Int<64>(), Int<4>());
}
#define NORM_MOST_BLOCKS 65536   // of k_norm; more rows are taken one after the other
template <typename T, typename TO>
void launch_norm(const NormArgs &a, hipStream_t st)
{
    norm_shape(a.C4, [&](auto g, auto iters) {
        constexpr int G = decltype(g)::value, GROUPS = BLOCK / G;
        const i64 blocks = std::min<i64>((a.n + GROUPS - 1) / GROUPS, NORM_MOST_BLOCKS);
        hipLaunchKernelGGL((k_norm<T, TO, G, decltype(iters)::value>), dim3((unsigned)blocks), dim3(BLOCK), 0, st, a);
    });
}
template <typename T, typename TD>
void launch_norm_grad(const NormGradArgs &a, hipStream_t st)
{
    norm_shape(a.C4, [&](auto g, auto iters) {
        hipLaunchKernelGGL((k_norm_grad<T, TD, decltype(g)::value, decltype(iters)::value>), dim3((unsigned)a.blocks), dim3(BLOCK), 0, st, a);
    });
}

}  // namespace

extern "C" {

int tensair_norm(const void *x, int32_t dtype, int64_t x_stride, int64_t n, int32_t dim, const float *weight, const float *bias, float eps, void *out,
                 int32_t out_dtype, int64_t out_stride, float *mean, float *rstd, void *stream)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = layer_matrix(out, n, out_stride, dim, out_dtype, "out"))) return rc;
    if ((rc = layer_floats(weight, "weight")) || (rc = layer_floats(bias, "bias"))) return rc;
    if (!(eps > 0.0f)) return tn_fail(TENSAIR_EINVAL, "eps must be positive");
    if (n > 0 && !mean != !rstd) return tn_fail(TENSAIR_EINVAL, "mean and rstd go together");
    if (((uintptr_t)mean | (uintptr_t)rstd) & 3) return tn_fail(TENSAIR_EINVAL, "mean and rstd must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    const NormArgs a = {x, out, x_stride, out_stride, n, dim / 4, 1.0f / (float)dim, eps, weight, bias, mean, rstd};
    hipStream_t st = (hipStream_t)stream;
    if (dtype == TENSAIR_F32 && out_dtype == TENSAIR_F32) launch_norm<float, float>(a, st);
    else if (dtype == TENSAIR_F32) launch_norm<float, bf16_t>(a, st);
    else if (out_dtype == TENSAIR_F32) launch_norm<bf16_t, float>(a, st);
    else launch_norm<bf16_t, bf16_t>(a, st);
    return layer_launched("norm");
}

size_t tensair_norm_workspace_bytes(int64_t n, int32_t dim)
{
    if (layer_sizes(n, dim)) return 0;
    int per;
    i64 blocks;
    norm_blocks(n, dim, &per, &blocks);
    // rows are spread over at most NORM_BLOCKS workgroups, a little fewer where `per` is rounded up, until every lane has the most rows it may add up
    return layer_up256((size_t)std::max<i64>(blocks, NORM_BLOCKS) * 8 * (size_t)dim);
}

int tensair_norm_grad(const void *d_out, int32_t d_dtype, int64_t d_stride, const void *x, int32_t dtype, int64_t x_stride, int64_t n, int32_t dim,
                      const float *weight, const float *mean, const float *rstd, const void *d_add, int64_t d_add_stride, void *d_x, int64_t d_x_stride,
                      float *d_weight, float *d_bias, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(d_out, n, d_stride, dim, d_dtype, "d_out")) || (rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) ||
        (rc = layer_matrix(d_x, n, d_x_stride, dim, dtype, "d_x")))
        return rc;
    if (d_add && (rc = layer_matrix(d_add, n, d_add_stride, dim, dtype, "d_add"))) return rc;
    if ((rc = layer_floats(weight, "weight")) || (rc = layer_floats(d_weight, "d_weight")) || (rc = layer_floats(d_bias, "d_bias"))) return rc;
    if (n > 0 && (!mean || !rstd)) return tn_fail(TENSAIR_EINVAL, "mean and rstd are NULL");
    if (((uintptr_t)mean | (uintptr_t)rstd) & 3) return tn_fail(TENSAIR_EINVAL, "mean and rstd must be 4-byte aligned");
    const bool sums = d_weight || d_bias;
    if (sums && (rc = layer_workspace(workspace, workspace_bytes, tensair_norm_workspace_bytes(n, dim), "tensair_norm_workspace_bytes"))) return rc;
    if (n == 0 && !sums) return TENSAIR_OK;
    NormGradArgs a;
    memset(&a, 0, sizeof(a));
    a.d = d_out;
    a.x = x;
    a.add = d_add;
    a.dx = d_x;
    a.d_stride = d_stride;
    a.x_stride = x_stride;
    a.add_stride = d_add_stride;
    a.dx_stride = d_x_stride;
    a.n = n;
    a.C4 = dim / 4;
    a.inv = 1.0f / (float)dim;
    a.w = weight;
    a.mean = mean;
    a.rstd = rstd;
    a.part = sums ? (float *)workspace : nullptr;
    i64 blocks;
    norm_blocks(n, dim, &a.per, &blocks);
    a.blocks = (int)blocks;
    hipStream_t st = (hipStream_t)stream;
    if (n > 0) {
        if (dtype == TENSAIR_F32 && d_dtype == TENSAIR_F32) launch_norm_grad<float, float>(a, st);
        else if (dtype == TENSAIR_F32) launch_norm_grad<float, bf16_t>(a, st);
        else if (d_dtype == TENSAIR_F32) launch_norm_grad<bf16_t, float>(a, st);
        else launch_norm_grad<bf16_t, bf16_t>(a, st);
    }
    if (sums) hipLaunchKernelGGL(k_norm_join, dim3((unsigned)((2 * a.C4 + 7) / 8)), dim3(JOIN_THREADS), 0, st, (const float *)workspace, a.blocks, a.C4, d_weight, d_bias);
    return layer_launched("norm_grad");
}

}  // extern "C"
