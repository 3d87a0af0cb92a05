// Checks and small helpers that the operators between and behind a table's two ends share (host side, and sums over the lanes of a row).
#pragma once
#include "../../include/tensair.h"
#include "dev_common.h"
#include "kernels.h"

// address and stride of four elements; rows > 0 only need an address
static inline int layer_matrix(const void *p, i64 rows, i64 stride, int32_t dim, int32_t dtype, const char *what)
{
    if (dtype != TENSAIR_F32 && dtype != TENSAIR_BF16) return tn_fail(TENSAIR_EINVAL, "%s: unknown dtype", what);
    if (rows > 0 && !p) return tn_fail(TENSAIR_EINVAL, "%s is NULL", what);
    if ((uintptr_t)p & (dtype == TENSAIR_F32 ? 15 : 7)) return tn_fail(TENSAIR_EINVAL, "%s must have the alignment of four elements", what);
    if (stride < dim || stride % 4) return tn_fail(TENSAIR_EINVAL, "%s: the row stride must be >= dim and a multiple of 4", what);
    return TENSAIR_OK;
}
static inline int layer_sizes(i64 n, int32_t dim)
{
    if (n < 0 || n > TENSAIR_MAX_ROWS) return tn_fail(TENSAIR_EINVAL, "n must be in 0..TENSAIR_MAX_ROWS");
    if (dim < 4 || dim > TENSAIR_MAX_DIM || dim % 4) return tn_fail(TENSAIR_EINVAL, "dim must be a multiple of 4 in 4..TENSAIR_MAX_DIM");
    return TENSAIR_OK;
}
// fp32 vectors and states; NULL is the caller's matter
static inline int layer_floats(const void *p, const char *what)
{
    return (uintptr_t)p & 15 ? tn_fail(TENSAIR_EINVAL, "%s must be 16-byte aligned", what) : TENSAIR_OK;
}
static inline int layer_workspace(const void *p, size_t have, size_t need, const char *what)
{
    if (!p || ((uintptr_t)p & 255)) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    if (have < need) return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see %s", what);
    return TENSAIR_OK;
}
static inline int layer_launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TENSAIR_OK : tn_fail(TENSAIR_EHIP, "%s: %s", what, hipGetErrorString(e));
}
static inline size_t layer_up256(size_t x) { return (x + 255) / 256 * 256; }
// x / c = (x * magic) >> 32 for x < c + 1024 (c <= 256 chunks of a row); 0 where c = 1
static inline u32 layer_magic(int c) { return c == 1 ? 0u : (u32)(((1ull << 32) + (u32)c - 1) / (u32)c); }

// sum over the G lanes (8, 16, 32 or 64, aligned) that hold a row; every lane gets it, the order is fixed
template <int G>
__device__ __forceinline__ float lanes_sum(float x)
{
    if (G == 64) return wave_sum_dpp(x);
    x += dpp_get<0xB1, 0xF>(x);                  // quad_perm [1,0,3,2]
    x += dpp_get<0x4E, 0xF>(x);                  // quad_perm [2,3,0,1]
    x += dpp_get<0x141, 0xF>(x);                 // row_half_mirror: every lane of 8
    if (G >= 16) x += dpp_get<0x140, 0xF>(x);    // row_mirror: every lane of 16
    if (G >= 32) x += __shfl_xor(x, 16, WAVE);
    return x;
}
__device__ __forceinline__ float4 mul4(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 plus4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float hsum4(float4 a) { return (a.x + a.y) + (a.z + a.w); }
// rounded to nearest even by the hardware's conversion of two
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void put4(float *p, float4 v) { st4(p, v); }
__device__ __forceinline__ void put4(bf16_t *p, float4 v)
{
    const bf16x2 lo = {(__bf16)v.x, (__bf16)v.y}, hi = {(__bf16)v.z, (__bf16)v.w};
    *reinterpret_cast<uint2 *>(p) = make_uint2(__builtin_bit_cast(u32, lo), __builtin_bit_cast(u32, hi));
}
