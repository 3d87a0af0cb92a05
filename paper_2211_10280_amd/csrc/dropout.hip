// Dropout from the counter-based generator: out = residual + (kept ? x / (1 - p) : 0).  The mask of four elements is one block of
// Philox4x32-10, whose counter is the elements' place, so that the gradient makes it again instead of reading it.
#include <hip/hip_runtime.h>

#include <cmath>

#include "layers.h"

namespace {

#define DROP_TAG 0x44524F50u
struct DropArgs {
    const void *x, *residual;
    void *out;
    i64 x_stride, r_stride, out_stride, n, step;
    const i64 *step_at;
    int C4;
    u32 magic, keep, k0, k1, tag;      // elements with a word below `keep` are dropped
    float scale;
};

// Chunks of 4 elements as one list; a thread takes one of every BLOCK.
template <typename T, typename TO>
__global__ void __launch_bounds__(BLOCK) k_dropout(DropArgs a)
{
    const u64 chunk = (u64)blockIdx.x * BLOCK;
    const u64 row0 = chunk / (u32)a.C4;
    const u32 x = (u32)(chunk - row0 * (u32)a.C4) + threadIdx.x, q = a.magic ? (u32)(((u64)x * a.magic) >> 32) : x;
    const i64 row = (i64)(row0 + q);
    const u32 col = x - q * (u32)a.C4;
    if (row >= a.n) return;
    const float4 v = ld4((const T *)a.x + row * a.x_stride + 4 * col);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.residual) o = ld4((const TO *)a.residual + row * a.r_stride + 4 * col);
    const u64 c = chunk + threadIdx.x;
    const u32 step = (u32)(a.step_at ? a.step + *a.step_at : a.step);
    const philox_out r = philox4x32_10((u32)c, (u32)(c >> 32), step, a.tag, a.k0, a.k1);
    o.x += r.r0 >= a.keep ? v.x * a.scale : 0.f;
    o.y += r.r1 >= a.keep ? v.y * a.scale : 0.f;
    o.z += r.r2 >= a.keep ? v.z * a.scale : 0.f;
    o.w += r.r3 >= a.keep ? v.w * a.scale : 0.f;
    st4((TO *)a.out + row * a.out_stride + 4 * col, o);
}

}  // namespace

extern "C" int tensair_dropout(const void *x, int32_t dtype, int64_t x_stride, int64_t n, int32_t dim, double p, uint64_t seed, uint32_t layer, int64_t step,
                               const int64_t *step_at, const void *residual, int64_t residual_stride, void *out, int32_t out_dtype, int64_t out_stride,
                               void *stream)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = layer_matrix(out, n, out_stride, dim, out_dtype, "out"))) return rc;
    if (residual && (rc = layer_matrix(residual, n, residual_stride, dim, out_dtype, "residual"))) return rc;
    if (!(p >= 0.0 && p < 1.0)) return tn_fail(TENSAIR_EINVAL, "p must be in [0, 1)");
    if ((uintptr_t)step_at & 7) return tn_fail(TENSAIR_EINVAL, "step_at must be 8-byte aligned");
    if (n == 0) return TENSAIR_OK;
    const u64 blocks = ((u64)n * (u64)(dim / 4) + BLOCK - 1) / BLOCK;
    if (blocks > TN_MAX_BLOCKS) return tn_fail(TENSAIR_EINVAL, "n * dim beyond what one launch covers");
    const DropArgs a = {x, residual, out, x_stride, residual_stride, out_stride, n, step, (const i64 *)step_at, dim / 4, layer_magic(dim / 4),
                        (u32)std::floor(p * 4294967296.0), (u32)seed, (u32)(seed >> 32), DROP_TAG + layer, (float)(1.0 / (1.0 - p))};
    const dim3 grid((unsigned)blocks), blk(BLOCK);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == TENSAIR_F32 && out_dtype == TENSAIR_F32) hipLaunchKernelGGL((k_dropout<float, float>), grid, blk, 0, st, a);
    else if (dtype == TENSAIR_F32) hipLaunchKernelGGL((k_dropout<float, bf16_t>), grid, blk, 0, st, a);
    else if (out_dtype == TENSAIR_F32) hipLaunchKernelGGL((k_dropout<bf16_t, float>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((k_dropout<bf16_t, bf16_t>), grid, blk, 0, st, a);
    return layer_launched("dropout");
}
