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

#define DROP_CHUNKS 4
// Chunks of 4 elements as one list; a thread takes one of every 256 of its workgroup's 1 024, all loads in flight before the first mask is made.
// Memory bounds it: 131 071 rows of 512 in bfloat16 54 us (268 MB, 4.9 TB/s), a chunk to a thread 61; loads and stores around the caches: no difference.  The masks, 10 rounds of two
// products for 4 elements, take half of that time on the vector units, beside the loads.
template <typename T, typename TO>
__global__ void __launch_bounds__(BLOCK) k_dropout(DropArgs a)
{
    const u64 chunk = (u64)blockIdx.x * (BLOCK * DROP_CHUNKS);
    const u64 row0 = chunk / (u32)a.C4;
    const u32 first = (u32)(chunk - row0 * (u32)a.C4);
    const u32 step = (u32)a.step + (a.step_at ? (u32)*a.step_at : 0u);
    typename Raw4<T>::type v[DROP_CHUNKS];
    typename Raw4<TO>::type add[DROP_CHUNKS];
    i64 row[DROP_CHUNKS];
    u32 col[DROP_CHUNKS];
#pragma unroll
    for (int j = 0; j < DROP_CHUNKS; ++j) {
        const u32 x = first + (u32)j * BLOCK + threadIdx.x, q = a.magic ? (u32)(((u64)x * a.magic) >> 32) : x;
        col[j] = x - q * (u32)a.C4;
        row[j] = (i64)(row0 + q);
        zero_raw(v[j]);
        zero_raw(add[j]);
        if (row[j] >= a.n) continue;
        v[j] = ldraw((const T *)a.x + row[j] * a.x_stride + 4 * col[j]);
        if (a.residual) add[j] = ldraw((const TO *)a.residual + row[j] * a.r_stride + 4 * col[j]);
    }
#pragma unroll
    for (int j = 0; j < DROP_CHUNKS; ++j) {
        if (row[j] >= a.n) continue;
        const u64 c = chunk + (u32)j * BLOCK + threadIdx.x;
        const philox_out r = philox4x32_10((u32)c, (u32)(c >> 32), step, a.tag, a.k0, a.k1);
        const float4 x = widen4(v[j]);
        float4 o = widen4(add[j]);
        o.x += r.r0 >= a.keep ? x.x * a.scale : 0.f;
        o.y += r.r1 >= a.keep ? x.y * a.scale : 0.f;
        o.z += r.r2 >= a.keep ? x.z * a.scale : 0.f;
        o.w += r.r3 >= a.keep ? x.w * a.scale : 0.f;
        put4((TO *)a.out + row[j] * a.out_stride + 4 * col[j], o);
    }
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
    const u64 blocks = ((u64)n * (u64)(dim / 4) + BLOCK * DROP_CHUNKS - 1) / (BLOCK * DROP_CHUNKS);
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
