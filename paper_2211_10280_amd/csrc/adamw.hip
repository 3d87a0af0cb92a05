// AdamW over many tensors at once: one launch for all tensors of the same types.  With t the step, g the gradient (times a
// scale), every operation in fp32 and rounded by itself, in this order:
//   m <- b1 m + (1 - b1) g        v <- b2 v + (1 - b2) (g g)        r = sqrt(v)
//   p <- p (1 - lr decay) - (m lr / (1 - b1^t)) / (r / sqrt(1 - b2^t) + eps)
// States in 8 bits: a group of 256 elements of a tensor shares a scale, the group's largest magnitude / 448.  m is kept as an
// 8-bit float (4 exponent, 3 mantissa bits), to nearest even.  Of v the root is kept, which halves the range it has to span;
// it is a slow average (0.1 % of the way a step at b2 = 0.999), which rounding to nearest to 3 bits would freeze, so what is cut
// off is carried with an offset that walks evenly through the steps and elements (a Weyl sequence): over the steps the average
// of what is kept is the average of what was computed.  Values below 2^-6 of a scale's unit are kept as that: a root
// is never rounded to zero, where the step would be divided by eps.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/tensair.h"
#include "dev_common.h"
#include "kernels.h"

namespace {

#define ADAMW_CHUNK 4096       // elements of a workgroup
#define ADAMW_GROUP 256        // elements that share a scale: a wave, four to a lane
#define ADAMW_STREAM_BYTES ((i64)256 << 20)
#define ADAMW_VECS (ADAMW_CHUNK / (BLOCK * 4))

struct AdamwTensor {
    void *param, *m, *v;
    const void *grad;
    float *m_scale, *v_scale;
    bf16_t *copy;              // bfloat16 copy of the new parameters (NULL: none)
    i64 n;
    float decay;
    u32 first;                 // its first chunk
    u32 vec;                   // 4 elements can be loaded at a time
    u32 pad;
};
// what a step's number and size come to: in the arguments, or, where they are read on the device, in the workspace
struct AdamwLive {
    float lr, size, fix;
    u32 walk;                  // the step's part of the offsets
};
struct AdamwStep {
    const AdamwTensor *tensors;
    const u32 *chunks;         // [chunks] the tensor of every chunk
    const float *grad_scale;
    float b1, c1, b2, c2, eps;
    AdamwLive now;
    const AdamwLive *live;     // NULL: as in `now`
};
// in 64 bits, each rounded once
__host__ __device__ __forceinline__ AdamwLive adamw_live(double lr, i64 step, double beta1, double beta2)
{
    return AdamwLive{(float)lr, (float)(lr / (1.0 - pow(beta1, (double)step))), (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step))), (u32)step * 0x85EBCA77u};
}
__global__ void k_adamw_live(AdamwLive *out, const double *lr, const i64 *step, double beta1, double beta2)
{
    *out = adamw_live(*lr, max((i64)1, *step), beta1, beta2);
}

typedef float v2f __attribute__((ext_vector_type(2)));

// 4 elements at p + i of n
template <bool STREAM>
__device__ __forceinline__ float4 get4(const float *p, i64 i, i64 n, bool vec)
{
    if (vec && i + 4 <= n) return STREAM ? ld4s(p + i) : ld4(p + i);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n) v.x = p[i];
    if (i + 1 < n) v.y = p[i + 1];
    if (i + 2 < n) v.z = p[i + 2];
    if (i + 3 < n) v.w = p[i + 3];
    return v;
}
template <bool STREAM>
__device__ __forceinline__ float4 get4(const bf16_t *p, i64 i, i64 n, bool vec)
{
    if (vec && i + 4 <= n) return STREAM ? ld4s(p + i) : ld4(p + i);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < n) v.x = bf16_to_f32(p[i]);
    if (i + 1 < n) v.y = bf16_to_f32(p[i + 1]);
    if (i + 2 < n) v.z = bf16_to_f32(p[i + 2]);
    if (i + 3 < n) v.w = bf16_to_f32(p[i + 3]);
    return v;
}
template <bool STREAM>
__device__ __forceinline__ u32 get4(const unsigned char *p, i64 i, i64 n, bool vec)
{
    if (vec && i + 4 <= n) return STREAM ? __builtin_nontemporal_load((const GLOBAL_AS u32 *)(p + i)) : *(const u32 *)(p + i);
    u32 v = 0;
    for (int k = 0; k < 4; ++k)
        if (i + k < n) v |= (u32)p[i + k] << (8 * k);
    return v;
}
__device__ __forceinline__ void put1(float *p, float v) { *p = v; }
__device__ __forceinline__ void put1(bf16_t *p, float v) { *p = f32_to_bf16(v); }
template <bool STREAM, typename T>
__device__ __forceinline__ void put4(T *p, i64 i, i64 n, bool vec, float4 v)
{
    if (vec && i + 4 <= n) {
        if (STREAM) st4s(p + i, v);
        else st4(p + i, v);
        return;
    }
    if (i < n) put1(p + i, v.x);
    if (i + 1 < n) put1(p + i + 1, v.y);
    if (i + 2 < n) put1(p + i + 2, v.z);
    if (i + 3 < n) put1(p + i + 3, v.w);
}
template <bool STREAM>
__device__ __forceinline__ void put4(unsigned char *p, i64 i, i64 n, bool vec, u32 v)
{
    if (vec && i + 4 <= n) {
        if (STREAM) __builtin_nontemporal_store(v, (GLOBAL_AS u32 *)(p + i));
        else *(u32 *)(p + i) = v;
        return;
    }
    for (int k = 0; k < 4; ++k)
        if (i + k < n) p[i + k] = (unsigned char)(v >> (8 * k));
}

// largest over the wave, as whole numbers: of magnitudes a NaN is the largest, then infinity
__device__ __forceinline__ u32 wave_max_bits(u32 x)
{
    x = max(x, (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));
    x = max(x, (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));
    x = max(x, (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, false));
    x = max(x, (u32)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, false));
    const u32 a = (u32)__builtin_amdgcn_readlane((int)x, 0), b = (u32)__builtin_amdgcn_readlane((int)x, 16);
    const u32 c = (u32)__builtin_amdgcn_readlane((int)x, 32), d = (u32)__builtin_amdgcn_readlane((int)x, 48);
    return max(max(a, b), max(c, d));
}
__device__ __forceinline__ u32 magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ __forceinline__ float4 from_fp8(u32 c, float s)
{
    const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    return make_float4(a.x * s, a.y * s, b.x * s, b.y * s);
}
// the factor that takes a group of this largest magnitude to the 8-bit float's range; below 2^-100 the group is zero
__device__ __forceinline__ float to_range(float largest) { return largest >= 0x1p-100f || largest != largest ? (1.0f / largest) * 448.0f : 0.0f; }

// the root's 8 bits: x in units of the scale, cut to 3 mantissa bits after `offset` (20 bits) was added below them
__device__ __forceinline__ u32 root_code(float x, u32 offset)
{
    const u32 bits = __float_as_uint(fminf(fmaxf(x, 0x1p-6f), 448.0f)) + offset;
    const u32 code = min(bits >> 20, 0x43Eu) - 0x3C0u;
    return x > 0.0f ? code : 0u;
}

__device__ __forceinline__ void adamw1(float &p, float g, float &m, float &v, float &r, const AdamwStep &a, const AdamwLive &now, float keep)
{
    m = a.b1 * m + a.c1 * g;
    v = a.b2 * v + a.c2 * (g * g);
    r = sqrtf(v);
    p = p * keep - (m * now.size) / (r * now.fix + a.eps);
}

// One pass over parameters, gradients and states, which memory bounds: 600 M fp32 parameters with bfloat16 gradients and 8-bit
// states 1.67 ms (8.4 GB, 5.0 TB/s, the rate of a large copy), 200 M with fp32 states 0.96 ms (5.8 TB/s), 96 tensors of 7 M in all 43 us.
// STREAM: around the caches, where the tensors do not fit the memory-side cache
template <typename TP, typename TG, bool EIGHT, bool STREAM>
__global__ void __launch_bounds__(BLOCK) k_adamw(AdamwStep a, u32 first_chunk)
{
    const u32 chunk = first_chunk + blockIdx.x;
    const AdamwTensor &t = a.tensors[a.chunks[chunk]];
    const i64 n = t.n, base = (i64)(chunk - t.first) * ADAMW_CHUNK + (i64)threadIdx.x * 4;
    const bool vec = t.vec != 0;
    const AdamwLive now = a.live ? *a.live : a.now;
    const float keep = 1.0f - t.decay * now.lr;
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
    TP *param = (TP *)t.param;
    const TG *grad = (const TG *)t.grad;
    float4 p[ADAMW_VECS], g[ADAMW_VECS];
#pragma unroll
    for (int j = 0; j < ADAMW_VECS; ++j) {
        p[j] = get4<STREAM>(param, base + j * (BLOCK * 4), n, vec);
        g[j] = get4<STREAM>(grad, base + j * (BLOCK * 4), n, vec);
    }
    if (a.grad_scale) {
#pragma unroll
        for (int j = 0; j < ADAMW_VECS; ++j) g[j] = make_float4(g[j].x * gs, g[j].y * gs, g[j].z * gs, g[j].w * gs);
    }
    if constexpr (!EIGHT) {
        float *m = (float *)t.m, *v = (float *)t.v;
        float4 mm[ADAMW_VECS], vv[ADAMW_VECS];
#pragma unroll
        for (int j = 0; j < ADAMW_VECS; ++j) {
            mm[j] = get4<STREAM>(m, base + j * (BLOCK * 4), n, vec);
            vv[j] = get4<STREAM>(v, base + j * (BLOCK * 4), n, vec);
        }
#pragma unroll
        for (int j = 0; j < ADAMW_VECS; ++j) {
            const i64 i = base + j * (BLOCK * 4);
            float r;
            adamw1(p[j].x, g[j].x, mm[j].x, vv[j].x, r, a, now, keep);
            adamw1(p[j].y, g[j].y, mm[j].y, vv[j].y, r, a, now, keep);
            adamw1(p[j].z, g[j].z, mm[j].z, vv[j].z, r, a, now, keep);
            adamw1(p[j].w, g[j].w, mm[j].w, vv[j].w, r, a, now, keep);
            put4<STREAM>(param, i, n, vec, p[j]);
            put4<STREAM>(m, i, n, vec, mm[j]);
            put4<STREAM>(v, i, n, vec, vv[j]);
            if (t.copy) put4<STREAM>(t.copy, i, n, vec, p[j]);
        }
    } else {
        unsigned char *m = (unsigned char *)t.m, *v = (unsigned char *)t.v;
        u32 mc[ADAMW_VECS], vc[ADAMW_VECS];
        float ms[ADAMW_VECS], vs[ADAMW_VECS];
#pragma unroll
        for (int j = 0; j < ADAMW_VECS; ++j) {
            const i64 i = base + j * (BLOCK * 4), group = i / ADAMW_GROUP;       // a wave's elements are one group
            mc[j] = get4<STREAM>(m, i, n, vec);
            vc[j] = get4<STREAM>(v, i, n, vec);
            const bool in = group * ADAMW_GROUP < n;
            ms[j] = in ? t.m_scale[group] : 0.0f;
            vs[j] = in ? t.v_scale[group] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < ADAMW_VECS; ++j) {
            const i64 i = base + j * (BLOCK * 4), group = i / ADAMW_GROUP;
            float4 mm = from_fp8(mc[j], ms[j]), vv = from_fp8(vc[j], vs[j]), r;
            vv = make_float4(vv.x * vv.x, vv.y * vv.y, vv.z * vv.z, vv.w * vv.w);
            adamw1(p[j].x, g[j].x, mm.x, vv.x, r.x, a, now, keep);
            adamw1(p[j].y, g[j].y, mm.y, vv.y, r.y, a, now, keep);
            adamw1(p[j].z, g[j].z, mm.z, vv.z, r.z, a, now, keep);
            adamw1(p[j].w, g[j].w, mm.w, vv.w, r.w, a, now, keep);
            const float mx = __uint_as_float(wave_max_bits(max(max(magnitude(mm.x), magnitude(mm.y)), max(magnitude(mm.z), magnitude(mm.w)))));
            const float rx = __uint_as_float(wave_max_bits(max(max(magnitude(r.x), magnitude(r.y)), max(magnitude(r.z), magnitude(r.w)))));
            const float mi = to_range(mx), ri = to_range(rx);
            int code = __builtin_amdgcn_cvt_pk_fp8_f32(mm.x * mi, mm.y * mi, 0, false);
            code = __builtin_amdgcn_cvt_pk_fp8_f32(mm.z * mi, mm.w * mi, code, true);
            const u32 off = (u32)i * 0x9E3779B1u + now.walk;
            const u32 root = root_code(r.x * ri, off >> 12) | root_code(r.y * ri, (off + 0x9E3779B1u) >> 12) << 8 |
                             root_code(r.z * ri, (off + 2u * 0x9E3779B1u) >> 12) << 16 | root_code(r.w * ri, (off + 3u * 0x9E3779B1u) >> 12) << 24;
            put4<STREAM>(param, i, n, vec, p[j]);
            put4<STREAM>(m, i, n, vec, (u32)code);
            put4<STREAM>(v, i, n, vec, root);
            if (t.copy) put4<STREAM>(t.copy, i, n, vec, p[j]);
            if (lane_id() == 0 && i < n) {
                t.m_scale[group] = mi == 0.0f && mx < 1.0f ? 0.0f : mx * (1.0f / 448.0f);
                t.v_scale[group] = ri == 0.0f && rx < 1.0f ? 0.0f : rx * (1.0f / 448.0f);
            }
        }
    }
}

int kind_of(const tensair_adamw_tensor &t) { return (t.param_dtype == TENSAIR_BF16 ? 2 : 0) + (t.grad_dtype == TENSAIR_BF16 ? 1 : 0); }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

int check_tensors(const tensair_adamw_tensor *t, int32_t n, int32_t state_dtype, i64 *chunks)
{
    *chunks = 0;
    if (n < 1 || !t) return tn_fail(TENSAIR_EINVAL, "no tensors");
    if (state_dtype != TENSAIR_F32 && state_dtype != TENSAIR_FP8) return tn_fail(TENSAIR_EINVAL, "state_dtype must be TENSAIR_F32 or TENSAIR_FP8");
    for (int32_t k = 0; k < n; ++k) {
        const tensair_adamw_tensor &x = t[k];
        if (x.n < 0 || x.n > TENSAIR_MAX_DENSE) return tn_fail(TENSAIR_EINVAL, "tensor %d: n out of range", k);
        if ((x.param_dtype != TENSAIR_F32 && x.param_dtype != TENSAIR_BF16) || (x.grad_dtype != TENSAIR_F32 && x.grad_dtype != TENSAIR_BF16))
            return tn_fail(TENSAIR_EINVAL, "tensor %d: unknown dtype", k);
        if (!(x.weight_decay >= 0.0f)) return tn_fail(TENSAIR_EINVAL, "tensor %d: weight_decay must not be negative", k);
        if (x.n == 0) continue;
        if (!x.param || !x.grad || !x.m || !x.v) return tn_fail(TENSAIR_EINVAL, "tensor %d: NULL pointer", k);
        if (state_dtype == TENSAIR_FP8 && (!x.m_scale || !x.v_scale)) return tn_fail(TENSAIR_EINVAL, "tensor %d: 8-bit states need scales", k);
        const uintptr_t pa = x.param_dtype == TENSAIR_F32 ? 3 : 1, ga = x.grad_dtype == TENSAIR_F32 ? 3 : 1, sa = state_dtype == TENSAIR_F32 ? 3 : 0;
        if (((uintptr_t)x.param & pa) || ((uintptr_t)x.grad & ga) || (((uintptr_t)x.m | (uintptr_t)x.v) & sa) ||
            (((uintptr_t)x.m_scale | (uintptr_t)x.v_scale) & 3) || ((uintptr_t)x.param_copy & 1))
            return tn_fail(TENSAIR_EINVAL, "tensor %d: a pointer is not aligned to its elements", k);
        *chunks += (x.n + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
    }
    if (*chunks > TN_MAX_BLOCKS) return tn_fail(TENSAIR_EINVAL, "more elements than one launch covers");
    return TENSAIR_OK;
}

}  // namespace

struct tensair_adamw {
    const AdamwTensor *tensors;
    const u32 *chunks;
    u32 first[4], count[4];    // chunks by types: parameters fp32 or bfloat16, gradients fp32 or bfloat16
    AdamwLive *live;
    bool eight, stream;
};

template <typename TP, typename TG>
static void launch_adamw(const tensair_adamw *h, const AdamwStep &a, int kind, hipStream_t st)
{
    if (!h->count[kind]) return;
    const dim3 grid(h->count[kind]), blk(BLOCK);
    if (h->eight && h->stream) hipLaunchKernelGGL((k_adamw<TP, TG, true, true>), grid, blk, 0, st, a, h->first[kind]);
    else if (h->eight) hipLaunchKernelGGL((k_adamw<TP, TG, true, false>), grid, blk, 0, st, a, h->first[kind]);
    else if (h->stream) hipLaunchKernelGGL((k_adamw<TP, TG, false, true>), grid, blk, 0, st, a, h->first[kind]);
    else hipLaunchKernelGGL((k_adamw<TP, TG, false, false>), grid, blk, 0, st, a, h->first[kind]);
}

static int check_step(const tensair_adamw *h, double beta1, double beta2, double eps, const float *grad_scale)
{
    if (!h) return tn_fail(TENSAIR_EINVAL, "handle is NULL");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return tn_fail(TENSAIR_EINVAL, "betas must be in [0, 1)");
    if (!((float)eps > 0.0f)) return tn_fail(TENSAIR_EINVAL, "eps must be positive");
    if ((uintptr_t)grad_scale & 3) return tn_fail(TENSAIR_EINVAL, "grad_scale must be 4-byte aligned");
    return TENSAIR_OK;
}
static int adamw_step(const tensair_adamw *h, const AdamwLive &now, const AdamwLive *live, double beta1, double beta2, double eps, const float *grad_scale,
                      hipStream_t st)
{
    const AdamwStep a = {h->tensors, h->chunks, grad_scale, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, now, live};
    launch_adamw<float, float>(h, a, 0, st);
    launch_adamw<float, bf16_t>(h, a, 1, st);
    launch_adamw<bf16_t, float>(h, a, 2, st);
    launch_adamw<bf16_t, bf16_t>(h, a, 3, st);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TENSAIR_OK : tn_fail(TENSAIR_EHIP, "adamw_step: %s", hipGetErrorString(e));
}

extern "C" {

size_t tensair_adamw_workspace_bytes(const tensair_adamw_tensor *tensors, int32_t n_tensors, int32_t state_dtype)
{
    i64 chunks;
    if (check_tensors(tensors, n_tensors, state_dtype, &chunks)) return 0;
    return up256(sizeof(AdamwTensor) * (size_t)n_tensors) + up256(4 * (size_t)(chunks > 0 ? chunks : 1)) + up256(sizeof(AdamwLive));
}

int tensair_adamw_init(tensair_adamw **out, const tensair_adamw_tensor *tensors, int32_t n_tensors, int32_t state_dtype, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    if (!out) return tn_fail(TENSAIR_EINVAL, "out is NULL");
    *out = nullptr;
    i64 chunks;
    int rc = check_tensors(tensors, n_tensors, state_dtype, &chunks);
    if (rc) return rc;
    const size_t head = up256(sizeof(AdamwTensor) * (size_t)n_tensors);
    if (!workspace || ((uintptr_t)workspace & 255)) return tn_fail(TENSAIR_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < tensair_adamw_workspace_bytes(tensors, n_tensors, state_dtype))
        return tn_fail(TENSAIR_ECAPACITY, "workspace too small: see tensair_adamw_workspace_bytes");
    tensair_adamw *h = nullptr;
    try {
        std::vector<char> image(head + 4 * (size_t)chunks, 0);
        AdamwTensor *dt = (AdamwTensor *)image.data();
        u32 *map = (u32 *)(image.data() + head);
        h = new tensair_adamw;
        memset(h, 0, sizeof(*h));
        h->eight = state_dtype == TENSAIR_FP8;
        i64 bytes = 0;
        u32 at = 0;
        for (int kind = 0; kind < 4; ++kind) {
            h->first[kind] = at;
            for (int32_t k = 0; k < n_tensors; ++k) {
                const tensair_adamw_tensor &x = tensors[k];
                if (x.n == 0 || kind_of(x) != kind) continue;
                const uintptr_t pa = x.param_dtype == TENSAIR_F32 ? 15 : 7, ga = x.grad_dtype == TENSAIR_F32 ? 15 : 7, sa = h->eight ? 3 : 15;
                bytes += x.n * ((x.param_dtype == TENSAIR_F32 ? 4 : 2) + (x.grad_dtype == TENSAIR_F32 ? 4 : 2) + (h->eight ? 2 : 8));
                AdamwTensor &d = dt[k];
                d.param = x.param;
                d.grad = x.grad;
                d.m = x.m;
                d.v = x.v;
                d.m_scale = x.m_scale;
                d.v_scale = x.v_scale;
                d.copy = (bf16_t *)x.param_copy;
                d.n = x.n;
                d.decay = x.weight_decay;
                d.first = at;
                d.vec = !(((uintptr_t)x.param & pa) || ((uintptr_t)x.grad & ga) || (((uintptr_t)x.m | (uintptr_t)x.v) & sa) ||
                          ((uintptr_t)x.param_copy & 7));
                for (i64 c = 0; c < (x.n + ADAMW_CHUNK - 1) / ADAMW_CHUNK; ++c) map[at++] = (u32)k;
            }
            h->count[kind] = at - h->first[kind];
        }
        h->stream = bytes > ADAMW_STREAM_BYTES;
        h->tensors = (const AdamwTensor *)workspace;
        h->chunks = (const u32 *)((char *)workspace + head);
        h->live = (AdamwLive *)((char *)workspace + head + up256(4 * (size_t)(chunks > 0 ? chunks : 1)));
        hipStream_t st = (hipStream_t)stream;
        hipError_t e = hipMemcpyAsync(workspace, image.data(), image.size(), hipMemcpyHostToDevice, st);
        if (e == hipSuccess) e = hipStreamSynchronize(st);
        if (e != hipSuccess) {
            delete h;
            return tn_fail(TENSAIR_EHIP, "adamw_init: %s", hipGetErrorString(e));
        }
    } catch (const std::bad_alloc &) {
        delete h;
        return tn_fail(TENSAIR_EHIP, "adamw_init: out of host memory");
    }
    *out = h;
    return TENSAIR_OK;
}

int tensair_adamw_step(tensair_adamw *h, double lr, int64_t step, double beta1, double beta2, double eps, const float *grad_scale, void *stream)
{
    if (int rc = check_step(h, beta1, beta2, eps, grad_scale)) return rc;
    if (step < 1) return tn_fail(TENSAIR_EINVAL, "steps count from 1");
    if (!(lr == lr)) return tn_fail(TENSAIR_EINVAL, "lr is NaN");
    return adamw_step(h, adamw_live(lr, step, beta1, beta2), nullptr, beta1, beta2, eps, grad_scale, (hipStream_t)stream);
}

int tensair_adamw_step_at(tensair_adamw *h, const double *lr, const int64_t *step, double beta1, double beta2, double eps, const float *grad_scale, void *stream)
{
    if (int rc = check_step(h, beta1, beta2, eps, grad_scale)) return rc;
    if (!lr || !step) return tn_fail(TENSAIR_EINVAL, "NULL pointer argument");
    if (((uintptr_t)lr | (uintptr_t)step) & 7) return tn_fail(TENSAIR_EINVAL, "lr and step must be 8-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(k_adamw_live, dim3(1), dim3(1), 0, st, h->live, lr, (const i64 *)step, beta1, beta2);
    return adamw_step(h, AdamwLive{}, h->live, beta1, beta2, eps, grad_scale, st);
}

int tensair_adamw_destroy(tensair_adamw *h)
{
    delete h;
    return TENSAIR_OK;
}

}  // extern "C"
