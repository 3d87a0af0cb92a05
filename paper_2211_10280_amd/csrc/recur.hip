// A gated linear recurrence over packed sequences, its gradient, and its form for single tokens:
//   h[t] = a[t] h[t - 1] + (1 - a[t]) x[t],  a = 1 / (1 + exp(-gate))
//   l[t] = d_out[t] + a[t + 1] l[t + 1],  d_x = (1 - a) l,  d_gate[t] = l[t] (h[t - 1] - x[t]) a[t] (1 - a[t])
// States are fp32.  The forward pass leaves the state before every RECUR_TILE'th token, from which the gradient makes the states of a tile again: that is
// 1 / 256 of x in memory, and exact, where the outputs are rounded to their type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "layers.h"

namespace {

#define RECUR_TILE 256

struct RecurArgs {
    const void *x, *gate, *d;
    void *out, *dx, *dg;
    i64 x_stride, g_stride, d_stride, out_stride, dx_stride, dg_stride, n, n_seq;
    int C4;
    const int *offsets;
    const float *h0, *d_last;
    float *h_last, *dh0, *states;
    const float *kept;           // states, as the gradient reads them
    int *status;
};

// a = 1 / (1 + exp(-g)) and b = 1 - a without the difference
__device__ __forceinline__ void gate2(float g, float &a, float &b)
{
    const float e = __expf(-(g < -87.f ? -87.f : g));
    a = 1.0f / (1.0f + e);
    b = e * a;
}
__device__ __forceinline__ void gate4(float4 g, float4 &a, float4 &b)
{
    gate2(g.x, a.x, b.x);
    gate2(g.y, a.y, b.y);
    gate2(g.z, a.z, b.z);
    gate2(g.w, a.w, b.w);
}
__device__ __forceinline__ float4 fma4(float4 a, float4 b, float4 c) { return make_float4(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w)); }

// tokens of sequence s; none, and the status bit, where the offsets are not in order
__device__ __forceinline__ void span_of(const RecurArgs &a, i64 s, i64 &lo, i64 &hi)
{
    lo = a.offsets[s];
    hi = a.offsets[s + 1];
    if (lo < 0 || hi < lo || hi > a.n) {
        if (a.status) atomicOr(a.status, ST_BAD_ORDER);
        lo = hi = 0;
    }
}

// A thread to four channels of a sequence, token after token.
template <typename T>
__global__ void __launch_bounds__(WAVE) k_recur(RecurArgs a)
{
    const i64 id = (i64)blockIdx.x * WAVE + threadIdx.x, s = id / a.C4;
    const int c = 4 * (int)(id - s * a.C4), D = 4 * a.C4;
    if (s >= a.n_seq) return;
    i64 lo, hi;
    span_of(a, s, lo, hi);
    float4 h = a.h0 ? ld4(a.h0 + s * D + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    for (i64 t = lo; t < hi; ++t) {
        if (a.states && t % RECUR_TILE == 0) st4(a.states + t / RECUR_TILE * D + c, h);
        float4 f, b;
        gate4(ld4((const T *)a.gate + t * a.g_stride + c), f, b);
        h = fma4(f, h, mul4(b, ld4((const T *)a.x + t * a.x_stride + c)));
        st4((T *)a.out + t * a.out_stride + c, h);
    }
    if (a.h_last) st4(a.h_last + s * D + c, h);
}

#define GRAD_THREADS 16
template <typename T>
__global__ void __launch_bounds__(GRAD_THREADS) k_recur_grad(RecurArgs a)
{
    __shared__ float4 before[RECUR_TILE][GRAD_THREADS];        // states of a tile: a column is one thread's
    const int me = (int)threadIdx.x;
    const i64 id = (i64)blockIdx.x * GRAD_THREADS + me, s = id / a.C4;
    const int c = 4 * (int)(id - s * a.C4), D = 4 * a.C4;
    if (s >= a.n_seq) return;
    i64 lo, hi;
    span_of(a, s, lo, hi);
    float4 l = a.d_last ? ld4(a.d_last + s * D + c) : make_float4(0.f, 0.f, 0.f, 0.f);   // a[t + 1] l[t + 1]
    for (i64 end = hi; end > lo;) {
        const i64 tile = (end - 1) / RECUR_TILE, begin = std::max(lo, tile * RECUR_TILE);
        float4 h, f, b;
        if (begin > lo) h = ld4(a.kept + tile * D + c);
        else h = a.h0 ? ld4(a.h0 + s * D + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        for (i64 t = begin; t < end; ++t) {
            before[t - begin][me] = h;
            gate4(ld4((const T *)a.gate + t * a.g_stride + c), f, b);
            h = fma4(f, h, mul4(b, ld4((const T *)a.x + t * a.x_stride + c)));
        }
        for (i64 t = end - 1; t >= begin; --t) {
            l = plus4(l, ld4((const T *)a.d + t * a.d_stride + c));
            gate4(ld4((const T *)a.gate + t * a.g_stride + c), f, b);
            const float4 x = ld4((const T *)a.x + t * a.x_stride + c), p = before[t - begin][me], dx = mul4(b, l);
            st4((T *)a.dx + t * a.dx_stride + c, dx);
            st4((T *)a.dg + t * a.dg_stride + c, mul4(make_float4(p.x - x.x, p.y - x.y, p.z - x.z, p.w - x.w), mul4(f, dx)));
            l = mul4(f, l);
        }
        end = begin;
    }
    if (a.dh0) st4(a.dh0 + s * D + c, l);
}

struct StepArgs {
    const void *x, *gate;
    void *out;
    i64 x_stride, g_stride, out_stride, state_stride, n, n_slots;
    int C4;
    const int *slots;
    float *state;
    int *status;
};

template <typename T>
__global__ void __launch_bounds__(BLOCK) k_recur_step(StepArgs a)
{
    const i64 id = (i64)blockIdx.x * BLOCK + threadIdx.x, i = id / a.C4;
    const int c = 4 * (int)(id - i * a.C4);
    if (i >= a.n) return;
    const i64 slot = a.slots ? a.slots[i] : i;
    if (slot < 0 || slot >= a.n_slots) {
        if (a.status && c == 0) atomicOr(a.status, ST_BAD_ID);
        if (a.out) st4((T *)a.out + i * a.out_stride + c, make_float4(0.f, 0.f, 0.f, 0.f));
        return;
    }
    if (a.slots)
        for (i64 j = 0; j < i; ++j)
            if (a.slots[j] == slot) return;                    // the slot's first row takes them all
    float4 h = ld4(a.state + slot * a.state_stride + c);
    for (i64 j = i; j < a.n; ++j) {
        if (j > i && (!a.slots || a.slots[j] != slot)) {
            if (!a.slots) break;
            continue;
        }
        float4 f, b;
        gate4(ld4((const T *)a.gate + j * a.g_stride + c), f, b);
        h = fma4(f, h, mul4(b, ld4((const T *)a.x + j * a.x_stride + c)));
        if (a.out) st4((T *)a.out + j * a.out_stride + c, h);
    }
    st4(a.state + slot * a.state_stride + c, h);
}

int check_recur(const void *x, i64 x_stride, const void *gate, i64 gate_stride, int32_t dtype, i64 n, int32_t dim, const int32_t *offsets, i64 n_seq,
                const void *workspace, size_t workspace_bytes, const int32_t *status)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = layer_matrix(gate, n, gate_stride, dim, dtype, "gate"))) return rc;
    if (n_seq < 0 || n_seq > TENSAIR_MAX_ROWS) return tn_fail(TENSAIR_EINVAL, "n_seq must be in 0..TENSAIR_MAX_ROWS");
    if (!offsets || ((uintptr_t)offsets & 3)) return tn_fail(TENSAIR_EINVAL, "offsets must be 4-byte aligned and not NULL");
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    return layer_workspace(workspace, workspace_bytes, tensair_recur_workspace_bytes(n, dim), "tensair_recur_workspace_bytes");
}

}  // namespace

extern "C" {

int64_t tensair_recur_state_rows(int64_t n)
{
    if (layer_sizes(n, 4)) return TENSAIR_EINVAL;
    return std::max<i64>(1, (n + RECUR_TILE - 1) / RECUR_TILE);
}

size_t tensair_recur_workspace_bytes(int64_t n, int32_t dim)
{
    if (layer_sizes(n, dim)) return 0;
    return 256;
}

int tensair_recur(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *offsets,
                  int64_t n_seq, const float *h0, void *out, int64_t out_stride, float *h_last, float *states, void *workspace, size_t workspace_bytes,
                  int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_recur(x, x_stride, gate, gate_stride, dtype, n, dim, offsets, n_seq, workspace, workspace_bytes, status))) return rc;
    if ((rc = layer_matrix(out, n, out_stride, dim, dtype, "out"))) return rc;
    if ((rc = layer_floats(h0, "h0")) || (rc = layer_floats(h_last, "h_last")) || (rc = layer_floats(states, "states"))) return rc;
    if (n_seq == 0) return TENSAIR_OK;
    RecurArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x;
    a.gate = gate;
    a.out = out;
    a.x_stride = x_stride;
    a.g_stride = gate_stride;
    a.out_stride = out_stride;
    a.n = n;
    a.n_seq = n_seq;
    a.C4 = dim / 4;
    a.offsets = offsets;
    a.h0 = h0;
    a.h_last = h_last;
    a.states = states;
    a.status = status;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)((n_seq * a.C4 + WAVE - 1) / WAVE)), blk(WAVE);
    if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_recur<float>, grid, blk, 0, st, a);
    else hipLaunchKernelGGL(k_recur<bf16_t>, grid, blk, 0, st, a);
    return layer_launched("recur");
}

int tensair_recur_grad(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *offsets,
                       int64_t n_seq, const float *h0, const float *states, const void *d_out, int64_t d_stride, const float *d_last, void *d_x,
                       int64_t d_x_stride, void *d_gate, int64_t d_gate_stride, float *d_h0, void *workspace, size_t workspace_bytes, int32_t *status, void *stream)
{
    int rc;
    if ((rc = check_recur(x, x_stride, gate, gate_stride, dtype, n, dim, offsets, n_seq, workspace, workspace_bytes, status))) return rc;
    if ((rc = layer_matrix(d_out, n, d_stride, dim, dtype, "d_out")) || (rc = layer_matrix(d_x, n, d_x_stride, dim, dtype, "d_x")) ||
        (rc = layer_matrix(d_gate, n, d_gate_stride, dim, dtype, "d_gate")))
        return rc;
    if ((rc = layer_floats(h0, "h0")) || (rc = layer_floats(states, "states")) || (rc = layer_floats(d_last, "d_last")) || (rc = layer_floats(d_h0, "d_h0"))) return rc;
    if (!states) return tn_fail(TENSAIR_EINVAL, "states is NULL");
    if (n_seq == 0) return TENSAIR_OK;
    RecurArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x;
    a.gate = gate;
    a.d = d_out;
    a.dx = d_x;
    a.dg = d_gate;
    a.x_stride = x_stride;
    a.g_stride = gate_stride;
    a.d_stride = d_stride;
    a.dx_stride = d_x_stride;
    a.dg_stride = d_gate_stride;
    a.n = n;
    a.n_seq = n_seq;
    a.C4 = dim / 4;
    a.offsets = offsets;
    a.h0 = h0;
    a.d_last = d_last;
    a.dh0 = d_h0;
    a.kept = states;
    a.status = status;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)((n_seq * a.C4 + GRAD_THREADS - 1) / GRAD_THREADS)), blk(GRAD_THREADS);
    if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_recur_grad<float>, grid, blk, 0, st, a);
    else hipLaunchKernelGGL(k_recur_grad<bf16_t>, grid, blk, 0, st, a);
    return layer_launched("recur_grad");
}

int tensair_recur_step(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, int32_t dtype, int64_t n, int32_t dim, const int32_t *slots,
                       int64_t n_slots, float *state, int64_t state_stride, void *out, int64_t out_stride, int32_t *status, void *stream)
{
    int rc;
    if ((rc = layer_sizes(n, dim))) return rc;
    if ((rc = layer_matrix(x, n, x_stride, dim, dtype, "x")) || (rc = layer_matrix(gate, n, gate_stride, dim, dtype, "gate"))) return rc;
    if (out && (rc = layer_matrix(out, n, out_stride, dim, dtype, "out"))) return rc;
    if ((rc = layer_matrix(state, n_slots, state_stride, dim, TENSAIR_F32, "state"))) return rc;
    if (n_slots < (n > 0) || n_slots > TENSAIR_MAX_ROWS) return tn_fail(TENSAIR_EINVAL, "n_slots must be in 1..TENSAIR_MAX_ROWS");
    if ((uintptr_t)slots & 3) return tn_fail(TENSAIR_EINVAL, "slots must be 4-byte aligned");
    if (slots ? n > TENSAIR_MAX_STEP_ROWS : n > n_slots) return tn_fail(TENSAIR_EINVAL, "n must be at most TENSAIR_MAX_STEP_ROWS with slots, n_slots without");
    if ((uintptr_t)status & 3) return tn_fail(TENSAIR_EINVAL, "status must be 4-byte aligned");
    if (n == 0) return TENSAIR_OK;
    const StepArgs a = {x, gate, out, x_stride, gate_stride, out_stride, state_stride, n, n_slots, dim / 4, slots, state, status};
    const u64 blocks = ((u64)n * (u64)a.C4 + BLOCK - 1) / BLOCK;
    if (blocks > TN_MAX_BLOCKS) return tn_fail(TENSAIR_EINVAL, "n * dim beyond what one launch covers");
    const dim3 grid((unsigned)blocks), blk(BLOCK);
    hipStream_t st = (hipStream_t)stream;
    if (dtype == TENSAIR_F32) hipLaunchKernelGGL(k_recur_step<float>, grid, blk, 0, st, a);
    else hipLaunchKernelGGL(k_recur_step<bf16_t>, grid, blk, 0, st, a);
    return layer_launched("recur_step");
}

}  // extern "C"
