// Global norm of many gradient tensors, and clipping.
//
//   N_k = |u| sqrt(sum_i g_ki^2),  N = sqrt(sum_k N_k^2),  c = u * (N > M ? M / N : 1)   (c = 0 where N is not finite)
//
// The tensors are cut into units of the same number of elements, one workgroup each; a map names every unit's tensor.
// norm_units_kernel writes one partial sum per unit, norm_finish_kernel adds them in the order of the units, per tensor
// and over all, so the result does not depend on the order in which workgroups run.
#include "solo_ops.h"

#include <math.h>

namespace solo {

constexpr int kNormThreads = 256;
constexpr uint64_t kNormUnit = 16384;                      // elements of a unit of a small table
constexpr uint64_t kNormUnits = 1 << 16;                   // a larger table has units of so many more elements that about this many are left
constexpr int kFinishThreads = 1024;

struct NormEntry {
    const void *grad;
    void *clipped;
    uint64_t n;
    uint64_t unit0;         // first unit of the tensor
    uint64_t unit_elems;    // elements of a unit, the same for all tensors of the table
    uint32_t bf16;
    uint32_t reserved;
};
static_assert(sizeof(NormEntry) == 48, "table layout");

struct NormArgs {
    const NormEntry *entries;
    const uint32_t *map;
    double *partial;        // one per unit
    const float *unscale;   // may be null
    float *norm, *scale, *tensor_norm;      // the last may be null
    float max_norm;
    uint32_t count, units;
};

// Sum of the squares of elements [begin, end) over the workgroup's threads (each thread's part of it).
// Squares and sums are binary64: the square of a finite binary32 value never overflows or vanishes there, and the kernel
// waits for memory, not for the additions.
template <bool BF16>
__device__ __forceinline__ double square_sum(const void *grad, uint64_t begin, uint64_t end)
{
    using E = Elements<BF16>;
    constexpr int kAhead = BF16 ? 8 : 4;
    constexpr uint64_t kStep = kNormThreads * 8;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    uint64_t i = begin + threadIdx.x * 8;
    for (; i + (kAhead - 1) * kStep + 8 <= end; i += kAhead * kStep) {
        typename E::Raw raw[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) raw[a] = E::load8(grad, i + a * kStep);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            float x[8];
            E::unpack(raw[a], x);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k & 3] = fma((double)x[k], (double)x[k], sum[k & 3]);
        }
    }
    for (; i + 8 <= end; i += kStep) {
        float x[8];
        E::unpack(E::load8(grad, i), x);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k & 3] = fma((double)x[k], (double)x[k], sum[k & 3]);
    }
    for (; i < end; ++i) {                                  // the last, shorter group of eight: one thread's
        const double x = E::load1(grad, i);
        sum[0] = fma(x, x, sum[0]);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

__global__ __launch_bounds__(kNormThreads) void norm_units_kernel(const NormArgs a)
{
    __shared__ double lds[kNormThreads / kLanes];
    const uint32_t unit = blockIdx.x;
    const NormEntry e = a.entries[a.map[unit]];
    const uint64_t begin = (unit - e.unit0) * e.unit_elems;
    const uint64_t end = min(begin + e.unit_elems, e.n);
    double sum = e.bf16 ? square_sum<true>(e.grad, begin, end) : square_sum<false>(e.grad, begin, end);
    sum = group_sum(sum, lds, kNormThreads / kLanes);
    if (threadIdx.x == 0) a.partial[unit] = sum;
}

__global__ __launch_bounds__(kFinishThreads) void norm_finish_kernel(const NormArgs a)
{
    __shared__ double lds[kFinishThreads / kLanes];
    const double u = a.unscale ? (double)*a.unscale : 1.0;
    double total = 0.0;
    for (uint32_t i = threadIdx.x; i < a.units; i += kFinishThreads) total += a.partial[i];
    total = group_sum(total, lds, kFinishThreads / kLanes);
    if (threadIdx.x == 0) {
        const float norm = (float)(sqrt(total) * fabs(u));
        *a.norm = norm;
        float c = 0.0f;
        if (isfinite(norm)) c = (float)(norm > a.max_norm ? u * ((double)a.max_norm / (double)norm) : u);
        *a.scale = c;
    }
    if (!a.tensor_norm) return;
    const int wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    for (uint32_t k = wave; k < a.count; k += kFinishThreads / kLanes) {
        const uint64_t first = a.entries[k].unit0, units = (a.entries[k].n + a.entries[k].unit_elems - 1) / a.entries[k].unit_elems;
        double sum = 0.0;
        for (uint64_t i = lane; i < units; i += kLanes) sum += a.partial[first + i];
        sum = wave_sum(sum);
        if (lane == 0) a.tensor_norm[k] = (float)(sqrt(sum) * fabs(u));
    }
}

// A factor of 0 (a norm that is not finite, max_norm = 0) writes zeros, also over gradients that are not finite.
template <bool BF16>
__device__ __forceinline__ void scale_unit(const void *grad, void *out, uint64_t begin, uint64_t end, float c)
{
    using E = Elements<BF16>;
    constexpr int kAhead = 4;
    constexpr uint64_t kStep = kNormThreads * 8;
    const bool zero = c == 0.0f;
    uint64_t i = begin + threadIdx.x * 8;
    for (; i + (kAhead - 1) * kStep + 8 <= end; i += kAhead * kStep) {
        typename E::Raw raw[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) raw[a] = E::load8(grad, i + a * kStep);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            float x[8];
            E::unpack(raw[a], x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = zero ? 0.0f : x[k] * c;
            E::store8(out, i + a * kStep, x);
        }
    }
    for (; i + 8 <= end; i += kStep) {
        float x[8];
        E::unpack(E::load8(grad, i), x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = zero ? 0.0f : x[k] * c;
        E::store8(out, i, x);
    }
    for (; i < end; ++i) E::store1(out, i, zero ? 0.0f : E::load1(grad, i) * c);
}

__global__ __launch_bounds__(kNormThreads) void clip_units_kernel(const NormArgs a)
{
    const uint32_t unit = blockIdx.x;
    const float c = *a.scale;
    const NormEntry e = a.entries[a.map[unit]];
    if (!e.clipped || (c == 1.0f && e.clipped == e.grad)) return;            // nothing to write
    const uint64_t begin = (unit - e.unit0) * e.unit_elems;
    const uint64_t end = min(begin + e.unit_elems, e.n);
    if (e.bf16) scale_unit<true>(e.grad, e.clipped, begin, end, c);
    else scale_unit<false>(e.grad, e.clipped, begin, end, c);
}

static uint64_t unit_elems(const solo_grad *grads, uint32_t count)
{
    uint64_t total = 0, unit = kNormUnit;
    for (uint32_t k = 0; k < count; ++k) total += grads[k].n;
    while (total / unit >= kNormUnits) unit *= 2;
    return unit;
}

static uint64_t units_of(uint64_t n, uint64_t unit) { return (n + unit - 1) / unit; }

static bool small_enough(const solo_grad *grads, uint32_t count)
{
    for (uint32_t k = 0; k < count; ++k)
        if (grads[k].n > (1ull << 40)) return false;
    return true;
}

static int norm_args(NormArgs &a, const void *table, uint32_t count, uint64_t units, const float *unscale, float max_norm,
                     float *norm, float *grad_scale, float *tensor_norm, void *workspace)
{
    if (!(max_norm >= 0.0f)) return SOLO_E_INVALID;
    if (count == 0 || !at_multiple(table, 16) || !at_multiple(norm, 4) || !at_multiple(grad_scale, 4) ||
        (unscale && !at_multiple(unscale, 4)) || (tensor_norm && !at_multiple(tensor_norm, 4)) || !at_multiple(workspace, 16))
        return SOLO_E_INVALID;
    if (units >= (1ull << 24)) return SOLO_E_UNSUPPORTED;  // (as many workgroups of 256 as one launch takes)
    a.entries = static_cast<const NormEntry *>(table);
    a.map = reinterpret_cast<const uint32_t *>(a.entries + count);
    a.partial = static_cast<double *>(workspace);
    a.unscale = unscale;
    a.norm = norm; a.scale = grad_scale; a.tensor_norm = tensor_norm;
    a.max_norm = max_norm;
    a.count = count; a.units = (uint32_t)units;
    return SOLO_OK;
}

static int norm(const NormArgs &a, hipStream_t stream)
{
    if (a.units) hipLaunchKernelGGL(norm_units_kernel, dim3(a.units), dim3(kNormThreads), 0, stream, a);
    hipLaunchKernelGGL(norm_finish_kernel, dim3(1), dim3(kFinishThreads), 0, stream, a);
    return launched();
}

}  // namespace solo

extern "C" {

uint64_t solo_norm_units(const solo_grad *grads, uint32_t count)
{
    if (!grads || !solo::small_enough(grads, count)) return 0;
    const uint64_t unit = solo::unit_elems(grads, count);
    uint64_t units = 0;
    for (uint32_t k = 0; k < count; ++k) units += solo::units_of(grads[k].n, unit);
    return units;
}

size_t solo_norm_table_bytes(uint32_t count, uint64_t units)
{
    return (size_t)count * sizeof(solo::NormEntry) + (size_t)units * sizeof(uint32_t);
}

size_t solo_norm_workspace_bytes(uint64_t units) { return (size_t)(units ? units : 1) * sizeof(double); }

int solo_norm_table_build(const solo_grad *grads, uint32_t count, void *table_host, size_t table_bytes)
{
    if (!grads || !table_host || count == 0) return SOLO_E_INVALID;
    if (!solo::small_enough(grads, count)) return SOLO_E_UNSUPPORTED;
    const uint64_t units = solo_norm_units(grads, count), unit = solo::unit_elems(grads, count);
    if (units >= (1ull << 24)) return SOLO_E_UNSUPPORTED;
    if (table_bytes < solo_norm_table_bytes(count, units)) return SOLO_E_INVALID;
    solo::NormEntry *entries = static_cast<solo::NormEntry *>(table_host);
    uint32_t *map = reinterpret_cast<uint32_t *>(entries + count);
    uint64_t unit0 = 0;
    for (uint32_t k = 0; k < count; ++k) {
        const solo_grad &g = grads[k];
        if (!solo::dtype_ok(g.dtype) || g.reserved != 0) return SOLO_E_INVALID;
        const uintptr_t size = solo::element_bytes(g.dtype);
        if (g.n != 0 && (!solo::at_multiple(g.grad, size) || (g.clipped && !solo::at_multiple(g.clipped, size)))) return SOLO_E_INVALID;
        entries[k] = solo::NormEntry{g.grad, g.clipped, g.n, unit0, unit, g.dtype == SOLO_BF16 ? 1u : 0u, 0u};
        for (uint64_t u = 0; u < solo::units_of(g.n, unit); ++u) map[unit0++] = k;
    }
    return SOLO_OK;
}

int solo_grad_norm(const void *table_device, uint32_t count, uint64_t units, const float *unscale, float max_norm, float *norm,
                   float *grad_scale, float *tensor_norm, void *workspace, void *stream)
{
    solo::NormArgs a;
    const int rc = solo::norm_args(a, table_device, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace);
    return rc != SOLO_OK ? rc : solo::norm(a, (hipStream_t)stream);
}

int solo_grad_clip(const void *table_device, uint32_t count, uint64_t units, const float *unscale, float max_norm, float *norm,
                   float *grad_scale, float *tensor_norm, void *workspace, void *stream)
{
    solo::NormArgs a;
    int rc = solo::norm_args(a, table_device, count, units, unscale, max_norm, norm, grad_scale, tensor_norm, workspace);
    if (rc == SOLO_OK) rc = solo::norm(a, (hipStream_t)stream);
    if (rc != SOLO_OK || units == 0) return rc;
    hipLaunchKernelGGL(solo::clip_units_kernel, dim3(a.units), dim3(solo::kNormThreads), 0, (hipStream_t)stream, a);
    return solo::launched();
}

}  // extern "C"
