// Global norm of many gradient tensors, and clipping.
//
//   N_k = |u| sqrt(sum_i g_ki^2),  N = sqrt(sum_k N_k^2),  c = u * (N > M ? M / N : 1)   (c = 0 where N is not finite)
//
// The tensors are cut into units of the same number of elements, one workgroup each; a map names every unit's tensor.
// norm_units_kernel writes one partial sum per unit, norm_finish_kernel adds them in the order of the units, per tensor
// and over all, so the result does not depend on the order in which workgroups run.
//
// Bound by memory: two operations per element beside 2 or 4 bytes.  The 291 tensors of the 7B shapes in bf16, 13.5 GB: 1.91 ms, 7.1 TB/s
// (a large copy reaches 5.4, reads alone through the caches 6.1), 9 us of them the sums of 51000 units.  Clipping reads twice,
// since no element can be scaled before the last one is known, and writes once: 1.31e9 bf16 elements 1.39 ms (7.9 GB), 1.24e8 fp32 elements
// 266 us (1.5 GB: the norm 75 us, the rest at the rate of a copy).
#include "solo_ops.h"

#include <math.h>

namespace solo {

constexpr int kNormThreads = 256;
constexpr uint64_t kNormUnit = 16384;                      // elements of a unit of a small table
constexpr uint64_t kNormUnits = 1 << 16;                   // a larger table has units of so many more elements that about this many are left
constexpr int kFinishThreads = 1024;
// Gradients of up to so many bytes are partly in the last-level cache (256 MiB) when the norm is known: the norm loads them
// through the caches, and clipping, which is the last to look at them, loads and writes past them.  Of more nothing is left by
// then: the norm loads past the caches, and clipping loads and writes through them.  Clipping 1.2e8 elements: bf16, 249 MB, 148 us with plain accesses throughout, 122 us;
// fp32, 498 MB, 296 and 276 us.  Norm of 4e9 bf16 elements: 1.33 ms, past the caches 1.24 ms (6.45 TB/s).  The two sides
// cross between 360 and 500 MB.  What reads the clipped gradients next loses nothing: clipping and a step of 1.05e8 bf16 elements 285 us,
// 295 us where clipping writes through the caches.
constexpr uint64_t kLargeBytes = 384ull << 20;

struct NormEntry {
    const void *grad;
    void *clipped;
    uint64_t n;
    uint64_t unit0;         // first unit of the tensor
    uint64_t unit_elems;    // elements of a unit, the same for all tensors of the table
    uint32_t bf16;
    uint32_t large;         // the table's tensors are more than the last-level cache keeps, see kLargeBytes
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
template <bool BF16, bool PAST>
__device__ __forceinline__ double square_sum(const void *grad, uint64_t begin, uint64_t end, uint32_t thread)
{
    using Lane = Lane16<BF16>;
    constexpr int kPer = Lane::kPer, kAhead = 8;
    constexpr uint64_t kStep = kNormThreads * kPer;
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    auto add = [&](const Quad &q) {
        float x[kPer];
        Lane::unpack(q, x);
#pragma unroll
        for (int k = 0; k < kPer; ++k) sum[k & 3] = fma((double)x[k], (double)x[k], sum[k & 3]);
    };
    uint64_t i = begin + thread * kPer;
    for (; i + (kAhead - 1) * kStep + kPer <= end; i += kAhead * kStep) {
        Quad q[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) q[a] = Lane::template load<PAST>(grad, i + a * kStep);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) add(q[a]);
    }
    for (; i + kPer <= end; i += kStep) add(Lane::template load<false>(grad, i));
    for (; i < end; ++i) {                                 // the last, shorter group: one thread's
        const double x = Elements<BF16>::load1(grad, i);
        sum[0] = fma(x, x, sum[0]);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

__device__ __forceinline__ double unit_square_sum(const NormEntry &e, uint32_t unit, uint32_t thread)
{
    const uint64_t begin = (unit - e.unit0) * e.unit_elems, end = min(begin + e.unit_elems, e.n);
    if (e.large) return e.bf16 ? square_sum<true, true>(e.grad, begin, end, thread) : square_sum<false, true>(e.grad, begin, end, thread);
    return e.bf16 ? square_sum<true, false>(e.grad, begin, end, thread) : square_sum<false, false>(e.grad, begin, end, thread);
}

__global__ __launch_bounds__(kNormThreads) void norm_units_kernel(const NormArgs a)
{
    __shared__ double lds[kNormThreads / kLanes];
    const uint32_t unit = blockIdx.x;
    double sum = unit_square_sum(a.entries[a.map[unit]], unit, threadIdx.x);
    sum = group_sum(sum, lds, kNormThreads / kLanes);
    if (threadIdx.x == 0) a.partial[unit] = sum;
}

__device__ __forceinline__ double unscale_of(const NormArgs &a) { return a.unscale ? (double)*a.unscale : 1.0; }

__device__ __forceinline__ void put_norm(const NormArgs &a, double total, double u)
{
    const float norm = (float)(sqrt(total) * fabs(u));
    *a.norm = norm;
    *a.scale = !isfinite(norm) ? 0.0f : (float)(norm > a.max_norm ? u * ((double)a.max_norm / (double)norm) : u);
}

// Sum of values[0 .. n), over every `step`-th from `first` on, with eight loads under way.
__device__ __forceinline__ double strided_sum(const double *values, uint64_t n, uint64_t first, uint64_t step)
{
    double sum[8] = {};
    for (uint64_t i = first; i < n; i += 8 * step) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const double x = values[min(i + k * step, n - 1)];
            sum[k] += i + k * step < n ? x : 0.0;
        }
    }
    return ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
}

// The first workgroup adds all units, the others those of a tensor per wavefront.
__global__ __launch_bounds__(kFinishThreads) void norm_finish_kernel(const NormArgs a)
{
    __shared__ double lds[kFinishThreads / kLanes];
    const double u = unscale_of(a);
    if (blockIdx.x == 0) {
        const double total = group_sum(strided_sum(a.partial, a.units, threadIdx.x, kFinishThreads), lds, kFinishThreads / kLanes);
        if (threadIdx.x == 0) put_norm(a, total, u);
        return;
    }
    const uint32_t waves = (gridDim.x - 1) * (kFinishThreads / kLanes);
    for (uint32_t k = (blockIdx.x - 1) * (kFinishThreads / kLanes) + threadIdx.x / kLanes; k < a.count; k += waves) {
        const NormEntry &e = a.entries[k];
        const double sum = wave_sum(strided_sum(a.partial + e.unit0, (e.n + e.unit_elems - 1) / e.unit_elems, threadIdx.x % kLanes, kLanes));
        if (threadIdx.x % kLanes == 0) a.tensor_norm[k] = (float)(sqrt(sum) * fabs(u));
    }
}

// All of it by one workgroup, a quarter of it for a unit: tables of up to four units.  A vector of 4096 elements takes 3.8 us a call
// (2.4 of them the kernel) instead of 6.9 with two launches; five units and more are read faster by as many compute units.
constexpr uint32_t kSmallUnits = kFinishThreads / kNormThreads;

__global__ __launch_bounds__(kFinishThreads) void norm_small_kernel(const NormArgs a)
{
    __shared__ double lds[kFinishThreads / kLanes];
    __shared__ double partial[kSmallUnits];
    const uint32_t unit = threadIdx.x / kNormThreads, thread = threadIdx.x % kNormThreads;
    const double u = unscale_of(a);
    double sum = 0.0;
    if (unit < a.units) sum = unit_square_sum(a.entries[a.map[unit]], unit, thread);
    sum = wave_sum(sum);
    if (threadIdx.x % kLanes == 0) lds[threadIdx.x / kLanes] = sum;
    __syncthreads();
    constexpr uint32_t kWaves = kNormThreads / kLanes;
    if (threadIdx.x < kSmallUnits) {
        double s = lds[threadIdx.x * kWaves];
        for (uint32_t w = 1; w < kWaves; ++w) s += lds[threadIdx.x * kWaves + w];
        partial[threadIdx.x] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double total = 0.0;
        for (uint32_t k = 0; k < a.units; ++k) total += partial[k];
        put_norm(a, total, u);
    }
    if (!a.tensor_norm) return;
    for (uint32_t k = threadIdx.x; k < a.count; k += kFinishThreads) {
        const NormEntry &e = a.entries[k];
        const uint32_t units = (uint32_t)((e.n + e.unit_elems - 1) / e.unit_elems);
        double s = 0.0;
        for (uint32_t i = 0; i < units; ++i) s += partial[e.unit0 + i];
        a.tensor_norm[k] = (float)(sqrt(s) * fabs(u));
    }
}

// A factor of 0 (a norm that is not finite, max_norm = 0) writes zeros, also over gradients that are not finite.
template <bool BF16, bool PAST>
__device__ __forceinline__ void scale_unit(const void *grad, void *out, uint64_t begin, uint64_t end, float c)
{
    using Lane = Lane16<BF16>;
    constexpr int kPer = Lane::kPer, kAhead = 8;
    constexpr uint64_t kStep = kNormThreads * kPer;
    const bool zero = c == 0.0f;
    auto scaled = [&](const Quad &q, float x[kPer]) {
        Lane::unpack(q, x);
#pragma unroll
        for (int k = 0; k < kPer; ++k) x[k] = zero ? 0.0f : x[k] * c;
    };
    uint64_t i = begin + threadIdx.x * kPer;
    for (; i + (kAhead - 1) * kStep + kPer <= end; i += kAhead * kStep) {
        Quad q[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) q[a] = Lane::template load<PAST>(grad, i + a * kStep);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            float x[kPer];
            scaled(q[a], x);
            Lane::template store<PAST>(out, i + a * kStep, x);
        }
    }
    for (; i + kPer <= end; i += kStep) {
        float x[kPer];
        scaled(Lane::template load<false>(grad, i), x);
        Lane::template store<false>(out, i, x);
    }
    for (; i < end; ++i) Elements<BF16>::store1(out, i, zero ? 0.0f : Elements<BF16>::load1(grad, i) * c);
}

__global__ __launch_bounds__(kNormThreads) void clip_units_kernel(const NormArgs a)
{
    const uint32_t unit = blockIdx.x;
    const float c = *a.scale;
    const NormEntry e = a.entries[a.map[unit]];
    if (!e.clipped || (c == 1.0f && e.clipped == e.grad)) return;            // nothing to write
    const uint64_t begin = (unit - e.unit0) * e.unit_elems;
    const uint64_t end = min(begin + e.unit_elems, e.n);
    if (e.large) {
        if (e.bf16) scale_unit<true, false>(e.grad, e.clipped, begin, end, c);
        else scale_unit<false, false>(e.grad, e.clipped, begin, end, c);
    } else {
        if (e.bf16) scale_unit<true, true>(e.grad, e.clipped, begin, end, c);
        else scale_unit<false, true>(e.grad, e.clipped, begin, end, c);
    }
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
    if (a.units <= kSmallUnits) return launch(norm_small_kernel, dim3(1), kFinishThreads, stream, a);
    const int rc = launch(norm_units_kernel, dim3(a.units), kNormThreads, stream, a);
    if (rc != SOLO_OK) return rc;
    const uint32_t tensors = a.tensor_norm ? (a.count + kFinishThreads / kLanes - 1) / (kFinishThreads / kLanes) : 0;
    return launch(norm_finish_kernel, dim3(1 + (tensors < 256 ? tensors : 256)), kFinishThreads, stream, a);
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
    uint64_t unit0 = 0, bytes = 0;
    for (uint32_t k = 0; k < count; ++k) bytes += grads[k].n * solo::element_bytes(grads[k].dtype);
    for (uint32_t k = 0; k < count; ++k) {
        const solo_grad &g = grads[k];
        if (!solo::dtype_ok(g.dtype) || g.reserved != 0) return SOLO_E_INVALID;
        const uintptr_t size = solo::element_bytes(g.dtype);
        if (g.n != 0 && (!solo::at_multiple(g.grad, size) || (g.clipped && !solo::at_multiple(g.clipped, size)))) return SOLO_E_INVALID;
        entries[k] = solo::NormEntry{g.grad, g.clipped, g.n, unit0, unit, g.dtype == SOLO_BF16 ? 1u : 0u, bytes > solo::kLargeBytes ? 1u : 0u};
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
    return solo::launch(solo::clip_units_kernel, dim3(a.units), solo::kNormThreads, (hipStream_t)stream, a);
}

}  // extern "C"
