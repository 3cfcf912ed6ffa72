// Log probabilities of given tokens, the entropy and the largest alternatives of every row of logits, and the gradient.
//
//   d_j = s (x_j - max x),  S = sum_j e^(d_j),  W = sum_j e^(d_j) d_j
//   logprob = d_t - ln S        entropy = ln S - W / S        log p_j = d_j - ln S
//   dx_j = s (a (delta_jt - p_j) - b p_j (log p_j + entropy))        a, b: gradients of logprob and entropy
//
// One workgroup takes a row, and one pass over it: every thread keeps a reference (a value near the largest one that it has
// seen) and its sums relative to that; the sums of the threads are brought to the row's maximum at the end.  Differences
// are taken before they are scaled, so a row of the type's lowest value is as good as any other.
//
// The alternatives come out of the same pass: a thread also remembers its largest logit and the group of eight that holds
// it.  The k threads with the largest of these hold the k largest logits of the row, and nothing that is smaller than the
// k-th of these is among them; only those threads' elements are read again.
#include "solo_ops.h"

#include <float.h>
#include <math.h>
#include <type_traits>

namespace solo {

constexpr int kCandidates = 1024;      // of a row, before the slower selection takes over
constexpr float kSlack = 8.0f;         // binary orders that a logit may lie above a thread's reference
constexpr float kFloor = -1000.0f;     // e^d is 0 far above this; below it d is -inf or would be no number times 0

struct RowArgs {
    const void *logits, *targets;
    void *grad;
    float *logprob, *entropy, *stats, *top_logprob;
    int32_t *rank, *top_token;
    const float *grad_logprob, *grad_entropy;
    uint64_t rows, stride, grad_stride;
    uint32_t cols, top;
    float scale;
    uint32_t wide;          // targets of 64 bits
};

// Sums of a part of a row: relative to a reference `at` in units of the logits; exponentials of base 2.
struct Sums { float at, s, w; };

__device__ __forceinline__ void rebase(Sums &a, float at, float k)
{
    // (a.s is 0 where nothing has been added, and then so is a.w)
    const float d = fmaxf((a.at - at) * k, kFloor), f = __builtin_amdgcn_exp2f(d);
    a.w = f * fmaf(a.s, d, a.w);
    a.s *= f;
    a.at = at;
}

__device__ __forceinline__ void add8(Sums &a, const float x[8], float k)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = (x[e] - a.at) * k, p = __builtin_amdgcn_exp2f(d);
        a.s += p;
        a.w = fmaf(p, fmaxf(d, kFloor), a.w);
    }
}

__device__ __forceinline__ float max8(const float x[8])
{
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}

// Logits in the order of their values, as whole numbers; -0 and +0 are the same.  Behind it the column: the lower one is the larger key.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t column)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xFFFFFFFFu - column);
}
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ uint32_t column_of(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }

__device__ __forceinline__ int64_t target_of(const RowArgs &a, uint64_t row)
{
    return a.wide ? static_cast<const int64_t *>(a.targets)[row] : (int64_t)static_cast<const int32_t *>(a.targets)[row];
}

// Group g of eight columns of a row; columns behind the last are -inf.
template <bool BF16>
__device__ __forceinline__ void read_group(const void *row, uint32_t g, uint32_t cols, float x[8])
{
    if (g * 8 + 8 <= cols) {
        Elements<BF16>::unpack(Elements<BF16>::load8(row, g * 8), x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = g * 8 + e < cols ? Elements<BF16>::load1(row, g * 8 + e) : -INFINITY;
    }
}

template <int THREADS>
struct RowLds {
    float at[THREADS / kLanes], s[THREADS / kLanes], w[THREADS / kLanes];
    uint32_t above[THREADS / kLanes];
    uint64_t key[THREADS];
    uint32_t owner[SOLO_TOP_MAX];
    uint64_t threshold, best;
    uint32_t candidates;
    uint64_t candidate[kCandidates];
};
template <int THREADS>
struct RowLdsSmall { float at[THREADS / kLanes], s[THREADS / kLanes], w[THREADS / kLanes]; uint32_t above[THREADS / kLanes]; };

// The sums of a row, for every thread; `largest` and `where`: this thread's largest logit and its group.
template <bool BF16, bool TOP, bool RANK, int THREADS, typename Lds>
__device__ __forceinline__ Sums row_sums(const void *row, uint32_t cols, float k, float target, Lds &lds, float &largest, uint32_t &where, uint32_t &above)
{
    Sums a = {-FLT_MAX, 0.0f, 0.0f};
    largest = -INFINITY;
    where = threadIdx.x;
    uint32_t count = 0;
    const uint32_t groups = (cols + 7) / 8;
    for (uint32_t g = threadIdx.x; g < groups; g += THREADS) {
        float x[8];
        read_group<BF16>(row, g, cols, x);
        const float m = max8(x);
        if ((m - a.at) * k > kSlack) rebase(a, m, k);
        if (TOP && m > largest) { largest = m; where = g; }
        if (RANK) {
#pragma unroll
            for (int e = 0; e < 8; ++e) count += x[e] > target;
        }
        add8(a, x, k);
    }
    // bring the sums of the wavefront, then of the workgroup, to one reference: the largest of the threads'
    float at = a.at;
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) at = fmaxf(at, __shfl_xor(at, d));
    rebase(a, at, k);
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    if (RANK) count = wave_sum(count);
    const int wave = threadIdx.x / kLanes;
    if (threadIdx.x % kLanes == 0) {
        lds.at[wave] = a.at; lds.s[wave] = a.s; lds.w[wave] = a.w;
        lds.above[wave] = count;
    }
    __syncthreads();
    at = lds.at[0];
    for (int w = 1; w < THREADS / kLanes; ++w) at = fmaxf(at, lds.at[w]);
    Sums all = {at, 0.0f, 0.0f};
    above = 0;
    for (int w = 0; w < THREADS / kLanes; ++w) {
        Sums part = {lds.at[w], lds.s[w], lds.w[w]};
        rebase(part, at, k);
        all.s += part.s;
        all.w += part.w;
        above += lds.above[w];
    }
    return all;
}

// The a.top largest logits of a row, by key; `mine` is this thread's largest (0 if it has none).
template <bool BF16, int THREADS>
__device__ __forceinline__ void row_top(const RowArgs &a, const void *row, uint64_t out, uint64_t mine, const Sums &all, RowLds<THREADS> &lds)
{
    const uint32_t groups = (a.cols + 7) / 8, found = min(a.top, a.cols);
    const float log_s = __builtin_amdgcn_logf(all.s);
    float *const value = a.top_logprob + out * a.top;
    int32_t *const token = a.top_token + out * a.top;
    auto put = [&](uint32_t at, uint64_t key) {
        const float x = value_of(key);
        value[at] = all.s == 0.0f ? -INFINITY : fmaf(x - all.at, a.scale, -log_s * kLn2);
        token[at] = (int32_t)column_of(key);
    };
    lds.key[threadIdx.x] = mine;
    if (threadIdx.x == 0) lds.candidates = 0;
    __syncthreads();
    uint32_t larger = 0;
    for (int t = 0; t < THREADS; ++t) larger += lds.key[t] > mine;
    const uint32_t owners = min(found, min(groups, (uint32_t)THREADS));        // threads that have a key at all, at most a.top of them
    if (mine != 0 && larger < owners) {
        lds.owner[larger] = threadIdx.x;
        if (larger == owners - 1) lds.threshold = owners == found ? mine : 0;  // (fewer threads than alternatives: every element is a candidate)
    }
    __syncthreads();
    const uint64_t threshold = lds.threshold;
    // groups of the owners: owner, owner + THREADS, ...
    const uint32_t each = (groups + THREADS - 1) / THREADS;
    for (uint32_t i = threadIdx.x; i < owners * each; i += THREADS) {
        const uint32_t g = lds.owner[i % owners] + i / owners * THREADS;
        if (g >= groups) continue;
        float x[8];
        read_group<BF16>(row, g, a.cols, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint64_t key = key_of(x[e], g * 8 + e);
            if (g * 8 + e < a.cols && key >= threshold) {
                const uint32_t at = atomicAdd(&lds.candidates, 1u);
                if (at < kCandidates) lds.candidate[at] = key;
            }
        }
    }
    __syncthreads();
    const uint32_t count = lds.candidates;
    if (count <= kCandidates) {
        for (uint32_t i = threadIdx.x; i < count; i += THREADS) {
            const uint64_t key = lds.candidate[i];
            uint32_t before = 0;
            for (uint32_t j = 0; j < count; ++j) before += lds.candidate[j] > key;
            if (before < found) put(before, key);
        }
    } else {                                               // large logits crowd in few threads: one alternative after the other
        uint64_t last = ~0ull;
        for (uint32_t r = 0; r < found; ++r) {
            uint64_t best = 0;
            for (uint32_t i = threadIdx.x; i < owners * each; i += THREADS) {
                const uint32_t g = lds.owner[i % owners] + i / owners * THREADS;
                if (g >= groups) continue;
                float x[8];
                read_group<BF16>(row, g, a.cols, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint64_t key = key_of(x[e], g * 8 + e);
                    if (g * 8 + e < a.cols && key < last && key > best) best = key;
                }
            }
            __syncthreads();
            lds.key[threadIdx.x] = best;
            __syncthreads();
            for (int t = 0; t < THREADS; ++t) best = lds.key[t] > best ? lds.key[t] : best;
            if (threadIdx.x == 0) put(r, best);
            last = best;
        }
    }
    for (uint32_t r = found + threadIdx.x; r < a.top; r += THREADS) {
        value[r] = -INFINITY;
        token[r] = -1;
    }
}

__device__ __forceinline__ float row_entropy(const Sums &all)
{
    return all.s == 0.0f ? 0.0f : (__builtin_amdgcn_logf(all.s) - all.w / all.s) * kLn2;
}
__device__ __forceinline__ float row_logprob(const Sums &all, float target, float scale)
{
    return all.s == 0.0f ? -INFINITY : fmaf(target - all.at, scale, -__builtin_amdgcn_logf(all.s) * kLn2);
}

template <bool BF16, bool TOP, bool RANK, int THREADS>
__global__ __launch_bounds__(THREADS) void logprob_kernel(const RowArgs a)
{
    __shared__ typename std::conditional<TOP, RowLds<THREADS>, RowLdsSmall<THREADS>>::type lds;
    const float k = a.scale * kLog2E;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const char *row = static_cast<const char *>(a.logits) + r * a.stride * Elements<BF16>::kBytes;
        const int64_t t = a.targets ? target_of(a, r) : 0;
        const bool has = a.targets != nullptr;
        if (has && (t < 0 || t >= (int64_t)a.cols)) {      // no target: the row is not read
            if (threadIdx.x == 0) {
                if (a.logprob) a.logprob[r] = 0.0f;
                if (a.entropy) a.entropy[r] = 0.0f;
                if (a.rank) a.rank[r] = -1;
                if (a.stats) { a.stats[2 * r] = 0.0f; a.stats[2 * r + 1] = 0.0f; }
            }
            if (TOP)
                for (uint32_t i = threadIdx.x; i < a.top; i += THREADS) {
                    a.top_logprob[r * a.top + i] = -INFINITY;
                    a.top_token[r * a.top + i] = -1;
                }
            continue;
        }
        const float target = has ? Elements<BF16>::load1(row, t) : 0.0f;
        float largest;
        uint32_t where, above;
        const Sums all = row_sums<BF16, TOP, RANK, THREADS>(row, a.cols, k, target, lds, largest, where, above);
        if (threadIdx.x == 0) {
            if (a.logprob && has) a.logprob[r] = row_logprob(all, target, a.scale);
            if (a.entropy) a.entropy[r] = row_entropy(all);
            if (RANK) a.rank[r] = (int32_t)above;
            if (a.stats) { a.stats[2 * r] = all.at; a.stats[2 * r + 1] = all.s; }
        }
        if constexpr (TOP) {
            uint64_t mine = 0;
            if (where * 8 < a.cols) {                       // the lowest column of the group that holds the largest one
                float x[8];
                read_group<BF16>(row, where, a.cols, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint64_t key = key_of(x[e], where * 8 + e);
                    if (where * 8 + e < a.cols && key > mine) mine = key;
                }
            }
            row_top<BF16, THREADS>(a, row, r, mine, all, lds);
        }
        __syncthreads();                                   // (the sums in lds)
    }
}

// dx of group g; `at` and `s` of the row's sums.
template <bool BF16>
__device__ __forceinline__ void put_gradient(const void *row, void *out, uint32_t g, uint32_t cols, uint32_t target, float at, float s, float k, float scale, float a, float b, float entropy)
{
    float x[8];
    read_group<BF16>(row, g, cols, x);
    const float inverse = s == 0.0f ? 0.0f : 1.0f / s, log_s = s == 0.0f ? 0.0f : __builtin_amdgcn_logf(s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = (x[e] - at) * k, p = __builtin_amdgcn_exp2f(d) * inverse;
        const float inner = fmaxf(d - log_s, kFloor) * kLn2 + entropy;
        x[e] = -p * fmaf(b, inner, a);
        if (g * 8 + e == target && s != 0.0f) x[e] += a;
        x[e] *= scale;
    }
    if (g * 8 + 8 <= cols) {
        Elements<BF16>::store8(out, g * 8, x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (g * 8 + e < cols) Elements<BF16>::store1(out, g * 8 + e, x[e]);
    }
}

template <bool BF16>
__device__ __forceinline__ void put_zeros(void *out, uint32_t g, uint32_t cols)
{
    const float none[8] = {};
    if (g * 8 + 8 <= cols) {
        Elements<BF16>::store8(out, g * 8, none);
    } else {
        for (uint32_t c = g * 8; c < cols; ++c) Elements<BF16>::store1(out, c, 0.0f);
    }
}

// FORWARD: the sums first, then the gradient, of a row that the caches still hold; else from the sums that are given.
template <bool BF16, bool FORWARD, int THREADS>
__global__ __launch_bounds__(THREADS) void logprob_grad_kernel(const RowArgs a)
{
    __shared__ RowLdsSmall<THREADS> lds;
    const float k = a.scale * kLog2E;
    const uint32_t groups = (a.cols + 7) / 8;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const char *row = static_cast<const char *>(a.logits) + r * a.stride * Elements<BF16>::kBytes;
        char *out = static_cast<char *>(a.grad) + r * a.grad_stride * Elements<BF16>::kBytes;
        const int64_t t = a.targets ? target_of(a, r) : -1;
        if (a.targets && (t < 0 || t >= (int64_t)a.cols)) {
            for (uint32_t g = threadIdx.x; g < groups; g += THREADS) put_zeros<BF16>(out, g, a.cols);
            if (FORWARD && threadIdx.x == 0) {
                if (a.logprob) a.logprob[r] = 0.0f;
                if (a.entropy) a.entropy[r] = 0.0f;
            }
            continue;
        }
        const float up = a.grad_logprob && a.targets ? a.grad_logprob[r] : 0.0f, up_entropy = a.grad_entropy ? a.grad_entropy[r] : 0.0f;
        Sums all;
        float entropy;
        if (FORWARD) {
            const float target = a.targets ? Elements<BF16>::load1(row, t) : 0.0f;
            float largest;
            uint32_t where, above;
            all = row_sums<BF16, false, false, THREADS>(row, a.cols, k, target, lds, largest, where, above);
            entropy = row_entropy(all);
            if (threadIdx.x == 0) {
                if (a.logprob && a.targets) a.logprob[r] = row_logprob(all, target, a.scale);
                if (a.entropy) a.entropy[r] = entropy;
            }
        } else {
            all.at = a.stats[2 * r];
            all.s = a.stats[2 * r + 1];
            entropy = a.entropy[r];
        }
        for (uint32_t g = threadIdx.x; g < groups; g += THREADS)
            put_gradient<BF16>(row, out, g, a.cols, (uint32_t)t, all.at, all.s, k, a.scale, up, up_entropy, entropy);
        if (FORWARD) __syncthreads();
    }
}

// ---- host ------------------------------------------------------------------------------------
static int rows_args(RowArgs &a, const void *logits, const void *targets, const solo_logits *s)
{
    if (!s || !dtype_ok(s->dtype) || (s->target_bits != 32 && s->target_bits != 64) || s->top > SOLO_TOP_MAX || s->reserved != 0 || s->reserved2 != 0 ||
        !(s->scale > 0.0f) || !isfinite(s->scale) || !isfinite(s->scale * kLog2E) || s->stride < s->cols)
        return SOLO_E_INVALID;
    if (s->rows != 0 && ((s->cols != 0 && !at_multiple(logits, element_bytes(s->dtype))) ||
                         (targets && !at_multiple(targets, s->target_bits / 8))))
        return SOLO_E_INVALID;
    if (s->cols >= (1ull << 31) || s->rows >= (1ull << 40) || s->stride >= (1ull << 40) || s->grad_stride >= (1ull << 40)) return SOLO_E_UNSUPPORTED;
    a = RowArgs{};
    a.logits = logits; a.targets = targets;
    a.rows = s->rows; a.cols = (uint32_t)s->cols; a.stride = s->stride; a.grad_stride = s->grad_stride;
    a.top = s->top; a.scale = s->scale; a.wide = s->target_bits == 64;
    return SOLO_OK;
}

static bool optional_at(const void *p, uintptr_t size) { return !p || at_multiple(p, size); }

static uint32_t row_grid(uint64_t rows) { return (uint32_t)(rows < (1u << 20) ? rows : 1u << 20); }

template <int THREADS>
static void logprob_launch(const RowArgs &a, bool bf16, hipStream_t stream)
{
    void (*kernel)(RowArgs);
    const bool top = a.top != 0, rank = a.rank != nullptr;
    if (bf16) kernel = top ? (rank ? logprob_kernel<true, true, true, THREADS> : logprob_kernel<true, true, false, THREADS>)
                           : (rank ? logprob_kernel<true, false, true, THREADS> : logprob_kernel<true, false, false, THREADS>);
    else kernel = top ? (rank ? logprob_kernel<false, true, true, THREADS> : logprob_kernel<false, true, false, THREADS>)
                      : (rank ? logprob_kernel<false, false, true, THREADS> : logprob_kernel<false, false, false, THREADS>);
    hipLaunchKernelGGL(kernel, dim3(row_grid(a.rows)), dim3(THREADS), 0, stream, a);
}

constexpr uint64_t kFewRows = 512;     // up to so many rows a workgroup has 1024 threads instead of 256

}  // namespace solo

extern "C" {

int solo_logprob(const void *logits, const void *targets, float *logprob, float *entropy, int32_t *rank, float *top_logprob, int32_t *top_token,
                 float *stats, const solo_logits *shape, void *stream)
{
    using namespace solo;
    RowArgs a;
    const int rc = rows_args(a, logits, targets, shape);
    if (rc != SOLO_OK) return rc;
    if (shape->rows == 0) return SOLO_OK;
    if (!optional_at(logprob, 4) || !optional_at(entropy, 4) || !optional_at(rank, 4) || !optional_at(stats, 4) ||
        ((logprob || rank) && !targets) || (shape->top != 0 && (!at_multiple(top_logprob, 4) || !at_multiple(top_token, 4))))
        return SOLO_E_INVALID;
    a.logprob = logprob; a.entropy = entropy; a.rank = rank; a.top_logprob = top_logprob; a.top_token = top_token; a.stats = stats;
    if (a.rows <= kFewRows) logprob_launch<1024>(a, shape->dtype == SOLO_BF16, (hipStream_t)stream);
    else logprob_launch<256>(a, shape->dtype == SOLO_BF16, (hipStream_t)stream);
    return launched();
}

int solo_logprob_grad(const void *logits, const void *targets, const float *entropy, const float *stats, const float *grad_logprob,
                      const float *grad_entropy, void *grad_logits, const solo_logits *shape, void *stream)
{
    using namespace solo;
    RowArgs a;
    const int rc = rows_args(a, logits, targets, shape);
    if (rc != SOLO_OK) return rc;
    if (shape->grad_stride < shape->cols) return SOLO_E_INVALID;
    if (shape->rows == 0 || shape->cols == 0) return SOLO_OK;
    if (!at_multiple(entropy, 4) || !at_multiple(stats, 4) || !optional_at(grad_logprob, 4) || !optional_at(grad_entropy, 4) ||
        (!grad_logprob && !grad_entropy) || (grad_logprob && !targets) || !at_multiple(grad_logits, element_bytes(shape->dtype)))
        return SOLO_E_INVALID;
    a.entropy = const_cast<float *>(entropy); a.stats = const_cast<float *>(stats);
    a.grad_logprob = grad_logprob; a.grad_entropy = grad_entropy; a.grad = grad_logits;
    hipLaunchKernelGGL((shape->dtype == SOLO_BF16 ? logprob_grad_kernel<true, false, 256> : logprob_grad_kernel<false, false, 256>),
                       dim3(row_grid(a.rows)), dim3(256), 0, (hipStream_t)stream, a);
    return launched();
}

int solo_logprob_with_grad(const void *logits, const void *targets, const float *grad_logprob, const float *grad_entropy, float *logprob,
                           float *entropy, void *grad_logits, const solo_logits *shape, void *stream)
{
    using namespace solo;
    RowArgs a;
    const int rc = rows_args(a, logits, targets, shape);
    if (rc != SOLO_OK) return rc;
    if (shape->grad_stride < shape->cols) return SOLO_E_INVALID;
    if (shape->rows == 0) return SOLO_OK;
    if (!optional_at(logprob, 4) || !optional_at(entropy, 4) || !optional_at(grad_logprob, 4) || !optional_at(grad_entropy, 4) ||
        (!grad_logprob && !grad_entropy) || ((logprob || grad_logprob) && !targets) ||
        (shape->cols != 0 && !at_multiple(grad_logits, element_bytes(shape->dtype))))
        return SOLO_E_INVALID;
    a.logprob = logprob; a.entropy = entropy;
    a.grad_logprob = grad_logprob; a.grad_entropy = grad_entropy; a.grad = grad_logits;
    hipLaunchKernelGGL((shape->dtype == SOLO_BF16 ? logprob_grad_kernel<true, true, 512> : logprob_grad_kernel<false, true, 512>),
                       dim3(row_grid(a.rows)), dim3(512), 0, (hipStream_t)stream, a);
    return launched();
}

}  // extern "C"
