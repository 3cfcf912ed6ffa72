// What the operators on rows of logits have in common: how a row is dealt out to the threads of its workgroup, the order of logits.
#pragma once
#include "solo_ops.h"

namespace solo {

// (NaN wins; three operands an instruction, where fmaxf first quiets each of its own)
template <int N>
__device__ __forceinline__ float max_of(const float x[N])
{
    float m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(x[0], x[1]), x[2]);
    if constexpr (N == 4) return __builtin_elementwise_maximum(m, x[3]);
    m = __builtin_elementwise_maximum(m, __builtin_elementwise_maximum(__builtin_elementwise_maximum(x[3 % N], x[4 % N]), x[5 % N]));
    return __builtin_elementwise_maximum(m, __builtin_elementwise_maximum(x[6 % N], x[7 % N]));
}

// Logits in the order of their values, as whole numbers; -0 and +0 are the same.  A key has the column behind it: the lower one is larger.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, uint32_t column) { return (uint64_t)order << 32 | (0xFFFFFFFFu - column); }
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ uint32_t column_of(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }

// A row is cut into groups of columns, 16 bytes each, dealt out to the threads in turn, and the few columns behind the last whole
// group, one each to the first threads.
template <bool BF16>
struct Row {
    using Lane = Lane16<BF16>;
    static constexpr uint32_t kPer = Lane::kPer;
    const void *at;
    uint32_t groups, rest;      // whole groups; columns behind them

    template <typename Args>
    __device__ __forceinline__ Row(const Args &a, uint64_t r)
        : at(static_cast<const char *>(a.logits) + r * a.stride * Lane::kBytes), groups(a.cols / kPer), rest(a.cols % kPer) {}
    __device__ __forceinline__ bool has_share(uint32_t thread) const { return thread < groups || thread < rest; }
    template <bool PAST = false>
    __device__ __forceinline__ Quad group(uint32_t g) const { return Lane::template load_near<PAST>(at, g * kPer); }
    __device__ __forceinline__ float one(uint32_t column) const { return Elements<BF16>::load1(at, column); }
    // The column behind the groups that a thread has (if it is less than `rest`).
    __device__ __forceinline__ uint32_t last_column(uint32_t thread) const { return groups * kPer + thread; }
};

// The first DEPTH groups of a thread; one that it does not have is another's.
template <bool BF16, bool PAST, int THREADS, int DEPTH>
__device__ __forceinline__ void first_groups(const Row<BF16> &row, Quad q[DEPTH])
{
    if (row.groups == 0) return;
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) q[j] = row.template group<PAST>(min(j * THREADS + threadIdx.x, row.groups - 1));
}

}  // namespace solo
