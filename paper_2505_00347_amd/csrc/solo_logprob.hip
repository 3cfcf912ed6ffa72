// Log probabilities of given tokens, the entropy and the largest alternatives of every row of logits, and the gradient.
//
//   d_j = s (x_j - max x),  S = sum_j e^(d_j),  W = sum_j e^(d_j) d_j
//   logprob = d_t - ln S        entropy = ln S - W / S        log p_j = d_j - ln S
//   dx_j = s (a (delta_jt - p_j) - b p_j (log p_j + entropy))        a, b: gradients of logprob and entropy
//
// One workgroup takes a row, and one pass over it: every thread keeps the largest logit that it has seen and its sums relative
// to that; the sums of the threads are brought to the row's maximum at the end.  S is then 1 or more, and d_t - ln S of a target with nearly all
// of the probability loses no digits.  (A reference that may lie up to 8 binary orders below the maximum saves few exponentials, sums of
// 4096 x 50304 bf16 67.1 us instead of 68.2, and costs up to 1e-6 of such a log probability.)  Differences
// are taken before they are scaled, so a row of the type's lowest value is as good as any other.
//
// The alternatives come out of the same pass: a thread also remembers its largest logit, the group that holds it and the largest
// one of its other groups.  From the threads' largest follows a value that the k largest logits of the row are not below, and that
// few others reach (row_top()); only the groups that can hold one are looked at again, one for most threads that have any.
//
// Bound by memory where there are many rows: sums of 4096 x 50304 bf16 68 us (6.0 TB/s), with rank and twenty alternatives 82 us; loss and
// gradient of 8192 x 32000 in one call 172 us (the row stays in registers: 1.05 GB, 6.1 TB/s), 168 us where a tenth of the rows has no target;
// of 1000 x 50257 fp32 in two calls 98 us.
// A logit costs some twelve instructions and an exponential, 36 us of vector issue for 4096 x 50304; the alternatives add what a row costs once.
// A single row of 50257 takes 9.8 us: one compute unit's exponentials, and loads of 4 us.
#include "solo_ops.h"

#include <float.h>
#include <math.h>
#include <type_traits>

namespace solo {

constexpr int kCandidates = 512;       // logits that are collected for the alternatives, before a slower selection takes over
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

// Sums of a part of a row: relative to its largest logit, `at`; exponentials of base 2.
struct Sums { float at, s, w; };

__device__ __forceinline__ void rebase(Sums &a, float at, float k)
{
    // (a.s is 0 where nothing has been added, and then so is a.w)
    const float d = fmaxf((a.at - at) * k, kFloor), f = __builtin_amdgcn_exp2f(d);
    a.w = f * fmaf(a.s, d, a.w);
    a.s *= f;
    a.at = at;
}

__device__ __forceinline__ void add1(Sums &a, float x, float k)
{
    const float d = (x - a.at) * k, p = __builtin_amdgcn_exp2f(d);
    a.s += p;
    a.w = fmaf(p, fmaxf(d, kFloor), a.w);
}

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

__device__ __forceinline__ int64_t target_of(const RowArgs &a, uint64_t row)
{
    return a.wide ? static_cast<const int64_t *>(a.targets)[row] : (int64_t)static_cast<const int32_t *>(a.targets)[row];
}

// A row is cut into groups of columns, 16 bytes each, dealt out to the threads in turn, and the few columns behind the last whole
// group, one each to the first threads.
template <bool BF16>
struct Row {
    using Lane = Lane16<BF16>;
    static constexpr uint32_t kPer = Lane::kPer;
    const void *at;
    uint32_t groups, rest;      // whole groups; columns behind them

    __device__ __forceinline__ Row(const RowArgs &a, uint64_t r)
        : at(static_cast<const char *>(a.logits) + r * a.stride * Lane::kBytes), groups(a.cols / kPer), rest(a.cols % kPer) {}
    __device__ __forceinline__ bool has_share(uint32_t thread) const { return thread < groups || thread < rest; }
    template <bool PAST = false>
    __device__ __forceinline__ Quad group(uint32_t g) const { return Lane::template load_near<PAST>(at, g * kPer); }
    __device__ __forceinline__ float one(uint32_t column) const { return Elements<BF16>::load1(at, column); }
    // The column behind the groups that a thread has (if it is less than `rest`).
    __device__ __forceinline__ uint32_t last_column(uint32_t thread) const { return groups * kPer + thread; }
};

template <int THREADS>
struct SumLds { float at[THREADS / kLanes], s[THREADS / kLanes], w[THREADS / kLanes]; uint32_t above[THREADS / kLanes]; };

template <int THREADS>
struct TopLds : SumLds<THREADS> {
    uint32_t largest[kLanes];                  // of the shares, as ordered whole numbers
    uint32_t column[THREADS];                  // where the threshold stands first among a thread's logits
    uint32_t threshold, last_column;
    uint32_t holders, owners, candidates;
    uint32_t owner[THREADS];
    uint64_t candidate[kCandidates];
    uint32_t before[kCandidates];              // candidates with a larger key
    uint64_t best[THREADS / kLanes];
};

// What a thread remembers of its logits for the alternatives: the largest one, the group that holds it, and the largest one of its
// other groups.  (The column behind the groups counts as a group, with the number behind theirs.)
struct Largest {
    float first = -INFINITY, second = -INFINITY;
    uint32_t group = 0xFFFFFFFFu;
    __device__ __forceinline__ void see(float m, uint32_t g)
    {
        second = __builtin_amdgcn_fmed3f(second, m, first);        // (of second <= first and m, the middle one)
        group = m > first ? g : group;
        first = m > first ? m : first;
    }
};

// The first DEPTH groups of a thread; one that it does not have is another's.
template <bool BF16, bool PAST, int THREADS, int DEPTH>
__device__ __forceinline__ void first_groups(const Row<BF16> &row, Quad q[DEPTH])
{
    if (row.groups == 0) return;
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) q[j] = row.template group<PAST>(min(j * THREADS + threadIdx.x, row.groups - 1));
}

// The sums of a row, for every thread.  `q`: first_groups() of the row, which with RESIDENT, for rows of no more than THREADS * DEPTH
// groups, are all of them; otherwise the loads of the next DEPTH groups are under way while DEPTH are added.  `last`: the thread's
// column behind the groups.
template <bool BF16, bool TOP, bool RANK, bool RESIDENT, bool PAST, int THREADS, int DEPTH>
__device__ __forceinline__ Sums row_sums(const Row<BF16> &row, float k, float target, SumLds<THREADS> &lds, Quad q[DEPTH],
                                         float last, Largest &largest, uint32_t &above)
{
    Sums a = {-FLT_MAX, 0.0f, 0.0f};
    uint32_t count = 0;
    constexpr int kPer = Row<BF16>::kPer;
    auto add = [&](const Quad &quad, uint32_t g) {
        float x[kPer];
        Lane16<BF16>::unpack(quad, x);
        const float m = max_of<kPer>(x);
        if (m > a.at) rebase(a, m, k);
        if (TOP) largest.see(m, g);
        if (RANK) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) count += x[e] > target;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) add1(a, x[e], k);
    };
    uint32_t g0 = 0;
    if (!RESIDENT)
        for (; g0 + THREADS * DEPTH <= row.groups; g0 += THREADS * DEPTH) {
            Quad now[DEPTH];
#pragma unroll
            for (int j = 0; j < DEPTH; ++j) {
                now[j] = q[j];
                q[j] = row.template group<PAST>(min(g0 + THREADS * DEPTH + j * THREADS + threadIdx.x, row.groups - 1));
            }
#pragma unroll
            for (int j = 0; j < DEPTH; ++j) add(now[j], g0 + j * THREADS + threadIdx.x);
        }
#pragma unroll
    for (int j = 0; j < DEPTH; ++j)
        if (g0 + j * THREADS + threadIdx.x < row.groups) add(q[j], g0 + j * THREADS + threadIdx.x);
    if (threadIdx.x < row.rest) {
        if (last > a.at) rebase(a, last, k);
        if (TOP) largest.see(last, row.groups);
        if (RANK) count += last > target;
        add1(a, last, k);
    }
    const float at = wave_max(a.at);
    rebase(a, at, k);
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    if (RANK) count = wave_sum(count);
    above = count;
    if (THREADS == kLanes) return a;
    const int wave = threadIdx.x / kLanes;
    if (threadIdx.x % kLanes == 0) {
        lds.at[wave] = a.at; lds.s[wave] = a.s; lds.w[wave] = a.w;
        lds.above[wave] = count;
    }
    __syncthreads();
    constexpr int kWaves = THREADS / kLanes;
    const int part = threadIdx.x % kWaves;                 // every wavefront adds the wavefronts' sums, several times over
    Sums all = {lds.at[part], lds.s[part], lds.w[part]};
    above = lds.above[part];
    rebase(all, wave_max<kWaves>(all.at), k);
    all.s = wave_sum<kWaves>(all.s);
    all.w = wave_sum<kWaves>(all.w);
    if (RANK) above = wave_sum<kWaves>(above);
    return all;
}

// The a.top largest logits of a row.  The threads of one lane number, one in each wavefront, have a share of the row; with T the
// a.top-th largest of the 64 shares' largest logits, a.top logits at least are no smaller than T, and only threads whose own
// largest is no smaller hold any.  These are few, unless many share the value T: then, C being the a.top-th lowest of the
// columns where threads hold T first, a logit T behind column C is none of the alternatives.
template <bool BF16, int THREADS>
__device__ __forceinline__ void row_top(const RowArgs &a, const Row<BF16> &row, uint64_t out, const Largest &largest, const Sums &all, TopLds<THREADS> &lds)
{
    const uint32_t found = min(a.top, a.cols), each = (row.groups + THREADS - 1) / THREADS + 1;      // (groups of a thread, and its column behind them)
    const float log_s = __builtin_amdgcn_logf(all.s) * kLn2;
    const uint32_t lane = threadIdx.x % kLanes;
    auto put = [&](uint32_t at, uint64_t key) {
        a.top_logprob[out * a.top + at] = all.s == 0.0f ? -INFINITY : fmaf(value_of(key) - all.at, a.scale, -log_s);
        a.top_token[out * a.top + at] = (int32_t)column_of(key);
    };
    auto put_none = [&](uint32_t at) {
        a.top_logprob[out * a.top + at] = -INFINITY;
        a.top_token[out * a.top + at] = -1;
    };
    const bool any = row.has_share(threadIdx.x);
    const uint32_t mine = any ? order_of(largest.first) : 0;
    if (THREADS == kLanes) lds.largest[lane] = mine;
    else atomicMax(&lds.largest[lane], mine);              // (0 from the row before)
    __syncthreads();
    if (threadIdx.x < kLanes) {
        const uint32_t own = lds.largest[lane];
        uint32_t larger = 0;
#pragma unroll 4
        for (int t = 0; t < kLanes; t += 4) {
            const uint4 o = *reinterpret_cast<const uint4 *>(&lds.largest[t]);
            larger += (o.x > own) + (o.y > own) + (o.z > own) + (o.w > own);
        }
        // the smallest that fewer than `found` exceed; 0 where there are fewer shares
        const uint32_t it = ~wave_max(larger < found ? ~own : 0u);
        if (lane == 0) lds.threshold = it;
    }
    __syncthreads();
    const uint32_t threshold = lds.threshold;
    const float at_least = threshold == 0 ? -INFINITY : value_of((uint64_t)threshold << 32);
    const bool holds = any && mine >= threshold;
    bool counts = holds;
    const uint64_t holding = __ballot(holds);
    if (lane == 0 && holding != 0) atomicAdd(&lds.holders, (uint32_t)__popcll(holding));
    __syncthreads();
    const uint32_t holders = lds.holders;
    uint32_t last_column = 0xFFFFFFFFu;
    if (holders > (THREADS == kLanes ? found : 2 * found) + 8) {            // several hold the same value: their columns decide
        uint32_t column = 0xFFFFFFFFu;
        if (any && mine == threshold) {
            for (uint32_t g = threadIdx.x; g < row.groups && column == 0xFFFFFFFFu; g += THREADS) {
                float x[Row<BF16>::kPer];
                Lane16<BF16>::unpack(row.group(g), x);
#pragma unroll
                for (int e = Row<BF16>::kPer - 1; e >= 0; --e)
                    if (order_of(x[e]) == threshold) column = g * Row<BF16>::kPer + e;
            }
            if (column == 0xFFFFFFFFu && threadIdx.x < row.rest) column = row.last_column(threadIdx.x);
        }
        lds.column[threadIdx.x] = column;
        __syncthreads();
        if (threadIdx.x == 0) lds.last_column = 0xFFFFFFFFu;
        uint32_t lower = 0;
        if (column != 0xFFFFFFFFu) {
#pragma unroll 2
            for (int t = 0; t < THREADS; t += 4) {
                const uint4 o = *reinterpret_cast<const uint4 *>(&lds.column[t]);
                lower += (o.x < column) + (o.y < column) + (o.z < column) + (o.w < column);
            }
        }
        __syncthreads();
        if (column != 0xFFFFFFFFu && lower == found - 1) lds.last_column = column;     // (none where fewer hold it: then all of them count)
        __syncthreads();
        last_column = lds.last_column;
        counts = holds && (mine > threshold || column <= last_column);
    }
    // the logits of a group, from column `column` on, that count (a NaN does not)
    auto look = [&](const float *x, int n, uint32_t column, auto &&use) {
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < n; ++e)
            hits |= (x[e] > at_least || (x[e] == at_least && column + e <= last_column) ? 1u : 0u) << e;
        while (hits != 0) {                                // (one, mostly)
            const uint32_t e = __builtin_ctz(hits);
            hits &= hits - 1;
            float it = x[0];
#pragma unroll
            for (int o = 1; o < n; ++o) it = (int)e == o ? x[o] : it;
            use(key_of(order_of(it), column + e));
        }
    };
    auto look_at_group = [&](uint32_t g, uint32_t thread, auto &&use) {
        float x[Row<BF16>::kPer];
        if (g < row.groups) {
            Lane16<BF16>::unpack(row.group(g), x);
            look(x, Row<BF16>::kPer, g * Row<BF16>::kPer, use);
        } else if (g == row.groups && thread < row.rest) {
            x[0] = row.one(row.last_column(thread));
            look(x, 1, row.last_column(thread), use);
        }
    };
    auto collect = [&](uint64_t key) {
        const uint32_t at = atomicAdd(&lds.candidates, 1u);
        if (at < kCandidates) lds.candidate[at] = key;
    };
    // most threads hold theirs in one group; all groups of the others are looked through by everyone
    const bool one_group = counts && order_of(largest.second) < threshold;
    if (one_group) look_at_group(largest.group, threadIdx.x, collect);
    else if (counts) lds.owner[atomicAdd(&lds.owners, 1u)] = threadIdx.x;
    __syncthreads();
    const uint32_t owners = lds.owners;
    auto keys_of = [&](uint32_t i, auto &&use) {
        const uint32_t turn = i / owners, owner = lds.owner[i - turn * owners];
        const uint32_t g = owner + turn * THREADS;
        if (turn == each - 1) look_at_group(row.groups, owner, use);
        else if (g < row.groups) look_at_group(g, owner, use);
    };
    for (uint32_t i = threadIdx.x; i < owners * each; i += THREADS) keys_of(i, collect);
    if (owners != 0) __syncthreads();
    const uint32_t count = lds.candidates;
    if (count <= kCandidates) {
        // a thread compares one candidate with every (THREADS / kLanes)-th
        constexpr uint32_t kParts = THREADS / kLanes;
        for (uint32_t i = lane; i < count; i += kLanes) {
            const uint64_t key = lds.candidate[i];
            uint32_t before = 0;
#pragma unroll 4
            for (uint32_t j = threadIdx.x / kLanes; j < count; j += kParts) before += lds.candidate[j] > key;
            if (kParts == 1) {
                if (before < found) put(before, key);
            } else if (before) {
                atomicAdd(&lds.before[i], before);         // (0 from the row before)
            }
        }
        if (kParts > 1) {
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < count; i += THREADS) {
                const uint32_t before = lds.before[i];
                lds.before[i] = 0;
                if (before < found) put(before, lds.candidate[i]);
            }
        }
    } else {                                               // large logits crowd in few threads: one alternative after the other
        uint64_t last = ~0ull;
        for (uint32_t r = 0; r < found; ++r) {
            uint64_t best = 0;
            auto better = [&](uint64_t key) { if (key < last && key > best) best = key; };
            if (one_group) look_at_group(largest.group, threadIdx.x, better);
            for (uint32_t i = threadIdx.x; i < owners * each; i += THREADS) keys_of(i, better);
            best = wave_max(best);
            __syncthreads();                               // (best of the round before)
            if (lane == 0) lds.best[threadIdx.x / kLanes] = best;
            __syncthreads();
            for (int w = 0; w < THREADS / kLanes; ++w) best = lds.best[w] > best ? lds.best[w] : best;
            if (threadIdx.x == 0) {
                if (best != 0) put(r, best);
                else put_none(r);
            }
            last = best;
        }
    }
    // behind the last column (and in a row of NaN)
    for (uint32_t r = min(found, count) + threadIdx.x; r < a.top; r += THREADS) put_none(r);
    __syncthreads();
    if (threadIdx.x < kLanes) lds.largest[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        lds.holders = 0;
        lds.owners = 0;
        lds.candidates = 0;
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

// Wavefronts per SIMD that the registers have to leave room for.
constexpr int forward_waves(bool top, int threads) { return !top ? 8 : threads < 512 ? 6 : 5; }

template <bool BF16, bool TOP, bool RANK, bool PAST, int THREADS, int DEPTH>
__global__ __launch_bounds__(THREADS, forward_waves(TOP, THREADS)) void logprob_kernel(const RowArgs a)
{
    __shared__ __align__(16) typename std::conditional<TOP, TopLds<THREADS>, SumLds<THREADS>>::type lds;
    const float k = a.scale * kLog2E;
    if constexpr (TOP) {                                   // (the barriers of row_sums stand between this and its first use)
        if (threadIdx.x < kLanes) lds.largest[threadIdx.x] = 0;
        for (uint32_t i = threadIdx.x; i < kCandidates; i += THREADS) lds.before[i] = 0;
        if (threadIdx.x == 0) {
            lds.holders = 0;
            lds.owners = 0;
            lds.candidates = 0;
        }
    }
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<BF16> row(a, r);
        const bool has = a.targets != nullptr;
        const int64_t t = has ? target_of(a, r) : 0;
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
        Quad q[DEPTH];
        first_groups<BF16, PAST, THREADS, DEPTH>(row, q);
        const float target = has ? row.one((uint32_t)t) : 0.0f;
        const float last = threadIdx.x < row.rest ? row.one(row.last_column(threadIdx.x)) : -INFINITY;
        Largest largest;
        uint32_t above;
        const Sums all = row_sums<BF16, TOP, RANK, false, PAST, THREADS, DEPTH>(row, k, target, lds, q, last, largest, above);
        if (threadIdx.x == 0) {
            if (a.logprob && has) a.logprob[r] = row_logprob(all, target, a.scale);
            if (a.entropy) a.entropy[r] = row_entropy(all);
            if (RANK) a.rank[r] = (int32_t)above;
            if (a.stats) { a.stats[2 * r] = all.at; a.stats[2 * r + 1] = all.s; }
        }
        if constexpr (TOP) row_top<BF16, THREADS>(a, row, r, largest, all, lds);
        __syncthreads();                                   // (the sums in lds)
    }
}

// What the gradient of a row needs: p_j = 2^((x_j - at) k - log_s), dx_j = p_j (a + b (ln p_j + entropy)), and what is added at the target.
struct Slope { float at, log_s, a, b, entropy, target; };

__device__ __forceinline__ Slope slope_of(float at, float s, float entropy, float up, float up_entropy, float scale)
{
    // (no column of a row without probabilities has one: 2^-inf)
    return Slope{at, s == 0.0f ? INFINITY : __builtin_amdgcn_logf(s), -scale * up, -scale * up_entropy, entropy, s == 0.0f ? 0.0f : scale * up};
}

template <bool ENTROPY>
__device__ __forceinline__ float gradient_of(float x, const Slope &s, float k)
{
    const float d = fmaf(x - s.at, k, -s.log_s), p = __builtin_amdgcn_exp2f(d);
    return p * (ENTROPY ? fmaf(s.b, fmaf(fmaxf(d, kFloor), kLn2, s.entropy), s.a) : s.a);
}

template <bool BF16, bool ENTROPY, bool PAST>
__device__ __forceinline__ void put_gradient(const Quad &q, void *out, uint32_t g, uint32_t target, const Slope &s, float k)
{
    constexpr int kPer = Row<BF16>::kPer;
    float x[kPer];
    Lane16<BF16>::unpack(q, x);
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = gradient_of<ENTROPY>(x[e], s, k);
    if (g == target / kPer) {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (e == (int)(target % kPer)) x[e] += s.target;
    }
    Lane16<BF16>::template store_near<PAST>(out, g * kPer, x);
}

// Wavefronts per SIMD that the registers have to leave room for.  Rows that stay in registers: two workgroups of 1024 threads, so that
// one loads while the other computes, where 64 registers are enough; else as many as the row's own registers allow.
constexpr int grad_waves(bool bf16, bool forward, bool resident, int threads, int depth)
{
    if (!forward || !resident) return 8;
    if (depth > (bf16 ? 4 : 8)) return 4;
    return bf16 ? 8 : threads == 1024 ? 4 : 5;
}

// FORWARD: the sums first, then the gradient; else from the sums that are given.  RESIDENT: the row has no more than THREADS * DEPTH
// groups, which stay in registers between the two.
template <bool BF16, bool FORWARD, bool RESIDENT, bool ENTROPY, int PAST, int THREADS, int DEPTH>
__global__ __launch_bounds__(THREADS, grad_waves(BF16, FORWARD, RESIDENT, THREADS, DEPTH)) void logprob_grad_kernel(const RowArgs a)
{
    __shared__ SumLds<THREADS> lds;
    const float k = a.scale * kLog2E;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<BF16> row(a, r);
        char *out = static_cast<char *>(a.grad) + r * a.grad_stride * Elements<BF16>::kBytes;
        const int64_t t = a.targets ? target_of(a, r) : -1;
        if (a.targets && (t < 0 || t >= (int64_t)a.cols)) {
            const float none[Row<BF16>::kPer] = {};
            for (uint32_t g = threadIdx.x; g < row.groups; g += THREADS) Lane16<BF16>::template store_near<(PAST > 0)>(out, g * Row<BF16>::kPer, none);
            if (threadIdx.x < row.rest) Elements<BF16>::store1(out, row.last_column(threadIdx.x), 0.0f);
            if (FORWARD && threadIdx.x == 0) {
                if (a.logprob) a.logprob[r] = 0.0f;
                if (a.entropy) a.entropy[r] = 0.0f;
            }
            continue;
        }
        const float up = a.grad_logprob && a.targets ? a.grad_logprob[r] : 0.0f, up_entropy = ENTROPY ? a.grad_entropy[r] : 0.0f;
        Quad raw[DEPTH];
        float at, s, entropy;
        const float last = threadIdx.x < row.rest ? row.one(row.last_column(threadIdx.x)) : -INFINITY;
        if (FORWARD) {
            const float target = a.targets ? row.one((uint32_t)t) : 0.0f;
            Largest largest;
            uint32_t above;
            first_groups<BF16, (PAST > 1), THREADS, DEPTH>(row, raw);
            const Sums all = row_sums<BF16, false, false, RESIDENT, (PAST > 1), THREADS, DEPTH>(row, k, target, lds, raw, last, largest, above);
            at = all.at;
            s = all.s;
            entropy = row_entropy(all);
            if (threadIdx.x == 0) {
                if (a.logprob && a.targets) a.logprob[r] = row_logprob(all, target, a.scale);
                if (a.entropy) a.entropy[r] = entropy;
            }
        } else {
            at = a.stats[2 * r];
            s = a.stats[2 * r + 1];
            entropy = a.entropy[r];
        }
        const Slope slope = slope_of(at, s, entropy, up, up_entropy, a.scale);
        for (uint32_t g0 = threadIdx.x; g0 < row.groups; g0 += THREADS * DEPTH) {
            if (!(FORWARD && RESIDENT)) {
#pragma unroll
                for (int j = 0; j < DEPTH; ++j)
                    if (g0 + j * THREADS < row.groups) raw[j] = row.template group<(PAST > 1)>(g0 + j * THREADS);
            }
#pragma unroll
            for (int j = 0; j < DEPTH; ++j)
                if (g0 + j * THREADS < row.groups) {
                    // (what has been unpacked for the sums is not kept: it would take twice the registers)
                    if (FORWARD && RESIDENT) forget(raw[j]);
                    put_gradient<BF16, ENTROPY, (PAST > 0)>(raw[j], out, g0 + j * THREADS, (uint32_t)t, slope, k);
                }
            if (FORWARD && RESIDENT) break;
        }
        if (threadIdx.x < row.rest) {
            const uint32_t column = row.last_column(threadIdx.x);
            Elements<BF16>::store1(out, column, gradient_of<ENTROPY>(last, slope, k) + (column == (uint32_t)t ? slope.target : 0.0f));
        }
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
    if (s->cols >= (1ull << 29) || s->rows >= (1ull << 40) || s->stride >= (1ull << 40) || s->grad_stride >= (1ull << 40)) return SOLO_E_UNSUPPORTED;
    a = RowArgs{};
    a.logits = logits; a.targets = targets;
    a.rows = s->rows; a.cols = (uint32_t)s->cols; a.stride = s->stride; a.grad_stride = s->grad_stride;
    a.top = s->top; a.scale = s->scale; a.wide = s->target_bits == 64;
    return SOLO_OK;
}

static bool optional_at(const void *p, uintptr_t size) { return !p || at_multiple(p, size); }

static uint32_t row_grid(uint64_t rows) { return (uint32_t)(rows < (1u << 20) ? rows : 1u << 20); }

// Logits of more bytes than the last-level cache (256 MiB) keeps are read past the caches (412 MB: 75 and 67 us; 80 MB that the head has
// just written: 25 and 27), and gradients that are not small are written past them (64 MB: 25.6 and 20.7 us; 524 MB, with the
// loads, 185 and 171).  The product that reads the gradient next finds less of it in the caches: call and product together are
// between 3.5 % faster and 3.5 % slower for it at 41 to 256 MB, by the product (bf16 1024 x 32000 with 768 columns 216.5 us past the caches, 216.3
// through them; 1000 x 50257 417 and 403; 1000 x 50304 323 and 327; fp32 512 x 32000 with 256 columns, the worst, 215 and 199).
constexpr uint64_t kPastLoads = 256ull << 20, kPastStores = 32ull << 20;

static uint64_t logits_bytes(const RowArgs &a, bool bf16) { return a.rows * a.cols * (bf16 ? 2 : 4); }

template <bool BF16, bool TOP, int THREADS, int DEPTH>
static int logprob_launch(const RowArgs &a, hipStream_t stream)
{
    const bool rank = a.rank != nullptr;
    void (*kernel)(RowArgs);
    if (logits_bytes(a, BF16) > kPastLoads)
        kernel = rank ? logprob_kernel<BF16, TOP, true, true, THREADS, DEPTH> : logprob_kernel<BF16, TOP, false, true, THREADS, DEPTH>;
    else
        kernel = rank ? logprob_kernel<BF16, TOP, true, false, THREADS, DEPTH> : logprob_kernel<BF16, TOP, false, false, THREADS, DEPTH>;
    return launch(kernel, dim3(row_grid(a.rows)), THREADS, stream, a);
}

template <bool BF16, bool FORWARD, bool RESIDENT, int THREADS, int DEPTH>
static int grad_launch(const RowArgs &a, hipStream_t stream)
{
    constexpr int kDepth = BF16 ? DEPTH : 2 * DEPTH;
    const uint64_t bytes = logits_bytes(a, BF16);
    void (*kernel)(RowArgs);
    constexpr int kBoth = FORWARD && !RESIDENT ? 1 : 2;    // (a row that is read twice stays in the caches)
    if (a.grad_entropy) kernel = bytes > kPastLoads    ? logprob_grad_kernel<BF16, FORWARD, RESIDENT, true, kBoth, THREADS, kDepth>
                                 : bytes > kPastStores ? logprob_grad_kernel<BF16, FORWARD, RESIDENT, true, 1, THREADS, kDepth>
                                                       : logprob_grad_kernel<BF16, FORWARD, RESIDENT, true, 0, THREADS, kDepth>;
    else kernel = bytes > kPastLoads    ? logprob_grad_kernel<BF16, FORWARD, RESIDENT, false, kBoth, THREADS, kDepth>
                  : bytes > kPastStores ? logprob_grad_kernel<BF16, FORWARD, RESIDENT, false, 1, THREADS, kDepth>
                                        : logprob_grad_kernel<BF16, FORWARD, RESIDENT, false, 0, THREADS, kDepth>;
    return launch(kernel, dim3(row_grid(a.rows)), THREADS, stream, a);
}

// A wavefront takes a row by itself where rows are short, or where there are enough of them that no compute unit waits and they
// are not so long that all wavefronts look for their alternatives at the same time; few rows get more threads each.  (16384 rows of
// 4096 columns, bf16, five alternatives: 40 us, with 256 threads 69; 4096 rows of 50304, twenty: 108 us, with 256 threads 82;
// one row of 50257: 31 us, with 256 threads 12, with 512 threads 10.)  With alternatives, 256 threads have one load of bf16 ahead instead of two: the
// registers leave room for another wavefront, 82 instead of 84 us.  (groups: of eight columns)
template <bool BF16, bool TOP>
static int logprob_rows(const RowArgs &a, hipStream_t stream)
{
    const uint32_t groups = a.cols / 8;
    constexpr int kDepth = BF16 ? 2 : 4;
    if (groups <= 256 || (a.rows >= 4096 && groups <= 2048)) return logprob_launch<BF16, TOP, 64, kDepth>(a, stream);
    if (a.rows >= 128 || groups <= 1024) return logprob_launch<BF16, TOP, 256, BF16 && TOP ? 1 : kDepth>(a, stream);
    return logprob_launch<BF16, TOP, 512, kDepth>(a, stream);
}

// The fewest threads that hold the row with four groups of eight columns each, so that two workgroups share a compute unit and one
// loads while the other computes; up to 65536 columns eight each, one workgroup.  (8192 x 32000 bf16: 1024 threads with four 172 us, 512 with
// eight 174, 256 with sixteen 219, reading the row twice 200; 20000 x 8000: 256 with four 107, twice 208; 4096 x 50304: 1024 with eight 165,
// 512 with sixteen 189.)  Longer rows are read twice, 1024 threads: 2000 x 100000 182 us, with 512 197.
template <bool BF16>
static int with_grad_launch(const RowArgs &a, hipStream_t stream)
{
    const uint32_t groups = (a.cols + 7) / 8;              // (all of them have to fit)
    if (groups <= 64 * 4) return grad_launch<BF16, true, true, 64, 4>(a, stream);
    if (groups <= 256 * 4) return grad_launch<BF16, true, true, 256, 4>(a, stream);
    if (groups <= 512 * 4) return grad_launch<BF16, true, true, 512, 4>(a, stream);
    if (groups <= 1024 * 4) return grad_launch<BF16, true, true, 1024, 4>(a, stream);
    if (groups <= 1024 * 8) return grad_launch<BF16, true, true, 1024, 8>(a, stream);
    return grad_launch<BF16, true, false, 1024, 2>(a, stream);
}

// Two or three groups of a row for each thread.  (8192 x 32000 bf16: 1024 threads 184 us, 512 197, 256 205; 20000 x 3000: 256 47, 1024 108;
// 40000 x 500: 64 17, 256 23.)
template <bool BF16>
static int only_grad_launch(const RowArgs &a, hipStream_t stream)
{
    const uint32_t groups = a.cols / 8;
    if (groups <= 128) return grad_launch<BF16, false, false, 64, 2>(a, stream);
    if (groups <= 256) return grad_launch<BF16, false, false, 128, 2>(a, stream);
    if (groups <= 640) return grad_launch<BF16, false, false, 256, 2>(a, stream);
    if (groups <= 1536) return grad_launch<BF16, false, false, 512, 2>(a, stream);
    return grad_launch<BF16, false, false, 1024, 2>(a, stream);
}

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
    const hipStream_t s = (hipStream_t)stream;
    if (shape->dtype == SOLO_BF16) return a.top ? logprob_rows<true, true>(a, s) : logprob_rows<true, false>(a, s);
    return a.top ? logprob_rows<false, true>(a, s) : logprob_rows<false, false>(a, s);
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
    return shape->dtype == SOLO_BF16 ? only_grad_launch<true>(a, (hipStream_t)stream) : only_grad_launch<false>(a, (hipStream_t)stream);
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
    return shape->dtype == SOLO_BF16 ? with_grad_launch<true>(a, (hipStream_t)stream) : with_grad_launch<false>(a, (hipStream_t)stream);
}

}  // extern "C"
