// Sampling: of every row of logits one column, by a given uniform number.
//
//   w_j = e^((x_j - max x) / temperature), the columns in the order of their logits, ties by the lower column
//   kept: the first top_k of those with w >= min_p, and of these the shortest beginning that has top_p of their sum
//   the token is the first column, in that order, at which the running sum of the kept w exceeds uniform * their sum
//
// Each of the three is a place in the order at which a running sum (of ones or of w) reaches a goal, and none needs the order itself: a
// histogram over the distance from the maximum gives the bucket that holds the place, and only that bucket's columns are looked at
// again: up to 64 by one wavefront, each against all others; more are listed and cut by whole keys, value and column, until the part that holds the place
// has no more than 64; more than the list holds (equal logits, mostly) are cut that way from the row itself.  Where top_k or min_p leave few columns, which a bound on their logits shows beforehand, only these are weighed and put in order.
//
// Which column it is hangs on comparisons of sums, so these are exact: w is computed in binary64 (the rate of its instructions is that of
// binary32), to 2e-13, and rounded to a whole multiple of 2^-shift of the largest; sums of such are whole numbers below 2^63, the same in every order, and atomic
// additions in LDS make them.
//
// A workgroup takes a row.  One row of 50257 fp32, nucleus of 0.95, 20 us: 3 until the maximum is known, 8.5 for weights and buckets (25 vector instructions for 64
// columns on each of four SIMDs), 1 to add up, 3.5 for each of two places, most of it the pass over the row.  One after the other, without the next one's chain of
// instructions beside its own, the weights took 13.  1024 x 32000 fp32, the whole distribution, 50 us: 2.6 TB/s, vector instructions and loads about half of it each,
// side by side only where two rows of a compute unit are at different stages.  1024 x 50257 bf16 with min_p and nucleus 57 to 67 us, from card to card.
#include "solo_rows.h"

#include <float.h>
#include <math.h>

namespace solo {

// Buckets of the distance from the maximum, 64 binary orders of w in all; columns above a bound that are kept instead of the row; columns of a bucket that are
// listed; parts that a list is cut into.  What a row has in LDS says how many rows a compute unit has under way, and what it clears and adds up is much of a
// short row's work: two workgroups of 512 threads, whose registers allow no more, five of 256 (5000 rows of 4000 bf16, nucleus: 56 us, with the long rows' sizes
// 118) and twenty of one wavefront (100000 rows of 300 fp32: 150, with lists twice as long 160).  With half the buckets a long row's places take 4 to 7 % longer;
// with half the list 1024 rows of 50257 bf16 of which min_p leaves up to 4000 columns take 75 us instead of 66 on the same card.
template <int THREADS>
struct Sizes {
    static constexpr bool kShort = THREADS == kLanes, kMiddle = THREADS == 256;
    static constexpr uint32_t kBuckets = kShort ? 256 : kMiddle ? 512 : 2048, kKept = kShort ? 128 : kMiddle ? 1024 : 4096, kListed = kShort ? 128 : 1024,
                              kSub = kShort ? 64 : 512;
};

// Up to this many columns their number says how fine weights can be, and a sum is off by 2^-25 of the largest weight at most: half of what a number of 24 bits
// tells apart.  In longer rows it would be 2^-23, 2^-21 and so on; there their sum says it, which takes a pass more (four rows of 1000000 fp32, nucleus: 973 us, 897 without).
constexpr uint32_t kCountedCols = 1u << 19;

// 2^(i / 32)
__constant__ const double kRoots[32] = {
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0,
};

struct SampleArgs {
    const void *logits;
    const float *uniform, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    void *token;
    float *logprob;
    uint64_t rows, stride;
    uint32_t cols, wide;
    float one_temperature, one_top_p, one_min_p;
    int32_t one_top_k;
    uint32_t shift;
};

typedef uint32_t Words __attribute__((ext_vector_type(2)));

template <int THREADS>
struct SampleLds {
    static constexpr uint32_t kBuckets = Sizes<THREADS>::kBuckets, kKept = Sizes<THREADS>::kKept, kListed = Sizes<THREADS>::kListed,
                              kSub = Sizes<THREADS>::kSub;
    uint64_t mass[kBuckets + 1];       // sums of the buckets, then of all in front of a bucket
    uint32_t count[kBuckets + 1];
    float sub_x[kListed];              // of those in a bucket
    uint32_t sub_column[kListed];
    float few_x[kLanes];               // of a part of those
    uint32_t few_column[kLanes];
    uint64_t sub_mass[kSub];
    uint32_t sub_count[kSub];
    uint64_t key[kLanes], weight[kLanes];
    Words root[32];                    // 2^(i / 32) times 2^shift, less what i adds to the exponent below
    uint64_t wave_mass[THREADS / kLanes], lowest, highest;
    uint32_t wave_count[THREADS / kLanes];
    float at[THREADS / kLanes], last[8];
    uint32_t listed, bucket;
    uint64_t found_key, found_mass;
    double inverse, below, nucleus;    // of temperature; uniform and top_p, within their ends
    float x[kKept];                    // of the columns above a bound (last: what lies beyond 64 KB costs address registers)
    uint32_t column[kKept];
};

// threadIdx.x, as something that the compiler does not know: addresses made of it are made where they are used.  Made in front of the loop
// over the places to find and kept, as they would be, they take forty registers.
__device__ __forceinline__ uint32_t this_thread()
{
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    return thread;
}

// w as a whole number of 2^-shift, its logarithm, and how far that lies below 0, in eighths of a 32nd (64 orders for all below).
struct Weight {
    uint64_t w;
    double order;
    uint32_t below;
    template <int THREADS>
    __device__ __forceinline__ uint32_t bucket() const { return below / (16384 / Sizes<THREADS>::kBuckets); }
};

// The weights of a row.
struct Weights {
    double max, per_order;             // (x - max) * per_order is log2 w
    double least;                      // of what counts: log2 min_p, or that of half a whole number
    const Words *root;

    __device__ __forceinline__ Weight operator()(float x) const
    {
        const double t = fmax(((double)x - max) * per_order, -64.0);
        const double z = t + 0x1.8p47, r = t - (z - 0x1.8p47);     // (to 32nds)
        const uint32_t n = (uint32_t)__builtin_bit_cast(uint64_t, z), bytes = n * 8;
        // (2^r - 1) / r, interpolated at Chebyshev's nodes of [-1/64, 1/64]
        double p = 0.009618166713972776;
        p = fma(p, r, 0.055504434191939005);
        p = fma(p, r, 0.24022650695795306);
        p = fma(p, r, 0.693147180550011);
        p = fma(p, r, 1.0);
        // n / 32 whole orders are added to the exponent: n << 47, and what n % 32 adds there has been taken from the root
        Words scale = *reinterpret_cast<const Words *>(reinterpret_cast<const char *>(root) + (bytes & 0xF8));
        scale[1] += n << 15;
        Words whole = __builtin_bit_cast(Words, fma(p, __builtin_bit_cast(double, scale), 0x1p52));
        whole[1] -= 0x43300000u;
        return Weight{__builtin_bit_cast(uint64_t, whole), t, 0 - bytes};
    }
    __device__ __forceinline__ bool counts(const Weight &w) const { return w.order >= least; }
    // A logit that none of `orders` binary orders below the maximum, or fewer, is below: with room for the rounding of all that is compared.
    __device__ __forceinline__ float lowest(double orders) const
    {
        const float x = (float)(max - (orders + 1e-6) / per_order);
        return x - (fabsf(x) + fabsf((float)max)) * 0x1p-21f;
    }
    __device__ __forceinline__ float highest(double orders) const
    {
        const float x = (float)(max - (orders - 1e-6) / per_order);
        return x + (fabsf(x) + fabsf((float)max)) * 0x1p-21f;
    }
};

// The binary orders below the maximum between which a bucket lies (a logarithm is rounded to a 32nd before it is cut into buckets).
template <int THREADS>
__device__ __forceinline__ double bucket_begin(uint32_t b) { return b * (64.0 / Sizes<THREADS>::kBuckets) - 1.0 / 64; }
template <int THREADS>
__device__ __forceinline__ double bucket_end(uint32_t b) { return (b + 1) * (64.0 / Sizes<THREADS>::kBuckets) - 1.0 / 64; }

// The columns of a row, each one thread's.  The first DEPTH groups of a thread stay in registers, the others (LONG: if there may be any) are loaded in every pass.
template <bool BF16, int THREADS, int DEPTH, bool LONG>
struct Columns {
    static constexpr int kPer = Row<BF16>::kPer, kAhead = DEPTH ? 2 : 4;
    const Row<BF16> &row;
    Quad q[DEPTH ? DEPTH : 1];
    float *last;                       // of LDS: the threads' columns behind the groups

    __device__ __forceinline__ Columns(const Row<BF16> &row, float *last) : row(row), last(last)
    {
        if (DEPTH && row.groups != 0) {
#pragma unroll
            for (int j = 0; j < DEPTH; ++j) q[j] = row.group(min(j * THREADS + threadIdx.x, row.groups - 1));
        }
        if (threadIdx.x < row.rest) last[threadIdx.x] = row.one(row.last_column(threadIdx.x));
    }
    // use(x, n, column): the n logits x from column `column` on
    template <typename Use>
    __device__ __forceinline__ void each(Use &&use)
    {
        float x[kPer];
        // (the compiler does not know the logits from here on either: it would unpack and convert them once, in front of all passes)
        const uint32_t thread = this_thread();
#pragma unroll
        for (int j = 0; j < DEPTH; ++j)
            if (j * THREADS + thread < row.groups) {
                Quad a = q[j];
                forget(a);
                Lane16<BF16>::unpack(a, x);
                use(x, std::integral_constant<int, kPer>(), (j * THREADS + thread) * kPer);
            }
        if (LONG) {
            for (uint32_t g0 = DEPTH * THREADS + this_thread(); g0 < row.groups; g0 += THREADS * kAhead) {
                Quad a[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) a[j] = row.group(min(g0 + j * THREADS, row.groups - 1));
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (g0 + j * THREADS < row.groups) {
                        Lane16<BF16>::unpack(a[j], x);
                        use(x, std::integral_constant<int, kPer>(), (g0 + j * THREADS) * kPer);
                    }
            }
        }
        if (threadIdx.x < row.rest) {
            x[0] = last[threadIdx.x];
            use(x, std::integral_constant<int, 1>(), row.last_column(threadIdx.x));
        }
    }
    // use(x, column) for the logits from `from` on: few
    template <typename Use>
    __device__ __forceinline__ void not_below(float from, Use &&use)
    {
        each([&](const float *x, auto n, uint32_t column) {
            float most = x[0];
            if constexpr (n > 1) most = max_of<n>(x);
            if (__ballot(most >= from) == 0) return;
#pragma unroll
            for (int e = 0; e < n; ++e)
                if (x[e] >= from) use(x[e], column + e);
        });
    }
    // use(x, column) for the logits from `from` to `to`: few
    template <typename Use>
    __device__ __forceinline__ void between(float from, float to, Use &&use)
    {
        each([&](const float *x, auto n, uint32_t column) {
            bool hit[n], any = false;
#pragma unroll
            for (int e = 0; e < n; ++e) any |= hit[e] = __builtin_amdgcn_fmed3f(x[e], from, to) == x[e];
            if (__ballot(any) == 0) return;
#pragma unroll
            for (int e = 0; e < n; ++e)
                if (hit[e]) use(x[e], column + e);
        });
    }
};

// A running sum over the lanes of a wavefront.
template <typename T, int CONTROL, int ROWS>
__device__ __forceinline__ T from_lane(T x)
{
    if constexpr (sizeof(T) == 4) {
        return (T)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, ROWS, 0xF, false);
    } else {
        const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CONTROL, ROWS, 0xF, false);
        const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CONTROL, ROWS, 0xF, false);
        return (uint64_t)high << 32 | low;
    }
}
template <typename T>
__device__ __forceinline__ T running_sum(T x)
{
    x += from_lane<T, 0x111, 0xF>(x);                      // 1, 2, 4 and 8 lanes before, in rows of 16; then the rows before
    x += from_lane<T, 0x112, 0xF>(x);
    x += from_lane<T, 0x114, 0xF>(x);
    x += from_lane<T, 0x118, 0xF>(x);
    x += from_lane<T, 0x142, 0xA>(x);
    x += from_lane<T, 0x143, 0xC>(x);
    return x;
}

template <int THREADS>
__device__ __forceinline__ void clear_buckets(SampleLds<THREADS> &lds)
{
    const uint32_t thread = this_thread();
    for (uint32_t b = thread; b <= SampleLds<THREADS>::kBuckets; b += THREADS) {
        lds.mass[b] = 0;
        lds.count[b] = 0;
    }
    __syncthreads();
}

// Sums of the buckets to sums of all in front of a bucket.  The last entry has the sums of all.
template <bool MASS, bool COUNT, int THREADS>
__device__ __forceinline__ void add_up_buckets(SampleLds<THREADS> &lds)
{
    const uint32_t thread = this_thread();
    constexpr uint32_t kEach = SampleLds<THREADS>::kBuckets / THREADS;
    constexpr int kWaves = THREADS / kLanes;
    const uint32_t lane = thread % kLanes, wave = thread / kLanes, first = thread * kEach;
    __syncthreads();
    uint64_t mass[kEach], mass_to = 0;
    uint32_t count[kEach], count_to = 0;
#pragma unroll
    for (uint32_t b = 0; b < kEach; ++b) {
        if (MASS) mass_to += mass[b] = lds.mass[first + b];
        if (COUNT) count_to += count[b] = lds.count[first + b];
    }
    const uint64_t own_mass = mass_to;
    const uint32_t own_count = count_to;
    if (MASS) mass_to = running_sum(mass_to);
    if (COUNT) count_to = running_sum(count_to);
    if (lane == kLanes - 1) {
        if (MASS) lds.wave_mass[wave] = mass_to;
        if (COUNT) lds.wave_count[wave] = count_to;
    }
    __syncthreads();
    const uint32_t part = lane % kWaves;
    if (MASS) mass_to += wave_sum<kWaves>(part < wave ? lds.wave_mass[part] : 0) - own_mass;
    if (COUNT) count_to += wave_sum<kWaves>(part < wave ? lds.wave_count[part] : 0) - own_count;
#pragma unroll
    for (uint32_t b = 0; b < kEach; ++b) {
        if (MASS) {
            lds.mass[first + b] = mass_to;
            mass_to += mass[b];
        }
        if (COUNT) {
            lds.count[first + b] = count_to;
            count_to += count[b];
        }
    }
    if (thread == THREADS - 1) {
        if (MASS) lds.mass[SampleLds<THREADS>::kBuckets] = mass_to;
        if (COUNT) lds.count[SampleLds<THREADS>::kBuckets] = count_to;
    }
    __syncthreads();
}

// The bucket in which the running sum reaches `goal`, for every thread.
template <int THREADS, typename Sum>
__device__ __forceinline__ uint32_t bucket_of(SampleLds<THREADS> &lds, const Sum *before, uint64_t goal)
{
    const uint32_t thread = this_thread();
    for (uint32_t b = thread; b < SampleLds<THREADS>::kBuckets; b += THREADS)
        if (before[b] < goal && goal <= before[b + 1]) lds.bucket = b;
    __syncthreads();
    return lds.bucket;
}

// The place in the order: the goal that a running sum, of ones (`by_count`) or of w, reaches there, and what stands in front of the listed columns.
struct Goal {
    uint64_t sum, mass_before, count_before;
    bool by_count;
};

// One of a wavefront's columns: its key, and the sum of w before it and up to and with it.
struct InOrder { uint64_t key, before, upto; uint32_t place; };

__device__ __forceinline__ void lds_in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

// By one wavefront: n <= 64 columns, one a lane.
template <int THREADS>
__device__ __forceinline__ InOrder order_by_wave(SampleLds<THREADS> &lds, uint64_t key, uint64_t w, uint32_t n)
{
    const uint32_t lane = this_thread() % kLanes;
    lds.key[lane] = key;
    lds.weight[lane] = w;
    lds_in_order();
    InOrder it = {key, 0, 0, 0};
#pragma unroll 4
    for (uint32_t j = 0; j < n; ++j) {
        const bool first = lds.key[j] > key;
        it.before += first ? lds.weight[j] : 0;
        it.place += first;
    }
    it.upto = it.before + w;
    return it;
}

// The key of the one at the goal, and the sum of w up to and with it.
__device__ __forceinline__ uint64_t pick_by_wave(const InOrder &it, uint32_t n, const Goal &goal, uint64_t &mass)
{
    const bool at = goal.by_count ? goal.count_before + it.place + 1 == goal.sum
                                  : goal.mass_before + it.before < goal.sum && goal.sum <= goal.mass_before + it.upto;
    const uint32_t lane = __builtin_ctzll(__ballot(at && threadIdx.x % kLanes < n) | 1ull << 63);
    auto of = [&](uint64_t x) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
    };
    mass = goal.mass_before + of(it.upto);
    return of(it.key);
}

template <int THREADS>
__device__ __forceinline__ void list_in_bucket(SampleLds<THREADS> &lds, float x, uint32_t column)
{
    const uint32_t i = atomicAdd(&lds.listed, 1u);
    if (i < SampleLds<THREADS>::kListed) {
        lds.sub_x[i] = x;
        lds.sub_column[i] = column;
    }
}

// The key and w of the i-th listed column; for one that does not count or is of another bucket than `only`, 0 and a key behind those of all others.
constexpr uint32_t kAnyBucket = 0xFFFFFFFFu;
template <int THREADS>
__device__ __forceinline__ uint64_t listed_key(const Weights &weights, float x, uint32_t column, uint32_t only, uint32_t i, uint64_t &w)
{
    const Weight it = weights(x);
    const bool counts = weights.counts(it) && (only == kAnyBucket || it.template bucket<THREADS>() == only);
    w = counts ? it.w : 0;
    return counts ? key_of(order_of(x), column) : i;
}

// picks(at) by one wavefront among n listed columns, no more than 64, of bucket `only`: at(goal) finds the column there, whose key is lds.found_key when
// it is the last, and returns the sum of w up to and with it.  Returns what picks() does, in every thread.
template <int THREADS, typename Picks>
__device__ __forceinline__ uint64_t among(SampleLds<THREADS> &lds, const Weights &weights, const float *x, const uint32_t *column, uint32_t n, uint32_t only,
                                          Picks &&picks)
{
    if (threadIdx.x < kLanes) {
        const uint32_t lane = this_thread();
        uint64_t w = 0, key = lane < n ? listed_key<THREADS>(weights, x[lane], column[lane], only, lane, w) : 0;
        const InOrder it = order_by_wave<THREADS>(lds, key, w, n);
        const uint64_t mass = picks([&](const Goal &goal) {
            uint64_t upto;
            key = pick_by_wave(it, n, goal, upto);
            return upto;
        });
        if (lane == 0) {
            lds.found_key = key;
            lds.found_mass = mass;
        }
    }
    __syncthreads();
    return scalar(lds.found_mass);
}

// Of the n columns listed as those of bucket `only`, no more than kListed, lists the part that holds the goal as lds.few_x and few_column: cut by keys until it
// has no more than 64; returns how many.  (The keys are made again where they are used: kept in registers, beside those of a long row, they would be spilled.)
template <int THREADS>
__device__ __forceinline__ uint32_t refine(SampleLds<THREADS> &lds, const Weights &weights, uint32_t n, uint32_t only, Goal &goal)
{
    constexpr uint32_t kPart = SampleLds<THREADS>::kSub / kLanes;
    constexpr int kCut = SampleLds<THREADS>::kSub == 512 ? 9 : 6;
    uint64_t low = 1ull << 32, high = ~0ull;               // (keys that count are not below 2^32)
    auto candidates = [&](auto &&use) {
#pragma unroll 1
        for (uint32_t i = this_thread(); i < n; i += THREADS) {
            uint64_t w;
            const uint64_t key = listed_key<THREADS>(weights, lds.sub_x[i], lds.sub_column[i], only, i, w);
            if (key >= low && key <= high) use(key, w, i);
        }
    };
    for (;;) {
        if (this_thread() == 0) {
            lds.lowest = ~0ull;
            lds.highest = 0;
        }
        for (uint32_t b = this_thread(); b < SampleLds<THREADS>::kSub; b += THREADS) {
            lds.sub_mass[b] = 0;
            lds.sub_count[b] = 0;
        }
        __syncthreads();
        if (this_thread() == 0) lds.listed = 0;            // (read in front of the barrier)
        uint64_t least = ~0ull, most = 0;
        candidates([&](uint64_t key, uint64_t, uint32_t) {
            least = min(least, key);
            most = max(most, key);
        });
        least = wave_reduce(least, [](uint64_t p, uint64_t q) { return p < q ? p : q; });
        most = wave_max(most);
        if (this_thread() % kLanes == 0 && most != 0) {
            atomicMin((unsigned long long *)&lds.lowest, (unsigned long long)least);
            atomicMax((unsigned long long *)&lds.highest, (unsigned long long)most);
        }
        __syncthreads();
        least = scalar(lds.lowest);
        most = scalar(lds.highest);
        const int bits = 64 - __builtin_clzll((most - least) | 1), shift = bits > kCut ? bits - kCut : 0;
        candidates([&](uint64_t key, uint64_t w, uint32_t) {
            const uint32_t b = (uint32_t)((most - key) >> shift);
            atomicAdd((unsigned long long *)&lds.sub_mass[b], (unsigned long long)w);
            atomicAdd(&lds.sub_count[b], 1u);
        });
        __syncthreads();
        const uint32_t thread = this_thread();
        if (thread < kLanes) {                             // which part has the goal
            uint64_t mass = 0, count = 0;
#pragma unroll
            for (uint32_t k = 0; k < kPart; ++k) {
                mass += lds.sub_mass[thread * kPart + k];
                count += lds.sub_count[thread * kPart + k];
            }
            uint64_t mass_to = goal.mass_before + running_sum(mass) - mass, count_to = goal.count_before + running_sum(count) - count;
#pragma unroll
            for (uint32_t k = 0; k < kPart; ++k) {
                const uint64_t m = lds.sub_mass[thread * kPart + k], c = lds.sub_count[thread * kPart + k];
                const uint64_t to = goal.by_count ? count_to : mass_to, upto = goal.by_count ? count_to + c : mass_to + m;
                if (to < goal.sum && goal.sum <= upto) {
                    lds.bucket = thread * kPart + k;
                    lds.wave_mass[0] = mass_to;
                    lds.found_mass = count_to;
                }
                mass_to += m;
                count_to += c;
            }
        }
        __syncthreads();
        goal.mass_before = scalar(lds.wave_mass[0]);
        goal.count_before = scalar(lds.found_mass);
        high = most - ((uint64_t)scalar(lds.bucket) << shift);
        const uint64_t width = (1ull << shift) - 1;
        low = high - least > width ? high - width : least;
        candidates([&](uint64_t, uint64_t, uint32_t i) {
            const uint32_t at = atomicAdd(&lds.listed, 1u);
            if (at < kLanes) {
                lds.few_x[at] = lds.sub_x[i];
                lds.few_column[at] = lds.sub_column[i];
            }
        });
        __syncthreads();
        const uint32_t few = scalar(lds.listed);
        if (few <= kLanes) return few;
    }
}

// Of a bucket with too many columns: cuts it by their keys until the part that holds the goal has few, and lists these; returns how many.
// The row's buckets are lost.  (Seldom: the row is read again.)
template <bool BF16, int THREADS>
__device__ __forceinline__ uint32_t narrow(const Row<BF16> &row, const Weights &weights, uint32_t only, Goal &goal, SampleLds<THREADS> &lds)
{
    Columns<BF16, THREADS, 0, true> columns(row, lds.last);
    const float lowest = weights.lowest(bucket_end<THREADS>(only)), highest = weights.highest(bucket_begin<THREADS>(only));
    uint64_t from = 0, to = ~0ull;
    auto candidates = [&](auto &&use) {
        columns.between(lowest, highest, [&](float x, uint32_t column) {
            const Weight it = weights(x);
            const uint64_t key = key_of(order_of(x), column);
            if (it.template bucket<THREADS>() == only && weights.counts(it) && key >= from && key <= to) use(key, it.w, x, column);
        });
        __syncthreads();
    };
    for (;;) {
        if (threadIdx.x == 0) {
            lds.lowest = ~0ull;
            lds.highest = 0;
        }
        clear_buckets<THREADS>(lds);
        candidates([&](uint64_t key, uint64_t, float, uint32_t) {
            atomicMin((unsigned long long *)&lds.lowest, (unsigned long long)key);
            atomicMax((unsigned long long *)&lds.highest, (unsigned long long)key);
        });
        from = lds.lowest;
        to = lds.highest;
        uint32_t shift = 0;
        while ((to - from) >> shift >= SampleLds<THREADS>::kBuckets) ++shift;
        candidates([&](uint64_t key, uint64_t w, float, uint32_t) {
            const uint32_t b = (uint32_t)((to - key) >> shift);
            atomicAdd((unsigned long long *)&lds.mass[b], (unsigned long long)w);
            atomicAdd(&lds.count[b], 1u);
        });
        add_up_buckets<true, true, THREADS>(lds);
        if (threadIdx.x == 0) lds.listed = 0;
        const uint32_t b = goal.by_count ? bucket_of<THREADS>(lds, lds.count, goal.sum - goal.count_before)
                                         : bucket_of<THREADS>(lds, lds.mass, goal.sum - goal.mass_before);
        goal.mass_before += lds.mass[b];
        goal.count_before += lds.count[b];
        to -= (uint64_t)b << shift;
        const uint64_t width = (1ull << shift) - 1;
        from = to - from > width ? to - width : from;
        candidates([&](uint64_t, uint64_t, float x, uint32_t column) { list_in_bucket<THREADS>(lds, x, column); });
        const uint32_t n = lds.listed;
        if (n <= SampleLds<THREADS>::kListed) return n;
        __syncthreads();                                   // (the buckets and the number, before they are cleared again)
    }
}

template <int THREADS>
__device__ __forceinline__ uint64_t goal_of(const SampleLds<THREADS> &lds, int step, uint32_t top_k, uint64_t mass)
{
    return step == 0   ? (uint64_t)top_k
           : step == 1 ? min(max((uint64_t)ceil(lds.nucleus * (double)mass), (uint64_t)1), mass)
                       : min((uint64_t)(lds.below * (double)mass), mass - 1) + 1;
}

// One place after the other: that of top_k (0), of top_p (1), of the token (2), whose key is lds.found_key then, `mass` the sum of what is kept.
// Of the `kept` columns in the list, or, where that is 0, of the row.  `clear`: the buckets are.  `all`: every column counts (or has a w of 0, which
// may be added).  Without NARROW a bucket with too many columns ends it: false.
template <bool NARROW, bool BF16, int THREADS, int DEPTH, bool LONG>
__device__ __forceinline__ bool find_places(Columns<BF16, THREADS, DEPTH, LONG> &columns, const Weights &weights, uint32_t top_k, bool nucleus, bool all, uint32_t kept,
                                            bool clear, SampleLds<THREADS> &lds, uint64_t &mass)
{
    const bool counted = top_k < (kept ? kept : columns.row.groups * Row<BF16>::kPer + columns.row.rest);
    bool filled = false;
#pragma unroll 1
    for (int step = 0; step < 3; ++step) {
        if (step == 1 && !nucleus) continue;
        if (!filled) {
            if (!clear) clear_buckets<THREADS>(lds);
            clear = false;
            // (the weights of a few columns side by side: one is a chain of twenty instructions that wait for each other)
            auto add = [&](const float *x, auto n) {
                Weight it[n];
#pragma unroll
                for (int e = 0; e < n; ++e) it[e] = weights(x[e]);
#pragma unroll
                for (int e = 0; e < n; ++e) asm volatile("" : "+v"(it[e].w));      // (all of them here, not each in front of its use)
                if (all) {
#pragma unroll
                    for (int e = 0; e < n; ++e) atomicAdd((unsigned long long *)&lds.mass[it[e].template bucket<THREADS>()], (unsigned long long)it[e].w);
                    return;
                }
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    if (!weights.counts(it[e])) continue;
                    const uint32_t b = it[e].template bucket<THREADS>();
                    atomicAdd((unsigned long long *)&lds.mass[b], (unsigned long long)it[e].w);
                    if (counted) atomicAdd(&lds.count[b], 1u);
                }
            };
            if (kept)
                for (uint32_t i = this_thread(); i < kept; i += THREADS) add(&lds.x[i], std::integral_constant<int, 1>());
            else
                columns.each([&](const float *x, auto n, uint32_t) {
                    constexpr int kMost = DEPTH > 8 ? 2 : 4, kSide = n < kMost ? n : kMost;       // (beside a long row there are registers for two)
#pragma unroll
                    for (int e = 0; e < n; e += kSide) add(x + e, std::integral_constant<int, kSide>());
                });
            add_up_buckets<true, true, THREADS>(lds);
            filled = true;
            if (step == 0) mass = scalar(lds.mass[SampleLds<THREADS>::kBuckets]);
        }
        if (step == 0 && (!counted || lds.count[SampleLds<THREADS>::kBuckets] <= top_k)) continue;
        Goal goal = {scalar(goal_of(lds, step, top_k, mass)), 0, 0, step == 0};
        if (threadIdx.x == 0) lds.listed = 0;
        const uint32_t only = scalar(goal.by_count ? bucket_of<THREADS>(lds, lds.count, goal.sum) : bucket_of<THREADS>(lds, lds.mass, goal.sum));
        goal.mass_before = scalar(lds.mass[only]);
        goal.count_before = goal.by_count ? scalar(lds.count[only]) : 0;
        const float lowest = scalar(weights.lowest(bucket_end<THREADS>(only))), highest = scalar(weights.highest(bucket_begin<THREADS>(only)));
        if (kept) {
            for (uint32_t i = this_thread(); i < kept; i += THREADS)
                if (lds.x[i] >= lowest && lds.x[i] <= highest) list_in_bucket<THREADS>(lds, lds.x[i], lds.column[i]);
        } else {
            columns.between(lowest, highest, [&](float x, uint32_t column) { list_in_bucket<THREADS>(lds, x, column); });
        }
        __syncthreads();
        uint32_t n = scalar(lds.listed);
        if (n > SampleLds<THREADS>::kListed) {
            if constexpr (!NARROW) return false;
            __syncthreads();                               // (lds.listed)
            n = narrow<BF16, THREADS>(columns.row, weights, only, goal, lds);
            filled = false;
        }
        const bool many = n > kLanes;
        if (many) n = refine<THREADS>(lds, weights, n, only, goal);
        mass = among<THREADS>(lds, weights, many ? lds.few_x : lds.sub_x, many ? lds.few_column : lds.sub_column, n, only, [&](auto &&at) {
            const uint64_t upto = at(goal);
            return step == 2 ? mass : upto;
        });
        if (NARROW) __syncthreads();                       // (the buckets may be cleared next)
    }
    return true;
}

__device__ __forceinline__ void put_roots(Words *root, uint32_t shift)
{
    if (threadIdx.x < 32)
        root[threadIdx.x] = __builtin_bit_cast(Words, __builtin_bit_cast(uint64_t, __builtin_amdgcn_ldexp(kRoots[threadIdx.x], (int)shift)) - ((uint64_t)threadIdx.x << 47));
}

// For a row whose sum of weights is far below the number of its columns: multiples of 2^-shift that are as fine as the sum allows.  The sum, of exponentials in
// binary32, is off by less than a thousandth; with a sixteenth more it is below 2^bits, and so the sum of the whole numbers, each half of one more, below 2^62.
template <int THREADS, typename Of>
__device__ __forceinline__ uint32_t shift_of_sum(Of &columns, const Weights &weights, SampleLds<THREADS> &lds)
{
    double sum = 0.0;
    columns.each([&](const float *x, auto n, uint32_t) {
#pragma unroll
        for (int e = 0; e < n; ++e) sum += (double)__builtin_amdgcn_exp2f((float)fmax(((double)x[e] - weights.max) * weights.per_order, -200.0));
    });
    sum = wave_sum(sum);
    if (threadIdx.x % kLanes == 0) lds.wave_mass[threadIdx.x / kLanes] = __builtin_bit_cast(uint64_t, sum);
    __syncthreads();
    sum = wave_sum<THREADS / kLanes>(__builtin_bit_cast(double, lds.wave_mass[threadIdx.x % (THREADS / kLanes)]));
    const uint32_t bits = scalar((uint32_t)__builtin_amdgcn_frexp_exp(sum * 1.0625));
    return bits < 11 ? 51 : 62 - bits;
}

template <bool BF16, int THREADS, int DEPTH, bool LONG>
__global__ __launch_bounds__(THREADS, THREADS < 512 ? 1 : 4) void sample_kernel(const SampleArgs a)
{
    __shared__ SampleLds<THREADS> lds;
    constexpr int kWaves = THREADS / kLanes;
    const uint64_t r = (uint64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (r >= a.rows) return;
    const Row<BF16> row(a, r);
    Columns<BF16, THREADS, DEPTH, LONG> columns(row, lds.last);
    const float own_temperature = a.temperature ? a.temperature[r] : a.one_temperature, top_p = a.top_p ? a.top_p[r] : a.one_top_p;
    const float min_p = a.min_p ? a.min_p[r] : a.one_min_p, uniform = a.uniform[r];
    const int32_t own_top_k = a.top_k ? a.top_k[r] : a.one_top_k;
    auto put = [&](int64_t token, float logprob) {
        if (threadIdx.x != 0) return;
        if (a.wide) static_cast<int64_t *>(a.token)[r] = token;
        else static_cast<int32_t *>(a.token)[r] = (int32_t)token;
        if (a.logprob) a.logprob[r] = logprob;
    };
    put_roots(lds.root, a.shift);
    float own_most = -INFINITY;
    columns.each([&](const float *x, auto n, uint32_t) {
#pragma unroll
        for (int e = 0; e < n; ++e) own_most = __builtin_elementwise_maximum(own_most, x[e]);
    });
    float most = wave_reduce(own_most, [](float p, float q) { return __builtin_elementwise_maximum(p, q); });
    if (threadIdx.x % kLanes == 0) lds.at[threadIdx.x / kLanes] = most;
    if (threadIdx.x == 0) {
        lds.listed = 0;
        // (temperature 0: the first of the largest)
        lds.inverse = own_temperature == 0.0f ? 1.0 : 1.0 / (double)own_temperature;
        lds.below = uniform > 0.0f ? fmin((double)uniform, 0x1.fffffep-1) : 0.0;       // (the number next to 1)
        lds.nucleus = fmax((double)top_p, 0.0);
    }
    clear_buckets<THREADS>(lds);
    most = scalar(wave_reduce<kWaves>(lds.at[threadIdx.x % kWaves], [](float p, float q) { return __builtin_elementwise_maximum(p, q); }));
    if (!(most < INFINITY) || !(own_temperature >= 0.0f) || top_p != top_p || min_p != min_p || uniform != uniform) return put(-1, NAN);
    if (most == -INFINITY) return put(-1, -INFINITY);

    // (a min_p above every w leaves the one column that is kept at least)
    const uint32_t top_k = own_temperature == 0.0f || min_p > 1.0f ? 1 : own_top_k > 0 ? (uint32_t)own_top_k : a.cols;
    Weights weights;
    weights.max = scalar((double)most);
    weights.per_order = scalar(lds.inverse * 1.4426950408889634);
    weights.root = lds.root;
    uint32_t shift = a.shift;
    if constexpr (LONG)
        if (a.cols > kCountedCols && top_k != 1) {
            shift = shift_of_sum<THREADS>(columns, weights, lds);
            __syncthreads();                               // (nothing of the roots has been read)
            put_roots(lds.root, shift);
            __syncthreads();
        }
    weights.least = -1.0 - (double)shift;
    // a logit that no kept column is below, where min_p or few columns give one
    float bound = -INFINITY;
    bool spoilt = false;               // the buckets
    if (min_p > 0.0f) {
        weights.least = scalar(fmax(log2((double)fminf(min_p, 1.0f)), weights.least));
        bound = weights.lowest(-weights.least);
    }
    if (top_k == 1) {
        bound = most;
    } else if (top_k <= THREADS / 2 && top_k < a.cols) {   // the top_k-th of the threads' largest, by its bucket
        if (own_most > -INFINITY) atomicAdd(&lds.count[min(weights(own_most).template bucket<THREADS>(), SampleLds<THREADS>::kBuckets - 1)], 1u);
        add_up_buckets<false, true, THREADS>(lds);
        spoilt = true;
        if (lds.count[SampleLds<THREADS>::kBuckets] >= top_k) {
            const uint32_t b = bucket_of<THREADS>(lds, lds.count, (uint64_t)top_k);
            if (b < SampleLds<THREADS>::kBuckets - 1) bound = fmaxf(bound, weights.lowest(bucket_end<THREADS>(b)));
        } else {
            __syncthreads();                               // (the buckets, before they are cleared)
        }
    }
    // The columns that are not below the bound, if they are few: kKept are kept instead of the row, 64 are put in order at once.
    uint32_t kept = 0;
    if (bound > -INFINITY) {
        // (counted first: an atomic addition for each is waited for, and these may be many)
        uint32_t own = 0;
        columns.each([&](const float *x, auto n, uint32_t) {
#pragma unroll
            for (int e = 0; e < n; ++e) own += x[e] >= bound;
        });
        const uint32_t upto = running_sum(own);
        uint32_t i = 0;
        if (threadIdx.x % kLanes == kLanes - 1) i = atomicAdd(&lds.listed, upto);
        i = (uint32_t)__builtin_amdgcn_readlane((int)i, kLanes - 1) + upto - own;
        columns.not_below(bound, [&](float x, uint32_t column) {
            if (i < SampleLds<THREADS>::kKept) {
                lds.x[i] = x;
                lds.column[i] = column;
            }
            ++i;
        });
        __syncthreads();
        kept = lds.listed;
    }
    uint64_t mass = 0;
    if (kept != 0 && kept <= kLanes) {
        mass = among<THREADS>(lds, weights, lds.x, lds.column, kept, kAnyBucket, [&](auto &&at) {
            uint64_t sum = at(Goal{top_k < kept ? top_k : kept, 0, 0, true});
            if (top_p < 1.0f) sum = at(Goal{goal_of(lds, 1, top_k, sum), 0, 0, false});
            at(Goal{goal_of(lds, 2, top_k, sum), 0, 0, false});
            return sum;
        });
    } else {
        if (kept > SampleLds<THREADS>::kKept) kept = 0;
        const bool all = min_p <= 0.0f && top_k >= a.cols;
        if (!find_places<false, BF16>(columns, weights, top_k, top_p < 1.0f, all, kept, !spoilt, lds, mass)) {
            // (seldom; the row does not stay in registers meanwhile)
            Columns<BF16, THREADS, 0, true> again(row, lds.last);
            __syncthreads();
            find_places<true, BF16>(again, weights, top_k, top_p < 1.0f, all, 0, false, lds, mass);
        }
    }
    const uint64_t key = lds.found_key;
    put(column_of(key), (float)(((double)value_of(key) - weights.max) * lds.inverse - log(__builtin_amdgcn_ldexp((double)mass, -(int)shift))));
}

// ---- host ------------------------------------------------------------------------------------
// The fewest threads that hold the row, by groups of 16 bytes, without many a thread; more where there are fewer rows than the card takes side by side and it is one
// row's time that counts.  (Nucleus: 20000 rows of 1000 fp32, 256 threads 123 us, 64 61, and 1000 of them 11 and 14; 5000 of 1900 fp32 43 and 36, 1200 of them 14
// and 21.  4000 rows of 16000 fp32: 512 threads 129, 256 with sixteen groups 110, 1200 of 12000 42 and 42; of bf16, twice the columns a group, 2000 of 32000 111 and 114.
// 1024 rows of 50257 bf16: 512 threads 102, 1024 128.)
template <bool BF16>
static int sample_launch(const SampleArgs &a, hipStream_t stream)
{
    const uint32_t across = (uint32_t)(a.rows < (1u << 20) ? a.rows : 1u << 20);
    const dim3 grid(across, (uint32_t)((a.rows + across - 1) / across));
    const uint32_t quads = (a.cols + (BF16 ? 7 : 3)) / (BF16 ? 8 : 4);
    const bool many = a.rows > 2048;
    if (quads <= 64 * 2 || (quads <= 64 * 4 && many)) return launch(sample_kernel<BF16, 64, 4, false>, grid, 64, stream, a);
    if (!BF16 && quads <= 64 * 8 && many) return launch(sample_kernel<false, 64, 8, false>, grid, 64, stream, a);
    if (quads <= 256 * 4) return launch(sample_kernel<BF16, 256, 4, false>, grid, 256, stream, a);
    if (quads <= 256 * 8) return launch(sample_kernel<BF16, 256, 8, false>, grid, 256, stream, a);
    if (!BF16 && quads <= 256 * 16 && a.rows >= 1024) return launch(sample_kernel<false, 256, 16, false>, grid, 256, stream, a);
    if (quads <= 512 * 8 && a.rows > 256) return launch(sample_kernel<BF16, 512, 8, false>, grid, 512, stream, a);
    if (quads <= 512 * 16 && a.rows > 256) return launch(sample_kernel<BF16, 512, 16, false>, grid, 512, stream, a);
    if (quads <= 1024 * 8) return launch(sample_kernel<BF16, 1024, 8, false>, grid, 1024, stream, a);
    if (quads <= 1024 * 16) return launch(sample_kernel<BF16, 1024, 16, false>, grid, 1024, stream, a);
    return launch(sample_kernel<BF16, 1024, 16, true>, grid, 1024, stream, a);
}

static bool optional_at(const void *p, uintptr_t size) { return !p || at_multiple(p, size); }

}  // namespace solo

extern "C" int solo_sample(const void *logits, const float *uniform, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                           void *token, float *logprob, const solo_sample_shape *s, void *stream)
{
    using namespace solo;
    if (!s || !dtype_ok(s->dtype) || (s->token_bits != 32 && s->token_bits != 64) || s->reserved != 0 || s->reserved2 != 0 || !(s->temperature >= 0.0f) || s->top_p != s->top_p ||
        s->min_p != s->min_p || s->stride < s->cols)
        return SOLO_E_INVALID;
    if (s->rows != 0 && ((s->cols != 0 && !at_multiple(logits, element_bytes(s->dtype))) || !at_multiple(uniform, 4) || !optional_at(temperature, 4) ||
                         !optional_at(top_k, 4) || !optional_at(top_p, 4) || !optional_at(min_p, 4) || !at_multiple(token, s->token_bits / 8) ||
                         !optional_at(logprob, 4)))
        return SOLO_E_INVALID;
    if (s->cols >= (1ull << 29) || s->rows >= (1ull << 35) || s->stride >= (1ull << 40)) return SOLO_E_UNSUPPORTED;
    if (s->rows == 0) return SOLO_OK;
    SampleArgs a = {};
    a.logits = logits; a.uniform = uniform; a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
    a.token = token; a.logprob = logprob;
    a.rows = s->rows; a.stride = s->stride; a.cols = (uint32_t)s->cols; a.wide = s->token_bits == 64;
    a.one_temperature = s->temperature; a.one_top_p = s->top_p; a.one_min_p = s->min_p; a.one_top_k = s->top_k;
    uint32_t bits = 0;
    while ((1ull << bits) < s->cols) ++bits;
    a.shift = bits < 11 ? 51 : 62 - bits;                  // a weight is below 2^52, and so are sums of all columns below 2^63
    return s->dtype == SOLO_BF16 ? sample_launch<true>(a, (hipStream_t)stream) : sample_launch<false>(a, (hipStream_t)stream);
}
