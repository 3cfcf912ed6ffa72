// Sampling: of every row of logits one column, by a given uniform number.
//
//   w_j = e^((x_j - max x) / temperature), the columns in the order of their logits, ties by the lower column
//   kept: the first top_k of those with w >= min_p, and of these the shortest beginning that has top_p of their sum
//   the token is the first column, in that order, at which the running sum of the kept w exceeds uniform * their sum
//
// Each of the three is a place in the order at which a running sum (of ones or of w) reaches a goal, and none needs the order itself: a
// histogram over the distance from the maximum gives the bucket that holds the place, and only that bucket's columns are looked at
// again, each against all others of them.  A bucket with too many (equal logits, mostly) is cut further by whole keys, value and column, until it has few.
//
// Which column it is hangs on comparisons of sums, so these are exact: w is computed in binary64 (the rate of its instructions is that of
// binary32), to 4e-14, and rounded to a whole multiple of 2^-shift; sums of such are whole numbers below 2^63, the same in every order, and atomic additions in
// LDS make them.
#include "solo_rows.h"

#include <float.h>
#include <math.h>

namespace solo {

constexpr uint32_t kBuckets = 2048;    // of the distance from the maximum
constexpr uint32_t kListed = 1024;     // columns of a bucket that are compared with each other

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

template <int THREADS>
struct SampleLds {
    uint64_t mass[kBuckets + 1];       // sums of the buckets, then of all in front of a bucket
    uint32_t count[kBuckets + 1];
    uint64_t key[kListed], weight[kListed], before[kListed];
    uint32_t places[kListed];
    uint64_t wave_mass[THREADS / kLanes], lowest, highest;
    uint32_t wave_count[THREADS / kLanes];
    float at[THREADS / kLanes];
    uint32_t listed, bucket, column;
    uint64_t found_key, found_mass;
};

// The weights of a row.  A whole number of 2^-shift; 0 where the column does not count (w below min_p, or nothing at all).
struct Weights {
    float max, per_bucket;             // (max - x) * per_bucket is the bucket
    double per_order, least;           // (x - max) * per_order is log2 w; least: min_p in whole numbers
    uint32_t shift;

    __device__ __forceinline__ float place(float x) const { return (max - x) * per_bucket; }
    __device__ __forceinline__ static bool counts(float place) { return place <= kBuckets * 1.001f; }     // (not a NaN)
    __device__ __forceinline__ static uint32_t bucket(float place) { return min((uint32_t)place, kBuckets - 1); }
    __device__ __forceinline__ uint64_t operator()(float x) const
    {
        const double t = fmax(((double)x - (double)max) * per_order, -2000.0);
        const double z = t + 0x1.8p52, r = t - (z - 0x1.8p52);
        const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, z);
        // 2^r - 1 over r, interpolated at Chebyshev's nodes of [-1/2, 1/2]
        double p = 1.0203121063391729e-07;
        p = fma(p, r, 1.3255224878668817e-06);
        p = fma(p, r, 1.525268684626772e-05);
        p = fma(p, r, 0.00015403455852453838);
        p = fma(p, r, 0.0013333558179043112);
        p = fma(p, r, 0.009618129159402558);
        p = fma(p, r, 0.055504108664760424);
        p = fma(p, r, 0.2402265069581299);
        p = fma(p, r, 0.6931471805599453);
        p = fma(p, r, 1.0);
        const double w = __builtin_amdgcn_ldexp(p, n + (int)shift);
        const uint64_t whole = __builtin_bit_cast(uint64_t, w + 0x1p52) - 0x4330000000000000ull;
        return w >= least ? whole : 0;
    }
};

// use(x, column) for every column of the row, each by one thread.
template <bool BF16, int THREADS, typename Use>
__device__ __forceinline__ void for_columns(const Row<BF16> &row, Use &&use)
{
    constexpr int kPer = Row<BF16>::kPer, kDepth = 4;
    for (uint32_t g0 = threadIdx.x; g0 < row.groups; g0 += THREADS * kDepth) {
        Quad q[kDepth];
#pragma unroll
        for (int j = 0; j < kDepth; ++j) q[j] = row.group(min(g0 + j * THREADS, row.groups - 1));
#pragma unroll
        for (int j = 0; j < kDepth; ++j)
            if (g0 + j * THREADS < row.groups) {
                float x[kPer];
                Lane16<BF16>::unpack(q[j], x);
#pragma unroll
                for (int e = 0; e < kPer; ++e) use(x[e], (g0 + j * THREADS) * kPer + e);
            }
    }
    if (threadIdx.x < row.rest) use(row.one(row.last_column(threadIdx.x)), row.last_column(threadIdx.x));
}

template <int THREADS>
__device__ __forceinline__ void clear_buckets(SampleLds<THREADS> &lds)
{
    for (uint32_t b = threadIdx.x; b <= kBuckets; b += THREADS) {
        lds.mass[b] = 0;
        lds.count[b] = 0;
    }
    __syncthreads();
}

// Sums of the buckets to sums of all in front of a bucket.  The last entry has the sums of all.
template <int THREADS>
__device__ __forceinline__ void add_up_buckets(SampleLds<THREADS> &lds)
{
    constexpr uint32_t kEach = kBuckets / THREADS;
    const uint32_t lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes, first = threadIdx.x * kEach;
    __syncthreads();
    uint64_t mass = 0;
    uint32_t count = 0;
    for (uint32_t b = 0; b < kEach; ++b) {
        mass += lds.mass[first + b];
        count += lds.count[first + b];
    }
    uint64_t mass_to = mass;
    uint32_t count_to = count;
    for (uint32_t d = 1; d < kLanes; d *= 2) {
        const uint64_t m = __shfl_up(mass_to, d);
        const uint32_t c = __shfl_up(count_to, d);
        if (lane >= d) {
            mass_to += m;
            count_to += c;
        }
    }
    if (lane == kLanes - 1) {
        lds.wave_mass[wave] = mass_to;
        lds.wave_count[wave] = count_to;
    }
    __syncthreads();
    mass_to -= mass;
    count_to -= count;
    for (uint32_t w = 0; w < wave; ++w) {
        mass_to += lds.wave_mass[w];
        count_to += lds.wave_count[w];
    }
    for (uint32_t b = 0; b < kEach; ++b) {
        const uint64_t m = lds.mass[first + b];
        const uint32_t c = lds.count[first + b];
        lds.mass[first + b] = mass_to;
        lds.count[first + b] = count_to;
        mass_to += m;
        count_to += c;
    }
    if (threadIdx.x == THREADS - 1) {
        lds.mass[kBuckets] = mass_to;
        lds.count[kBuckets] = count_to;
    }
    __syncthreads();
}

// The column at which the running sum (BY_COUNT: of ones) reaches `goal`, 1 to the sum of all: its key and the sum of w up to and with
// it, in lds.found_key and found_mass.  The buckets are those of the whole row when it begins; `spoilt` is set where they no longer are at the end.
template <bool BF16, bool BY_COUNT, int THREADS>
__device__ __forceinline__ void find_place(const Row<BF16> &row, const Weights &weights, uint64_t goal, SampleLds<THREADS> &lds, bool &spoilt)
{
    uint64_t from = 0, to = ~0ull, mass_before = 0;        // keys of the columns that can be it; of those in front of them, the sum of w
    uint64_t count_before = 0;
    uint32_t only = kBuckets, narrowed = 0;                // the bucket they are in
    for (;;) {
        for (uint32_t b = threadIdx.x; b < kBuckets; b += THREADS) {
            const uint64_t before = BY_COUNT ? count_before + lds.count[b] : mass_before + lds.mass[b];
            const uint64_t upto = BY_COUNT ? count_before + lds.count[b + 1] : mass_before + lds.mass[b + 1];
            if (before < goal && goal <= upto) lds.bucket = b;
        }
        if (threadIdx.x == 0) lds.listed = 0;
        __syncthreads();
        const uint32_t b = lds.bucket;
        mass_before += lds.mass[b];
        count_before += lds.count[b];
        if (only == kBuckets) {
            only = b;
        } else {                                           // (bucket b of the keys: narrowed is their shift)
            const uint64_t last = to - ((uint64_t)b << narrowed);
            const uint64_t width = (1ull << narrowed) - 1;
            from = last - from > width ? last - width : from;
            to = last;
        }
        auto in_bucket = [&](float x, uint32_t column, auto &&use) {
            const float place = weights.place(x);
            if (!Weights::counts(place) || Weights::bucket(place) != only) return;
            const uint64_t key = key_of(order_of(x), column);
            if (key < from || key > to) return;
            const uint64_t w = weights(x);
            if (w != 0) use(key, w);
        };
        for_columns<BF16, THREADS>(row, [&](float x, uint32_t column) {
            in_bucket(x, column, [&](uint64_t key, uint64_t w) {
                const uint32_t i = atomicAdd(&lds.listed, 1u);
                if (i < kListed) {
                    lds.key[i] = key;
                    lds.weight[i] = w;
                    lds.before[i] = 0;
                    lds.places[i] = 0;
                }
            });
        });
        __syncthreads();
        const uint32_t n = lds.listed;
        if (n <= kListed) {
            // a thread compares one column with a part of the others
            const uint32_t across = min((n + kLanes - 1) / kLanes * kLanes, (uint32_t)THREADS), parts = THREADS / across, part = threadIdx.x / across;
            for (uint32_t i = part < parts ? threadIdx.x % across : n; i < n; i += across) {
                const uint64_t key = lds.key[i];
                uint64_t before = 0;
                uint32_t places = 0;
                for (uint32_t j = part; j < n; j += parts)
                    if (lds.key[j] > key) {
                        before += lds.weight[j];
                        ++places;
                    }
                if (places) {
                    atomicAdd((unsigned long long *)&lds.before[i], (unsigned long long)before);
                    atomicAdd(&lds.places[i], places);
                }
            }
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < n; i += THREADS) {
                const uint64_t before = BY_COUNT ? count_before + lds.places[i] : mass_before + lds.before[i];
                if (before < goal && goal <= before + (BY_COUNT ? 1 : lds.weight[i])) {
                    lds.found_key = lds.key[i];
                    lds.found_mass = mass_before + lds.before[i] + lds.weight[i];
                }
            }
            __syncthreads();
            return;
        }
        // too many: their keys, cut into buckets
        if (threadIdx.x == 0) {
            lds.lowest = ~0ull;
            lds.highest = 0;
        }
        spoilt = true;
        clear_buckets<THREADS>(lds);
        for_columns<BF16, THREADS>(row, [&](float x, uint32_t column) {
            in_bucket(x, column, [&](uint64_t key, uint64_t) {
                atomicMin((unsigned long long *)&lds.lowest, (unsigned long long)key);
                atomicMax((unsigned long long *)&lds.highest, (unsigned long long)key);
            });
        });
        __syncthreads();
        from = lds.lowest;
        to = lds.highest;
        narrowed = 0;
        while ((to - from) >> narrowed >= kBuckets) ++narrowed;
        for_columns<BF16, THREADS>(row, [&](float x, uint32_t column) {
            in_bucket(x, column, [&](uint64_t key, uint64_t w) {
                const uint32_t at = (uint32_t)((to - key) >> narrowed);
                atomicAdd((unsigned long long *)&lds.mass[at], (unsigned long long)w);
                atomicAdd(&lds.count[at], 1u);
            });
        });
        add_up_buckets<THREADS>(lds);
    }
}

template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(const SampleArgs a)
{
    __shared__ SampleLds<THREADS> lds;
    constexpr int kWaves = THREADS / kLanes;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<BF16> row(a, r);
        const float temperature = a.temperature ? a.temperature[r] : a.one_temperature, top_p = a.top_p ? a.top_p[r] : a.one_top_p;
        const float min_p = a.min_p ? a.min_p[r] : a.one_min_p, uniform = a.uniform[r];
        const int32_t top_k = a.top_k ? a.top_k[r] : a.one_top_k;
        auto put = [&](int64_t token, float logprob) {
            if (threadIdx.x != 0) return;
            if (a.wide) static_cast<int64_t *>(a.token)[r] = token;
            else static_cast<int32_t *>(a.token)[r] = (int32_t)token;
            if (a.logprob) a.logprob[r] = logprob;
        };
        float most = -INFINITY;
        for_columns<BF16, THREADS>(row, [&](float x, uint32_t) { most = __builtin_elementwise_maximum(most, x); });
        most = wave_reduce(most, [](float p, float q) { return __builtin_elementwise_maximum(p, q); });
        if (threadIdx.x % kLanes == 0) lds.at[threadIdx.x / kLanes] = most;
        if (threadIdx.x == 0) lds.column = 0xFFFFFFFFu;
        __syncthreads();
        most = wave_reduce<kWaves>(lds.at[threadIdx.x % kWaves], [](float p, float q) { return __builtin_elementwise_maximum(p, q); });
        if (!(most < INFINITY) || !(temperature >= 0.0f) || top_p != top_p || min_p != min_p || uniform != uniform) {
            put(-1, NAN);
        } else if (most == -INFINITY) {
            put(-1, -INFINITY);
        } else if (temperature == 0.0f || top_k == 1) {
            for_columns<BF16, THREADS>(row, [&](float x, uint32_t column) {
                if (x == most) atomicMin(&lds.column, column);
            });
            __syncthreads();
            put(lds.column, 0.0f);
        } else {
            Weights weights;
            const double inverse = 1.0 / (double)temperature;
            weights.max = most;
            weights.shift = a.shift;
            weights.per_order = inverse * 1.4426950408889634;
            const float least = fminf(min_p, 1.0f);
            weights.least = least > 0.0f ? __builtin_amdgcn_ldexp((double)least, (int)a.shift) : 0.0;
            // w is half of 2^-shift behind the last bucket, or below min_p
            const float orders = fminf(least > 0.0f ? 0.01f - 1.001f * __builtin_amdgcn_logf(fmaxf(least, FLT_MIN)) : FLT_MAX, (float)(a.shift + 1));
            weights.per_bucket = fminf((float)weights.per_order * (kBuckets / orders), 1e30f);
            const bool cut = top_k > 1 && (uint32_t)top_k < a.cols;
            auto fill = [&] {
                clear_buckets<THREADS>(lds);
                for_columns<BF16, THREADS>(row, [&](float x, uint32_t) {
                    const float place = weights.place(x);
                    if (!Weights::counts(place)) return;
                    const uint64_t w = weights(x);
                    if (w == 0) return;
                    atomicAdd((unsigned long long *)&lds.mass[Weights::bucket(place)], (unsigned long long)w);
                    if (cut) atomicAdd(&lds.count[Weights::bucket(place)], 1u);
                });
                add_up_buckets<THREADS>(lds);
            };
            bool spoilt = false;
            fill();
            uint64_t mass = lds.mass[kBuckets];
            if (cut && lds.count[kBuckets] > (uint32_t)top_k) {
                find_place<BF16, true, THREADS>(row, weights, (uint64_t)top_k, lds, spoilt);
                mass = lds.found_mass;
            }
            if (top_p < 1.0f) {
                if (spoilt) fill();
                spoilt = false;
                const uint64_t goal = (uint64_t)ceil(fmax((double)top_p, 0.0) * (double)mass);
                find_place<BF16, false, THREADS>(row, weights, min(max(goal, (uint64_t)1), mass), lds, spoilt);
                mass = lds.found_mass;
            }
            if (spoilt) fill();
            const uint64_t goal = (uint64_t)(fmax((double)uniform, 0.0) * (double)mass);
            find_place<BF16, false, THREADS>(row, weights, min(goal, mass - 1) + 1, lds, spoilt);
            const uint64_t key = lds.found_key;
            put(column_of(key), (float)(((double)value_of(key) - (double)most) * inverse - log(__builtin_amdgcn_ldexp((double)mass, -(int)a.shift))));
        }
        __syncthreads();                                   // (what the next row writes to lds)
    }
}

// ---- host ------------------------------------------------------------------------------------
template <bool BF16>
static int sample_launch(const SampleArgs &a, hipStream_t stream)
{
    const dim3 grid((uint32_t)(a.rows < (1u << 20) ? a.rows : 1u << 20));
    if (a.cols <= 8192) return launch(sample_kernel<BF16, 256>, grid, 256, stream, a);
    return launch(sample_kernel<BF16, 1024>, grid, 1024, stream, a);
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
    if (s->cols >= (1ull << 29) || s->rows >= (1ull << 40) || s->stride >= (1ull << 40)) return SOLO_E_UNSUPPORTED;
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
