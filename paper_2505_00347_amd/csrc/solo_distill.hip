// Distillation: the divergence of every row of a student's logits from a teacher of which a few alternatives are known, and the gradient.
//
//   e_j = e^(s (x_j - m)),  m = max x,  S = sum_j e_j,  q_j = e_j / S;   the teacher's p_k at columns c_k, and what they leave of 1, r
//   of the columns that are not among the c_k:  f_j = e^(s (x_j - o)),  R = sum of f_j;   g = e^(s (o - m)), so that e_j = g f_j
//   loss = sum_k p_k (ln p_k - ln q_(c_k)) + r (ln r - (s (o - m) + ln R - ln S))
//   dx_j = s a (e_j T / S - sum over k with c_k = j of p_k)  among the c_k,   s a f_j (g T / S - r / R)  elsewhere,   T = sum_k p_k + r
//
// (r is 0 where the p_k are brought to a sum of 1.)  R is summed by itself: as 1 minus the rest of the q it would have no digits left in a
// student that is sure of an alternative.  So the columns c_k are taken out in front of the sums.  o is m, or, where R would be below 2^-64, the largest logit
// of those columns: beside an alternative that leads by 88 / s their e_j are 0 in binary32, their shares f_j / R of what the teacher leaves are not.  One wavefront reads the teacher's row while
// the logits are on their way and hangs every alternative into a list of the thread that has its column; a thread knows by one bit for each of its
// groups whether it has any there.  The gradient is written as if there were none; then the threads write those of their alternatives over it.
//
// Otherwise as the log probabilities: a workgroup takes a row, one pass for the sums, the row stays in registers for the gradient.
//
// Bound by memory: loss and gradient of 8192 x 32000 bf16, a tenth without a teacher, 181 us (5.5 TB/s of what it needs; rows without a teacher are
// read, too, since the logits are under way before the teacher is known); loss of 512 x 50304 bf16 12.7 us; 1000 x 50257 fp32 in
// two calls 104 us.  The alternatives' logits as they come by in both passes, inside the loops, took 313 us of the first: four times the registers, one workgroup a
// compute unit instead of two.  Short rows, one a wavefront, are bound by vector instructions: 608462 x 154 fp32 with 32 alternatives 328 us, 372 a row.
#include "solo_rows.h"

#include <float.h>
#include <math.h>

namespace solo {

constexpr int kMostTop = SOLO_DISTILL_MAX;
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr double kNoRest = 1.0 / (1 << 20);    // what is left of 1 below this is the probabilities' rounding
constexpr float kSmallRest = 0x1p-64f;         // R below this, relative to the row's largest: its smallest terms may be 0, and so may soon all of it

struct DistillArgs {
    const void *logits, *value, *token;
    void *grad;
    float *loss, *stats;
    const float *grad_loss;
    uint64_t rows, stride, grad_stride, value_stride, token_stride;
    uint32_t cols, top;
    float scale, teacher_scale;
    uint32_t wide, value_bf16, rest;
};

template <int THREADS>
struct TeacherLds {
    uint32_t head[THREADS];            // a thread's first alternative; kNone: it has none
    uint32_t column[kMostTop];         // of an alternative; kNone: none, or an earlier one has the same
    uint32_t next[kMostTop], same[kMostTop];       // same: the first alternative with its column
    float p[kMostTop], log_p[kMostTop];
    float all_p[kMostTop];             // of all alternatives of the column
    float logit[kMostTop];
    float total, left;                 // T and r
    uint32_t any;
    float at[THREADS / kLanes], s[THREADS / kLanes];
};

__device__ __forceinline__ void lds_in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

// By the first wavefront: the teacher's row, and the lists.  A lane has alternatives `lane`, `lane` + 64, ... of PER * 64.  A barrier has to follow.
template <int PER, bool BF16, int THREADS>
__device__ __forceinline__ void read_alternatives(const DistillArgs &a, const Row<BF16> &row, uint64_t r, TeacherLds<THREADS> &lds)
{
    const uint32_t lane = threadIdx.x;
    uint32_t column[PER];
    float value[PER], p[PER], log_p[PER];
    bool live[PER];
#pragma unroll
    for (int h = 0; h < PER; ++h) {
        const uint32_t i = lane + h * kLanes;
        int64_t id = -1;
        value[h] = -INFINITY;
        if (i < a.top) {
            id = a.wide ? static_cast<const int64_t *>(a.token)[r * a.token_stride + i] : (int64_t)static_cast<const int32_t *>(a.token)[r * a.token_stride + i];
            value[h] = a.value_bf16 ? Elements<true>::load1(a.value, r * a.value_stride + i) : Elements<false>::load1(a.value, r * a.value_stride + i);
        }
        live[h] = id >= 0 && id < (int64_t)a.cols && value[h] != -INFINITY;      // (a NaN counts, and shows)
        column[h] = live[h] ? (uint32_t)id : kNone;
    }
    float most = -INFINITY;
    bool some = false;
#pragma unroll
    for (int h = 0; h < PER; ++h) {
        some = some || live[h];
        if (live[h]) most = fmaxf(most, value[h]);
    }
    const bool any = __ballot(some) != 0;
    float total, left = 0.0f;
    if (a.rest) {
        double sum = 0.0;
#pragma unroll
        for (int h = 0; h < PER; ++h) {
            const double exact = live[h] ? exp((double)value[h]) : 0.0;
            p[h] = (float)exact;
            log_p[h] = value[h];
            sum += exact;
        }
        sum = wave_sum(sum);
        if (!(1.0 - sum < kNoRest)) left = (float)(1.0 - sum);
        total = (float)sum + left;
    } else {
        most = wave_max(most);
        float sum = 0.0f;
#pragma unroll
        for (int h = 0; h < PER; ++h) {
            log_p[h] = (value[h] - most) * a.teacher_scale;
            p[h] = live[h] ? __builtin_amdgcn_exp2f(log_p[h] * kLog2E) : 0.0f;
            sum += p[h];
        }
        sum = wave_sum(sum);
        const float log_sum = __builtin_amdgcn_logf(sum) * kLn2;
#pragma unroll
        for (int h = 0; h < PER; ++h) {
            p[h] /= any ? sum : 1.0f;
            log_p[h] -= log_sum;
        }
        total = any ? 1.0f : 0.0f;
    }
    // every alternative into the list of the thread that has its column
    auto hang = [&](int h) {
        const uint32_t i = lane + h * kLanes, g = column[h] / Row<BF16>::kPer;
        lds.next[i] = atomicExch(&lds.head[g < row.groups ? g % THREADS : column[h] - row.groups * Row<BF16>::kPer], i);
    };
    for (uint32_t t = lane; t < THREADS; t += kLanes) lds.head[t] = kNone;
    lds_in_order();
#pragma unroll
    for (int h = 0; h < PER; ++h) {
        const uint32_t i = lane + h * kLanes;
        lds.column[i] = column[h];
        lds.p[i] = lds.all_p[i] = p[h];
        lds.log_p[i] = log_p[h];
        lds.same[i] = i;
        if (live[h]) hang(h);
    }
    if (lane == 0) {
        lds.total = total;
        lds.left = left;
        lds.any = any;
    }
    lds_in_order();
    bool twice = false;                                    // (of two with one column the one that came later sees the other)
#pragma unroll
    for (int h = 0; h < PER; ++h)
        if (live[h])
            for (uint32_t k = lds.next[lane + h * kLanes]; k != kNone; k = lds.next[k]) twice = twice || lds.column[k] == column[h];
    if (__ballot(twice) == 0) return;
    // Seldom: the first of each column stays in the lists, with the probabilities of all of them, added in their order.
    uint32_t same[PER];
#pragma unroll
    for (int h = 0; h < PER; ++h) {
        p[h] = 0.0f;
        same[h] = lane + h * kLanes;
    }
    for (uint32_t i = 0; i < a.top; ++i) {
        const uint32_t c = lds.column[i];
        const float pi = lds.p[i];
#pragma unroll
        for (int h = 0; h < PER; ++h)
            if (c == column[h]) {
                p[h] += pi;
                same[h] = min(same[h], i);
            }
    }
    lds_in_order();
    for (uint32_t t = lane; t < THREADS; t += kLanes) lds.head[t] = kNone;
    lds_in_order();
#pragma unroll
    for (int h = 0; h < PER; ++h) {
        const uint32_t i = lane + h * kLanes;
        lds.all_p[i] = p[h];
        lds.same[i] = same[h];
        if (same[h] != i) lds.column[i] = kNone;
        else if (live[h]) hang(h);
    }
}

template <bool BF16, int THREADS>
__device__ __forceinline__ void read_teacher(const DistillArgs &a, const Row<BF16> &row, uint64_t r, TeacherLds<THREADS> &lds)
{
    if (a.top <= kLanes) read_alternatives<1, BF16, THREADS>(a, row, r, lds);
    else read_alternatives<kMostTop / kLanes, BF16, THREADS>(a, row, r, lds);
}

// The bits of a thread's groups that hold an alternative (group g has bit g / THREADS, of 32), and the one of its last column.
template <bool BF16, int THREADS>
__device__ __forceinline__ uint32_t own_alternatives(const Row<BF16> &row, const TeacherLds<THREADS> &lds, uint32_t &at_last)
{
    uint32_t mask = 0;
    at_last = kNone;
    for (uint32_t k = lds.head[threadIdx.x]; k != kNone; k = lds.next[k]) {
        const uint32_t g = lds.column[k] / Row<BF16>::kPer;
        if (g < row.groups) mask |= 1u << (g / THREADS % 32);
        else at_last = k;
    }
    return mask;
}

// The logits of group g without those of the alternatives, which go to lds; `most` is no less than any of them.
template <bool BF16, int THREADS>
__device__ __forceinline__ void take_out(Quad &quad, uint32_t g, TeacherLds<THREADS> &lds, float &most)
{
    for (uint32_t k = lds.head[threadIdx.x]; k != kNone; k = lds.next[k]) {
        const uint32_t c = lds.column[k], e = c % Row<BF16>::kPer;
        if (c / Row<BF16>::kPer != g) continue;
        const uint32_t at = BF16 ? e / 2 : e;
        uint32_t word = quad[0];
#pragma unroll
        for (uint32_t o = 1; o < 4; ++o) word = at == o ? quad[o] : word;
        const float x = __uint_as_float(!BF16 ? word : e % 2 ? word & 0xFFFF0000u : word << 16);
        const uint32_t without = !BF16 ? 0xFF800000u : e % 2 ? (word & 0xFFFFu) | 0xFF800000u : (word & 0xFFFF0000u) | 0xFF80u;
#pragma unroll
        for (uint32_t o = 0; o < 4; ++o)
            if (at == o) quad[o] = without;
        lds.logit[k] = x;
        most = __builtin_elementwise_maximum(most, x);
    }
}

struct RowSums { float at, rest_at, all, rest; };          // m, o, S and R
struct OwnSum { float at, s; };                            // a thread's largest logit of the rest and its sum relative to it

// The sum of all threads' relative to the largest of all, from wavefronts' sums relative to theirs.
template <int THREADS>
__device__ __forceinline__ float join_waves(float wave_at, float wave_s, float k, TeacherLds<THREADS> &lds, float &all_at)
{
    constexpr int kWaves = THREADS / kLanes;
    if (threadIdx.x % kLanes == 0) {
        lds.at[threadIdx.x / kLanes] = wave_at;
        lds.s[threadIdx.x / kLanes] = wave_s;
    }
    __syncthreads();
    all_at = wave_at;
    if (kWaves > 1) {
        const int part = threadIdx.x % kWaves;
        const float part_at = lds.at[part];
        all_at = wave_max<kWaves>(part_at);
        wave_s = wave_sum<kWaves>(lds.s[part] * __builtin_amdgcn_exp2f((part_at - all_at) * k));
    }
    return wave_s;
}

// The sums of a row, for every thread; the alternatives' logits go to lds.  `q`, `last`: as for the sums of the log probabilities.
template <bool BF16, bool RESIDENT, bool PAST, int THREADS, int DEPTH>
__device__ __forceinline__ RowSums student_sums(const Row<BF16> &row, float k, TeacherLds<THREADS> &lds, Quad q[DEPTH], float last, uint32_t top,
                                                uint32_t mask, uint32_t at_last, OwnSum &own)
{
    constexpr int kPer = Row<BF16>::kPer;
    float at = -FLT_MAX, s = 0.0f, most = -FLT_MAX;        // the largest logit of the rest and its sum relative to it; the alternatives' largest
    auto rebase = [&](float to) {
        s *= __builtin_amdgcn_exp2f((at - to) * k);        // (0 where nothing has been added)
        at = to;
    };
    auto add = [&](Quad &quad, uint32_t g) {
        if (mask >> (g / THREADS % 32) & 1) take_out<BF16, THREADS>(quad, g, lds, most);
        float x[kPer];
        Lane16<BF16>::unpack(quad, x);
        const float m = max_of<kPer>(x);
        if (m > at) rebase(m);
#pragma unroll
        for (int e = 0; e < kPer; ++e) s += __builtin_amdgcn_exp2f((x[e] - at) * k);
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
        if (at_last != kNone) {
            lds.logit[at_last] = last;
            most = __builtin_elementwise_maximum(most, last);
        } else {
            if (last > at) rebase(last);
            s += __builtin_amdgcn_exp2f((last - at) * k);
        }
    }
    own = OwnSum{at, s};
    // (an alternative that is NaN shows in its own term below)
    const float wave_at = wave_max(fmaxf(at, most));
    rebase(wave_at);
    RowSums sums;
    sums.rest = join_waves<THREADS>(wave_at, wave_sum(s), k, lds, sums.at);
    sums.rest_at = sums.at;
    float among = 0.0f;
    for (uint32_t i = threadIdx.x % kLanes; i < top; i += kLanes)
        if (lds.column[i] != kNone) among += __builtin_amdgcn_exp2f((lds.logit[i] - sums.at) * k);
    sums.all = sums.rest + wave_sum(among);
    return sums;
}

// The rest once more, relative to its own largest.
template <int THREADS>
__device__ __forceinline__ void rest_by_itself(RowSums &sums, const OwnSum &own, float k, TeacherLds<THREADS> &lds)
{
    const float rest_at = wave_max(own.at);
    __syncthreads();                                       // (lds.at and lds.s have been read)
    sums.rest = join_waves<THREADS>(rest_at, wave_sum(own.s * __builtin_amdgcn_exp2f((own.at - rest_at) * k)), k, lds, sums.rest_at);
}

// By the first wavefront, behind the sums: the row's loss and, if asked for, stats.  APART: o is not m.
template <bool APART, int THREADS>
__device__ __forceinline__ void put_loss(const DistillArgs &a, uint64_t r, const RowSums &sums, const TeacherLds<THREADS> &lds)
{
    const float log_s = __builtin_amdgcn_logf(sums.all) * kLn2;
    float loss = 0.0f;
    for (uint32_t i = threadIdx.x; i < a.top; i += kLanes) {
        const float p = lds.p[i];
        if (!(p <= 0.0f)) loss = fmaf(p, lds.log_p[i] - fmaf(lds.logit[lds.same[i]] - sums.at, a.scale, -log_s), loss);
    }
    loss = wave_sum(loss);
    if (lds.left > 0.0f)
        loss = fmaf(lds.left, (__builtin_amdgcn_logf(lds.left) - __builtin_amdgcn_logf(sums.rest)) * kLn2 + (APART ? fmaf(sums.at - sums.rest_at, a.scale, log_s) : log_s),
                    loss);
    if (threadIdx.x == 0) {
        if (a.loss) a.loss[r] = sums.all == 0.0f ? INFINITY : loss;
        if (a.stats) { a.stats[3 * r] = sums.rest_at; a.stats[3 * r + 1] = APART ? -sums.all : sums.all; a.stats[3 * r + 2] = sums.rest; }
    }
}

// What the gradient of a row needs: dx_j = (f_j rest) factor, or (e_j all - p) factor at an alternative.
struct DistillSlope { float at, rest_at, all, rest, factor; };

// `lowered`: g.
__device__ __forceinline__ DistillSlope distill_slope(const RowSums &sums, float lowered, float total, float left, float factor)
{
    // (no column of a student's row without probabilities has a gradient)
    const float all = sums.all == 0.0f ? 0.0f : total / sums.all, rest = sums.rest == 0.0f ? 0.0f : fmaf(all, lowered, -(left / sums.rest));
    return DistillSlope{sums.at, sums.rest_at, all, rest, sums.all == 0.0f ? 0.0f : factor};
}

// Wavefronts per SIMD that the registers have to leave room for: two workgroups of 1024 threads, so that one loads while the other computes, where 64
// registers are enough.
constexpr int distill_waves(bool forward, bool grad, bool resident, int depth)
{
    return forward && grad && resident && depth > 8 ? 4 : 8;
}

// FORWARD: the sums and the loss; GRAD: the gradient, from the sums or, without FORWARD, from those that are given.  RESIDENT: the row has no more
// than THREADS * DEPTH groups, which stay in registers between the two.  PAST: 1 stores past the caches, 2 loads as well.
template <bool BF16, bool FORWARD, bool GRAD, bool RESIDENT, int PAST, int THREADS, int DEPTH>
__global__ __launch_bounds__(THREADS, distill_waves(FORWARD, GRAD, RESIDENT, DEPTH)) void distill_kernel(const DistillArgs a)
{
    __shared__ TeacherLds<THREADS> lds;
    constexpr int kPer = Row<BF16>::kPer;
    const float k = a.scale * kLog2E;
    const uint64_t r = (uint64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (r >= a.rows) return;
    const Row<BF16> row(a, r);
    Quad raw[DEPTH];
    if (FORWARD) first_groups<BF16, (PAST > 1), THREADS, DEPTH>(row, raw);
    const float last = threadIdx.x < row.rest ? row.one(row.last_column(threadIdx.x)) : -INFINITY;
    if (threadIdx.x < kLanes) read_teacher<BF16, THREADS>(a, row, r, lds);
    __syncthreads();
    char *out = static_cast<char *>(a.grad) + r * a.grad_stride * Elements<BF16>::kBytes;
    if (!lds.any) {                                        // no teacher
        if (GRAD) {
            const float none[kPer] = {};
            for (uint32_t g = threadIdx.x; g < row.groups; g += THREADS) Lane16<BF16>::template store_near<(PAST > 0)>(out, g * kPer, none);
            if (threadIdx.x < row.rest) Elements<BF16>::store1(out, row.last_column(threadIdx.x), 0.0f);
        }
        if (FORWARD && threadIdx.x == 0) {
            if (a.loss) a.loss[r] = 0.0f;
            if (a.stats) { a.stats[3 * r] = 0.0f; a.stats[3 * r + 1] = 0.0f; a.stats[3 * r + 2] = 0.0f; }
        }
        return;
    }
    RowSums sums;
    float lowered = 1.0f;
    const uint32_t head = FORWARD ? kNone : lds.head[threadIdx.x];        // (once, not again behind a barrier that few rows come to)
    if (FORWARD) {
        uint32_t at_last;
        OwnSum own;
        const uint32_t mask = own_alternatives<BF16, THREADS>(row, lds, at_last);
        sums = student_sums<BF16, RESIDENT, (PAST > 1), THREADS, DEPTH>(row, k, lds, raw, last, a.top, mask, at_last, own);
        if (threadIdx.x < kLanes) put_loss<false, THREADS>(a, r, sums, lds);
        // Seldom.  (The sum is bit by bit the same in all threads, so all of them come here or none; it is not below +0, and its bits are in the order of its value.)
        if (scalar(__float_as_uint(sums.rest)) < __float_as_uint(kSmallRest) && scalar(lds.left) > 0.0f) {
            rest_by_itself<THREADS>(sums, own, k, lds);
            if (threadIdx.x < kLanes && sums.rest != 0.0f) put_loss<true, THREADS>(a, r, sums, lds);
            lowered = scalar(__builtin_amdgcn_exp2f((sums.rest_at - sums.at) * k));
        }
    } else {
        sums = RowSums{a.stats[3 * r], a.stats[3 * r], a.stats[3 * r + 1], a.stats[3 * r + 2]};
        // (the gradient may be written over them)
        for (uint32_t i = head; i != kNone; i = lds.next[i]) lds.logit[i] = row.one(lds.column[i]);
        if (scalar(sums.all) < 0.0f) {                     // (an alternative is the row's largest)
            __syncthreads();
            float at = -FLT_MAX;
            for (uint32_t i = threadIdx.x % kLanes; i < a.top; i += kLanes)
                if (lds.column[i] != kNone) at = fmaxf(at, lds.logit[i]);
            sums.at = wave_max(at);
            sums.all = -sums.all;
            lowered = scalar(__builtin_amdgcn_exp2f((sums.rest_at - sums.at) * k));
        }
    }
    if (!GRAD) return;
    const DistillSlope slope = distill_slope(sums, lowered, lds.total, lds.left, a.scale * a.grad_loss[r]);
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
                float x[kPer];
                Lane16<BF16>::unpack(raw[j], x);
#pragma unroll
                for (int e = 0; e < kPer; ++e) x[e] = __builtin_amdgcn_exp2f((x[e] - slope.rest_at) * k) * slope.rest * slope.factor;
                Lane16<BF16>::template store_near<(PAST > 0)>(out, (g0 + j * THREADS) * kPer, x);
            }
        if (FORWARD && RESIDENT) break;
    }
    if (threadIdx.x < row.rest)
        Elements<BF16>::store1(out, row.last_column(threadIdx.x), __builtin_amdgcn_exp2f((last - slope.rest_at) * k) * slope.rest * slope.factor);
    // over what the same thread has just written (of an alternative's logit, where the row has been read again, anything)
    for (uint32_t i = FORWARD ? lds.head[threadIdx.x] : head; i != kNone; i = lds.next[i])
        Elements<BF16>::store1(out, lds.column[i], fmaf(__builtin_amdgcn_exp2f((lds.logit[i] - slope.at) * k), slope.all, -lds.all_p[i]) * slope.factor);
}

// ---- host ------------------------------------------------------------------------------------
static int distill_args(DistillArgs &a, const void *logits, const void *value, const void *token, const solo_distill_shape *s)
{
    if (!s || !dtype_ok(s->dtype) || !dtype_ok(s->value_dtype) || (s->token_bits != 32 && s->token_bits != 64) || (s->flags & ~SOLO_DISTILL_REST) ||
        s->top < 1 || s->top > SOLO_DISTILL_MAX || s->reserved != 0 || !(s->scale > 0.0f) || !isfinite(s->scale) || !isfinite(s->scale * kLog2E) ||
        !(s->teacher_scale > 0.0f) || !isfinite(s->teacher_scale) || ((s->flags & SOLO_DISTILL_REST) && s->teacher_scale != 1.0f) ||
        s->stride < s->cols || s->value_stride < s->top || s->token_stride < s->top)
        return SOLO_E_INVALID;
    if (s->rows != 0 && ((s->cols != 0 && !at_multiple(logits, element_bytes(s->dtype))) || !at_multiple(value, element_bytes(s->value_dtype)) ||
                         !at_multiple(token, s->token_bits / 8)))
        return SOLO_E_INVALID;
    if (s->cols >= (1ull << 29) || s->rows >= (1ull << 35) || s->stride >= (1ull << 40) || s->grad_stride >= (1ull << 40) || s->value_stride >= (1ull << 40) ||
        s->token_stride >= (1ull << 40))
        return SOLO_E_UNSUPPORTED;
    a = DistillArgs{};
    a.logits = logits; a.value = value; a.token = token;
    a.rows = s->rows; a.cols = (uint32_t)s->cols; a.stride = s->stride; a.grad_stride = s->grad_stride;
    a.value_stride = s->value_stride; a.token_stride = s->token_stride;
    a.top = s->top; a.scale = s->scale; a.teacher_scale = s->teacher_scale;
    a.wide = s->token_bits == 64; a.value_bf16 = s->value_dtype == SOLO_BF16; a.rest = (s->flags & SOLO_DISTILL_REST) != 0;
    return SOLO_OK;
}

static bool optional_at(const void *p, uintptr_t size) { return !p || at_multiple(p, size); }

// As for the log probabilities: what is larger than the last-level cache is read past it, gradients that are not small are written past it.
constexpr uint64_t kDistillPastLoads = 256ull << 20, kDistillPastStores = 32ull << 20;

template <bool BF16, bool FORWARD, bool GRAD, bool RESIDENT, int THREADS, int DEPTH>
static int distill_launch(const DistillArgs &a, hipStream_t stream)
{
    constexpr int kDepth = BF16 ? DEPTH : 2 * DEPTH;
    const uint64_t bytes = a.rows * a.cols * (BF16 ? 2 : 4);
    const uint32_t across = (uint32_t)(a.rows < (1u << 20) ? a.rows : 1u << 20);
    const dim3 grid(across, (uint32_t)((a.rows + across - 1) / across));
    if constexpr (GRAD) {
        constexpr int kBoth = FORWARD && !RESIDENT ? 1 : 2;        // (a row that is read twice stays in the caches)
        return launch(bytes > kDistillPastLoads    ? distill_kernel<BF16, FORWARD, GRAD, RESIDENT, kBoth, THREADS, kDepth>
                      : bytes > kDistillPastStores ? distill_kernel<BF16, FORWARD, GRAD, RESIDENT, 1, THREADS, kDepth>
                                                   : distill_kernel<BF16, FORWARD, GRAD, RESIDENT, 0, THREADS, kDepth>,
                      grid, THREADS, stream, a);
    } else {
        return launch(bytes > kDistillPastLoads ? distill_kernel<BF16, FORWARD, GRAD, RESIDENT, 2, THREADS, kDepth>
                                                : distill_kernel<BF16, FORWARD, GRAD, RESIDENT, 0, THREADS, kDepth>,
                      grid, THREADS, stream, a);
    }
}

template <bool BF16>
static int distill_forward(const DistillArgs &a, hipStream_t stream)
{
    const uint32_t groups = a.cols / 8;
    if (groups <= 256) return distill_launch<BF16, true, false, false, 64, 2>(a, stream);
    if (a.rows >= 128 || groups <= 1024) return distill_launch<BF16, true, false, false, 256, 2>(a, stream);
    return distill_launch<BF16, true, false, false, 512, 2>(a, stream);
}

template <bool BF16>
static int distill_with_grad(const DistillArgs &a, hipStream_t stream)
{
    const uint32_t groups = (a.cols + 7) / 8;              // (all of them have to fit)
    if (groups <= 64 * 4) return distill_launch<BF16, true, true, true, 64, 4>(a, stream);
    if (groups <= 256 * 4) return distill_launch<BF16, true, true, true, 256, 4>(a, stream);
    if (groups <= 512 * 4) return distill_launch<BF16, true, true, true, 512, 4>(a, stream);
    if (groups <= 1024 * 4) return distill_launch<BF16, true, true, true, 1024, 4>(a, stream);
    if (groups <= 1024 * 8) return distill_launch<BF16, true, true, true, 1024, 8>(a, stream);
    return distill_launch<BF16, true, true, false, 1024, 2>(a, stream);
}

template <bool BF16>
static int distill_only_grad(const DistillArgs &a, hipStream_t stream)
{
    const uint32_t groups = a.cols / 8;
    if (groups <= 128) return distill_launch<BF16, false, true, false, 64, 2>(a, stream);
    if (groups <= 640) return distill_launch<BF16, false, true, false, 256, 2>(a, stream);
    return distill_launch<BF16, false, true, false, 1024, 2>(a, stream);
}

}  // namespace solo

extern "C" {

int solo_distill(const void *logits, const void *teacher_value, const void *teacher_token, float *loss, float *stats, const solo_distill_shape *shape, void *stream)
{
    using namespace solo;
    DistillArgs a;
    const int rc = distill_args(a, logits, teacher_value, teacher_token, shape);
    if (rc != SOLO_OK) return rc;
    if (shape->rows == 0) return SOLO_OK;
    if (!optional_at(loss, 4) || !optional_at(stats, 4)) return SOLO_E_INVALID;
    a.loss = loss; a.stats = stats;
    return shape->dtype == SOLO_BF16 ? distill_forward<true>(a, (hipStream_t)stream) : distill_forward<false>(a, (hipStream_t)stream);
}

int solo_distill_grad(const void *logits, const void *teacher_value, const void *teacher_token, const float *stats, const float *grad_loss, void *grad_logits,
                      const solo_distill_shape *shape, void *stream)
{
    using namespace solo;
    DistillArgs a;
    const int rc = distill_args(a, logits, teacher_value, teacher_token, shape);
    if (rc != SOLO_OK) return rc;
    if (shape->grad_stride < shape->cols) return SOLO_E_INVALID;
    if (shape->rows == 0 || shape->cols == 0) return SOLO_OK;
    if (!at_multiple(stats, 4) || !at_multiple(grad_loss, 4) || !at_multiple(grad_logits, element_bytes(shape->dtype))) return SOLO_E_INVALID;
    a.stats = const_cast<float *>(stats); a.grad_loss = grad_loss; a.grad = grad_logits;
    return shape->dtype == SOLO_BF16 ? distill_only_grad<true>(a, (hipStream_t)stream) : distill_only_grad<false>(a, (hipStream_t)stream);
}

int solo_distill_with_grad(const void *logits, const void *teacher_value, const void *teacher_token, const float *grad_loss, float *loss, void *grad_logits,
                           const solo_distill_shape *shape, void *stream)
{
    using namespace solo;
    DistillArgs a;
    const int rc = distill_args(a, logits, teacher_value, teacher_token, shape);
    if (rc != SOLO_OK) return rc;
    if (shape->grad_stride < shape->cols) return SOLO_E_INVALID;
    if (shape->rows == 0) return SOLO_OK;
    if (!optional_at(loss, 4) || !at_multiple(grad_loss, 4) || (shape->cols != 0 && !at_multiple(grad_logits, element_bytes(shape->dtype)))) return SOLO_E_INVALID;
    a.loss = loss; a.grad_loss = grad_loss; a.grad = grad_logits;
    return shape->dtype == SOLO_BF16 ? distill_with_grad<true>(a, (hipStream_t)stream) : distill_with_grad<false>(a, (hipStream_t)stream);
}

}  // extern "C"
