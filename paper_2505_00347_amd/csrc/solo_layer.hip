// Layer norm of rows, and its gradient with the reductions of weight and bias over the rows.
//
//   mean = sum x / n (0 for the root mean square alone)    rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)    h = (x - mean) rstd
//   y = h w + b
//   g = dy w        dx = rstd (g - sum g / n - h sum(g h) / n)        dw = sum over rows of dy h        db = sum over rows of dy
//
// (without the term in sum g for the root mean square).  A row stays in registers between its sums and its results, so it is read
// once; the squares are those of the differences from the mean, and what the mean's own rounding leaves of the differences' sum is taken out
// as well, so a row far from zero loses no digits.  The gradient has the mean rounded to binary32; where that is half a millionth of a deviation or
// more, what it leaves in h is summed and taken out.  The gradient's threads keep
// their columns: each adds dy h and dy of all its rows in registers, the workgroups' sums go to the workspace, and a second launch
// adds those in the order of the workgroups.
//
// Bound by memory where rows are wide: 16384 x 4096 bf16 forward 50 us (5.4 TB/s), gradient 80 us (5.0), sums of the parts 4 us.  Loads of the next row in
// front of the work on this one gain nothing (80 us with them, 41 instead of 36 for 8192 x 2048 fp32): the other wavefronts have theirs under way.  Accesses past the
// caches take 3 to 8 % off calls of more than 256 MiB (32768 x 4096 bf16, both, 247 and 227 us), which the product that reads the output next would lose.  Rows
// that do not fill their threads (560 bf16: 70 of 128 groups) are bound by instructions, 2.9 TB/s.
#include "solo_ops.h"

#include <math.h>

namespace solo {

struct LayerArgs {
    const void *x, *w, *b, *dy;
    void *y, *dx;
    float *stats, *part, *centre;
    uint64_t rows, x_stride, y_stride, dx_stride;
    uint32_t cols;
    float eps;
    uint32_t w_bf16, rms;
};

// PER elements as they lie in memory: 16 or 8 bytes.
template <bool BF16, int PER>
struct Raw {
    static constexpr int kWords = PER * (BF16 ? 2 : 4) / 4;
    typedef uint32_t Words __attribute__((ext_vector_type(kWords), aligned(2)));
    Words w;

    __device__ __forceinline__ void load(const void *base, uint64_t i)
    {
        w = *reinterpret_cast<const Words *>(static_cast<const char *>(base) + i * (BF16 ? 2 : 4));
    }
    // the first `n` of them; zeros behind
    __device__ __forceinline__ void load_part(const void *base, uint64_t i, uint32_t n)
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            if (BF16) {
                const uint32_t low = 2 * k < (int)n ? static_cast<const uint16_t *>(base)[i + 2 * k] : 0;
                const uint32_t high = 2 * k + 1 < (int)n ? static_cast<const uint16_t *>(base)[i + 2 * k + 1] : 0;
                w[k] = high << 16 | low;
            } else {
                w[k] = k < (int)n ? static_cast<const uint32_t *>(base)[i + k] : 0;
            }
        }
    }
    __device__ __forceinline__ void unpack(float x[PER]) const
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            if (BF16) {
                x[2 * k % PER] = bf16_low(w[k]);
                x[(2 * k + 1) % PER] = bf16_high(w[k]);
            } else {
                x[k % PER] = __uint_as_float(w[k]);
            }
        }
    }
    __device__ __forceinline__ static void store(void *base, uint64_t i, const float x[PER], uint32_t n)
    {
        char *at = static_cast<char *>(base) + i * (BF16 ? 2 : 4);
        if (n == PER) {
            Words q;
#pragma unroll
            for (int k = 0; k < kWords; ++k) q[k] = BF16 ? to_bf16(x[2 * k % PER], x[(2 * k + 1) % PER]) : __float_as_uint(x[k % PER]);
            *reinterpret_cast<Words *>(at) = q;
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e)
                if (e < (int)n) Elements<BF16>::store1(at, e, x[e]);
        }
    }
};

// How a row of up to LANES * E elements is dealt out: groups of kPer elements, in turn, to LANES threads, which have E each.
// Rows of up to 64 lanes share a workgroup of 256 threads.  16 bytes a lane and access of the wider type.
template <bool XB, bool YB, int LANES, int E>
struct Deal {
    static constexpr int kPer = XB && YB ? 8 : 4, kDepth = E / kPer;
    static constexpr int kThreads = LANES < 256 ? 256 : LANES, kRows = kThreads / LANES;
    uint32_t lane, cols;

    __device__ __forceinline__ explicit Deal(uint32_t cols) : lane(threadIdx.x % LANES), cols(cols) {}
    __device__ __forceinline__ uint32_t column(int j) const { return (j * LANES + lane) * kPer; }
    __device__ __forceinline__ uint32_t count(int j) const        // elements of group j
    {
        const uint32_t c = column(j);
        return c >= cols ? 0 : min(cols - c, (uint32_t)kPer);
    }
    template <bool BF16>
    __device__ __forceinline__ void load(Raw<BF16, kPer> q[kDepth], const void *base, uint64_t at) const
    {
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            const uint32_t n = count(j);
            if (n == kPer) q[j].load(base, at + column(j));
            else q[j].load_part(base, at + column(j), n);
        }
    }
    // weights of either type, or `none` where there are none
    __device__ __forceinline__ void load_weights(float w[E], const void *base, bool bf16, float none) const
    {
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            const uint32_t n = count(j);
            if (!base) {
#pragma unroll
                for (int e = 0; e < kPer; ++e) w[j * kPer + e] = none;
            } else if (bf16) {
                Raw<true, kPer> q;
                if (n == kPer) q.load(base, column(j));
                else q.load_part(base, column(j), n);
                q.unpack(w + j * kPer);
            } else {
#pragma unroll
                for (int h = 0; h < kPer; h += 4) {
                    Raw<false, 4> q;
                    if (n == kPer) q.load(base, column(j) + h);
                    else q.load_part(base, column(j) + h, n > (uint32_t)h ? n - h : 0);
                    q.unpack(w + j * kPer + h);
                }
            }
        }
    }
};

// Sums of V values over the LANES threads of a row, for each of them.  Two halves of `lds` are used in turn: a thread that writes one
// again has passed the barrier of the sum in between, behind which nobody reads it any more.
template <int LANES, int V>
__device__ __forceinline__ void row_total(float v[V], float (*halves)[32], uint32_t &turn)
{
    constexpr int kWaves = LANES / kLanes;
    static_assert(V * kWaves <= 32, "");
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = wave_sum<(LANES < kLanes ? LANES : kLanes)>(v[k]);
    if constexpr (kWaves > 1) {
        float *const lds = halves[turn];
        turn ^= 1;
        if (threadIdx.x % kLanes == 0) {
#pragma unroll
            for (int k = 0; k < V; ++k) lds[k * kWaves + threadIdx.x / kLanes] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = wave_sum<kWaves>(lds[k * kWaves + threadIdx.x % kWaves]);
    }
}

template <bool XB, bool YB, int LANES, int E>
__global__ __launch_bounds__((Deal<XB, YB, LANES, E>::kThreads)) void layer_forward_kernel(const LayerArgs a)
{
    using D = Deal<XB, YB, LANES, E>;
    constexpr int kPer = D::kPer, kDepth = D::kDepth;
    __shared__ float lds[2][32];
    uint32_t turn = 0;
    const D deal(a.cols);
    const float inverse = 1.0f / (float)a.cols;
    float w[E], b[E];
    deal.load_weights(w, a.w, a.w_bf16, 1.0f);
    deal.load_weights(b, a.b, a.w_bf16, 0.0f);
    for (uint64_t r = blockIdx.x * (uint64_t)D::kRows + threadIdx.x / LANES; r < a.rows; r += gridDim.x * (uint64_t)D::kRows) {
        Raw<XB, kPer> q[kDepth];
        deal.template load<XB>(q, a.x, r * a.x_stride);
        float x[E], sum[1] = {0.0f}, left[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kDepth; ++j) q[j].unpack(x + j * kPer);
        if (!a.rms) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += x[e];
            row_total<LANES, 1>(sum, lds, turn);
        }
        float mean = sum[0] * inverse;
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            const uint32_t n = deal.count(j);
#pragma unroll
            for (int e = j * kPer; e < (j + 1) * kPer; ++e) x[e] -= mean;
            if (n != kPer) {                               // (nothing behind the row)
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (e >= (int)n) x[j * kPer + e] = 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            left[0] += x[e];
            left[1] = fmaf(x[e], x[e], left[1]);
        }
        row_total<LANES, 2>(left, lds, turn);
        // what the mean's rounding has left of it: of rows far from zero more than the spread
        const float shift = a.rms ? 0.0f : left[0] * inverse;
        const float variance = fmaf(-shift, shift, left[1] * inverse);
        const float rstd = 1.0f / sqrtf((variance < 0.0f ? 0.0f : variance) + a.eps);        // (NaN stays)
        mean += shift;
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            float y[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) y[e] = fmaf((x[j * kPer + e] - shift) * rstd, w[j * kPer + e], b[j * kPer + e]);
            const uint32_t n = deal.count(j);
            if (n != 0) Raw<YB, kPer>::store(a.y, r * a.y_stride + deal.column(j), y, n);
        }
        if (a.stats && deal.lane == 0) {
            a.stats[2 * r] = mean;
            a.stats[2 * r + 1] = rstd;
        }
    }
}

// A row of a mean this many deviations away from zero: 16 * 2^-24, what rounding the mean leaves in h, is 2^-20, and sums over a row leave as much.
__device__ __forceinline__ bool far_from_zero(float mean, float rstd) { return fabsf(mean) * rstd > 16.0f; }

// The gradients of rows blockIdx.x, blockIdx.x + gridDim.x, ... and the workgroup's sums for weight and bias: part[0][group][cols] and
// part[1][group][cols].
template <bool XB, bool YB, int LANES, int E>
__global__ __launch_bounds__((Deal<XB, YB, LANES, E>::kThreads)) void layer_backward_kernel(const LayerArgs a)
{
    using D = Deal<XB, YB, LANES, E>;
    constexpr int kPer = D::kPer, kDepth = D::kDepth;
    __shared__ float lds[2][32];
    uint32_t turn = 0;
    const D deal(a.cols);
    const float inverse = 1.0f / (float)a.cols;
    float w[E], dw[E] = {}, db[E] = {};
    deal.load_weights(w, a.w, a.w_bf16, 1.0f);
    for (uint64_t r = blockIdx.x * (uint64_t)D::kRows + threadIdx.x / LANES; r < a.rows; r += gridDim.x * (uint64_t)D::kRows) {
        Raw<XB, kPer> qx[kDepth];
        Raw<YB, kPer> qy[kDepth];
        deal.template load<XB>(qx, a.x, r * a.x_stride);
        deal.template load<YB>(qy, a.dy, r * a.y_stride);
        const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1];
        float h[E], g[E], sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            qx[j].unpack(h + j * kPer);
            qy[j].unpack(g + j * kPer);
            const uint32_t n = deal.count(j);
#pragma unroll
            for (int e = j * kPer; e < (j + 1) * kPer; ++e) h[e] = (h[e] - mean) * rstd;
            if (n != kPer) {
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (e >= (int)n) h[j * kPer + e] = 0.0f;
            }
        }
        // (rows of a wavefront may differ in it, threads that meet at a barrier have one row; behind the row g is 0)
        const bool far = far_from_zero(mean, rstd);
        if (__ballot(far) != 0) {
            float left[1] = {0.0f};
#pragma unroll
            for (int e = 0; e < E; ++e) left[0] += h[e];
            row_total<LANES, 1>(left, lds, turn);
            const float centre = far ? left[0] * inverse : 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) h[e] -= centre;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            dw[e] = fmaf(g[e], h[e], dw[e]);
            db[e] += g[e];
            g[e] *= w[e];
            sums[0] += g[e];
            sums[1] = fmaf(g[e], h[e], sums[1]);
        }
        if (!a.dx) continue;
        row_total<LANES, 2>(sums, lds, turn);
        const float shift = a.rms ? 0.0f : sums[0] * inverse, slope = sums[1] * inverse;
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            float dx[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) dx[e] = (fmaf(-h[j * kPer + e], slope, g[j * kPer + e]) - shift) * rstd;
            const uint32_t n = deal.count(j);
            if (n != 0) Raw<XB, kPer>::store(a.dx, r * a.dx_stride + deal.column(j), dx, n);
        }
    }
    if (!a.part) return;
    float *const part_w = a.part + (uint64_t)blockIdx.x * a.cols, *const part_b = part_w + (uint64_t)gridDim.x * a.cols;
    if constexpr (D::kRows == 1) {
#pragma unroll
        for (int j = 0; j < kDepth; ++j) {
            const uint32_t n = deal.count(j);
            if (n == 0) continue;
            Raw<false, 4>::store(part_w, deal.column(j), dw + j * kPer, min(n, 4u));
            Raw<false, 4>::store(part_b, deal.column(j), db + j * kPer, min(n, 4u));
            if (kPer == 8 && n > 4) {
                Raw<false, 4>::store(part_w, deal.column(j) + 4, dw + (j * kPer + 4) % E, n - 4);
                Raw<false, 4>::store(part_b, deal.column(j) + 4, db + (j * kPer + 4) % E, n - 4);
            }
        }
    } else {
        // the sums of a wavefront's rows, then those of the wavefronts in their order
        constexpr int kWaves = D::kThreads / kLanes;
        __shared__ float all[2][kWaves][LANES * E];
        const uint32_t wave = threadIdx.x / kLanes;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (LANES < kLanes) {
                dw[e] = wave_reduce<kLanes, LANES>(dw[e], [](float p, float q) { return p + q; });
                db[e] = wave_reduce<kLanes, LANES>(db[e], [](float p, float q) { return p + q; });
            }
            if (threadIdx.x % kLanes < LANES) {
                // (element e of each lane side by side: no two lanes in one bank)
                all[0][wave][e * LANES + deal.lane] = dw[e];
                all[1][wave][e * LANES + deal.lane] = db[e];
            }
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.cols; c += D::kThreads) {
            const uint32_t group = c / kPer, at = (group / LANES * kPer + c % kPer) * LANES + group % LANES;
            float sum_w = all[0][0][at], sum_b = all[1][0][at];
#pragma unroll
            for (int k = 1; k < kWaves; ++k) {
                sum_w += all[0][k][at];
                sum_b += all[1][k][at];
            }
            part_w[c] = sum_w;
            part_b[c] = sum_b;
        }
    }
}

// Rows too long for registers.  One workgroup a row; every sum is a pass over it (from the caches, behind the first).  (2000 x 20000 bf16, forward and gradient, 238 us.)
template <bool XB, bool YB>
__global__ __launch_bounds__(1024) void layer_forward_long_kernel(const LayerArgs a)
{
    __shared__ float lds[2][32];
    uint32_t turn = 0;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const uint64_t at = r * a.x_stride;
        float sum[1] = {0.0f}, left[2] = {0.0f, 0.0f};
        if (!a.rms) {
            for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) sum[0] += Elements<XB>::load1(a.x, at + c);
            row_total<1024, 1>(sum, lds, turn);
        }
        const float mean = sum[0] / (float)a.cols;
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
            const float d = Elements<XB>::load1(a.x, at + c) - mean;
            left[0] += d;
            left[1] = fmaf(d, d, left[1]);
        }
        row_total<1024, 2>(left, lds, turn);
        const float shift = a.rms ? 0.0f : left[0] / (float)a.cols;
        const float variance = fmaf(-shift, shift, left[1] / (float)a.cols);
        const float rstd = 1.0f / sqrtf((variance < 0.0f ? 0.0f : variance) + a.eps);
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
            const float w = !a.w ? 1.0f : a.w_bf16 ? Elements<true>::load1(a.w, c) : Elements<false>::load1(a.w, c);
            const float b = !a.b ? 0.0f : a.w_bf16 ? Elements<true>::load1(a.b, c) : Elements<false>::load1(a.b, c);
            Elements<YB>::store1(a.y, r * a.y_stride + c, fmaf((Elements<XB>::load1(a.x, at + c) - mean - shift) * rstd, w, b));
        }
        if (a.stats && threadIdx.x == 0) {
            a.stats[2 * r] = mean + shift;
            a.stats[2 * r + 1] = rstd;
        }
    }
}

// What the mean's rounding leaves in h, of a long row.
template <bool XB>
__device__ __forceinline__ float long_centre(const LayerArgs &a, uint64_t r, float (*lds)[32], uint32_t &turn)
{
    const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1];
    if (!far_from_zero(mean, rstd)) return 0.0f;
    float sum[1] = {0.0f};
    for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) sum[0] += (Elements<XB>::load1(a.x, r * a.x_stride + c) - mean) * rstd;
    row_total<1024, 1>(sum, lds, turn);
    return sum[0] / (float)a.cols;
}

// The same for the columns' sums.
template <bool XB>
__global__ __launch_bounds__(1024) void layer_centre_kernel(const LayerArgs a)
{
    __shared__ float lds[2][32];
    uint32_t turn = 0;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const float centre = long_centre<XB>(a, r, lds, turn);
        if (threadIdx.x == 0) a.centre[r] = centre;
    }
}

template <bool XB, bool YB>
__global__ __launch_bounds__(1024) void layer_backward_long_kernel(const LayerArgs a)
{
    __shared__ float lds[2][32];
    uint32_t turn = 0;
    for (uint64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const uint64_t at = r * a.x_stride, at_y = r * a.y_stride;
        const float mean = a.stats[2 * r], rstd = a.stats[2 * r + 1], centre = long_centre<XB>(a, r, lds, turn);
        float sums[2] = {0.0f, 0.0f};
        auto weighted = [&](uint32_t c) {
            const float w = !a.w ? 1.0f : a.w_bf16 ? Elements<true>::load1(a.w, c) : Elements<false>::load1(a.w, c);
            return Elements<YB>::load1(a.dy, at_y + c) * w;
        };
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = weighted(c), h = (Elements<XB>::load1(a.x, at + c) - mean) * rstd - centre;
            sums[0] += g;
            sums[1] = fmaf(g, h, sums[1]);
        }
        row_total<1024, 2>(sums, lds, turn);
        const float shift = a.rms ? 0.0f : sums[0] / (float)a.cols, slope = sums[1] / (float)a.cols;
        for (uint32_t c = threadIdx.x; c < a.cols; c += 1024) {
            const float g = weighted(c), h = (Elements<XB>::load1(a.x, at + c) - mean) * rstd - centre;
            Elements<XB>::store1(a.dx, r * a.dx_stride + c, (fmaf(-h, slope, g) - shift) * rstd);
        }
    }
}

// Sums of blockIdx.y's share of the rows for 256 columns: in front of the rows' gradients, which may be written over the inputs.
template <bool XB, bool YB>
__global__ __launch_bounds__(256) void layer_columns_kernel(const LayerArgs a)
{
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float dw = 0.0f, db = 0.0f;
    for (uint64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float dy = Elements<YB>::load1(a.dy, r * a.y_stride + c);
        dw = fmaf(dy, (Elements<XB>::load1(a.x, r * a.x_stride + c) - a.stats[2 * r]) * a.stats[2 * r + 1] - a.centre[r], dw);
        db += dy;
    }
    a.part[(uint64_t)blockIdx.y * a.cols + c] = dw;
    a.part[((uint64_t)gridDim.y + blockIdx.y) * a.cols + c] = db;
}

struct LayerSumArgs {
    const float *part;
    void *dw, *db;
    uint32_t cols, parts, bf16, accumulate;
};

// The parts' sums, 64 columns a workgroup: 16 threads have four columns each, 64 of those every 64th part.
__global__ __launch_bounds__(1024) void layer_parts_kernel(const LayerSumArgs a)
{
    __shared__ float lds[64][64];
    void *const out = blockIdx.y ? a.db : a.dw;
    if (!out) return;
    const float *const part = a.part + (blockIdx.y ? (uint64_t)a.parts * a.cols : 0);
    const uint32_t c = blockIdx.x * 64 + threadIdx.x % 16 * 4, n = c < a.cols ? min(a.cols - c, 4u) : 0;
    float sum[4] = {};
    if (n == 4) {
#pragma unroll 8
        for (uint32_t p = threadIdx.x / 16; p < a.parts; p += 64) {
            float x[4];
            Raw<false, 4> q;
            q.load(part, (uint64_t)p * a.cols + c);
            q.unpack(x);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += x[e];
        }
    } else if (n != 0) {
        for (uint32_t p = threadIdx.x / 16; p < a.parts; p += 64)
            for (uint32_t e = 0; e < 4; ++e)
                if (e < n) sum[e] += part[(uint64_t)p * a.cols + c + e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[threadIdx.x / 16][threadIdx.x % 16 * 4 + e] = sum[e];
    __syncthreads();
    const uint32_t own = threadIdx.x % 64, rows = threadIdx.x / 64 * 4;    // a wavefront adds four rows, then the first one the wavefronts' sums
    lds[rows][own] = (lds[rows][own] + lds[rows + 1][own]) + (lds[rows + 2][own] + lds[rows + 3][own]);
    __syncthreads();
    const uint32_t column = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || column >= a.cols) return;
    float total = lds[0][own];
#pragma unroll
    for (int k = 4; k < 64; k += 4) total += lds[k][own];
    if (a.bf16) Elements<true>::store1(out, column, a.accumulate ? Elements<true>::load1(out, column) + total : total);
    else Elements<false>::store1(out, column, a.accumulate ? Elements<false>::load1(out, column) + total : total);
}

// ---- host ------------------------------------------------------------------------------------
static int layer_check(const solo_layernorm_shape *s)
{
    if (!s || !dtype_ok(s->x_dtype) || !dtype_ok(s->y_dtype) || !dtype_ok(s->weight_dtype) ||
        (s->flags & ~(SOLO_LAYERNORM_RMS | SOLO_LAYERNORM_ACCUMULATE)) || !(s->eps > 0.0f) || !isfinite(s->eps) || s->reserved != 0 ||
        s->x_stride < s->cols || s->y_stride < s->cols || s->grad_stride < s->cols)
        return SOLO_E_INVALID;
    if (s->cols >= (1ull << 24) || s->rows >= (1ull << 31) || s->x_stride >= (1ull << 31) || s->y_stride >= (1ull << 31) || s->grad_stride >= (1ull << 31))
        return SOLO_E_UNSUPPORTED;
    return SOLO_OK;
}

static LayerArgs layer_args(const solo_layernorm_shape *s)
{
    LayerArgs a = {};
    a.rows = s->rows; a.cols = (uint32_t)s->cols; a.x_stride = s->x_stride; a.y_stride = s->y_stride; a.dx_stride = s->grad_stride;
    a.eps = s->eps; a.w_bf16 = s->weight_dtype == SOLO_BF16; a.rms = (s->flags & SOLO_LAYERNORM_RMS) != 0;
    return a;
}

constexpr uint32_t kLongCols = 16384;      // rows of more do not stay in registers

// Threads of a row and elements of a thread.  More threads with fewer elements leave registers for more rows under way, and take more barriers and idle lanes:
// forward and gradient of 8192 x 2048 fp32 (bf16 out) with 256 x 8 17 and 34 us, 256 x 16 20 and 43, 512 x 8 21 and 41; of 16384 x 4096 bf16 with 256 x 16
// 45 and 79, 512 x 8 49 and 80; of 8192 x 8192 bf16 with 1024 x 8 51 and 84, 512 x 16 45 and 90, 256 x 32 46 and 88; of 20000 x 1024 fp32 with
// 64 x 16 21 and 38, 256 x 8 25 and 49; of 100000 x 256 bf16 with 32 x 8 18 and 32, 64 x 8 29 and 57.
struct LayerForm { uint32_t lanes, elements; };
static LayerForm layer_form(uint32_t cols)
{
    if (cols <= 64) return {8, 8};
    if (cols <= 256) return {32, 8};
    if (cols <= 512) return {64, 8};
    if (cols <= 1024) return {64, 16};
    if (cols <= 2048) return {256, 8};
    if (cols <= 4096) return {256, 16};
    if (cols <= 8192) return {1024, 8};
    return {1024, 16};
}
static uint32_t layer_rows_of(uint32_t lanes) { return lanes < 256 ? 256 / lanes : 1; }

// Workgroups of the gradient, each of which leaves sums of its own: never fewer for more rows.  Two of 256 threads a compute unit: more have more rows under
// way, but write more sums (16384 x 4096 bf16: 256 workgroups 108 us, 512 79, 768 83, 1024 93).
static uint32_t layer_parts(uint64_t rows, uint32_t cols)
{
    if (cols > kLongCols) {
        const uint64_t most = cols > (1u << 18) ? 8 : 64;  // (these rows have enough columns for every compute unit)
        return (uint32_t)(rows < most ? rows : most);
    }
    const LayerForm f = layer_form(cols);
    const uint64_t groups = (rows + layer_rows_of(f.lanes) - 1) / layer_rows_of(f.lanes), most = f.lanes <= 256 ? 512 : 256;
    return (uint32_t)(groups < most ? groups : most);
}

// Workgroups of the forward pass: each reads the weights once.  (16384 x 4096 bf16: 1024 workgroups 45 us, 2048 51, one for each row 61; 100000 x 256
// bf16: 1024 18.7, 2048 18.3)
static uint32_t layer_groups(uint64_t rows, uint32_t lanes)
{
    const uint64_t groups = (rows + layer_rows_of(lanes) - 1) / layer_rows_of(lanes), most = lanes < 256 ? 2048 : lanes == 256 ? 1024 : 512;
    return (uint32_t)(groups < most ? groups : most);
}

template <bool XB, bool YB>
static int layer_forward_launch(const LayerArgs &a, hipStream_t stream)
{
    if (a.cols > kLongCols) return launch(layer_forward_long_kernel<XB, YB>, dim3((uint32_t)(a.rows < (1u << 20) ? a.rows : 1u << 20)), 1024, stream, a);
    const LayerForm f = layer_form(a.cols);
    const dim3 grid(layer_groups(a.rows, f.lanes));
    const uint32_t threads = f.lanes < 256 ? 256 : f.lanes;
    if (f.lanes == 8) return launch(layer_forward_kernel<XB, YB, 8, 8>, grid, threads, stream, a);
    if (f.lanes == 32) return launch(layer_forward_kernel<XB, YB, 32, 8>, grid, threads, stream, a);
    if (f.lanes == 64 && f.elements == 8) return launch(layer_forward_kernel<XB, YB, 64, 8>, grid, threads, stream, a);
    if (f.lanes == 64) return launch(layer_forward_kernel<XB, YB, 64, 16>, grid, threads, stream, a);
    if (f.lanes == 256 && f.elements == 8) return launch(layer_forward_kernel<XB, YB, 256, 8>, grid, threads, stream, a);
    if (f.lanes == 256) return launch(layer_forward_kernel<XB, YB, 256, 16>, grid, threads, stream, a);
    if (f.elements == 8) return launch(layer_forward_kernel<XB, YB, 1024, 8>, grid, threads, stream, a);
    return launch(layer_forward_kernel<XB, YB, 1024, 16>, grid, threads, stream, a);
}

template <bool XB, bool YB>
static int layer_backward_launch(const LayerArgs &a, uint32_t parts, hipStream_t stream)
{
    if (a.cols > kLongCols) {
        int rc = SOLO_OK;
        const dim3 rows((uint32_t)(a.rows < (1u << 20) ? a.rows : 1u << 20));
        if (a.part) rc = launch(layer_centre_kernel<XB>, rows, 1024, stream, a);
        if (rc == SOLO_OK && a.part) rc = launch(layer_columns_kernel<XB, YB>, dim3((a.cols + 255) / 256, parts), 256, stream, a);
        if (rc == SOLO_OK && a.dx) rc = launch(layer_backward_long_kernel<XB, YB>, rows, 1024, stream, a);
        return rc;
    }
    const LayerForm f = layer_form(a.cols);
    const dim3 grid(parts);
    const uint32_t threads = f.lanes < 256 ? 256 : f.lanes;
    if (f.lanes == 8) return launch(layer_backward_kernel<XB, YB, 8, 8>, grid, threads, stream, a);
    if (f.lanes == 32) return launch(layer_backward_kernel<XB, YB, 32, 8>, grid, threads, stream, a);
    if (f.lanes == 64 && f.elements == 8) return launch(layer_backward_kernel<XB, YB, 64, 8>, grid, threads, stream, a);
    if (f.lanes == 64) return launch(layer_backward_kernel<XB, YB, 64, 16>, grid, threads, stream, a);
    if (f.lanes == 256 && f.elements == 8) return launch(layer_backward_kernel<XB, YB, 256, 8>, grid, threads, stream, a);
    if (f.lanes == 256) return launch(layer_backward_kernel<XB, YB, 256, 16>, grid, threads, stream, a);
    if (f.elements == 8) return launch(layer_backward_kernel<XB, YB, 1024, 8>, grid, threads, stream, a);
    return launch(layer_backward_kernel<XB, YB, 1024, 16>, grid, threads, stream, a);
}

static bool optional_at(const void *p, uintptr_t size) { return !p || at_multiple(p, size); }

}  // namespace solo

extern "C" {

int solo_layernorm(const void *x, const void *weight, const void *bias, void *y, float *stats, const solo_layernorm_shape *shape, void *stream)
{
    using namespace solo;
    const int rc = layer_check(shape);
    if (rc != SOLO_OK) return rc;
    if (shape->flags & SOLO_LAYERNORM_ACCUMULATE) return SOLO_E_INVALID;
    if (shape->rows == 0 || shape->cols == 0) return SOLO_OK;
    const uintptr_t weights = element_bytes(shape->weight_dtype);
    if (!at_multiple(x, element_bytes(shape->x_dtype)) || !at_multiple(y, element_bytes(shape->y_dtype)) || !optional_at(weight, weights) ||
        !optional_at(bias, weights) || !optional_at(stats, 4))
        return SOLO_E_INVALID;
    LayerArgs a = layer_args(shape);
    a.x = x; a.w = weight; a.b = bias; a.y = y; a.stats = stats;
    const hipStream_t s = (hipStream_t)stream;
    if (shape->x_dtype == SOLO_BF16) return shape->y_dtype == SOLO_BF16 ? layer_forward_launch<true, true>(a, s) : layer_forward_launch<true, false>(a, s);
    return shape->y_dtype == SOLO_BF16 ? layer_forward_launch<false, true>(a, s) : layer_forward_launch<false, false>(a, s);
}

size_t solo_layernorm_workspace_bytes(const solo_layernorm_shape *shape)
{
    using namespace solo;
    if (layer_check(shape) != SOLO_OK) return 0;
    const uint64_t parts = layer_parts(shape->rows, (uint32_t)shape->cols);
    return 16 + parts * shape->cols * 8 + (shape->cols > kLongCols ? shape->rows * 4 : 0);
}

int solo_layernorm_grad(const void *grad_y, const void *x, const void *weight, const float *stats, void *grad_x, void *grad_weight, void *grad_bias,
                        void *workspace, size_t workspace_bytes, const solo_layernorm_shape *shape, void *stream)
{
    using namespace solo;
    const int rc = layer_check(shape);
    if (rc != SOLO_OK) return rc;
    if (shape->cols == 0) return SOLO_OK;
    const uintptr_t weights = element_bytes(shape->weight_dtype);
    const bool sums = grad_weight || grad_bias, accumulate = (shape->flags & SOLO_LAYERNORM_ACCUMULATE) != 0;
    if (!optional_at(weight, weights) || !optional_at(grad_weight, weights) || !optional_at(grad_bias, weights) ||
        !optional_at(grad_x, element_bytes(shape->x_dtype)) || (!grad_x && !sums))
        return SOLO_E_INVALID;
    if (shape->rows != 0 && (!at_multiple(grad_y, element_bytes(shape->y_dtype)) || !at_multiple(x, element_bytes(shape->x_dtype)) || !at_multiple(stats, 4)))
        return SOLO_E_INVALID;
    if (sums && shape->rows != 0 && (!at_multiple(workspace, 16) || workspace_bytes < solo_layernorm_workspace_bytes(shape))) return SOLO_E_INVALID;
    const uint32_t cols = (uint32_t)shape->cols, parts = layer_parts(shape->rows, cols);
    const hipStream_t s = (hipStream_t)stream;
    if (shape->rows != 0) {
        LayerArgs a = layer_args(shape);
        a.x = x; a.w = weight; a.dy = grad_y; a.dx = grad_x; a.stats = const_cast<float *>(stats); a.part = sums ? static_cast<float *>(workspace) : nullptr;
        if (sums) a.centre = a.part + 2 * (uint64_t)parts * cols;      // (of long rows)
        int done;
        if (shape->x_dtype == SOLO_BF16)
            done = shape->y_dtype == SOLO_BF16 ? layer_backward_launch<true, true>(a, parts, s) : layer_backward_launch<true, false>(a, parts, s);
        else
            done = shape->y_dtype == SOLO_BF16 ? layer_backward_launch<false, true>(a, parts, s) : layer_backward_launch<false, false>(a, parts, s);
        if (done != SOLO_OK) return done;
    }
    if (!sums || (parts == 0 && accumulate)) return SOLO_OK;
    LayerSumArgs t = {};
    t.part = static_cast<const float *>(workspace); t.dw = grad_weight; t.db = grad_bias;
    t.cols = cols; t.parts = parts; t.bf16 = shape->weight_dtype == SOLO_BF16; t.accumulate = accumulate;
    return launch(layer_parts_kernel, dim3((cols + 63) / 64, 2), 1024, s, t);
}

}  // extern "C"
