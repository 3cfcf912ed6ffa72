// Embedding lookup with scaling, and the gradient of the table by sorted tokens.
//
//   out[i] = s E[t_i]            dE[v] = s sum_{i: t_i = v} dy[i]          (t_i outside the table: a row of zeros, no gradient)
//
// The gradient never adds atomically: a stable sort of the tokens puts the rows of dy that belong together next to each
// other, in the order of their positions, and the sorted list is cut into pieces of the same length, whatever the tokens
// are.  The sums and their order are therefore the same on every call.
//
// Sorting takes one launch: a workgroup owns a bucket of consecutive table rows, reads all tokens twice (they lie in the
// caches) and needs nothing from the others: the first time it counts the tokens of every row of its bucket, by wavefront, and
// those below the bucket, which is where its part of the sorted list begins; the second time it places them.
#include "solo_ops.h"

#include <math.h>

namespace solo {

constexpr int kSortWaves = 16;
constexpr uint32_t kBuckets = 512;                         // buckets of a table, about (a bucket has 16 rows at least, 512 at most)
constexpr uint32_t kMinBucketBits = 4, kMaxBucketBits = 9;
constexpr int kEmbedThreads = 256;
constexpr int kAheadRows = 8;                              // rows of dy that a team has under way

struct EmbedArgs {
    const void *in;         // table, or gradient of the looked-up rows
    const void *tokens;
    void *out;              // looked-up rows, or gradient of the table
    uint32_t *order;        // positions of the tokens inside the table, sorted by token
    uint32_t *sorted;       // their tokens
    uint32_t *start;        // first place of every row's tokens in both, and their number behind it: [vocab + 1]
    float *partial;         // two rows of sums per piece, see embed_sum_kernel
    uint64_t in_stride, out_stride;
    uint32_t vocab, dim, n;
    float scale;
    uint32_t bucket_bits, piece, team_bits, tiles;
    uint32_t pieces;        // pieces of n sorted tokens
    uint32_t add;           // the gradient is added to what is there
    uint32_t zero_groups;   // workgroups that write the rows without a token
};

template <bool WIDE>
__device__ __forceinline__ uint32_t token_at(const void *tokens, uint64_t i, uint32_t vocab)
{
    if (WIDE) {
        const uint64_t t = static_cast<const uint64_t *>(tokens)[i];
        return t < vocab ? (uint32_t)t : 0xFFFFFFFFu;
    }
    const uint32_t t = static_cast<const uint32_t *>(tokens)[i];
    return t < vocab ? t : 0xFFFFFFFFu;
}

// ---- lookup ----------------------------------------------------------------------------------
// Teams of 2^team_bits lanes take one token each; a lane copies eight elements at a time.
template <bool IN16, bool OUT16, bool WIDE>
__global__ __launch_bounds__(kEmbedThreads) void embed_lookup_kernel(const EmbedArgs a)
{
    const uint32_t team = 1u << a.team_bits, lane = threadIdx.x & (team - 1);
    const uint64_t teams = (uint64_t)gridDim.x * kEmbedThreads >> a.team_bits;
    const uint32_t whole = a.dim / 8 * 8;
    for (uint64_t i = ((uint64_t)blockIdx.x * kEmbedThreads + threadIdx.x) >> a.team_bits; i < a.n; i += teams) {
        const uint32_t t = token_at<WIDE>(a.tokens, i, a.vocab);
        const bool known = t != 0xFFFFFFFFu;
        const char *from = static_cast<const char *>(a.in) + (known ? t : 0) * a.in_stride * Elements<IN16>::kBytes;
        char *to = static_cast<char *>(a.out) + i * a.out_stride * Elements<OUT16>::kBytes;
        for (uint32_t c = lane * 8; c < whole; c += team * 8) {
            float x[8] = {};
            if (known) Elements<IN16>::unpack(Elements<IN16>::load8(from, c), x);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] *= a.scale;
            Elements<OUT16>::store8(to, c, x);
        }
        const uint32_t c = whole + lane;
        if (c < a.dim) Elements<OUT16>::store1(to, c, known ? Elements<IN16>::load1(from, c) * a.scale : 0.0f);
        if (team < 8 && lane == 0)                        // (fewer lanes than a shorter group of eight has elements)
            for (uint32_t e = whole + team; e < a.dim; ++e) Elements<OUT16>::store1(to, e, known ? Elements<IN16>::load1(from, e) * a.scale : 0.0f);
    }
}

// ---- sort ------------------------------------------------------------------------------------
// Lanes of the wavefront whose token lies in the same row of the bucket as this lane's (of those in it).
__device__ __forceinline__ uint64_t same_row(uint32_t row, bool in, uint32_t bits)
{
    uint64_t same = __ballot(in);
    for (uint32_t b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot((row >> b) & 1u);
        same &= (row >> b) & 1u ? ones : ~ones;
    }
    return same;
}

template <bool WIDE>
__global__ __launch_bounds__(kSortWaves * kLanes) void embed_sort_kernel(const EmbedArgs a)
{
    extern __shared__ uint32_t count[];                    // [wavefront][row of the bucket], then one word per wavefront
    const uint32_t rows = 1u << a.bucket_bits;
    uint32_t *const below_of = count + kSortWaves * rows;
    const uint32_t wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const uint32_t first = blockIdx.x << a.bucket_bits;    // the bucket's first row
    const uint32_t share = (a.n + kSortWaves * kLanes - 1) / (kSortWaves * kLanes) * kLanes;        // tokens of a wavefront
    const uint64_t begin = (uint64_t)wave * share, end = min(begin + share, (uint64_t)a.n);
    uint32_t *const mine = count + wave * rows;
    for (uint32_t r = threadIdx.x; r < kSortWaves * rows; r += kSortWaves * kLanes) count[r] = 0;
    __syncthreads();
    uint32_t below = 0;
    for (uint64_t i = begin + lane; i < end; i += 4 * kLanes) {
        uint32_t t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = i + k * kLanes < end ? token_at<WIDE>(a.tokens, i + k * kLanes, a.vocab) : 0xFFFFFFFFu;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            below += t[k] < first;
            if (t[k] != 0xFFFFFFFFu && t[k] - first < rows) atomicAdd(&mine[t[k] - first], 1u);
        }
    }
    below = wave_sum(below);
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    below = 0;
    for (int w = 0; w < kSortWaves; ++w) below += below_of[w];
    // where the tokens of row r that wavefront w has found go: behind the rows before it, and the wavefronts before this one
    __shared__ uint32_t sums[kSortWaves];
    const uint32_t r = threadIdx.x;
    uint32_t total = 0;
    if (r < rows)
        for (int w = 0; w < kSortWaves; ++w) total += count[w * rows + r];
    uint32_t upto = total;
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) {
        const uint32_t left = __shfl_up(upto, d);
        if (lane >= (uint32_t)d) upto += left;
    }
    if (lane == kLanes - 1) sums[wave] = upto;
    __syncthreads();
    uint32_t place = below + upto - total;
    for (uint32_t w = 0; w < wave; ++w) place += sums[w];
    if (r < rows) {
        if (first + r < a.vocab) a.start[first + r] = place;
        if (first + r + 1 == a.vocab) a.start[a.vocab] = place + total;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = count[w * rows + r];
            count[w * rows + r] = place;
            place += c;
        }
    }
    __syncthreads();
    for (uint64_t i0 = begin; i0 < end; i0 += 4 * kLanes) {
        uint32_t t[4];
        const uint64_t i = i0 + lane;
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = i + k * kLanes < end ? token_at<WIDE>(a.tokens, i + k * kLanes, a.vocab) : 0xFFFFFFFFu;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t row = t[k] - first;
            const bool in = t[k] != 0xFFFFFFFFu && row < rows;
            if (!__any(in)) continue;
            const uint64_t same = same_row(row, in, a.bucket_bits);
            const uint32_t before = __popcll(same & ((1ull << lane) - 1));
            if (in) {
                const uint32_t at = mine[row] + before;
                a.order[at] = (uint32_t)(i + k * kLanes);
                a.sorted[at] = t[k];
            }
            __builtin_amdgcn_wave_barrier();
            if (in && before == 0) mine[row] += __popcll(same);
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// ---- sums ------------------------------------------------------------------------------------
// A team of 2^team_bits lanes owns eight columns per lane of one piece: `piece` places of the sorted list.  It adds the rows
// that begin inside the piece, to their ends where they have no more than `piece` tokens.  A longer row ("hot") is added
// piece by piece: the part in the piece where it begins goes to that piece's second row of `partial`, the part in every
// later piece to that one's first, and embed_join_kernel adds these.
template <bool IN16, bool OUT16>
__device__ __forceinline__ void put_row(const EmbedArgs &a, uint32_t row, uint32_t c, const float sum[8])
{
    char *to = static_cast<char *>(a.out) + row * a.out_stride * Elements<OUT16>::kBytes;
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = sum[k] * a.scale;
    if (c + 8 <= a.dim) {
        if (a.add) {
            float old[8];
            Elements<OUT16>::unpack(Elements<OUT16>::load8(to, c), old);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] += old[k];
        }
        Elements<OUT16>::store8(to, c, x);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (c + k < a.dim) Elements<OUT16>::store1(to, c + k, x[k] + (a.add ? Elements<OUT16>::load1(to, c + k) : 0.0f));
}

__device__ __forceinline__ void put_partial(const EmbedArgs &a, uint64_t slot, uint32_t c, const float sum[8])
{
    float *to = a.partial + slot * (((uint64_t)a.dim + 7) / 8 * 8) + c;     // (rows of whole groups of eight)
    Elements<false>::store8(to, 0, sum);
}

template <bool IN16>
__device__ __forceinline__ void row_part(const EmbedArgs &a, uint32_t position, uint32_t c, typename Elements<IN16>::Raw &raw, float tail[8], bool whole)
{
    const char *from = static_cast<const char *>(a.in) + position * a.in_stride * Elements<IN16>::kBytes;
    if (whole) {
        raw = Elements<IN16>::load8(from, c);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) tail[k] = c + k < a.dim ? Elements<IN16>::load1(from, c + k) : 0.0f;
    }
}

template <bool IN16, bool OUT16>
__device__ __forceinline__ void sum_piece(const EmbedArgs &a, uint32_t piece, uint32_t c, uint32_t total)
{
    const uint32_t begin = piece * a.piece, edge = min(begin + a.piece, total);
    if (begin >= edge) return;
    uint32_t lo = begin, hi = edge;
    bool head = false, tail = false;                       // the first row is the rest of a hot one; the last row is the beginning of one
    uint32_t row = a.sorted[begin];
    if (a.start[row] < begin) {
        if (a.start[row + 1] - a.start[row] > a.piece) head = true;
        else lo = a.start[row + 1];
    }
    const uint32_t last = a.sorted[edge - 1];
    if (a.start[last + 1] > edge) {
        if (a.start[last + 1] - a.start[last] > a.piece) tail = a.start[last] >= begin;
        else if (a.start[last] >= begin) hi = a.start[last + 1];
    }
    if (lo >= hi) return;
    row = a.sorted[lo];
    const bool whole = c + 8 <= a.dim;
    float sum[8] = {};
    for (uint32_t s = lo; s < hi; s += kAheadRows) {
        typename Elements<IN16>::Raw raw[kAheadRows];
        uint32_t next[kAheadRows];
        float x[8];
        if (whole) {
#pragma unroll
            for (int k = 0; k < kAheadRows; ++k) {
                const uint32_t at = min(s + k, hi - 1);
                next[k] = a.sorted[at];
                row_part<IN16>(a, a.order[at], c, raw[k], x, true);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kAheadRows; ++k) next[k] = a.sorted[min(s + k, hi - 1)];
        }
#pragma unroll
        for (int k = 0; k < kAheadRows; ++k) {
            if (s + k >= hi) break;
            if (next[k] != row) {
                if (head) put_partial(a, 2ull * piece, c, sum);
                else put_row<IN16, OUT16>(a, row, c, sum);
                head = false;
                row = next[k];
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
            }
            if (whole) Elements<IN16>::unpack(raw[k], x);
            else row_part<IN16>(a, a.order[s + k], c, raw[k], x, false);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[e];
        }
    }
    if (head) put_partial(a, 2ull * piece, c, sum);
    else if (tail) put_partial(a, 2ull * piece + 1, c, sum);
    else put_row<IN16, OUT16>(a, row, c, sum);
}

template <bool OUT16>
__device__ __forceinline__ void zero_rows(const EmbedArgs &a, uint32_t group)
{
    const float none[8] = {};
    for (uint32_t row = group; row < a.vocab; row += a.zero_groups) {
        if (a.n != 0 && a.start[row] != a.start[row + 1]) continue;
        char *to = static_cast<char *>(a.out) + row * a.out_stride * Elements<OUT16>::kBytes;
        uint32_t c = threadIdx.x * 8;
        for (; c + 8 <= a.dim; c += kEmbedThreads * 8) Elements<OUT16>::store8(to, c, none);
        for (; c < a.dim; ++c) Elements<OUT16>::store1(to, c, 0.0f);
    }
}

template <bool IN16, bool OUT16>
__global__ __launch_bounds__(kEmbedThreads) void embed_sum_kernel(const EmbedArgs a)
{
    const uint64_t teams = (uint64_t)(gridDim.x - a.zero_groups) * kEmbedThreads >> a.team_bits;
    if (blockIdx.x >= gridDim.x - a.zero_groups) {
        zero_rows<OUT16>(a, blockIdx.x - (gridDim.x - a.zero_groups));
        return;
    }
    const uint32_t lane = threadIdx.x & ((1u << a.team_bits) - 1), total = a.start[a.vocab];
    for (uint64_t item = ((uint64_t)blockIdx.x * kEmbedThreads + threadIdx.x) >> a.team_bits; item < (uint64_t)a.pieces * a.tiles; item += teams) {
        const uint32_t piece = (uint32_t)(item / a.tiles), c = ((uint32_t)(item % a.tiles) << a.team_bits | lane) * 8;
        if (c < a.dim) sum_piece<IN16, OUT16>(a, piece, c, total);
    }
}

// The rows with more than `piece` tokens: the piece where such a row begins adds its parts.
template <bool IN16, bool OUT16>
__global__ __launch_bounds__(kEmbedThreads) void embed_join_kernel(const EmbedArgs a)
{
    const uint32_t piece = blockIdx.x, total = a.start[a.vocab];
    const uint64_t edge = (uint64_t)(piece + 1) * a.piece;
    if (edge >= total) return;
    const uint32_t row = a.sorted[edge - 1], from = a.start[row], to = a.start[row + 1];
    if (to <= edge || to - from <= a.piece || from < piece * a.piece) return;
    const uint32_t last = (to - 1) / a.piece;
    const uint64_t stride = ((uint64_t)a.dim + 7) / 8 * 8;
    const uint32_t c = (blockIdx.y * kEmbedThreads + threadIdx.x) * 8;
    if (c >= a.dim) return;
    float sum[8];
    Elements<false>::unpack(Elements<false>::load8(a.partial + (2ull * piece + 1) * stride, c), sum);
    for (uint32_t p = piece + 1; p <= last; p += kAheadRows) {
        Elements<false>::Raw raw[kAheadRows];
#pragma unroll
        for (int k = 0; k < kAheadRows; ++k) raw[k] = Elements<false>::load8(a.partial + 2ull * min(p + k, last) * stride, c);
#pragma unroll
        for (int k = 0; k < kAheadRows; ++k) {
            if (p + k > last) break;
            float x[8];
            Elements<false>::unpack(raw[k], x);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[e];
        }
    }
    put_row<IN16, OUT16>(a, row, c, sum);
}

// ---- host ------------------------------------------------------------------------------------
static bool shape_ok(const solo_embedding_shape *s)
{
    return s && dtype_ok(s->table_dtype) && dtype_ok(s->rows_dtype) && (s->token_bits == 32 || s->token_bits == 64) &&
           isfinite(s->scale) && s->reserved == 0 && (s->flags & ~SOLO_EMBEDDING_ACCUMULATE) == 0 && s->table_stride >= s->dim && s->rows_stride >= s->dim;
}

// Offsets of a row are 64 bits wide, counts and places 32.
static bool shape_fits(const solo_embedding_shape *s)
{
    return s->vocab < (1ull << 31) && s->dim < (1ull << 24) && s->tokens < (1ull << 28) && s->table_stride < (1ull << 31) && s->rows_stride < (1ull << 31);
}

static uint32_t bits_for(uint64_t n) { uint32_t b = 0; while ((1ull << b) < n) ++b; return b; }

struct EmbedPlan { uint32_t bucket_bits, buckets, piece, pieces, team_bits, tiles; size_t order, sorted, start, partial, bytes; };

static EmbedPlan embed_plan(const solo_embedding_shape *s)
{
    EmbedPlan p;
    const uint64_t n = s->tokens, groups = (s->dim + 7) / 8;
    p.bucket_bits = bits_for((s->vocab + kBuckets - 1) / kBuckets);
    p.bucket_bits = p.bucket_bits < kMinBucketBits ? kMinBucketBits : p.bucket_bits > kMaxBucketBits ? kMaxBucketBits : p.bucket_bits;
    p.buckets = (uint32_t)((s->vocab + (1u << p.bucket_bits) - 1) >> p.bucket_bits);
    p.team_bits = bits_for(groups);
    if (p.team_bits > 6) p.team_bits = 6;
    p.tiles = (uint32_t)((groups + (1u << p.team_bits) - 1) >> p.team_bits);
    p.piece = 32;
    p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
    size_t at = 0;
    auto take = [&](uint64_t bytes) { const size_t was = at; at += (size_t)((bytes + 255) / 256 * 256); return was; };
    p.order = take(4 * n);
    p.sorted = take(4 * n);
    p.start = take(4 * (s->vocab + 1));
    p.partial = take(n > p.piece ? 2ull * p.pieces * groups * 8 * sizeof(float) : 0);
    p.bytes = at;
    return p;
}

template <bool IN16, bool OUT16>
static void sum_rows(const EmbedArgs &a, const EmbedPlan &p, uint32_t sum_groups, hipStream_t stream)
{
    const uint32_t grid = sum_groups + a.zero_groups;
    if (grid) hipLaunchKernelGGL((embed_sum_kernel<IN16, OUT16>), dim3(grid), dim3(kEmbedThreads), 0, stream, a);
    if (p.pieces > 1)
        hipLaunchKernelGGL((embed_join_kernel<IN16, OUT16>), dim3(p.pieces, (a.dim + kEmbedThreads * 8 - 1) / (kEmbedThreads * 8)),
                           dim3(kEmbedThreads), 0, stream, a);
}

}  // namespace solo

extern "C" {

int solo_embedding(const void *table, const void *tokens, void *rows, const solo_embedding_shape *shape, void *stream)
{
    using namespace solo;
    if (!shape_ok(shape) || shape->flags != 0) return SOLO_E_INVALID;
    if (shape->tokens == 0 || shape->dim == 0) return SOLO_OK;
    if (!at_multiple(rows, element_bytes(shape->rows_dtype)) || !at_multiple(tokens, shape->token_bits / 8) ||
        (shape->vocab != 0 && !at_multiple(table, element_bytes(shape->table_dtype))))
        return SOLO_E_INVALID;
    if (!shape_fits(shape)) return SOLO_E_UNSUPPORTED;
    EmbedArgs a = {};
    a.in = table; a.tokens = tokens; a.out = rows;
    a.in_stride = shape->table_stride; a.out_stride = shape->rows_stride;
    a.vocab = (uint32_t)shape->vocab; a.dim = (uint32_t)shape->dim; a.n = (uint32_t)shape->tokens;
    a.scale = shape->scale;
    a.team_bits = bits_for((shape->dim + 7) / 8);
    if (a.team_bits > 8) a.team_bits = 8;
    uint64_t grid = ((shape->tokens << a.team_bits) + kEmbedThreads - 1) / kEmbedThreads;
    if (grid > (1u << 20)) grid = 1u << 20;
    const bool in16 = shape->table_dtype == SOLO_BF16, out16 = shape->rows_dtype == SOLO_BF16, wide = shape->token_bits == 64;
    void (*kernel)(EmbedArgs) =
        in16 ? (out16 ? (wide ? embed_lookup_kernel<true, true, true> : embed_lookup_kernel<true, true, false>)
                      : (wide ? embed_lookup_kernel<true, false, true> : embed_lookup_kernel<true, false, false>))
             : (out16 ? (wide ? embed_lookup_kernel<false, true, true> : embed_lookup_kernel<false, true, false>)
                      : (wide ? embed_lookup_kernel<false, false, true> : embed_lookup_kernel<false, false, false>));
    hipLaunchKernelGGL(kernel, dim3((uint32_t)grid), dim3(kEmbedThreads), 0, (hipStream_t)stream, a);
    return launched();
}

size_t solo_embedding_workspace_bytes(const solo_embedding_shape *shape)
{
    if (!solo::shape_ok(shape) || !solo::shape_fits(shape)) return 0;
    return solo::embed_plan(shape).bytes;
}

int solo_embedding_grad(const void *grad_rows, const void *tokens, void *grad_table, void *workspace, size_t workspace_bytes,
                        const solo_embedding_shape *shape, void *stream)
{
    using namespace solo;
    if (!shape_ok(shape)) return SOLO_E_INVALID;
    const bool add = (shape->flags & SOLO_EMBEDDING_ACCUMULATE) != 0;
    if (shape->vocab == 0 || shape->dim == 0 || (add && shape->tokens == 0)) return SOLO_OK;
    if (!at_multiple(grad_table, element_bytes(shape->table_dtype)) ||
        (shape->tokens != 0 && (!at_multiple(grad_rows, element_bytes(shape->rows_dtype)) || !at_multiple(tokens, shape->token_bits / 8))) ||
        !at_multiple(workspace, 16))
        return SOLO_E_INVALID;
    if (!shape_fits(shape)) return SOLO_E_UNSUPPORTED;
    const EmbedPlan p = embed_plan(shape);
    if (workspace_bytes < p.bytes) return SOLO_E_INVALID;
    EmbedArgs a = {};
    a.in = grad_rows; a.tokens = tokens; a.out = grad_table;
    char *const ws = static_cast<char *>(workspace);
    a.order = reinterpret_cast<uint32_t *>(ws + p.order); a.sorted = reinterpret_cast<uint32_t *>(ws + p.sorted);
    a.start = reinterpret_cast<uint32_t *>(ws + p.start); a.partial = reinterpret_cast<float *>(ws + p.partial);
    a.in_stride = shape->rows_stride; a.out_stride = shape->table_stride;
    a.vocab = (uint32_t)shape->vocab; a.dim = (uint32_t)shape->dim; a.n = (uint32_t)shape->tokens;
    a.scale = shape->scale;
    a.bucket_bits = p.bucket_bits; a.piece = p.piece; a.pieces = p.pieces; a.team_bits = p.team_bits; a.tiles = p.tiles;
    a.add = add ? 1u : 0u;
    a.zero_groups = add ? 0 : a.vocab < 4096 ? a.vocab : 4096;
    hipStream_t s = (hipStream_t)stream;
    if (a.n != 0) {
        const uint32_t lds = (kSortWaves * (1u << p.bucket_bits) + kSortWaves) * (uint32_t)sizeof(uint32_t);
        if (shape->token_bits == 64) hipLaunchKernelGGL(embed_sort_kernel<true>, dim3(p.buckets), dim3(kSortWaves * kLanes), lds, s, a);
        else hipLaunchKernelGGL(embed_sort_kernel<false>, dim3(p.buckets), dim3(kSortWaves * kLanes), lds, s, a);
    }
    uint64_t items = (uint64_t)p.pieces * p.tiles, groups = ((items << p.team_bits) + kEmbedThreads - 1) / kEmbedThreads;
    if (groups > (1u << 22)) groups = 1u << 22;
    const bool in16 = shape->rows_dtype == SOLO_BF16, out16 = shape->table_dtype == SOLO_BF16;
    if (in16) out16 ? sum_rows<true, true>(a, p, (uint32_t)groups, s) : sum_rows<true, false>(a, p, (uint32_t)groups, s);
    else out16 ? sum_rows<false, true>(a, p, (uint32_t)groups, s) : sum_rows<false, false>(a, p, (uint32_t)groups, s);
    return launched();
}

}  // extern "C"
