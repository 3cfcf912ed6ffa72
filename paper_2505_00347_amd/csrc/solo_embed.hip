// Embedding lookup with scaling, and the gradient of the table by sorted tokens.
//
//   out[i] = s E[t_i]            dE[v] = s sum_{i: t_i = v} dy[i]          (t_i outside the table: a row of zeros, no gradient)
//
// The gradient never adds atomically: a stable sort of the tokens puts the rows of dy that belong together next to each
// other, in the order of their positions, and the sorted list is cut into pieces of the same length, whatever the tokens
// are.  The sums and their order are therefore the same on every call.
//
// Sorting takes one launch: a workgroup owns a bucket of table rows, every 256th one or so (the frequent tokens of a vocabulary
// are neighbours, and half of a text is a few hundred of them), reads all tokens (they lie in the caches) and needs nothing from the
// others.  It counts the tokens of the buckets before its own, which is where its part of the sorted list begins, and its own by row
// and wavefront; then it places them.
//
// Bound by memory.  16384 tokens of a bf16 table of 32000 x 4096: lookup 31 us (178 MB with every row that occurs once), gradient 84 us
// (396 MB; the sort 8.9, the sums and zeros 67, the parts of frequent tokens 8 us); 396 MB take 72 us at the rate of a large copy.
#include "solo_ops.h"

#include <math.h>

namespace solo {

constexpr int kSortWaves = 16;
constexpr uint32_t kListed = 256;                          // tokens of its bucket that a wavefront keeps in LDS
constexpr int kSortDepth = 8;                             // tokens of a lane that are under way, and in registers, together
constexpr uint32_t kMinBuckets = 256;                      // workgroups that sort: one for each compute unit
constexpr uint32_t kMaxRowBits = 9;                        // rows of a bucket: 512 at most (counters by wavefront: 32 KB of LDS)
constexpr int kEmbedThreads = 256;
// Looked-up rows of more bytes than this are written past the caches, and gradients of more are read past them: a quarter of the
// last-level cache.  Lookup of 134 MB of a text's tokens 43 us through the caches, 32 us past them, of evenly drawn tokens 50 and 42 (with
// the product that reads the rows next, 4096 columns, 445 and 451), of 16 MB no difference; gradient of 134 MB 94 and 84 us,
// but of 40 MB, which the backward pass has left in the caches, 38 and 51 us.
constexpr uint64_t kPastBytes = 64ull << 20;
constexpr int kAheadRows = 8;                              // rows of dy that a team has under way

struct EmbedArgs {
    const void *in;         // table, or gradient of the looked-up rows
    const void *tokens;
    void *out;              // looked-up rows, or gradient of the table
    uint32_t *order;        // positions of the tokens inside the table, sorted by token
    uint32_t *sorted;       // their tokens
    uint2 *span;            // where the tokens of every row begin and end in both; behind the last row: the number of all
    float *partial;         // two rows of sums per piece, see embed_sum_kernel
    uint64_t in_stride, out_stride;
    uint32_t vocab, dim, n;
    float scale;
    uint32_t bucket_bits, row_bits, piece, team_bits, tiles;
    uint32_t pieces;        // pieces of n sorted tokens
    uint32_t add;           // the gradient is added to what is there
    uint32_t zero_groups;   // workgroups that write the rows without a token,
    uint32_t zero_rows;     // so many a wavefront, 64 at most
    uint32_t zero_team_bits;
};

// A token as a number of 32 bits; what is negative or does not fit becomes one that no table has (tables have fewer than 2^31 rows).
template <bool WIDE>
__device__ __forceinline__ uint32_t token_at(const void *tokens, uint64_t i)
{
    if (!WIDE) return static_cast<const uint32_t *>(tokens)[i];
    const uint2 t = static_cast<const uint2 *>(tokens)[i];
    return t.y == 0 ? t.x : 0xFFFFFFFFu;
}
template <bool WIDE>
__device__ __forceinline__ uint32_t token_at(const void *tokens, uint64_t i, uint32_t vocab)
{
    const uint32_t t = token_at<WIDE>(tokens, i);
    return t < vocab ? t : 0xFFFFFFFFu;
}

// ---- lookup ----------------------------------------------------------------------------------
// Teams of 2^team_bits lanes take one token each; a lane writes 16 bytes at a time.
template <bool IN16, bool OUT16, bool WIDE, bool PAST>
__global__ __launch_bounds__(kEmbedThreads) void embed_lookup_kernel(const EmbedArgs a)
{
    using Out = Lane16<OUT16>;
    constexpr uint32_t kPer = Out::kPer;
    const uint32_t team = 1u << a.team_bits, lane = threadIdx.x & (team - 1);
    const uint64_t teams = (uint64_t)gridDim.x * kEmbedThreads >> a.team_bits;
    const uint32_t whole = a.dim / kPer * kPer;
    for (uint64_t i = ((uint64_t)blockIdx.x * kEmbedThreads + threadIdx.x) >> a.team_bits; i < a.n; i += teams) {
        const uint32_t t = token_at<WIDE>(a.tokens, i, a.vocab);
        const bool known = t != 0xFFFFFFFFu;
        const char *from = static_cast<const char *>(a.in) + (known ? t : 0) * a.in_stride * Elements<IN16>::kBytes;
        char *to = static_cast<char *>(a.out) + i * a.out_stride * Out::kBytes;
        for (uint32_t c = lane * kPer; c < whole; c += 2 * team * kPer) {      // two loads in front of their stores
            const uint32_t d = c + team * kPer;
            float x[kPer] = {}, y[kPer] = {};
            if (known) {
                load_floats<IN16, (int)kPer>(from, c, x);
                if (d < whole) load_floats<IN16, (int)kPer>(from, d, y);
            }
#pragma unroll
            for (uint32_t k = 0; k < kPer; ++k) {
                x[k] *= a.scale;
                y[k] *= a.scale;
            }
            Out::template store<PAST>(to, c, x);
            if (d < whole) Out::template store<PAST>(to, d, y);
        }
        for (uint32_t c = whole + lane; c < a.dim; c += team)
            Elements<OUT16>::store1(to, c, known ? Elements<IN16>::load1(from, c) * a.scale : 0.0f);
    }
}

// ---- sort ------------------------------------------------------------------------------------
// Lanes of the wavefront, of those with `in`, whose token lies in the same row of the bucket as this lane's.
__device__ __forceinline__ uint64_t same_row(uint32_t row, bool in, uint32_t bits)
{
    uint64_t same = __ballot(in);
    if (same != 0 && !__any(in && row != (uint32_t)__builtin_amdgcn_readlane(row, __builtin_ctzll(same)))) return same;        // (one token all over)
#pragma unroll
    for (uint32_t b = 0; b < kMaxRowBits; ++b) {
        if (b < bits) {
            const uint32_t own = (uint32_t)((int32_t)(row << (31 - b)) >> 31); // all ones where the bit is set
            const uint64_t ones = __ballot(own != 0);
            same &= ~(ones ^ ((uint64_t)own << 32 | own));
        }
    }
    return same;
}

template <bool WIDE>
__global__ __launch_bounds__(kSortWaves * kLanes) void embed_sort_kernel(const EmbedArgs a)
{
    extern __shared__ uint32_t count[];                    // [wavefront][row of the bucket]
    __shared__ uint32_t below_of[kSortWaves], sums[kSortWaves];
    __shared__ uint32_t list[kSortWaves][kListed];         // a wavefront's tokens of the bucket: where they are, from its first on
    __shared__ uint16_t list_row[kSortWaves][kListed];
    const uint32_t wave = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    const uint32_t bucket = blockIdx.x, bits = a.bucket_bits, low = (1u << bits) - 1, rows = 1u << a.row_bits;
    const uint32_t share = (a.n + kSortWaves * kLanes - 1) / (kSortWaves * kLanes) * kLanes;        // tokens of a wavefront
    const uint64_t begin = (uint64_t)wave * share, end = min(begin + share, (uint64_t)a.n);
    uint32_t *const mine = count + wave * rows;
    for (uint32_t r = threadIdx.x; r < kSortWaves * rows; r += kSortWaves * kLanes) count[r] = 0;
    __syncthreads();
    uint32_t below = 0, listed = 0;
    for (uint64_t i0 = begin; i0 < end; i0 += kSortDepth * kLanes) {
        uint32_t t[kSortDepth];
#pragma unroll
        for (int k = 0; k < kSortDepth; ++k) t[k] = token_at<WIDE>(a.tokens, min(i0 + k * kLanes + lane, end - 1));
#pragma unroll
        for (int k = 0; k < kSortDepth; ++k) {
            const uint64_t i = i0 + k * kLanes + lane;
            const bool known = t[k] < a.vocab && i < end;
            below += __popcll(__ballot(known && (t[k] & low) < bucket));
            const bool in = known && (t[k] & low) == bucket;
            const uint64_t all = __ballot(in);
            if (all == 0) continue;
            if (in) {
                const uint32_t row = t[k] >> bits, at = listed + __popcll(all & ((1ull << lane) - 1));
                atomicAdd(&mine[row], 1u);
                if (at < kListed) {
                    list[wave][at] = (uint32_t)(i - begin);
                    list_row[wave][at] = (uint16_t)row;
                }
            }
            listed += __popcll(all);
        }
    }
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    below = 0;
    for (int w = 0; w < kSortWaves; ++w) below += below_of[w];
    // where the tokens of row r that wavefront w has found go: behind the rows before it, and the wavefronts before this one
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
        const uint64_t row = (uint64_t)r << bits | bucket;
        if (row < a.vocab) a.span[row] = make_uint2(place, place + total);
        if (r == rows - 1 && bucket == gridDim.x - 1) a.span[a.vocab] = make_uint2(place + total, 0);
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = count[w * rows + r];
            count[w * rows + r] = place;
            place += c;
        }
    }
    __syncthreads();
    auto put = [&](bool in, uint32_t row, uint32_t position) {
        const uint64_t same = same_row(row, in, a.row_bits);
        const uint32_t before = __popcll(same & ((1ull << lane) - 1));
        if (in) {
            const uint32_t at = mine[row] + before;
            a.order[at] = position;
            a.sorted[at] = row << bits | bucket;
        }
        __builtin_amdgcn_wave_barrier();
        if (in && before == 0) mine[row] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    };
    auto put_listed = [&](uint32_t k, uint32_t n) {        // entries k .. k + 63 of the first n, of a list that begins again behind its end
        const bool in = k + lane < n;
        const uint32_t at = (k + lane) % kListed;
        put(in, in ? list_row[wave][at] : 0, (uint32_t)begin + (in ? list[wave][at] : 0));
    };
    uint32_t done = 0;
    if (listed > kListed) {                                // more than the list holds: from the beginning, 64 at a time
        listed = 0;
        for (uint64_t i0 = begin; i0 < end; i0 += kSortDepth * kLanes) {
            uint32_t t[kSortDepth];
#pragma unroll
            for (int k = 0; k < kSortDepth; ++k) t[k] = token_at<WIDE>(a.tokens, min(i0 + k * kLanes + lane, end - 1));
#pragma unroll
            for (int k = 0; k < kSortDepth; ++k) {
                const uint64_t i = i0 + k * kLanes + lane;
                const bool in = t[k] < a.vocab && (t[k] & low) == bucket && i < end;
                const uint64_t all = __ballot(in);
                if (in) {
                    const uint32_t at = (listed + __popcll(all & ((1ull << lane) - 1))) % kListed;
                    list[wave][at] = (uint32_t)(i - begin);
                    list_row[wave][at] = (uint16_t)(t[k] >> bits);
                }
                listed += __popcll(all);
                __builtin_amdgcn_wave_barrier();
                if (listed - done >= kLanes) {
                    put_listed(done, listed);
                    done += kLanes;
                }
            }
        }
    }
    for (; done < listed; done += kLanes) put_listed(done, listed);
}

// ---- sums ------------------------------------------------------------------------------------
// A team of 2^team_bits lanes owns 16 bytes of columns per lane of one piece: `piece` places of the sorted list.  It adds the rows
// that begin inside the piece, to their ends where they have no more than `piece` tokens.  A longer row ("hot") is added
// piece by piece: the part in the piece where it begins goes to that piece's second row of `partial`, the part in every
// later piece to that one's first, and embed_join_kernel adds these.
// N columns a lane: 16 bytes of a row of the rows' gradient.
template <bool OUT16, int N>
__device__ __forceinline__ void put_row(const EmbedArgs &a, uint32_t row, uint32_t c, const float sum[N])
{
    char *to = static_cast<char *>(a.out) + (uint64_t)row * a.out_stride * Elements<OUT16>::kBytes;
    float x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = sum[k] * a.scale;
    if (c + N <= a.dim) {
        if (a.add) {
            float old[N];
            load_floats<OUT16, N>(to, c, old);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] += old[k];
        }
        store_floats<OUT16, N>(to, c, x);
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (c + k < a.dim) Elements<OUT16>::store1(to, c + k, x[k] + (a.add ? Elements<OUT16>::load1(to, c + k) : 0.0f));
}

// Columns c .. c + N - 1 of a row, of the sums of columns from .. from + N - 1 (from < c only in the shorter last group).
template <bool OUT16, int N>
__device__ __forceinline__ void put_columns(const EmbedArgs &a, uint32_t row, uint32_t c, uint32_t from, const float sum[N])
{
    if (from == c) {
        put_row<OUT16, N>(a, row, c, sum);
        return;
    }
    char *to = static_cast<char *>(a.out) + row * a.out_stride * Elements<OUT16>::kBytes;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (from + k >= c) Elements<OUT16>::store1(to, from + k, sum[k] * a.scale + (a.add ? Elements<OUT16>::load1(to, from + k) : 0.0f));
}

// Where a piece's part of a hot row lies, columns c on: first or second row of the piece.  The parts of neighbouring pieces are
// neighbours, for the columns of a team: join reads them one behind the other.
template <int N>
__device__ __forceinline__ float *partial_at(const EmbedArgs &a, uint32_t piece, bool second, uint32_t c)
{
    const uint32_t width = (uint32_t)N << a.team_bits, tile = c / width;
    return a.partial + (((uint64_t)tile * 2 + second) * a.pieces + piece) * width + c % width;
}

template <int N>
__device__ __forceinline__ void put_partial(const EmbedArgs &a, uint32_t piece, bool second, uint32_t c, const float sum[N])
{
    store_floats<false, N>(partial_at<N>(a, piece, second, c), 0, sum);
}

// The lane with the shorter last group of a row takes the last N columns instead, where there are that many.
template <int N>
__device__ __forceinline__ uint32_t first_column(const EmbedArgs &a, uint32_t c) { return a.dim >= N ? min(c, a.dim - N) : 0; }

template <bool IN16, bool PAST = false>
__device__ __forceinline__ Quad load_columns(const EmbedArgs &a, uint32_t position, uint32_t from)
{
    using Lane = Lane16<IN16>;
    const char *at = static_cast<const char *>(a.in) + ((uint64_t)position * a.in_stride + from) * Lane::kBytes;
    if (a.dim >= (uint32_t)Lane::kPer) return Lane::template load<PAST>(at, 0);
    float x[Lane::kPer];
#pragma unroll
    for (int k = 0; k < Lane::kPer; ++k) x[k] = k < (int)a.dim ? Elements<IN16>::load1(at, k) : 0.0f;
    Quad q;
    Lane::template store<false>(&q, 0, x);
    return q;
}

template <bool IN16, bool OUT16>
__device__ __forceinline__ void sum_piece(const EmbedArgs &a, uint32_t piece, uint32_t c, uint32_t total)
{
    const uint32_t begin = piece * a.piece, edge = min(begin + a.piece, total);
    if (begin >= edge) return;
    constexpr int N = Lane16<IN16>::kPer;
    uint32_t lo = begin, hi = edge;
    bool head = false, tail = false;                       // the first row is the rest of a hot one; the last row is the beginning of one
    uint32_t row = a.sorted[begin];
    const uint32_t last = a.sorted[edge - 1];
    const uint2 first_span = a.span[row], last_span = a.span[last];
    if (first_span.x < begin) {
        if (first_span.y - first_span.x > a.piece) head = true;
        else lo = first_span.y;
    }
    if (last_span.y > edge && last_span.x >= begin) {
        if (last_span.y - last_span.x > a.piece) tail = true;
        else hi = last_span.y;
    }
    if (lo >= hi) return;
    const uint32_t from = first_column<N>(a, c);
    float sum[N] = {};
    auto put = [&](bool to_head, bool to_tail) {
        if (to_head || to_tail) put_partial<N>(a, piece, to_tail, c, sum);
        else put_columns<OUT16, N>(a, row, c, from, sum);
    };
    row = a.sorted[lo];
    for (uint32_t s = lo; s < hi; s += kAheadRows) {
        Quad raw[kAheadRows];
        uint32_t next[kAheadRows];
#pragma unroll
        for (int k = 0; k < kAheadRows; ++k) {
            const uint32_t at = min(s + k, hi - 1);
            next[k] = a.sorted[at];
            raw[k] = load_columns<IN16>(a, a.order[at], from);
        }
#pragma unroll
        for (int k = 0; k < kAheadRows; ++k) {
            if (s + k >= hi) break;
            if (next[k] != row) {
                put(head, false);
                head = false;
                row = next[k];
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] = 0.0f;
            }
            float x[N];
            Lane16<IN16>::unpack(raw[k], x);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += x[e];
        }
    }
    put(head, tail);
}

// The same by a whole wavefront, for rows of more than 256 columns (fp32: 128): the places of the list are a lane each, so that rows and
// positions are scalars, and a batch of rows is under way while the one before is added and written.  (A wait for loads also waits
// for the stores in front of them: stores of a batch come behind the loads of the next.)
template <bool IN16, bool OUT16, bool PAST>
__device__ __forceinline__ void sum_piece_wave(const EmbedArgs &a, uint32_t piece, uint32_t c)
{
    constexpr int N = Lane16<IN16>::kPer, kBatch = 8;
    const uint32_t begin = piece * a.piece, lane = threadIdx.x % kLanes, total = a.span[a.vocab].x;
    const uint32_t at = min(begin + lane, a.n - 1);
    const uint32_t token = a.sorted[at], position = a.order[at];               // (behind `total`: not set, and not used)
    const uint32_t edge = min(begin + a.piece, total);
    if (begin >= edge) return;
    const uint32_t first = __builtin_amdgcn_readfirstlane(token), last = __builtin_amdgcn_readlane(token, edge - 1 - begin);
    const uint2 first_span = a.span[first], last_span = a.span[last];
    const uint32_t first_start = first_span.x, first_end = first_span.y, last_start = last_span.x, last_end = last_span.y;
    const bool head = first_start < begin && first_end - first_start > a.piece;
    const bool tail = last_end > edge && last_end - last_start > a.piece && last_start >= begin;
    const uint32_t lo = first_start < begin && !head ? first_end : begin;
    const uint32_t hi = last_end > edge && last_end - last_start <= a.piece && last_start >= begin ? last_end : edge;
    if (lo >= hi) return;
    const uint32_t from = first_column<N>(a, c);
    const bool writes = c < a.dim;                          // (the last team's lanes behind the row take part, and write nothing)
    const char *const in = static_cast<const char *>(a.in) + (uint64_t)from * Elements<IN16>::kBytes;
    const uint32_t k0 = lo - begin, k1 = hi - begin;        // at most 64 places: `piece`, and one less of the last row
    float sum[N] = {};
    uint32_t row = __builtin_amdgcn_readlane(token, k0);
    bool in_head = head;
    Quad raw[2][kBatch];
    auto load = [&](Quad *r, uint32_t k) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint64_t at_row = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(position, min(k + j, k1 - 1)) * a.in_stride;
            const char *const at = in + at_row * Elements<IN16>::kBytes;
            r[j] = Lane16<IN16>::template load<PAST>(at, 0);
        }
    };
    auto put = [&](uint32_t row, bool head, bool tail) {
        if (!writes) return;
        if (head || tail) put_partial<N>(a, piece, tail && !head, c, sum);
        else put_columns<OUT16, N>(a, row, c, from, sum);
    };
    auto add = [&](const Quad *r, uint32_t k) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (k + j >= k1) break;
            const uint32_t next = __builtin_amdgcn_readlane(token, k + j);
            if (next != row) {
                put(row, in_head, false);
                in_head = false;
                row = next;
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] = 0.0f;
            }
            float x[N];
            Lane16<IN16>::unpack(r[j], x);
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += x[e];
        }
    };
    load(raw[0], k0);
    for (uint32_t k = k0; k < k1; k += 2 * kBatch) {
        if (k + kBatch < k1) load(raw[1], k + kBatch);
        add(raw[0], k);
        if (k + kBatch >= k1) break;
        if (k + 2 * kBatch < k1) load(raw[0], k + 2 * kBatch);
        add(raw[1], k + kBatch);
    }
    put(row, in_head, tail && !in_head);
}

// Rows without a token, past the caches: a wavefront looks at up to 64 rows, a lane each, and its teams write those that are empty,
// 16 bytes a lane.  (Gradient of 96 tokens, 154 MB of zeros in rows of 3 KB: 62 us through the caches, 41 us past them, by the sort.)
__device__ __forceinline__ void zero_row(char *to, uint32_t bytes, uint32_t lane, uint32_t lanes)
{
    const Quad none = {};
    uint32_t i = lane * 16;
    for (; i + 16 <= bytes; i += lanes * 16) __builtin_nontemporal_store(none, reinterpret_cast<Quad *>(to + i));
    for (; i < bytes; i += 2) *reinterpret_cast<uint16_t *>(to + i) = 0;       // (one lane's: what is left is less than 16 bytes)
}

// A launch has fewer than 2^32 threads, 2^30 at most for the sums: tables of more than 2^25 rows of 2 KB and more have more rows a wavefront.
// (2^30 rows, 64 for each wavefront, are 2^24 wavefronts.)
constexpr uint32_t kZeroWaves = 1u << 25;

// `empty`: bit r is set where row first + r has no token.
template <bool OUT16>
__device__ __forceinline__ void zero_rows(const EmbedArgs &a, uint32_t first, uint64_t empty)
{
    const uint32_t lanes = 1u << a.zero_team_bits, lane = threadIdx.x & (lanes - 1), team = threadIdx.x % kLanes >> a.zero_team_bits;
    for (uint32_t r = team; r < a.zero_rows; r += kLanes >> a.zero_team_bits)
        if (empty >> r & 1)
            zero_row(static_cast<char *>(a.out) + (uint64_t)(first + r) * a.out_stride * Elements<OUT16>::kBytes, a.dim * Elements<OUT16>::kBytes, lane, lanes);
}

template <bool IN16, bool OUT16, bool WAVE, bool PAST>
__global__ __launch_bounds__(kEmbedThreads) void embed_sum_kernel(const EmbedArgs a)
{
    const uint32_t lane = threadIdx.x % kLanes;
    if (blockIdx.x >= gridDim.x - a.zero_groups) {
        const uint64_t wave = ((uint64_t)(blockIdx.x - (gridDim.x - a.zero_groups)) * kEmbedThreads + threadIdx.x) / kLanes;
        const uint64_t first = wave * a.zero_rows, mine = first + lane;
        const bool empty = lane < a.zero_rows && mine < a.vocab && (a.n == 0 || a.span[mine].x == a.span[mine].y);
        zero_rows<OUT16>(a, (uint32_t)first, __ballot(empty));
        return;
    }
    const uint64_t items = (uint64_t)a.pieces * a.tiles, teams = (uint64_t)(gridDim.x - a.zero_groups) * kEmbedThreads >> a.team_bits;
    const uint64_t team = ((uint64_t)blockIdx.x * kEmbedThreads + threadIdx.x) >> a.team_bits;
    if (WAVE) {
        for (uint64_t item = __builtin_amdgcn_readfirstlane((uint32_t)team); item < items; item += teams) {
            const uint32_t piece = (uint32_t)(item / a.tiles), c = ((uint32_t)(item % a.tiles) << 6 | lane) * Lane16<IN16>::kPer;
            sum_piece_wave<IN16, OUT16, PAST>(a, piece, c);
        }
        return;
    }
    const uint32_t total = a.span[a.vocab].x, c = (threadIdx.x & ((1u << a.team_bits) - 1)) * Lane16<IN16>::kPer;        // (one tile)
    for (uint64_t item = team; item < items; item += teams)
        if (c < a.dim) sum_piece<IN16, OUT16>(a, (uint32_t)item, c, total);
}

// ---- few tokens ------------------------------------------------------------------------------
// One launch without a sort: every workgroup holds all tokens in LDS.  The wavefront of a token's first position adds the rows of
// all its positions; the zeros go to the rows that no token names.  96 tokens of a table of 50257 x 768: 27 us instead of
// 41 with the sort.  The line is where one wavefront's run over all tokens, if they are the same, takes as long as the launches saved.
constexpr uint32_t kFewTokens = 256;

template <bool IN16, bool OUT16, bool WIDE>
__global__ __launch_bounds__(kEmbedThreads) void embed_few_kernel(const EmbedArgs a)
{
    __shared__ uint32_t tokens[kFewTokens];
    __shared__ uint32_t named[kEmbedThreads / kLanes][2];
    constexpr int N = Lane16<IN16>::kPer;
    const uint32_t lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
    tokens[threadIdx.x] = threadIdx.x < a.n ? token_at<WIDE>(a.tokens, threadIdx.x, a.vocab) : 0xFFFFFFFFu;
    if (lane < 2) named[wave][lane] = 0;
    __syncthreads();
    if (blockIdx.x >= gridDim.x - a.zero_groups) {
        const uint64_t first = ((uint64_t)(blockIdx.x - (gridDim.x - a.zero_groups)) * (kEmbedThreads / kLanes) + wave) * a.zero_rows;
#pragma unroll
        for (uint32_t k = 0; k < kFewTokens; k += kLanes) {
            const uint32_t r = tokens[k + lane] - (uint32_t)first;             // (no token: larger than any row number)
            if (tokens[k + lane] >= first && r < a.zero_rows) atomicOr(&named[wave][r / 32], 1u << r % 32);
        }
        __builtin_amdgcn_wave_barrier();
        const uint64_t mask = (uint64_t)*(volatile uint32_t *)&named[wave][1] << 32 | *(volatile uint32_t *)&named[wave][0];
        zero_rows<OUT16>(a, (uint32_t)first, __ballot(lane < a.zero_rows && first + lane < a.vocab) & ~mask);
        return;
    }
    const uint32_t item = __builtin_amdgcn_readfirstlane(blockIdx.x * (kEmbedThreads / kLanes) + wave), i = item / a.tiles;
    if (i >= a.n) return;
    const uint32_t row = __builtin_amdgcn_readfirstlane(tokens[i]), c = (item % a.tiles * kLanes + lane) * N;
    if (row == 0xFFFFFFFFu) return;
    uint64_t same[kFewTokens / kLanes];
#pragma unroll
    for (uint32_t k = 0; k < kFewTokens / kLanes; ++k) same[k] = __ballot(tokens[k * kLanes + lane] == row);
#pragma unroll
    for (uint32_t k = 0; k < kFewTokens / kLanes; ++k) {                       // an earlier position has it all
        const uint64_t before = k < i / kLanes ? ~0ull : k == i / kLanes ? (1ull << i % kLanes) - 1 : 0;
        if (same[k] & before) return;
    }
    const uint32_t from = first_column<N>(a, c);
    float sum[N] = {};
#pragma unroll
    for (uint32_t k = 0; k < kFewTokens / kLanes; ++k) {
        uint64_t left = same[k];
        while (left) {
            constexpr int kBatch = 4;
            Quad raw[kBatch];
            int count = 0;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (left == 0) break;
                const uint32_t position = k * kLanes + __builtin_ctzll(left);
                left &= left - 1;
                raw[j] = load_columns<IN16>(a, position, from);
                count = j + 1;
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                if (j >= count) break;
                float x[N];
                Lane16<IN16>::unpack(raw[j], x);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += x[e];
            }
        }
    }
    if (c < a.dim) put_columns<OUT16, N>(a, row, c, from, sum);
}

// The rows with more than `piece` tokens: the piece where such a row begins adds its parts, each wavefront of the workgroup a
// run of them.
constexpr int kJoinWaves = 8;
constexpr uint32_t kJoinPieces = 4;                        // pieces of a workgroup
template <bool IN16, bool OUT16>
__global__ __launch_bounds__(kJoinWaves * kLanes) void embed_join_kernel(const EmbedArgs a)
{
    constexpr int N = Lane16<IN16>::kPer;
    __shared__ float lds[kJoinWaves][N][kLanes];
    const uint32_t lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes, total = a.span[a.vocab].x;
    for (uint32_t group = blockIdx.x; group < (a.pieces + kJoinPieces - 1) / kJoinPieces; group += gridDim.x) {
        // a lane looks at a piece
        const uint64_t at = (uint64_t)group * kJoinPieces + lane, at_edge = (at + 1) * a.piece;
        uint32_t its_row = 0, its_start = 0, its_end = 0;
        bool begins = lane < kJoinPieces && at_edge < total;
        if (begins) {
            its_row = a.sorted[at_edge - 1];
            const uint2 span = a.span[its_row];
            its_start = span.x;
            its_end = span.y;
            begins = its_end > at_edge && its_end - its_start > a.piece && its_start >= at * a.piece;
        }
        for (uint64_t left = __ballot(begins); left != 0; left &= left - 1) {
            const uint32_t which = __builtin_ctzll(left), piece = group * kJoinPieces + which;
            const uint32_t row = __builtin_amdgcn_readlane(its_row, which), to = __builtin_amdgcn_readlane(its_end, which);
            const uint32_t parts = (to - 1) / a.piece - piece + 1;                 // the first is the second row of its piece
            const uint32_t run = (parts + kJoinWaves - 1) / kJoinWaves, begin = wave * run, end = min(begin + run, parts);
            for (uint32_t c0 = blockIdx.y * kLanes * N; c0 < a.dim; c0 += gridDim.y * kLanes * N) {
                const uint32_t c = min(c0 + lane * N, (a.dim - 1) / N * N), from = first_column<N>(a, c);
                float sum[N] = {};
                for (uint32_t p = begin; p < end; p += kAheadRows) {
                    float raw[kAheadRows][N];
#pragma unroll
                    for (int k = 0; k < kAheadRows; ++k) {
                        const uint32_t part = min(p + k, end - 1);
                        load_floats<false, N>(partial_at<N>(a, piece + part, part == 0, c), 0, raw[k]);
                    }
#pragma unroll
                    for (int k = 0; k < kAheadRows; ++k) {
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[e] += p + k < end ? raw[k][e] : 0.0f;       // (no branch: behind one a load would be moved)
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) lds[wave][e][lane] = sum[e];
                __syncthreads();
                if (wave == 0) {
                    const uint32_t waves = (parts + run - 1) / run;
                    for (uint32_t w = 1; w < waves; ++w)
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[e] += lds[w][e][lane];
                    if (c0 + lane * N < a.dim) put_columns<OUT16, N>(a, row, c, from, sum);
                }
                __syncthreads();
            }
        }
    }
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
    return s->vocab < (1ull << 30) && s->dim < (1ull << 24) && s->tokens < (1ull << 28) && s->table_stride < (1ull << 31) && s->rows_stride < (1ull << 31);
}

static uint32_t bits_for(uint64_t n) { uint32_t b = 0; while ((1ull << b) < n) ++b; return b; }

struct EmbedPlan { uint32_t bucket_bits, row_bits, piece, pieces, team_bits, tiles; size_t order, sorted, span, partial, bytes; };

static EmbedPlan embed_plan(const solo_embedding_shape *s)
{
    EmbedPlan p;
    const uint64_t n = s->tokens, per = s->rows_dtype == SOLO_BF16 ? 8 : 4, groups = (s->dim + per - 1) / per;      // (columns of a lane)
    const uint64_t rows = s->vocab ? s->vocab : 1;
    p.bucket_bits = bits_for(kMinBuckets);
    while (((rows - 1) >> p.bucket_bits) >> kMaxRowBits) ++p.bucket_bits;
    p.row_bits = bits_for(((rows - 1) >> p.bucket_bits) + 1);
    p.team_bits = bits_for(groups);
    if (p.team_bits > 6) p.team_bits = 6;
    p.tiles = (uint32_t)((groups + (1u << p.team_bits) - 1) >> p.team_bits);
    // (wide rows: pieces of 16 write twice as many parts of frequent tokens, bf16 16384 x 4096 takes 90 us with 16 and 84 us with 32, and
    // pieces of 64 are too few wavefronts; narrow ones have few lanes a piece: 40000 tokens of a bf16 table of 5000 x 100 take 54 us
    // with 32, 41 us with 16 and 37 us with 8)
    p.piece = p.team_bits == 6 ? 32 : 8;
    p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
    size_t at = 0;
    auto take = [&](uint64_t bytes) { const size_t was = at; at += (size_t)((bytes + 255) / 256 * 256); return was; };
    p.order = take(4 * n);
    p.sorted = take(4 * n);
    p.span = take(8 * (s->vocab + 1));
    p.partial = take(n > p.piece ? 2ull * p.pieces * p.tiles * (per << p.team_bits) * sizeof(float) : 0);
    p.bytes = at;
    return p;
}

static bool past_caches(const solo_embedding_shape *s) { return s->tokens * s->dim * element_bytes(s->rows_dtype) > kPastBytes; }

template <bool IN16, bool OUT16>
static int lookup(const EmbedArgs &a, bool wide, bool past, uint64_t grid, void *stream)
{
    void (*kernel)(EmbedArgs) = wide ? (past ? embed_lookup_kernel<IN16, OUT16, true, true> : embed_lookup_kernel<IN16, OUT16, true, false>)
                                     : (past ? embed_lookup_kernel<IN16, OUT16, false, true> : embed_lookup_kernel<IN16, OUT16, false, false>);
    return launch(kernel, dim3((uint32_t)grid), kEmbedThreads, (hipStream_t)stream, a);
}

template <bool IN16, bool OUT16>
static int few_tokens(const EmbedArgs &a, bool wide, hipStream_t stream)
{
    const uint32_t waves = kEmbedThreads / kLanes, grid = (a.n * a.tiles + waves - 1) / waves + a.zero_groups;
    return launch(wide ? embed_few_kernel<IN16, OUT16, true> : embed_few_kernel<IN16, OUT16, false>, dim3(grid), kEmbedThreads, stream, a);
}

template <bool IN16, bool OUT16>
static int sum_rows(const EmbedArgs &a, const EmbedPlan &p, uint32_t sum_groups, bool past, hipStream_t stream)
{
    const uint32_t grid = sum_groups + a.zero_groups;
    void (*const sum)(EmbedArgs) = p.team_bits < 6 ? embed_sum_kernel<IN16, OUT16, false, false>
                                   : past          ? embed_sum_kernel<IN16, OUT16, true, true>
                                                   : embed_sum_kernel<IN16, OUT16, true, false>;
    const int rc = grid ? launch(sum, dim3(grid), kEmbedThreads, stream, a) : SOLO_OK;
    if (rc != SOLO_OK || p.pieces <= 1) return rc;
    constexpr uint32_t kColumns = kLanes * Lane16<IN16>::kPer;
    const uint32_t tiles = (a.dim + kColumns - 1) / kColumns, join_groups = (p.pieces + kJoinPieces - 1) / kJoinPieces;
    return launch(embed_join_kernel<IN16, OUT16>, dim3(join_groups < (1u << 22) ? join_groups : 1u << 22, tiles < 16 ? tiles : 16), kJoinWaves * kLanes, stream, a);
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
    const bool in16 = shape->table_dtype == SOLO_BF16, out16 = shape->rows_dtype == SOLO_BF16, wide = shape->token_bits == 64;
    a.team_bits = bits_for(out16 ? (shape->dim + 7) / 8 : (shape->dim + 3) / 4);
    if (a.team_bits > 8) a.team_bits = 8;
    uint64_t grid = ((shape->tokens << a.team_bits) + kEmbedThreads - 1) / kEmbedThreads;
    if (grid > (1u << 20)) grid = 1u << 20;
    const bool past = past_caches(shape);
    if (in16) return out16 ? lookup<true, true>(a, wide, past, grid, stream) : lookup<true, false>(a, wide, past, grid, stream);
    return out16 ? lookup<false, true>(a, wide, past, grid, stream) : lookup<false, false>(a, wide, past, grid, stream);
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
    a.span = reinterpret_cast<uint2 *>(ws + p.span); a.partial = reinterpret_cast<float *>(ws + p.partial);
    a.in_stride = shape->rows_stride; a.out_stride = shape->table_stride;
    a.vocab = (uint32_t)shape->vocab; a.dim = (uint32_t)shape->dim; a.n = (uint32_t)shape->tokens;
    a.scale = shape->scale;
    a.bucket_bits = p.bucket_bits; a.row_bits = p.row_bits;
    a.piece = p.piece; a.pieces = p.pieces; a.team_bits = p.team_bits; a.tiles = p.tiles;
    a.add = add ? 1u : 0u;
    if (!add) {
        const uint32_t row_bytes = a.dim * (uint32_t)element_bytes(shape->table_dtype);
        a.zero_team_bits = bits_for((row_bytes + 15) / 16);
        if (a.zero_team_bits > 6) a.zero_team_bits = 6;
        a.zero_rows = row_bytes >= 4096 ? 1 : 4096 / row_bytes < kLanes ? 4096 / row_bytes : kLanes;
        while ((a.vocab + a.zero_rows - 1) / a.zero_rows > kZeroWaves) a.zero_rows *= 2;
        const uint32_t waves = (a.vocab + a.zero_rows - 1) / a.zero_rows;
        a.zero_groups = (waves + kEmbedThreads / kLanes - 1) / (kEmbedThreads / kLanes);
    }
    hipStream_t s = (hipStream_t)stream;
    const bool in16 = shape->rows_dtype == SOLO_BF16, out16 = shape->table_dtype == SOLO_BF16, wide = shape->token_bits == 64;
    if (a.n != 0 && a.n <= kFewTokens) {
        const uint32_t columns = kLanes * (in16 ? 8 : 4);
        a.tiles = (a.dim + columns - 1) / columns;
        if (in16) return out16 ? few_tokens<true, true>(a, wide, s) : few_tokens<true, false>(a, wide, s);
        return out16 ? few_tokens<false, true>(a, wide, s) : few_tokens<false, false>(a, wide, s);
    }
    if (a.n != 0) {
        const uint32_t lds = kSortWaves * (1u << p.row_bits) * (uint32_t)sizeof(uint32_t);
        const int rc = launch(wide ? embed_sort_kernel<true> : embed_sort_kernel<false>, dim3(1u << p.bucket_bits), kSortWaves * kLanes, s, a, lds);
        if (rc != SOLO_OK) return rc;                      // (what follows reads what the sort writes)
    }
    uint64_t items = (uint64_t)p.pieces * p.tiles, groups = ((items << p.team_bits) + kEmbedThreads - 1) / kEmbedThreads;
    if (groups > (1u << 22)) groups = 1u << 22;
    const bool past = past_caches(shape);
    if (in16) return out16 ? sum_rows<true, true>(a, p, (uint32_t)groups, past, s) : sum_rows<true, false>(a, p, (uint32_t)groups, past, s);
    return out16 ? sum_rows<false, true>(a, p, (uint32_t)groups, past, s) : sum_rows<false, false>(a, p, (uint32_t)groups, past, s);
}

}  // extern "C"
