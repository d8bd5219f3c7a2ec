// C-ABI entry points cx_embed_lookup*, cx_embed_grad*, cx_embed_workspace: embedding tables that lie in the workers'
// flat rows, and their gradient by sorted tokens (see include/cx_lm.h).
//
//   out[w][n] = round(scale * table_w[token[w][n]])               g[w][v] = round(g_in[w][v] + scale * sum_{n: token = v} dout[w][n])
//
// Both are bound by memory: 16 workers' 4,096 tokens of 768 float32 columns take 49 to 51 us (5.7 to 6.0 TB/s), the gradient of as many in bfloat16 into
// tables of 32,768 rows 166 to 190 us for the sums and the filling, by where the buffers lie (medians of 169 and 178, 5.4 and 5.1 TB/s), 14 for
// the sort before and 8 for the joining behind.  A group of lanes
// (a power of two, as many as one row's 16-byte vectors, 64 at most) handles one vector column each of one row, so a short row does not leave a wavefront's lanes idle.
//
// The gradient adds in a fixed order, which atomics would not, and writes each row of the table once (where nearly all are zeros, the others twice).
// Three launches:
//   sort_kernel   a stable counting sort of each worker's tokens.  A workgroup owns 1,024 ids and reads all N tokens
//                 itself instead of exchanging counts with the others: no passes, no atomics on memory, and where the
//                 table has 32,768 rows 32 workgroups a worker read 32 x 16 KB of tokens from the cache.
//   grad_kernel   the sorted list in pieces of equal length, one to a group of lanes, so that a frequent token keeps no group longer than
//                 a rare one: it adds up the rows of dout that its piece names, list by list, and writes what lists lie inside the
//                 piece; what reaches beyond goes to the workspace.  Other workgroups of the same launch write the rows that no
//                 token names, unless workgroups beside the sort have filled all rows.
//   join_kernel   adds up the lists that reach over several pieces, in order; the sort has noted where these begin.
#include "lm_common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kBins = 1024;                 // ids of a workgroup of the sort
constexpr int kSortWaves = 16, kSortThreads = kSortWaves * kWave;
static_assert(kBins == kSortThreads, "a thread for every id");
constexpr int kHeld = 4;                    // tokens a lane of the sort loads at once; the first ones stay for the second walk
constexpr int kFewPieces = 8;               // a list of no more is joined by one group of lanes
constexpr int64_t kMaxTokens = CX_MAX_TOKENS;
constexpr int32_t kMaxVocab = CX_MAX_VOCAB, kMaxWidth = CX_MAX_WIDTH;

// Elements [0, n) of a vector.
template <class E>
__device__ __forceinline__ u4 load_part(const typename E::T *p, int n)
{
    u4 w{};
#pragma unroll
    for (int j = 0; j < E::kPer16; ++j)
        if (j < n) {
            if constexpr (E::kPer16 == 4) w[j] = __float_as_uint(p[j]);
            else w[j / 2] |= static_cast<unsigned>(p[j]) << (16 * (j & 1));
        }
    return w;
}

template <class E>
struct Columns {                            // the columns of a row that a lane handles
    int64_t first;
    int n;                                  // of kPer16; 0 beyond the row
    int back;                               // the row's last columns are read as a whole vector that begins so many columns earlier
    bool narrow;                            // unless the row is shorter than a vector
    // Reads a row's columns; place() before their use moves those of a row's end where they belong, so that no read waits for another: read
    // one by one, 3 workers' 2,438 tokens of 503 binary16 columns were added up in 23 us instead of 13.
    __device__ __forceinline__ u4 raw(const typename E::T *row) const
    {
        return narrow ? load_part<E>(row + first, n) : load16<E>(row + (first - back));
    }
    __device__ __forceinline__ void place(u4 &w) const
    {
        if (back == 0) return;
        uint64_t lo = static_cast<uint64_t>(w[1]) << 32 | w[0], hi = static_cast<uint64_t>(w[3]) << 32 | w[2];
        int bits = back * 8 * static_cast<int>(sizeof(typename E::T));
        if (bits >= 64) { lo = hi; hi = 0; bits -= 64; }
        lo = lo >> bits | hi << 1 << (63 - bits);
        hi >>= bits;
        w = u4{static_cast<unsigned>(lo), static_cast<unsigned>(lo >> 32), static_cast<unsigned>(hi), static_cast<unsigned>(hi >> 32)};
    }
    template <bool THROUGH = false>
    __device__ __forceinline__ void store(typename E::T *row, const float (&v)[E::kPer16]) const
    {
        if (n == E::kPer16) {
            if (THROUGH) store16_through<E>(row + first, E::pack(v)); else store16<E>(row + first, E::pack(v));
        } else {
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j)
                if (j < n) row[first + j] = E::narrow(v[j]);
        }
    }
};

template <class E>
__device__ __forceinline__ typename E::T element(const u4 &w, int j)
{
    if constexpr (E::kPer16 == 4) return __uint_as_float(w[j]);
    else return static_cast<typename E::T>(w[j / 2] >> (16 * (j & 1)));
}

template <class E>
__device__ __forceinline__ Columns<E> columns_of(int lane, int lanes, int slab, int D)
{
    const int64_t first = (static_cast<int64_t>(slab) * lanes + lane) * E::kPer16;
    const int64_t left = D - first;
    const int n = left >= E::kPer16 ? E::kPer16 : left > 0 ? static_cast<int>(left) : 0;
    const bool narrow = D < E::kPer16;
    return {first, n, narrow || n == 0 ? 0 : E::kPer16 - n, narrow};
}

// ROWS tokens a group of lanes: as many reads of the table in flight.  THROUGH: the results are larger than the caches.
template <class E, int ROWS, bool THROUGH>
__global__ __launch_bounds__(kThreads) void lookup_kernel(const typename E::T *table, int64_t ld, int32_t V, int32_t D, const int32_t *tokens,
                                                          int64_t N, float scale, typename E::T *out, int64_t ld_out, int shift)
{
    const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
    const Columns<E> c = columns_of<E>(lane, lanes, blockIdx.y, D);
    const int64_t n0 = (static_cast<int64_t>(blockIdx.x) * (kThreads >> shift) + (threadIdx.x >> shift)) * ROWS;
    if (c.n == 0 || n0 >= N) return;
    const int64_t w = blockIdx.z;
    table += w * ld;
    int token[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) token[r] = n0 + r < N ? tokens[w * N + n0 + r] : -1;
    u4 rows[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        rows[r] = u4{};
        if (static_cast<uint32_t>(token[r]) < static_cast<uint32_t>(V)) rows[r] = c.raw(table + static_cast<int64_t>(token[r]) * D);
    }
    if (c.back > 0)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) c.place(rows[r]);
    float v[ROWS][E::kPer16];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const bool known = static_cast<uint32_t>(token[r]) < static_cast<uint32_t>(V);
        E::unpack(rows[r], v[r]);
#pragma unroll
        for (int j = 0; j < E::kPer16; ++j) v[r][j] = known ? v[r][j] * scale : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (n0 + r < N) c.template store<THROUGH>(out + (w * N + n0 + r) * ld_out, v[r]);
}

struct Sorted {
    int32_t id, n;                          // a token and its place
};

struct Crossing {
    int32_t id, pieces;                     // the list that begins in a piece and goes on behind it, and how many it reaches over; 0: none does
};

// sorted[w]: the tokens of worker w by id, then by place; named[w]: a bit for every id, set if a token is that id;
// total[w]: the tokens that are an id at all;  crossing[w]: for every piece that is followed by another one.
__device__ __forceinline__ void sort_tokens(const int32_t *tokens, int64_t N, int32_t V, Sorted *sorted, uint64_t *named, int32_t *total, Crossing *crossing,
                                            int piece, int chunks, unsigned blocks)
{
    __shared__ unsigned count[kSortWaves][kBins];
    __shared__ unsigned below_of[kSortWaves], sum_of[kSortWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
    const int32_t lo = static_cast<int32_t>(blockIdx.x) * kBins;
    const unsigned ids = V - lo < kBins ? V - lo : kBins;
    tokens += blockIdx.y * N;
    sorted += blockIdx.y * N;
    // every wavefront has a contiguous part of the tokens
    const int64_t part = (N + kSortThreads - 1) / kSortThreads * kWave;
    const int64_t from = wave * part, to = from + part < N ? from + part : N;
    int held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) held[k] = from + k * kWave + lane < to ? tokens[from + k * kWave + lane] : -1;
    for (int k = threadIdx.x; k < kSortWaves * kBins; k += kSortThreads) (&count[0][0])[k] = 0;
    __syncthreads();
    int below = 0;
    const auto tally = [&](int token) {
        below += __popcll(__ballot(token >= 0 && token < lo));
        const unsigned bin = static_cast<unsigned>(token) - static_cast<unsigned>(lo);
        if (token >= 0 && bin < ids) atomicAdd(&count[wave][bin], 1u);                 // in LDS, integers
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) tally(held[k]);
    for (int64_t n = from + kHeld * kWave; n < to; n += kHeld * kWave) {
        int token[kHeld];
#pragma unroll
        for (int k = 0; k < kHeld; ++k) token[k] = n + k * kWave + lane < to ? tokens[n + k * kWave + lane] : -1;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) tally(token[k]);
    }
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    // a thread for every id: exclusive sums over the wavefronts, then over the ids
    unsigned own = 0;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
        const unsigned c = count[k][threadIdx.x];
        count[k][threadIdx.x] = own;
        own += c;
    }
    unsigned sum = own;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const unsigned other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == kWave - 1) sum_of[wave] = sum;
    __syncthreads();
    unsigned first = sum - own;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) first += below_of[k];
    for (int k = 0; k < wave; ++k) first += sum_of[k];
    if (blockIdx.x + 1 == blocks && threadIdx.x + 1 == kSortThreads) total[blockIdx.y] = static_cast<int32_t>(first + own);
    const uint64_t word = __ballot(own != 0);
    if (lane == 0 && static_cast<unsigned>(wave * kWave) < ids) named[blockIdx.y * ((static_cast<int64_t>(V) + 63) / 64) + lo / 64 + wave] = word;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) count[k][threadIdx.x] += first;
    // the list [first, end) says what crosses the end of each piece whose last token is in it
    if (own) {
        const int end = static_cast<int>(first + own), begins = static_cast<int>(first / static_cast<unsigned>(piece));
        for (int chunk = begins; (chunk + 1) * piece <= end; ++chunk) {
            const bool crosses = chunk == begins && (chunk + 1) * piece < end;
            crossing[blockIdx.y * static_cast<int64_t>(chunks) + chunk] = {lo + static_cast<int>(threadIdx.x), crosses ? (end - 1) / piece - begins + 1 : 0};
        }
    }
    __syncthreads();
    // the same walk again: the lanes of a wavefront that hold one id take consecutive places
    const auto put = [&](int token, int64_t n) {
        const unsigned bin = static_cast<unsigned>(token) - static_cast<unsigned>(lo);
        const bool here = token >= 0 && bin < ids;
        unsigned long long same = __ballot(here);
        if (same == 0) return;
#pragma unroll
        for (int bit = 1; bit < kBins; bit *= 2) {
            const unsigned long long set = __ballot((bin & bit) != 0);
            same &= (bin & bit) != 0 ? set : ~set;
        }
        const int leader = here ? __ffsll(same) - 1 : lane;
        unsigned at = 0;
        if (here && lane == leader) at = atomicAdd(&count[wave][bin], static_cast<unsigned>(__popcll(same)));
        at = __shfl(at, leader);
        if (here) sorted[at + __popcll(same & ((1ull << lane) - 1))] = {token, static_cast<int32_t>(n + lane)};
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k) put(held[k], from + k * kWave);
    for (int64_t n = from + kHeld * kWave; n < to; n += kHeld * kWave) {
        int token[kHeld];
#pragma unroll
        for (int k = 0; k < kHeld; ++k) token[k] = n + k * kWave + lane < to ? tokens[n + k * kWave + lane] : -1;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) put(token[k], n + k * kWave);
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_kernel(const int32_t *tokens, int64_t N, int32_t V, Sorted *sorted, uint64_t *named, int32_t *total,
                                                            Crossing *crossing, int piece, int chunks)
{
    sort_tokens(tokens, N, V, sorted, named, total, crossing, piece, chunks, gridDim.x);
}

// The same, and zeros for the table's whole gradient from other workgroups, behind the `blocks` that sort.
constexpr int kFillVectors = 4;             // of a thread
template <class E>
__global__ __launch_bounds__(kSortThreads) void sort_fill_kernel(const int32_t *tokens, int64_t N, int32_t V, Sorted *sorted, uint64_t *named, int32_t *total,
                                                                 Crossing *crossing, int piece, int chunks, unsigned blocks, typename E::T *g_out, int64_t ld,
                                                                 int64_t elements)
{
    if (blockIdx.x < blocks) return sort_tokens(tokens, N, V, sorted, named, total, crossing, piece, chunks, blocks);
    g_out += blockIdx.y * ld;
    const int64_t first = ((static_cast<int64_t>(blockIdx.x) - blocks) * kFillVectors * kSortThreads + threadIdx.x) * E::kPer16;
#pragma unroll
    for (int k = 0; k < kFillVectors; ++k) {
        const int64_t at = first + k * kSortThreads * E::kPer16;
        if (at + E::kPer16 <= elements) {
            store16<E>(g_out + at, u4{});
        } else {
            for (int64_t j = at; j < elements; ++j) g_out[j] = E::narrow(0.0f);
        }
    }
}

template <class E>
struct GradArgs {
    const typename E::T *dout;
    int64_t ld_dout;
    const Sorted *sorted;
    const uint64_t *named;
    const int32_t *total;
    const Crossing *crossing;               // [W][chunks]
    float *pieces;                          // [W][chunks][2][piece_ld]: a piece's sums of the list that begins before it, of the one that goes on behind it
    const typename E::T *g_in;              // first element of the table's columns, or NULL
    typename E::T *g_out;
    int64_t ld, N, piece_ld;                // piece_ld: D in whole vectors
    int32_t V, D, chunks, chunk_blocks;
    float scale;
    uint32_t per_row;                       // 2^32 / D, rounded down
    int shift, piece, slabs, fills, turn;   // lanes of a group (log2), tokens of a piece, groups to a row, workgroups to 64 rows
};

// A lane's sums, in fp32, 16 bytes at a time.
template <int N>
__device__ __forceinline__ void store_wide(float *to, const float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        const float part[4] = {v[j], v[j + 1], v[j + 2], v[j + 3]};
        store16<F32>(to + j, F32::pack(part));
    }
}
template <int N>
__device__ __forceinline__ void load_wide(const float *from, float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        float part[4];
        F32::unpack(load16<F32>(from + j), part);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j + i] = part[i];
    }
}

template <class E>
__device__ __forceinline__ int64_t place_of(const GradArgs<E> &a, int64_t w, int32_t v) { return w * a.ld + static_cast<int64_t>(v) * a.D; }

// g: the row of g_in, where there is one
template <class E>
__device__ __forceinline__ void finish(const GradArgs<E> &a, const Columns<E> &c, int64_t w, int32_t v, const float (&sum)[E::kPer16], u4 g_row)
{
    float g[E::kPer16];
    c.place(g_row);
    E::unpack(g_row, g);
#pragma unroll
    for (int j = 0; j < E::kPer16; ++j) g[j] = a.g_in ? __builtin_fmaf(a.scale, sum[j], g[j]) : a.scale * sum[j];
    c.store(a.g_out + place_of(a, w, v), g);
}

// One piece of the sorted list; `list` holds it and its neighbours (id -1: none).
template <class E>
__device__ __forceinline__ void sum_piece(const GradArgs<E> &a, const Columns<E> &c, int64_t w, int chunk, int tokens, const Sorted *list)
{
    constexpr int kRows = 8;                // rows of dout in flight, and of g_in where a list ends
    const typename E::T *rows = a.dout + w * a.N * a.ld_dout;
    float sum[E::kPer16] = {};
    bool began = list[-1].id != list[0].id; // in this piece
    for (int i = 0; i < tokens; i += kRows) {
        u4 v[kRows], g[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            v[k] = g[k] = u4{};
            if (i + k >= tokens) continue;
            v[k] = c.raw(rows + list[i + k].n * a.ld_dout);
            if (a.g_in && list[i + k].id != list[i + k + 1].id) g[k] = c.raw(a.g_in + place_of(a, w, list[i + k].id));
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (i + k >= tokens) break;
            float one[E::kPer16];
            c.place(v[k]);
            E::unpack(v[k], one);
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) sum[j] += one[j];
            const bool ends = list[i + k].id != list[i + k + 1].id;
            if (!ends && i + k + 1 < tokens) continue;
            if (began && ends) {
                finish<E>(a, c, w, list[i + k].id, sum, g[k]);
            } else {
                store_wide(a.pieces + ((w * a.chunks + chunk) * 2 + (began ? 1 : 0)) * a.piece_ld + c.first, sum);
            }
            began = true;
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) sum[j] = 0.0f;
        }
    }
}

// IN_PLACE: rows that no token names stay as they are: g_out is g_in, or filled.
template <class E, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void grad_kernel(const GradArgs<E> a)
{
    extern __shared__ Sorted list[];        // the pieces of this workgroup, one more on either side
    const int lanes = 1 << a.shift, groups = kThreads >> a.shift, group = threadIdx.x >> a.shift;
    const int64_t w = blockIdx.y;
    // workgroups of both kinds in turn, one that adds up for every a.turn of all: adding up waits, filling streams
    const int x = blockIdx.x, turns = a.chunk_blocks * a.slabs;
    if (x % a.turn == 0 && x / a.turn < turns) {
        const int block = x / a.turn / a.slabs, slab = x / a.turn % a.slabs;
        const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, slab, a.D);
        const int all = a.total[w], p0 = block * groups * a.piece;
        if (p0 >= all) return;
        const Sorted *sorted = a.sorted + w * a.N;
        for (int k = threadIdx.x; k < groups * a.piece + 2; k += kThreads) {
            const int p = p0 - 1 + k;
            list[k] = p >= 0 && p < all ? sorted[p] : Sorted{-1, 0};
        }
        __syncthreads();
        const int left = all - p0 - group * a.piece;
        if (left > 0 && c.n) sum_piece<E>(a, c, w, block * groups + group, left < a.piece ? left : a.piece, list + 1 + group * a.piece);
        return;
    }
    if constexpr (!IN_PLACE) {
        // 64 rows, one word of bits, in a.fills workgroups that have a contiguous part of their vectors each, whichever rows these lie in
        const int before = (x + a.turn - 1) / a.turn, block = x - (before < turns ? before : turns);
        const int64_t v0 = static_cast<int64_t>(block / a.fills) * 64;
        const int rows = a.V - v0 < 64 ? static_cast<int>(a.V - v0) : 64, elements = rows * a.D;
        const uint64_t word = a.named[w * ((static_cast<int64_t>(a.V) + 63) / 64) + v0 / 64];
        const typename E::T *from = a.g_in ? a.g_in + w * a.ld + v0 * a.D : nullptr;
        typename E::T *to = a.g_out + w * a.ld + v0 * a.D;
        constexpr int kPer = E::kPer16, kAhead = 4;
        // at / D by a product that is at most one too small
        const auto row_of = [&](int at) {
            const int r = static_cast<int>(__umulhi(static_cast<unsigned>(at), a.per_row));
            return (r + 1) * a.D <= at ? r + 1 : r;
        };
        const int vectors = (elements + kPer - 1) / kPer, each = (vectors + a.fills - 1) / a.fills;
        int q = block % a.fills * each;
        const int end = q + each < vectors ? q + each : vectors;
        q += threadIdx.x;
        if (word == 0) {
            const int whole = elements / kPer < end ? elements / kPer : end;            // the last vector may hang over the rows' end
            for (; q + (kAhead - 1) * kThreads < whole; q += kAhead * kThreads) {
                u4 v[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) v[k] = from ? load16<E>(from + (q + k * kThreads) * kPer) : u4{};
#pragma unroll
                for (int k = 0; k < kAhead; ++k) store16<E>(to + (q + k * kThreads) * kPer, v[k]);
            }
        }
        for (; q < end; q += kAhead * kThreads) {
            u4 v[kAhead];
            unsigned wanted[kAhead];                    // bit j: element j of the vector is of a row that no token names
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int first = (q + k * kThreads) * kPer, left = elements - first;
                v[k] = u4{};
                wanted[k] = 0;
                if (q + k * kThreads >= end) continue;
                if (left >= kPer) {
                    if (from) v[k] = load16<E>(from + first);
                    wanted[k] = (1u << kPer) - 1;
                } else {                                // the last vector hangs over the rows' end
                    if (from) v[k] = load_part<E>(from + first, left);
                    wanted[k] = (1u << left) - 1;
                }
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int first = (q + k * kThreads) * kPer;
                if (wanted[k] == 0) continue;
                const int r0 = row_of(first), r1 = first + kPer <= (r0 + 1) * a.D ? r0 : row_of((first + kPer < elements ? first + kPer : elements) - 1);
                const uint64_t rows_of_it = (2ull << (r1 - r0)) - 1, hit = (word >> r0) & rows_of_it;
                if (hit == rows_of_it) continue;
                if (hit != 0) {
                    int row = 0, next = (r0 + 1) * a.D;
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        if (first + j == next) { ++row; next += a.D; }
                        if ((hit >> row) & 1) wanted[k] &= ~(1u << j);
                    }
                }
                if (wanted[k] == (1u << kPer) - 1) {
                    store16<E>(to + first, v[k]);
                } else if (wanted[k] != 0) {
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if ((wanted[k] >> j) & 1) to[first + j] = element<E>(v[k], j);
                }
            }
        }
    }
}

// The lists that reach over several pieces: their sums, in order.  A group of lanes for every piece that one may begin in; those of many pieces
// are left to all groups together.
template <class E>
__global__ __launch_bounds__(kThreads) void join_kernel(const GradArgs<E> a)
{
    __shared__ float lds[E::kPer16][kThreads];
    __shared__ Crossing here[kThreads / 4];
    const int64_t w = blockIdx.z;
    const int lanes = 1 << a.shift, groups = kThreads >> a.shift, group = threadIdx.x >> a.shift, chunk0 = blockIdx.x * groups;
    if (static_cast<int>(threadIdx.x) < groups) {
        const int chunk = chunk0 + threadIdx.x;
        const bool full = (static_cast<int64_t>(chunk) + 1) * a.piece <= a.total[w];
        here[threadIdx.x] = full ? a.crossing[w * a.chunks + chunk] : Crossing{-1, 0};
    }
    __syncthreads();
    const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, blockIdx.y, a.D);
    // pieces [from, to) of a list, the first one's slot 1, slot 0 of the others
    const auto add = [&](int chunk, int from, int to, float (&sum)[E::kPer16]) {
        constexpr int kAhead = 4;
        const float *row = a.pieces + (w * a.chunks + chunk) * 2 * a.piece_ld + c.first;
        for (int k0 = from; k0 < to; k0 += kAhead) {
            float v[kAhead][E::kPer16];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = k0 + i < to ? k0 + i : to - 1;
                load_wide(row + (static_cast<int64_t>(k) * 2 + (k == 0)) * a.piece_ld, v[i]);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (k0 + i < to)
#pragma unroll
                    for (int j = 0; j < E::kPer16; ++j) sum[j] += v[i][j];
        }
    };
    const auto old = [&](int id) { return a.g_in ? c.raw(a.g_in + place_of(a, w, id)) : u4{}; };
    const Crossing own = here[group];
    if (own.pieces > 0 && own.pieces <= kFewPieces && c.n) {
        float sum[E::kPer16] = {};
        const u4 g = old(own.id);
        add(chunk0 + group, 0, own.pieces, sum);
        finish<E>(a, c, w, own.id, sum, g);
    }
    for (int f = 0; f < groups; ++f) {
        const Crossing list = here[f];
        if (list.pieces <= kFewPieces) continue;        // the same for the workgroup
        const int each = (list.pieces + groups - 1) / groups, from = group * each, to = from + each < list.pieces ? from + each : list.pieces;
        float sum[E::kPer16] = {};
        if (c.n) add(chunk0 + f, from, to, sum);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < E::kPer16; ++j) lds[j][threadIdx.x] = sum[j];
        __syncthreads();
        if (group == 0 && c.n) {
            for (int at = threadIdx.x + lanes; at < kThreads; at += lanes)
#pragma unroll
                for (int j = 0; j < E::kPer16; ++j) sum[j] += lds[j][at];
            finish<E>(a, c, w, list.id, sum, old(list.id));
        }
    }
}

// log2 of the lanes of a group: enough for a row, or 64, 32 or 16 of them several times, whichever leaves fewest idle.
template <class E>
int lanes_shift(int32_t D)
{
    const int64_t vectors = ceil_div(D, E::kPer16);
    int shift = 2;
    while (shift < 6 && (1 << shift) < vectors) ++shift;
    if (shift < 6 || vectors <= 64) return shift;
    for (int smaller = 5; smaller >= 4; --smaller)
        if (round_up(vectors, 1 << smaller) < round_up(vectors, 1 << shift)) shift = smaller;
    return shift;
}

int check_shape(int64_t ld, int32_t W, int64_t offset, int32_t V, int32_t D, int64_t N)
{
    if (W < 1 || W > CX_MAX_ROWS || V < 1 || V > kMaxVocab || D < 1 || D > kMaxWidth || N < 0 || N > kMaxTokens) return CX_ERR_SHAPE;
    if (offset < 0 || offset > kMaxExtent || bad_matrix(W, ld, offset + static_cast<int64_t>(V) * D)) return CX_ERR_SHAPE;
    return CX_OK;
}

template <class E>
int lookup(const typename E::T *x, int64_t ld, int32_t W, int64_t offset, int32_t V, int32_t D, const int32_t *tokens, int64_t N,
           float scale, typename E::T *out, int64_t ld_out, void *stream)
{
    if (!x || (N > 0 && (!tokens || !out))) return CX_ERR_NULL;
    const int rc = check_shape(ld, W, offset, V, D, N);
    if (rc != CX_OK) return rc;
    if (N == 0) return CX_OK;
    if (bad_matrix(W * N, ld_out, D)) return CX_ERR_SHAPE;
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(x, kElem) || misaligned_to(out, kElem) || misaligned_to(tokens, 4)) return CX_ERR_ALIGN;
    const Extent in[2] = {matrix_of(x, W, ld, offset + static_cast<int64_t>(V) * D, kElem), dense_of(tokens, W * N * 4)};
    const Extent result[1] = {matrix_of(out, W * N, ld_out, D, kElem)};
    if (outputs_share(in, result, -1, -1)) return CX_ERR_ALIAS;
    const int shift = lanes_shift<E>(D), groups = kThreads >> shift;
    const int64_t slabs = ceil_div(ceil_div(D, E::kPer16), 1 << shift);
    // Four rows a group from 4,096 workgroups of one row on; from 64 MB on, results that go past the caches, and two rows: 16 x 4,096 tokens
    // of 768 columns take 35 us with ordinary stores and 26 without in bfloat16, in float32 63 and 61, 56 with two rows, 65 with one
    const bool many = W * N * slabs >= int64_t(4096) * groups, large = many && W * N * D * kElem >= int64_t(64) << 20;
    const dim3 grid(static_cast<unsigned>(ceil_div(N, static_cast<int64_t>(groups) * (large ? 2 : many ? 4 : 1))), static_cast<unsigned>(slabs), W);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const auto launch = [&](auto rows, auto through) {
        hipLaunchKernelGGL((lookup_kernel<E, decltype(rows)::value, decltype(through)::value>), grid, dim3(kThreads), 0, st, x + offset, ld, V, D,
                           tokens, N, scale, out, ld_out, shift);
    };
    if (large) launch(std::integral_constant<int, 2>{}, std::true_type{});
    else if (many) launch(std::integral_constant<int, 4>{}, std::false_type{});
    else launch(std::integral_constant<int, 1>{}, std::false_type{});
    return launched();
}

struct GradSpace {
    int64_t named, total, sorted, crossing, pieces, bytes, chunks;
    int piece;
};

GradSpace grad_space(int32_t W, int64_t N, int32_t V, int32_t D)
{
    GradSpace s{};
    // tokens of a piece: few, so that there are many; more of them where long lists would leave thousands of sums to join.  Calls of 8, 16, 32 and
    // 64 tokens a piece, us, 768 bfloat16 columns and tables of 32,768 rows unless noted: four workers' 1,000 (129 float32 columns) 18, 20, 26, 39;
    // one worker's 4,096 28, 29, 36, 49, sixteen's 193, 191, 195, 211; one worker's 16,000 (129 float32 columns) 43, 39, 42, 54; 32,768 82, 72,
    // 72, 82, all of them one token 383, 233, 155, 123; sixteen workers' 32,768 491, 435, 414, 414; one worker's 131,072 (float32) 384, 322, 283,
    // 275.  Above 16,384 it is the frequent token that 64 are for: one worker's ordinary text would take less with 16 or 32
    s.piece = N <= 2048 ? 8 : N <= 16384 ? 16 : 64;
    s.chunks = ceil_div(N, s.piece);
    s.named = 0;
    s.total = round_up(W * ceil_div(V, 64) * 8, 256);
    s.sorted = s.total + round_up(W * 4, 256);
    s.crossing = s.sorted + round_up(W * N * static_cast<int64_t>(sizeof(Sorted)), 256);
    s.pieces = s.crossing + round_up(W * s.chunks * static_cast<int64_t>(sizeof(Crossing)), 256);
    s.bytes = s.pieces + W * s.chunks * 2 * round_up(D, 8) * 4;
    return s;
}

template <class E>
int grad(const typename E::T *dout, int64_t ld_dout, const int32_t *tokens, int32_t W, int64_t N, const typename E::T *g_in,
         typename E::T *g_out, int64_t ld, int64_t offset, int32_t V, int32_t D, float scale, void *workspace, int64_t workspace_bytes,
         void *stream)
{
    if (!g_out || !workspace || (N > 0 && (!dout || !tokens))) return CX_ERR_NULL;
    const int rc = check_shape(ld, W, offset, V, D, N);
    if (rc != CX_OK) return rc;
    if (N > 0 && bad_matrix(W * N, ld_dout, D)) return CX_ERR_SHAPE;
    const GradSpace space = grad_space(W, N, V, D);
    if (workspace_bytes < space.bytes) return CX_ERR_SHAPE;
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(dout, kElem) || misaligned_to(g_in, kElem) || misaligned_to(g_out, kElem) || misaligned_to(tokens, 4) ||
        misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const int64_t columns = offset + static_cast<int64_t>(V) * D;
    const Extent in[3] = {matrix_of(dout, W * N, ld_dout, D, kElem), dense_of(tokens, W * N * 4), matrix_of(g_in, W, ld, columns, kElem)};
    const Extent out[2] = {matrix_of(g_out, W, ld, columns, kElem), dense_of(workspace, space.bytes)};
    if (outputs_share(in, out, 0, 2)) return CX_ERR_ALIAS;
    char *base = static_cast<char *>(workspace);
    Sorted *sorted = reinterpret_cast<Sorted *>(base + space.sorted);
    uint64_t *named = reinterpret_cast<uint64_t *>(base + space.named);
    int32_t *total = reinterpret_cast<int32_t *>(base + space.total);
    Crossing *crossing = reinterpret_cast<Crossing *>(base + space.crossing);
    GradArgs<E> a{dout, ld_dout, sorted, named, total, crossing, reinterpret_cast<float *>(base + space.pieces), g_in ? g_in + offset : nullptr, g_out + offset,
                  ld, N, round_up(D, 8), V, D, static_cast<int32_t>(space.chunks), 0, scale, static_cast<uint32_t>(0xffffffffu / static_cast<uint32_t>(D)), lanes_shift<E>(D), space.piece, 0, 1, 1};
    const int groups = kThreads >> a.shift;
    a.slabs = static_cast<int>(ceil_div(ceil_div(D, E::kPer16), 1 << a.shift));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // Where tokens name few rows at most and nothing is added, all rows are filled while the tokens are sorted, and those few are written again:
    // 16 workers' tables of 32,768 x 768 in bfloat16 take 173 us instead of 192 with 2,048 tokens, but 198 instead of 190 with 4,096; 3 tables of
    // 23,182 x 375 in float32 30 instead of 37 with 790.  Rows of g_in would be read twice (2,048 tokens: 346 us instead of 320).
    const bool filled = !g_in && N <= V / 16;
    const unsigned sorters = static_cast<unsigned>(ceil_div(V, kBins));
    if (filled) {
        const int64_t elements = static_cast<int64_t>(V) * D, each = kFillVectors * kSortThreads * E::kPer16;
        hipLaunchKernelGGL((sort_fill_kernel<E>), dim3(sorters + static_cast<unsigned>(ceil_div(elements, each)), W), dim3(kSortThreads), 0, st, tokens, N, V,
                           sorted, named, total, crossing, space.piece, static_cast<int32_t>(space.chunks), sorters, a.g_out, ld, elements);
    } else {
        hipLaunchKernelGGL(sort_kernel, dim3(sorters, W), dim3(kSortThreads), 0, st, tokens, N, V, sorted, named, total, crossing, space.piece,
                           static_cast<int32_t>(space.chunks));
    }
    if (launched() != CX_OK) return CX_ERR_HIP;
    a.chunk_blocks = static_cast<int32_t>(ceil_div(space.chunks, groups));
    int64_t fill_blocks = 0;
    if (g_in != g_out && !filled) {
        // a workgroup to four vectors a thread: short ones keep what is written at a time close together in memory
        const int64_t words = ceil_div(V, 64);
        a.fills = static_cast<int>(ceil_div(64 * static_cast<int64_t>(D), E::kPer16 * kThreads * 4));
        fill_blocks = words * a.fills;
    }
    const int64_t sums = static_cast<int64_t>(a.chunk_blocks) * a.slabs;
    if (sums > 0) a.turn = static_cast<int>((sums + fill_blocks) / sums);
    const dim3 grid(static_cast<unsigned>(sums + fill_blocks), W);
    const unsigned list_bytes = (groups * a.piece + 2) * sizeof(Sorted);
    if (grid.x > 0) {
        if (g_in == g_out || filled) hipLaunchKernelGGL((grad_kernel<E, true>), grid, dim3(kThreads), list_bytes, st, a);
        else hipLaunchKernelGGL((grad_kernel<E, false>), grid, dim3(kThreads), list_bytes, st, a);
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    if (space.chunks <= 1) return CX_OK;
    hipLaunchKernelGGL(join_kernel<E>, dim3(static_cast<unsigned>(ceil_div(space.chunks - 1, groups)), a.slabs, W), dim3(kThreads), 0, st, a);
    return launched();
}

}  // namespace

extern "C" {

int cx_lm_abi_version(void) { return 1; }

#define CX_LM_EMBED(SUFFIX, E)                                                                                                        \
    int cx_embed_lookup##SUFFIX(const E::T *x, int64_t ld, int32_t W, int64_t offset, int32_t V, int32_t D, const int32_t *tokens,   \
                                int64_t N, float scale, E::T *out, int64_t ld_out, void *stream)                                      \
    {                                                                                                                                 \
        return lookup<E>(x, ld, W, offset, V, D, tokens, N, scale, out, ld_out, stream);                                              \
    }                                                                                                                                 \
    int cx_embed_grad##SUFFIX(const E::T *dout, int64_t ld_dout, const int32_t *tokens, int32_t W, int64_t N, const E::T *g_in,       \
                              E::T *g_out, int64_t ld, int64_t offset, int32_t V, int32_t D, float scale, void *workspace,            \
                              int64_t workspace_bytes, void *stream)                                                                  \
    {                                                                                                                                 \
        return grad<E>(dout, ld_dout, tokens, W, N, g_in, g_out, ld, offset, V, D, scale, workspace, workspace_bytes, stream);        \
    }
CX_LM_EMBED(, F32)
CX_LM_EMBED(_bf16, Bf16)
CX_LM_EMBED(_f16, F16)
#undef CX_LM_EMBED

int cx_embed_workspace(int32_t W, int64_t N, int32_t V, int32_t D, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    if (W < 1 || W > CX_MAX_ROWS || V < 1 || V > kMaxVocab || D < 1 || D > kMaxWidth || N < 0 || N > kMaxTokens) return CX_ERR_SHAPE;
    *bytes = grad_space(W, N, V, D).bytes;
    return CX_OK;
}

}  // extern "C"
