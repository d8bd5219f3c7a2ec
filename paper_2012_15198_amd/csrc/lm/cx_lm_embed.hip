// C-ABI entry points cx_embed_lookup*, cx_embed_grad*, cx_embed_workspace: embedding tables that lie in the workers'
// flat rows, and their gradient by sorted tokens (see include/cx_lm.h).
//
//   out[w][n] = round(scale * table_w[token[w][n]])               g[w][v] = round(g_in[w][v] + scale * sum_{n: token = v} dout[w][n])
//
// Both are bound by memory.  A group of lanes (a power of two, as many as one row's 16-byte vectors, 64 at most) handles one
// vector column each of one row, so a short row does not leave a wavefront's lanes idle.
//
// The gradient writes each row of the table once and adds in a fixed order, which atomics would not.  Three launches:
//   sort_kernel   a stable counting sort of each worker's tokens.  A workgroup owns 1,024 ids and reads all N tokens
//                 itself instead of exchanging counts with the others: no passes, no atomics on memory, and where the
//                 table has 32,768 rows 32 workgroups a worker read 32 x 16 KB of tokens from the cache.
//   grad_kernel   the sorted list in pieces of equal length, one to a group of lanes, so that a frequent token keeps no group longer than
//                 a rare one: it adds up the rows of dout that its piece names, list by list, and writes what lists lie inside the
//                 piece; what reaches beyond goes to the workspace.  Other workgroups of the same launch write the rows that no
//                 token names.
//   join_kernel   adds up the lists that reach over several pieces, in order.
#include "lm_common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kBins = 1024;                 // ids of a workgroup of the sort
constexpr int kSortWaves = 8, kSortThreads = kSortWaves * kWave;
constexpr int kBinsEach = kBins / kSortThreads;
constexpr int kHeld = 8;                    // tokens a lane of the sort keeps in registers between its two walks
constexpr int kJoinThreads = kWave;         // few: most workgroups of the join find nothing to do
constexpr int64_t kMaxTokens = CX_MAX_TOKENS;
constexpr int32_t kMaxVocab = CX_MAX_VOCAB, kMaxWidth = CX_MAX_WIDTH;

template <class E>
struct Columns {                            // the columns of a row that a lane handles
    int64_t first;
    int n;                                  // of kPer16; 0 beyond the row
    __device__ __forceinline__ void load(const typename E::T *row, float (&v)[E::kPer16]) const
    {
        if (n == E::kPer16) {
            E::unpack(load16<E>(row + first), v);
        } else {
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) v[j] = j < n ? E::widen(row[first + j]) : 0.0f;
        }
    }
    __device__ __forceinline__ void store(typename E::T *row, const float (&v)[E::kPer16]) const
    {
        if (n == E::kPer16) {
            store16<E>(row + first, E::pack(v));
        } else {
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j)
                if (j < n) row[first + j] = E::narrow(v[j]);
        }
    }
};

template <class E>
__device__ __forceinline__ Columns<E> columns_of(int lane, int lanes, int slab, int D)
{
    const int64_t first = (static_cast<int64_t>(slab) * lanes + lane) * E::kPer16;
    const int64_t left = D - first;
    return {first, left >= E::kPer16 ? E::kPer16 : left > 0 ? static_cast<int>(left) : 0};
}

// ROWS tokens a group of lanes: as many reads of the table in flight.
template <class E, int ROWS>
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
    float v[ROWS][E::kPer16];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (static_cast<uint32_t>(token[r]) < static_cast<uint32_t>(V)) {
            c.load(table + static_cast<int64_t>(token[r]) * D, v[r]);
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) v[r][j] *= scale;
        } else {
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) v[r][j] = 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
        if (n0 + r < N) c.store(out + (w * N + n0 + r) * ld_out, v[r]);
}

struct Sorted {
    int32_t id, n;                          // a token and its place
};

// sorted[w]: the tokens of worker w by id, then by place; named[w]: a bit for every id, set if a token is that id;
// total[w]: the tokens that are an id at all.
__global__ __launch_bounds__(kSortThreads) void sort_kernel(const int32_t *tokens, int64_t N, int32_t V, Sorted *sorted, uint64_t *named, int32_t *total)
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
    for (int64_t n = from + kHeld * kWave; n < to; n += kWave) tally(n + lane < to ? tokens[n + lane] : -1);
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    // a thread for every kBinsEach ids: exclusive sums over the wavefronts, then over the ids
    unsigned mine[kBinsEach], own = 0;
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) {
        const int bin = threadIdx.x * kBinsEach + i;
        mine[i] = 0;
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const unsigned c = count[k][bin];
            count[k][bin] = mine[i];
            mine[i] += c;
        }
        own += mine[i];
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
    if (blockIdx.x + 1 == gridDim.x && threadIdx.x + 1 == kSortThreads) total[blockIdx.y] = static_cast<int32_t>(first + own);
    static_assert(kBinsEach == 2, "a wavefront's bits make two words");
    const uint64_t even = __ballot(mine[0] != 0), odd = __ballot(mine[1] != 0);
    if (lane < kBinsEach) {
        uint64_t word = 0;                                  // of ids 2 * (64 * wave + 32 * lane) and on
        for (int k = 0; k < 32; ++k) word |= ((even >> (32 * lane + k)) & 1) << (2 * k) | ((odd >> (32 * lane + k)) & 1) << (2 * k + 1);
        const unsigned at = (2 * wave + lane) * 64;
        if (at < ids) named[blockIdx.y * ((static_cast<int64_t>(V) + 63) / 64) + (lo + at) / 64] = word;
    }
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) {
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) count[k][threadIdx.x * kBinsEach + i] += first;
        first += mine[i];
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
    for (int64_t n = from + kHeld * kWave; n < to; n += kWave) put(n + lane < to ? tokens[n + lane] : -1, n);
}

template <class E>
struct GradArgs {
    const typename E::T *dout;
    int64_t ld_dout;
    const Sorted *sorted;
    const uint64_t *named;
    const int32_t *total;
    float *pieces;                          // [W][chunks][2][D]: a piece's sums of the list that begins before it, of the one that goes on behind it
    const typename E::T *g_in;              // first element of the table's columns, or NULL
    typename E::T *g_out;
    int64_t ld, N;
    int32_t V, D, chunks, chunk_blocks;
    float scale;
    int shift, piece;                       // lanes of a group (log2), tokens of a piece
};

template <class E>
__device__ __forceinline__ void finish(const GradArgs<E> &a, const Columns<E> &c, int64_t w, int32_t v, const float (&sum)[E::kPer16])
{
    const int64_t at = w * a.ld + static_cast<int64_t>(v) * a.D;
    float g[E::kPer16];
    if (a.g_in) c.load(a.g_in + at, g);
#pragma unroll
    for (int j = 0; j < E::kPer16; ++j) g[j] = a.g_in ? __builtin_fmaf(a.scale, sum[j], g[j]) : a.scale * sum[j];
    c.store(a.g_out + at, g);
}

// One piece of the sorted list; `list` holds it and its neighbours (id -1: none).
template <class E>
__device__ __forceinline__ void sum_piece(const GradArgs<E> &a, const Columns<E> &c, int64_t w, int chunk, int tokens, const Sorted *list)
{
    constexpr int kRows = 4;                // rows of dout in flight
    const typename E::T *rows = a.dout + w * a.N * a.ld_dout;
    float sum[E::kPer16] = {};
    int id = list[0].id;
    bool began = list[-1].id != id;         // in this piece
    const auto close = [&](bool ends) {
        if (began && ends) {
            finish<E>(a, c, w, id, sum);
        } else {
            float *to = a.pieces + ((w * a.chunks + chunk) * 2 + (began ? 1 : 0)) * a.D + c.first;
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j)
                if (j < c.n) to[j] = sum[j];
        }
    };
    for (int i = 0; i < tokens; i += kRows) {
        float v[kRows][E::kPer16];
#pragma unroll
        for (int k = 0; k < kRows; ++k) c.load(rows + list[i + k < tokens ? i + k : tokens - 1].n * a.ld_dout, v[k]);
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (i + k >= tokens) break;
            const int next = list[i + k].id;
            if (next != id) {
                close(true);
                id = next;
                began = true;
#pragma unroll
                for (int j = 0; j < E::kPer16; ++j) sum[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) sum[j] += v[k][j];
        }
    }
    close(list[tokens].id != id);
}

// IN_PLACE: g_out is g_in, rows that no token names stay as they are.
template <class E, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void grad_kernel(const GradArgs<E> a)
{
    extern __shared__ Sorted list[];        // the pieces of this workgroup, one more on either side
    const int lanes = 1 << a.shift, groups = kThreads >> a.shift, group = threadIdx.x >> a.shift;
    const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, blockIdx.y, a.D);
    const int64_t w = blockIdx.z;
    if (static_cast<int>(blockIdx.x) < a.chunk_blocks) {
        const int all = a.total[w], p0 = static_cast<int>(blockIdx.x) * groups * a.piece;
        if (p0 >= all) return;
        const Sorted *sorted = a.sorted + w * a.N;
        for (int k = threadIdx.x; k < groups * a.piece + 2; k += kThreads) {
            const int p = p0 - 1 + k;
            list[k] = p >= 0 && p < all ? sorted[p] : Sorted{-1, 0};
        }
        __syncthreads();
        const int left = all - p0 - group * a.piece;
        if (left > 0 && c.n) sum_piece<E>(a, c, w, blockIdx.x * groups + group, left < a.piece ? left : a.piece, list + 1 + group * a.piece);
        return;
    }
    if constexpr (!IN_PLACE) {
        // 64 rows, one word of bits; the slabs of the grid share its vectors, whichever rows these lie in
        const int64_t v0 = static_cast<int64_t>(blockIdx.x - a.chunk_blocks) * 64;
        const int rows = a.V - v0 < 64 ? static_cast<int>(a.V - v0) : 64, elements = rows * a.D;
        const uint64_t word = a.named[w * ((static_cast<int64_t>(a.V) + 63) / 64) + v0 / 64];
        const typename E::T *from = a.g_in ? a.g_in + w * a.ld + v0 * a.D : nullptr;
        typename E::T *to = a.g_out + w * a.ld + v0 * a.D;
        constexpr int kPer = E::kPer16, kAhead = 4;
        const int stride = gridDim.y * kThreads;
        int q = blockIdx.y * kThreads + threadIdx.x;
        if (word == 0) {
            for (; (q + (kAhead - 1) * stride + 1) * kPer <= elements; q += kAhead * stride) {
                u4 v[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) v[k] = from ? load16<E>(from + (q + k * stride) * kPer) : u4{};
#pragma unroll
                for (int k = 0; k < kAhead; ++k) store16<E>(to + (q + k * stride) * kPer, v[k]);
            }
        }
        for (; q * kPer < elements; q += stride) {
            const int first = q * kPer, last = (first + kPer < elements ? first + kPer : elements) - 1;
            const int r0 = first / a.D, r1 = last / a.D;
            if (first + kPer <= elements && ((word >> r0) & ((2ull << (r1 - r0)) - 1)) == 0) {
                store16<E>(to + first, from ? load16<E>(from + first) : u4{});
            } else {
                for (int at = first; at <= last; ++at)
                    if (!((word >> (at / a.D)) & 1)) to[at] = from ? from[at] : E::narrow(0.0f);
            }
        }
    }
}

// The list that begins in this piece and goes on behind it, if one does: its sums, in order.
template <class E>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const GradArgs<E> a)
{
    __shared__ float lds[E::kPer16][kJoinThreads];
    const int64_t w = blockIdx.z;
    const Sorted *sorted = a.sorted + w * a.N;
    const int chunk = blockIdx.x, all = a.total[w], p0 = chunk * a.piece, p1 = p0 + a.piece;
    if (p1 >= all) return;
    const int id = sorted[p1 - 1].id;
    if (sorted[p1].id != id || (sorted[p0].id == id && p0 > 0 && sorted[p0 - 1].id == id)) return;
    int pieces = 1;                         // and those whose first token is of the list
    for (;; pieces += kJoinThreads) {
        const int64_t p = static_cast<int64_t>(chunk + pieces + static_cast<int>(threadIdx.x)) * a.piece;
        const int more = __popcll(__ballot(p < all && sorted[p].id == id));
        if (more < kJoinThreads) { pieces += more; break; }
    }
    const int lanes = 1 << a.shift, groups = kJoinThreads >> a.shift, group = threadIdx.x >> a.shift;
    const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, blockIdx.y, a.D);
    const int each = (pieces + groups - 1) / groups;
    const int from = group * each, to = from + each < pieces ? from + each : pieces;
    const float *row = a.pieces + (w * a.chunks + chunk) * 2 * a.D + c.first;
    float sum[E::kPer16] = {};
    constexpr int kAhead = 4;
    for (int k0 = from; k0 < to; k0 += kAhead) {
        float v[kAhead][E::kPer16];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = k0 + i < to ? k0 + i : to - 1;
            const float *piece = row + (static_cast<int64_t>(k) * 2 + (k == 0)) * a.D;
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) v[i][j] = j < c.n ? piece[j] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (k0 + i < to)
#pragma unroll
                for (int j = 0; j < E::kPer16; ++j) sum[j] += v[i][j];
    }
#pragma unroll
    for (int j = 0; j < E::kPer16; ++j) lds[j][threadIdx.x] = sum[j];
    __syncthreads();
    if (group == 0 && c.n) {
        for (int at = threadIdx.x + lanes; at < kJoinThreads; at += lanes)
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) sum[j] += lds[j][at];
        finish<E>(a, c, w, id, sum);
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
    const uint64_t out_bytes = span(W * N, ld_out, D, kElem);
    if (overlap(out, out_bytes, x, span(W, ld, offset + static_cast<int64_t>(V) * D, kElem)) || overlap(out, out_bytes, tokens, W * N * 4)) return CX_ERR_ALIAS;
    const int shift = lanes_shift<E>(D), groups = kThreads >> shift;
    const int64_t slabs = ceil_div(ceil_div(D, E::kPer16), 1 << shift);
    // Four rows a group from 4,096 workgroups of one row on
    const bool many = W * N * slabs >= int64_t(4096) * groups;
    const int64_t blocks = ceil_div(N, static_cast<int64_t>(groups) * (many ? 4 : 1));
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(slabs), W);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (many) hipLaunchKernelGGL((lookup_kernel<E, 4>), grid, dim3(kThreads), 0, st, x + offset, ld, V, D, tokens, N, scale, out, ld_out, shift);
    else hipLaunchKernelGGL((lookup_kernel<E, 1>), grid, dim3(kThreads), 0, st, x + offset, ld, V, D, tokens, N, scale, out, ld_out, shift);
    return launched();
}

struct GradSpace {
    int64_t named, total, sorted, pieces, bytes, chunks;
    int piece;
};

GradSpace grad_space(int32_t W, int64_t N, int32_t V, int32_t D)
{
    GradSpace s{};
    // tokens of a piece: few, so that there are many; more of them where a list of all tokens would leave thousands of sums to join
    s.piece = N <= 16384 ? 16 : 64;
    s.chunks = ceil_div(N, s.piece);
    s.named = 0;
    s.total = round_up(W * ceil_div(V, 64) * 8, 256);
    s.sorted = s.total + round_up(W * 4, 256);
    s.pieces = s.sorted + round_up(W * N * static_cast<int64_t>(sizeof(Sorted)), 256);
    s.bytes = s.pieces + W * s.chunks * 2 * D * 4;
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
    const uint64_t g_bytes = span(W, ld, offset + static_cast<int64_t>(V) * D, kElem), dout_bytes = span(W * N, ld_dout, D, kElem), token_bytes = W * N * 4;
    if (overlap(g_out, g_bytes, dout, dout_bytes) || overlap(g_out, g_bytes, tokens, token_bytes) ||
        (g_in != g_out && overlap(g_out, g_bytes, g_in, g_bytes))) return CX_ERR_ALIAS;
    if (overlap(workspace, space.bytes, g_out, g_bytes) || overlap(workspace, space.bytes, dout, dout_bytes) ||
        overlap(workspace, space.bytes, g_in, g_bytes) || overlap(workspace, space.bytes, tokens, token_bytes)) return CX_ERR_ALIAS;
    char *base = static_cast<char *>(workspace);
    Sorted *sorted = reinterpret_cast<Sorted *>(base + space.sorted);
    uint64_t *named = reinterpret_cast<uint64_t *>(base + space.named);
    int32_t *total = reinterpret_cast<int32_t *>(base + space.total);
    GradArgs<E> a{dout, ld_dout, sorted, named, total, reinterpret_cast<float *>(base + space.pieces), g_in ? g_in + offset : nullptr, g_out + offset,
                  ld, N, V, D, static_cast<int32_t>(space.chunks), 0, scale, lanes_shift<E>(D), space.piece};
    const int groups = kThreads >> a.shift;
    const unsigned slabs = static_cast<unsigned>(ceil_div(ceil_div(D, E::kPer16), 1 << a.shift));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(sort_kernel, dim3(static_cast<unsigned>(ceil_div(V, kBins)), W), dim3(kSortThreads), 0, st, tokens, N, V, sorted, named,
                       total);
    if (launched() != CX_OK) return CX_ERR_HIP;
    a.chunk_blocks = static_cast<int32_t>(ceil_div(space.chunks, groups));
    const int64_t empty_blocks = g_in == g_out ? 0 : ceil_div(V, 64);
    const dim3 grid(static_cast<unsigned>(a.chunk_blocks + empty_blocks), slabs, W);
    const unsigned list_bytes = (groups * a.piece + 2) * sizeof(Sorted);
    if (grid.x > 0) {
        if (g_in == g_out) hipLaunchKernelGGL((grad_kernel<E, true>), grid, dim3(kThreads), list_bytes, st, a);
        else hipLaunchKernelGGL((grad_kernel<E, false>), grid, dim3(kThreads), list_bytes, st, a);
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    if (space.chunks <= 1) return CX_OK;
    hipLaunchKernelGGL(join_kernel<E>, dim3(static_cast<unsigned>(space.chunks - 1), slabs, W), dim3(kJoinThreads), 0, st, a);
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
