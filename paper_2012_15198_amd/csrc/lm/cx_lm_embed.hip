// C-ABI entry points cx_embed_lookup*, cx_embed_grad*, cx_embed_workspace: embedding tables that lie in the workers'
// flat rows, and their gradient by sorted tokens (see include/cx_lm.h).
//
//   out[w][n] = round(scale * table_w[token[w][n]])               g[w][v] = round(g_in[w][v] + scale * sum_{n: token = v} dout[w][n])
//
// Both are bound by memory.  A group of lanes (a power of two, as many as one row's 16-byte vectors, 64 at most) handles one
// vector column each of one row, so a short row does not leave a wavefront's lanes idle.
//
// The gradient writes each row of the table once and adds in a fixed order, which atomics would not.  Three launches:
//   sort_kernel   a stable counting sort of each worker's tokens.  A workgroup owns 512 ids and reads all N tokens
//                 itself, twice, instead of exchanging counts with the others: no passes, no atomics on memory, and where the
//                 table has 32,768 rows 64 workgroups a worker read 64 x 16 KB of tokens from the cache.
//   grad_kernel   a group of lanes for every row of the table: sums the rows of dout that the sorted list names (none: zeros).
//                 Lists longer than kLong would make one group work long after the others, so those are cut at every
//                 kLong-th place of the sorted list into pieces that other workgroups of the same launch sum up;
//   join_kernel   adds the pieces of such a list in order.
#include "lm_common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kBins = 512;                  // ids of a workgroup of the sort
constexpr int kSortWaves = 8;
constexpr int kSortAhead = 4;               // tokens a lane loads before it looks at them
constexpr int kLong = 64;                   // tokens of one id from which its list is cut; also the length of a piece
constexpr int kRowsPerGroup = 4;            // rows of the table a group of lanes handles one after the other
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

// starts[w][v]: where the list of id v begins in order[w]; order[w]: places of the tokens, by id, then ascending.
__global__ __launch_bounds__(kSortWaves *kWave) void sort_kernel(const int32_t *tokens, int64_t N, int32_t V, int32_t *starts, int32_t *order)
{
    __shared__ unsigned count[kSortWaves][kBins];
    __shared__ unsigned below_of[kSortWaves], total_of[kSortWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
    const int32_t lo = static_cast<int32_t>(blockIdx.x) * kBins;
    const unsigned ids = V - lo < kBins ? V - lo : kBins;
    tokens += blockIdx.y * N;
    order += blockIdx.y * N;
    starts += blockIdx.y * (static_cast<int64_t>(V) + 1) + lo;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) count[k][threadIdx.x] = 0;
    __syncthreads();
    // every wavefront counts a contiguous part of the tokens
    const int64_t part = (N + kSortWaves * kWave - 1) / (kSortWaves * kWave) * kWave;
    const int64_t from = wave * part, to = from + part < N ? from + part : N;
    int below = 0;
    for (int64_t n = from; n < to; n += kSortAhead * kWave) {
        int token[kSortAhead];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) token[k] = n + k * kWave + lane < to ? tokens[n + k * kWave + lane] : -1;
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            below += __popcll(__ballot(token[k] >= 0 && token[k] < lo));
            const unsigned bin = static_cast<unsigned>(token[k]) - static_cast<unsigned>(lo);
            if (token[k] >= 0 && bin < ids) atomicAdd(&count[wave][bin], 1u);          // in LDS, integers
        }
    }
    if (lane == 0) below_of[wave] = below;
    __syncthreads();
    // exclusive sums: over the wavefronts of a bin, then over the bins
    unsigned mine = 0, first = 0;
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) {
        const unsigned c = count[k][threadIdx.x];
        count[k][threadIdx.x] = mine;
        mine += c;
        first += below_of[k];
    }
    unsigned sum = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const unsigned other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == kWave - 1) total_of[wave] = sum;
    __syncthreads();
    for (int k = 0; k < wave; ++k) first += total_of[k];
    first += sum - mine;
    if (threadIdx.x < ids) starts[threadIdx.x] = static_cast<int32_t>(first);
    if (threadIdx.x + 1 == ids && lo + static_cast<int32_t>(ids) == V) starts[ids] = static_cast<int32_t>(first + mine);
#pragma unroll
    for (int k = 0; k < kSortWaves; ++k) count[k][threadIdx.x] += first;
    __syncthreads();
    // the same walk again: the lanes of a wavefront that hold one id take consecutive places
    for (int64_t n = from; n < to; n += kSortAhead * kWave) {
        int token[kSortAhead];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) token[k] = n + k * kWave + lane < to ? tokens[n + k * kWave + lane] : -1;
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            const unsigned bin = static_cast<unsigned>(token[k]) - static_cast<unsigned>(lo);
            const bool here = token[k] >= 0 && bin < ids;
            unsigned long long same = __ballot(here);
            if (same == 0) continue;
#pragma unroll
            for (int bit = 1; bit < kBins; bit *= 2) {
                const unsigned long long set = __ballot((bin & bit) != 0);
                same &= (bin & bit) != 0 ? set : ~set;
            }
            const int leader = here ? __ffsll(same) - 1 : lane;
            unsigned at = 0;
            if (here && lane == leader) at = atomicAdd(&count[wave][bin], static_cast<unsigned>(__popcll(same)));
            at = __shfl(at, leader);
            if (here) order[at + __popcll(same & ((1ull << lane) - 1))] = static_cast<int32_t>(n + k * kWave + lane);
        }
    }
}

template <class E>
struct GradArgs {
    const typename E::T *dout;
    int64_t ld_dout;
    const int32_t *tokens, *starts, *order;
    float *pieces;                          // [W][chunks][2][D]
    const typename E::T *g_in;              // first element of the table's columns, or NULL
    typename E::T *g_out;
    int64_t ld, N;
    int32_t V, D, chunks;
    float scale;
    int shift;
};

// sum over i in [s, e) of rows[order[i]], in that order
template <class E>
__device__ __forceinline__ void add_rows(const Columns<E> &c, const typename E::T *rows, int64_t ld, const int32_t *order, int s, int e,
                                         float (&sum)[E::kPer16])
{
    constexpr int kAhead = 4;
    for (int i = s; i < e; i += kAhead) {
        float v[kAhead][E::kPer16];
        int at[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) at[k] = order[i + k < e ? i + k : e - 1];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) c.load(rows + at[k] * ld, v[k]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k < e)
#pragma unroll
                for (int j = 0; j < E::kPer16; ++j) sum[j] += v[k][j];
    }
}

template <class E>
__device__ __forceinline__ void finish(const GradArgs<E> &a, const Columns<E> &c, int64_t w, int32_t v, float (&sum)[E::kPer16])
{
    const int64_t at = w * a.ld + static_cast<int64_t>(v) * a.D;
    float g[E::kPer16];
    if (a.g_in) c.load(a.g_in + at, g);
#pragma unroll
    for (int j = 0; j < E::kPer16; ++j) g[j] = a.g_in ? __builtin_fmaf(a.scale, sum[j], g[j]) : a.scale * sum[j];
    c.store(a.g_out + at, g);
}

// The groups' sums added in order of the groups; the first group holds the result.
template <class E>
__device__ __forceinline__ void add_groups(float (&sum)[E::kPer16], float *lds, int shift)
{
    const int lanes = 1 << shift;
#pragma unroll
    for (int j = 0; j < E::kPer16; ++j) lds[j * kThreads + threadIdx.x] = sum[j];
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < lanes)
        for (int at = threadIdx.x + lanes; at < kThreads; at += lanes)
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j) sum[j] += lds[j * kThreads + at];
    __syncthreads();
}

// A piece: places [kLong * chunk, kLong * (chunk + 1)) of the sorted list.  At most two lists longer than that reach into it: the
// one that its first place belongs to (slot 0) and, if it is another, the one of its last place (slot 1).
template <class E>
__device__ void sum_piece(const GradArgs<E> &a, int chunk, float *lds)
{
    const int64_t w = blockIdx.z;
    const int32_t *starts = a.starts + w * (static_cast<int64_t>(a.V) + 1), *order = a.order + w * a.N, *tokens = a.tokens + w * a.N;
    const int all = starts[a.V], p0 = chunk * kLong;
    if (p0 >= all) return;
    const int p1 = p0 + kLong < all ? p0 + kLong : all;
    const int lanes = 1 << a.shift, groups = kThreads >> a.shift, group = threadIdx.x >> a.shift;
    const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, blockIdx.y, a.D);
    const int first = tokens[order[p0]], last = tokens[order[p1 - 1]];
    for (int slot = 0; slot < (first == last ? 1 : 2); ++slot) {
        const int id = slot ? last : first;
        const int s = starts[id], e = starts[id + 1];
        if (e - s <= kLong) continue;                                  // the same for every thread of the workgroup
        const int lo = s > p0 ? s : p0, hi = e < p1 ? e : p1, each = (hi - lo + groups - 1) / groups;
        const int from = lo + group * each, to = from + each < hi ? from + each : hi;
        float sum[E::kPer16] = {};
        if (c.n) add_rows<E>(c, a.dout + w * a.N * a.ld_dout, a.ld_dout, order, from, to, sum);
        add_groups<E>(sum, lds, a.shift);
        if (group == 0 && c.n) {
            float *to_row = a.pieces + ((w * a.chunks + chunk) * 2 + slot) * a.D + c.first;
#pragma unroll
            for (int j = 0; j < E::kPer16; ++j)
                if (j < c.n) to_row[j] = sum[j];
        }
    }
}

// IN_PLACE: g_out is g_in, rows that no token names stay as they are.
template <class E, bool IN_PLACE>
__global__ __launch_bounds__(kThreads) void grad_kernel(const GradArgs<E> a)
{
    __shared__ float lds[kThreads * E::kPer16];
    if (static_cast<int>(blockIdx.x) < a.chunks) { sum_piece<E>(a, blockIdx.x, lds); return; }
    const int lanes = 1 << a.shift;
    const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, blockIdx.y, a.D);
    const int64_t w = blockIdx.z;
    const int64_t v0 = (static_cast<int64_t>(blockIdx.x - a.chunks) * (kThreads >> a.shift) + (threadIdx.x >> a.shift)) * kRowsPerGroup;
    if (c.n == 0 || v0 >= a.V) return;
    const int32_t *starts = a.starts + w * (static_cast<int64_t>(a.V) + 1) + v0;
    const int rows = a.V - v0 < kRowsPerGroup ? static_cast<int>(a.V - v0) : kRowsPerGroup;
    int edge[kRowsPerGroup + 1];
#pragma unroll
    for (int r = 0; r <= kRowsPerGroup; ++r) edge[r] = starts[r < rows ? r : rows];
#pragma unroll
    for (int r = 0; r < kRowsPerGroup; ++r) {
        const int s = edge[r], e = edge[r + 1];
        if (r >= rows || (IN_PLACE && s == e) || e - s > kLong) continue;
        float sum[E::kPer16] = {};
        add_rows<E>(c, a.dout + w * a.N * a.ld_dout, a.ld_dout, a.order + w * a.N, s, e, sum);
        finish<E>(a, c, w, static_cast<int32_t>(v0) + r, sum);
    }
}

// The long list that begins in this chunk, if one does: its pieces, in order.
template <class E>
__global__ __launch_bounds__(kThreads) void join_kernel(const GradArgs<E> a)
{
    __shared__ float lds[kThreads * E::kPer16];
    const int64_t w = blockIdx.z;
    const int32_t *starts = a.starts + w * (static_cast<int64_t>(a.V) + 1), *order = a.order + w * a.N, *tokens = a.tokens + w * a.N;
    const int chunk = blockIdx.x, all = starts[a.V], p0 = chunk * kLong;
    if (p0 >= all) return;
    const int p1 = p0 + kLong < all ? p0 + kLong : all;
    const int first = tokens[order[p0]], id = tokens[order[p1 - 1]];
    const int s = starts[id], e = starts[id + 1];
    if (e - s <= kLong || s < p0) return;
    const int lanes = 1 << a.shift, groups = kThreads >> a.shift, group = threadIdx.x >> a.shift;
    const Columns<E> c = columns_of<E>(threadIdx.x & (lanes - 1), lanes, blockIdx.y, a.D);
    const int pieces = (e - 1) / kLong - chunk + 1, each = (pieces + groups - 1) / groups;
    const int from = group * each, to = from + each < pieces ? from + each : pieces;
    const float *row = a.pieces + (w * a.chunks + chunk) * 2 * a.D + c.first;
    float sum[E::kPer16] = {};
    for (int k = from; k < to; ++k) {
        const float *piece = row + (static_cast<int64_t>(k) * 2 + (k == 0 && id != first)) * a.D;
#pragma unroll
        for (int j = 0; j < E::kPer16; ++j)
            if (j < c.n) sum[j] += piece[j];
    }
    add_groups<E>(sum, lds, a.shift);
    if (group == 0 && c.n) finish<E>(a, c, w, id, sum);
}

// log2 of the lanes that handle one row
template <class E>
int lanes_shift(int32_t D)
{
    int shift = 0;
    while (shift < 6 && (1 << shift) * E::kPer16 < D) ++shift;
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
    int64_t starts, order, pieces, bytes, chunks;
};

GradSpace grad_space(int32_t W, int64_t N, int32_t V, int32_t D)
{
    GradSpace s{};
    s.chunks = N > kLong ? ceil_div(N, kLong) : 0;         // shorter: no list is long
    s.starts = 0;
    s.order = round_up(W * (static_cast<int64_t>(V) + 1) * 4, 256);
    s.pieces = s.order + round_up(W * N * 4, 256);
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
    GradArgs<E> a{dout, ld_dout, tokens, reinterpret_cast<int32_t *>(base + space.starts), reinterpret_cast<int32_t *>(base + space.order),
                  reinterpret_cast<float *>(base + space.pieces), g_in ? g_in + offset : nullptr, g_out + offset, ld, N, V, D,
                  static_cast<int32_t>(space.chunks), scale, lanes_shift<E>(D)};
    const int groups = kThreads >> a.shift;
    const unsigned slabs = static_cast<unsigned>(ceil_div(ceil_div(D, E::kPer16), 1 << a.shift));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(sort_kernel, dim3(static_cast<unsigned>(ceil_div(V, kBins)), W), dim3(kSortWaves * kWave), 0, st, tokens, N, V,
                       const_cast<int32_t *>(a.starts), const_cast<int32_t *>(a.order));
    if (launched() != CX_OK) return CX_ERR_HIP;
    const int64_t row_blocks = ceil_div(V, static_cast<int64_t>(groups) * kRowsPerGroup);
    const dim3 grid(static_cast<unsigned>(space.chunks + row_blocks), slabs, W);
    if (g_in == g_out) hipLaunchKernelGGL((grad_kernel<E, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((grad_kernel<E, false>), grid, dim3(kThreads), 0, st, a);
    if (launched() != CX_OK) return CX_ERR_HIP;
    if (space.chunks == 0) return CX_OK;
    hipLaunchKernelGGL(join_kernel<E>, dim3(static_cast<unsigned>(space.chunks), slabs, W), dim3(kThreads), 0, st, a);
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
