// C-ABI entry points cx_gated_scan*, cx_gated_scan_grad*, cx_scan_workspace: the gated linear recurrence (see include/cx_lm.h)
//
//   a = sigmoid(f)    h_t = a_t * (reset_t ? 0 : h_{t-1}) + (1 - a_t) * x_t    y = round(h)
//   r_t = dL/dh_t = dy_t + keep_{t+1} a_{t+1} r_{t+1}    dx = (1 - a) r    df = r (keep h_{t-1} - x) a (1 - a)
//
// One column's steps are a composition of affine maps h -> A h + S, and compositions associate: the steps are cut into pieces
// of kSteps, a lane composes the maps of its piece in registers, the pieces' maps are joined through LDS, and the lane then
// walks its piece once more with the state that enters it.  So the data are read once, whatever the length.
//
//   lane       kCols neighbouring columns (4 bytes of every row) and kSteps consecutive steps: 64 lanes read whole lines of
//              a row, the walk needs no exchange between lanes, and a wavefront keeps 2 (gradient: 3) x 16 loads in flight
//   wavefront  one piece of a tile;  workgroup: up to 8 wavefronts = a tile of 128 steps, tile after tile, the loads of the
//              next one issued before the present one is computed
//   split      where columns are few (workgroups < kSplitBelow) the steps are also split over workgroups: a first launch composes
//              the map of each span (it reads what the second reads again, from the last-level cache where the call fits there)
//
// States, maps and gates are fp32 throughout; y, df and dx are rounded once.  1 - a comes as exp(-f) a, which keeps its
// relative accuracy where a is near one.  A reset makes a map forget its input: such a map's A carries a sign bit (a
// product of gates has none), and what enters is dropped rather than multiplied by zero, so no NaN or infinity crosses it.
#include "lm_common.hpp"

namespace {

constexpr int kSteps = CX_SCAN_CHUNK;                   // steps of a lane's piece
constexpr int kMaxWaves = 8;
constexpr int kTile = kSteps * kMaxWaves;
constexpr int kMaxSpans = 64;                           // workgroups that the steps of one column are split over
constexpr int64_t kMaxColumns = CX_MAX_WIDTH, kMaxSeq = CX_MAX_TOKENS;

template <class E>
struct Cols {                                           // what a lane loads of a row: 4 bytes
    static constexpr int kCols = 4 / sizeof(typename E::T);
    static constexpr int kSlab = kCols * kWave;
};

struct Map {
    float A, S;
};
__device__ __forceinline__ bool forgets(float A) { return (__float_as_uint(A) >> 31) != 0; }
// the map of `earlier` followed by `later`
__device__ __forceinline__ Map then(const Map &earlier, const Map &later)
{
    const bool cut = forgets(later.A);
    return {cut ? later.A : earlier.A * later.A, cut ? later.S : __builtin_fmaf(later.A, earlier.S, later.S)};
}
__device__ __forceinline__ float apply(const Map &m, float h) { return forgets(m.A) ? m.S : __builtin_fmaf(m.A, h, m.S); }

struct Gate {
    float a, b;                                         // sigmoid(f), sigmoid(-f)
};
__device__ __forceinline__ Gate gate(float f)
{
    // exp(-f) is held at 2^115: a < 2^-114 either way, and b = exp(-f) a stays 1 instead of inf * 0.  A NaN passes the comparison.
    float t = f * -kLog2e;
    t = t > 115.0f ? 115.0f : t;
    const float e = exp2_fast(t), a = rcp_fast(1.0f + e);
    return {a, e * a};
}

// A lane's columns.  16-bit rows: two, loaded as one pair.  The pair of the last lane of an odd row begins one column earlier, at its neighbour's,
// whose results it does not store.
template <class E>
struct LaneColumns;
template <>
struct LaneColumns<F32> {
    static constexpr int N = 1;
    int64_t first;
    bool any;
    __device__ __forceinline__ LaneColumns(int64_t column, int D) : first(column < D ? column : D - 1), any(column < D) {}
    __device__ __forceinline__ unsigned load(const float *row) const { return __float_as_uint(row[first]); }
    static __device__ __forceinline__ float value(unsigned w, int) { return __uint_as_float(w); }
    __device__ __forceinline__ void store(float *row, const float (&v)[1]) const { if (any) row[first] = v[0]; }
    __device__ __forceinline__ void load_wide(const float *row, float (&v)[1]) const { v[0] = row[first]; }
    __device__ __forceinline__ void store_wide(float *row, const float (&v)[1]) const { if (any) row[first] = v[0]; }
};
template <class E>
struct LaneColumns {
    static constexpr int N = 2;
    int64_t first;
    bool any, both, single;                             // single: rows of one column
    __device__ __forceinline__ LaneColumns(int64_t column, int D)
        : first(column + 2 <= D ? column : D >= 2 ? D - 2 : 0), any(column < D), both(column + 2 <= D), single(D < 2) {}
    __device__ __forceinline__ unsigned load(const uint16_t *row) const
    {
        return single ? static_cast<unsigned>(row[0]) << 16 : *reinterpret_cast<const u1_at2 *>(row + first);
    }
    static __device__ __forceinline__ float value(unsigned w, int j) { return j ? E::high(w) : E::low(w); }
    __device__ __forceinline__ void store(uint16_t *row, const float (&v)[2]) const
    {
        if (both) *reinterpret_cast<u1_at2 *>(row + first) = E::two(v[0], v[1]);
        else if (any) row[single ? 0 : first + 1] = E::narrow(v[1]);
    }
    __device__ __forceinline__ void load_wide(const float *row, float (&v)[2]) const
    {
        const int64_t own = single ? 0 : first + 1;     // another workgroup may own the one before it
        v[0] = row[both ? first : own];
        v[1] = row[own];
    }
    __device__ __forceinline__ void store_wide(float *row, const float (&v)[2]) const
    {
        if (both) row[first] = v[0];
        if (any) row[single ? 0 : first + 1] = v[1];
    }
};

template <class E>
struct ScanArgs {
    using T = typename E::T;
    const T *f, *x, *dy;
    T *y, *df, *dx;
    int64_t ldf, ldx, ldy, lddy, lddf, lddx;
    const uint8_t *reset;
    const float *h0, *dh_last;
    float *h_last, *dh0, *states;
    const float *states_in;
    float *maps;                                        // split: [B][spans][2][D] (A, S) of each span, [B][D] what enters the first one
    int64_t T_;
    int32_t D, spans;
    int64_t span_steps;                                 // a multiple of kTile; the steps of one workgroup
};

// The gate's factor of each step's map and whether it forgets, for steps of one piece; steps beyond the end change nothing.
__device__ __forceinline__ unsigned reset_bits(const uint8_t *reset, int64_t row, int steps)
{
    if (!reset) return 0;
    const int lane = threadIdx.x & (kWave - 1);
    const bool here = lane < steps && reset[row + lane] != 0;
    return static_cast<unsigned>(__ballot(here));       // bit i: step i of the piece; the same for the wavefront
}

template <int N>
struct Exchange {                                       // the maps of the pieces of a tile, two tiles in turn
    float2 map[2][kMaxWaves][N][kWave];
};

// The map that leads to this wavefront's piece and that of the whole tile, in the order of the walk.
template <int N>
__device__ __forceinline__ void join_pieces(Exchange<N> &lds, int turn, int wave, int waves, bool backwards, const Map (&mine)[N],
                                            const float (&carry)[N], float (&enters)[N], float (&leaves)[N])
{
    const int lane = threadIdx.x & (kWave - 1);
    if (waves == 1) {
#pragma unroll
        for (int j = 0; j < N; ++j) { enters[j] = carry[j]; leaves[j] = apply(mine[j], carry[j]); }
        return;
    }
    const int place = backwards ? waves - 1 - wave : wave;
#pragma unroll
    for (int j = 0; j < N; ++j) lds.map[turn][place][j][lane] = float2{mine[j].A, mine[j].S};
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float h = carry[j];
        enters[j] = h;
        for (int k = 0; k < waves; ++k) {
            const float2 m = lds.map[turn][k][j][lane];
            h = apply({m.x, m.y}, h);
            enters[j] = k + 1 == place ? h : enters[j];
        }
        leaves[j] = h;
    }
}

// What enters this workgroup's span: the maps of the spans on the way to it, applied to what enters the first.
template <class E, int N>
__device__ __forceinline__ void entering(const ScanArgs<E> &a, const LaneColumns<E> &c, int64_t b, int span, bool backwards, const float *first,
                                         float (&h)[N])
{
    if (a.spans == 1) {
        if (first) c.load_wide(first + b * a.D, h);
        else
#pragma unroll
            for (int j = 0; j < N; ++j) h[j] = 0.0f;
        return;
    }
    const float *maps = a.maps + b * a.spans * 2 * a.D;
    c.load_wide(a.maps + (static_cast<int64_t>(gridDim.x) * a.spans * 2 + b) * a.D, h);
    const int before = backwards ? a.spans - 1 - span : span;
    for (int k = 0; k < before; k += 4) {
        float A[4][N], S[4][N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = k + i < before ? k + i : before - 1;
            const float *m = maps + static_cast<int64_t>(backwards ? a.spans - 1 - at : at) * 2 * a.D;
            c.load_wide(m, A[i]);
            c.load_wide(m + a.D, S[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < before)
#pragma unroll
                for (int j = 0; j < N; ++j) h[j] = apply({A[i][j], S[i][j]}, h[j]);
    }
}

// Loads of a piece: rows [t, t + kSteps) of the sequence, those beyond `end` as zeros.
template <class E>
__device__ __forceinline__ void load_piece(const LaneColumns<E> &c, const typename E::T *m, int64_t ld, int64_t row, int steps, unsigned (&v)[kSteps])
{
    const typename E::T *p = m + row * ld;
    if (steps >= kSteps) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) v[i] = c.load(p + i * ld);
    } else {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) v[i] = i < steps ? c.load(p + i * ld) : 0u;
    }
}

__device__ __forceinline__ int steps_at(int64_t t, int64_t end)
{
    const int64_t left = end - t;
    return left >= kSteps ? kSteps : left > 0 ? static_cast<int>(left) : 0;
}

// Grid (sequences, spans, slabs of columns).  ONLY_MAP: the first launch of a split call.
template <class E, bool ONLY_MAP>
__global__ __launch_bounds__(kMaxWaves *kWave) void scan_kernel(const ScanArgs<E> a)
{
    constexpr int N = LaneColumns<E>::N;
    __shared__ Exchange<N> lds;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int64_t b = blockIdx.x;
    const int span = blockIdx.y;
    const LaneColumns<E> c(static_cast<int64_t>(blockIdx.z) * Cols<E>::kSlab + lane * N, a.D);
    const int64_t row0 = b * a.T_, begin = span * a.span_steps, end = begin + a.span_steps < a.T_ ? begin + a.span_steps : a.T_;
    const int tile = waves * kSteps;
    float carry[N];
    Map whole[N];
    if constexpr (ONLY_MAP) {
        if (span == 0 && wave == 0) {                   // what enters the first span: the second launch may be given h_last = h0
            float h[N] = {};
            if (a.h0) c.load_wide(a.h0 + b * a.D, h);
            c.store_wide(a.maps + (static_cast<int64_t>(gridDim.x) * a.spans * 2 + b) * a.D, h);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) whole[j] = {1.0f, 0.0f};
    } else {
        entering<E, N>(a, c, b, span, false, a.h0, carry);
    }
    unsigned fw[kSteps], xw[kSteps];
    int64_t t = begin + wave * kSteps;
    int steps = steps_at(t, end);
    load_piece<E>(c, a.f, a.ldf, row0 + t, steps, fw);
    load_piece<E>(c, a.x, a.ldx, row0 + t, steps, xw);
    int turn = 0;
    for (int64_t tile0 = begin; tile0 < end; tile0 += tile, turn ^= 1) {
        const unsigned resets = reset_bits(a.reset, row0 + t, steps);
        float keep[kSteps][N], in[kSteps][N];
        Map mine[N];
#pragma unroll
        for (int j = 0; j < N; ++j) mine[j] = {1.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool there = i < steps, cut = (resets >> i) & 1u;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const Gate g = gate(c.value(fw[i], j));
                keep[i][j] = there ? g.a : 1.0f;
                in[i][j] = there ? g.b * c.value(xw[i], j) : 0.0f;
                mine[j].S = cut ? in[i][j] : __builtin_fmaf(keep[i][j], mine[j].S, in[i][j]);
                mine[j].A = cut ? -1.0f : keep[i][j] * mine[j].A;
            }
        }
        const int64_t t_now = t;
        const int steps_now = steps;
        t += tile;
        steps = steps_at(t, end);
        load_piece<E>(c, a.f, a.ldf, row0 + t, steps, fw);
        load_piece<E>(c, a.x, a.ldx, row0 + t, steps, xw);
        if constexpr (ONLY_MAP) {
            // the composition of maps, one wavefront's piece after the other
            Map piece[N];
            if (waves > 1) {
#pragma unroll
                for (int j = 0; j < N; ++j) lds.map[turn][wave][j][lane] = float2{mine[j].A, mine[j].S};
                __syncthreads();
                for (int k = 0; k < waves; ++k)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float2 m = lds.map[turn][k][j][lane];
                        piece[j] = {m.x, m.y};
                        whole[j] = then(whole[j], piece[j]);
                    }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) whole[j] = then(whole[j], mine[j]);
            }
        } else {
            float h[N], leaves[N];
            join_pieces<N>(lds, turn, wave, waves, false, mine, carry, h, leaves);
            if (a.states && steps_now > 0) c.store_wide(a.states + (b * ceil_div(a.T_, kSteps) + t_now / kSteps) * a.D, h);
            typename E::T *out = a.y + (row0 + t_now) * a.ldy;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (i >= steps_now) break;
                const bool cut = (resets >> i) & 1u;
#pragma unroll
                for (int j = 0; j < N; ++j) h[j] = cut ? in[i][j] : __builtin_fmaf(keep[i][j], h[j], in[i][j]);
                c.store(out + i * a.ldy, h);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) carry[j] = leaves[j];
        }
    }
    if constexpr (ONLY_MAP) {
        if (wave == 0) {
            float A[N], S[N];
#pragma unroll
            for (int j = 0; j < N; ++j) { A[j] = whole[j].A; S[j] = whole[j].S; }
            float *m = a.maps + (b * a.spans + span) * 2 * a.D;
            c.store_wide(m, A);
            c.store_wide(m + a.D, S);
        }
    } else if (a.h_last && end == a.T_ && wave == waves - 1) {
        c.store_wide(a.h_last + b * a.D, carry);
    }
}

// The gradient, from the last step to the first.  What a piece hands to the one before it is keep a r of its first step.
template <class E, bool ONLY_MAP>
__global__ __launch_bounds__(kMaxWaves *kWave) void scan_grad_kernel(const ScanArgs<E> a)
{
    constexpr int N = LaneColumns<E>::N;
    __shared__ Exchange<N> lds;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int64_t b = blockIdx.x;
    const int span = blockIdx.y;
    const LaneColumns<E> c(static_cast<int64_t>(blockIdx.z) * Cols<E>::kSlab + lane * N, a.D);
    const int64_t row0 = b * a.T_, begin = span * a.span_steps, end = begin + a.span_steps < a.T_ ? begin + a.span_steps : a.T_;
    const int tile = waves * kSteps;
    float carry[N];
    Map whole[N];
    if constexpr (ONLY_MAP) {
        if (span == 0 && wave == 0) {
            float r[N] = {};
            if (a.dh_last) c.load_wide(a.dh_last + b * a.D, r);
            c.store_wide(a.maps + (static_cast<int64_t>(gridDim.x) * a.spans * 2 + b) * a.D, r);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) whole[j] = {1.0f, 0.0f};
    } else {
        entering<E, N>(a, c, b, span, true, a.dh_last, carry);
    }
    int64_t tile0 = begin + (end - 1 - begin) / tile * tile;
    int64_t t = tile0 + wave * kSteps;
    int steps = steps_at(t, end);
    unsigned fw[kSteps], xw[kSteps], gw[kSteps];
    load_piece<E>(c, a.f, a.ldf, row0 + t, steps, fw);
    if constexpr (!ONLY_MAP) load_piece<E>(c, a.x, a.ldx, row0 + t, steps, xw);
    load_piece<E>(c, a.dy, a.lddy, row0 + t, steps, gw);
    int turn = 0;
    for (; tile0 >= begin; tile0 -= tile, turn ^= 1) {
        const unsigned resets = reset_bits(a.reset, row0 + t, steps);
        float keep[kSteps][N], open[kSteps][N], before[kSteps][N];
        unsigned x_now[kSteps], dy_now[kSteps];
        Map mine[N];
        float h[N] = {};
        if constexpr (!ONLY_MAP)
            if (steps > 0) c.load_wide(a.states_in + (b * ceil_div(a.T_, kSteps) + t / kSteps) * a.D, h);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool there = i < steps, cut = (resets >> i) & 1u;
            dy_now[i] = gw[i];
            if constexpr (!ONLY_MAP) x_now[i] = xw[i];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const Gate g = gate(c.value(fw[i], j));
                keep[i][j] = there ? g.a : 1.0f;
                if constexpr (!ONLY_MAP) {
                    open[i][j] = g.b;
                    before[i][j] = cut ? 0.0f : h[j];
                    const float in = g.b * c.value(xw[i], j);
                    h[j] = cut ? in : __builtin_fmaf(g.a, h[j], in);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) mine[j] = {1.0f, 0.0f};
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            const bool cut = (resets >> i) & 1u;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                mine[j].S = cut ? 0.0f : keep[i][j] * (c.value(dy_now[i], j) + mine[j].S);
                mine[j].A = cut ? -1.0f : keep[i][j] * mine[j].A;
            }
        }
        const int64_t t_now = t;
        const int steps_now = steps;
        t -= tile;
        steps = tile0 > begin ? kSteps : 0;
        load_piece<E>(c, a.f, a.ldf, row0 + t, steps, fw);
        if constexpr (!ONLY_MAP) load_piece<E>(c, a.x, a.ldx, row0 + t, steps, xw);
        load_piece<E>(c, a.dy, a.lddy, row0 + t, steps, gw);
        if constexpr (ONLY_MAP) {
            if (waves > 1) {
#pragma unroll
                for (int j = 0; j < N; ++j) lds.map[turn][wave][j][lane] = float2{mine[j].A, mine[j].S};
                __syncthreads();
                for (int k = waves - 1; k >= 0; --k)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float2 m = lds.map[turn][k][j][lane];
                        whole[j] = then(whole[j], {m.x, m.y});
                    }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) whole[j] = then(whole[j], mine[j]);
            }
        } else {
            float r[N], leaves[N];
            join_pieces<N>(lds, turn, wave, waves, true, mine, carry, r, leaves);
            typename E::T *df = a.df + (row0 + t_now) * a.lddf, *dx = a.dx + (row0 + t_now) * a.lddx;
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                if (i >= steps_now) continue;
                const bool cut = (resets >> i) & 1u;
                float f_out[N], x_out[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float g = c.value(dy_now[i], j) + r[j];
                    x_out[j] = open[i][j] * g;
                    f_out[j] = (before[i][j] - c.value(x_now[i], j)) * keep[i][j] * x_out[j];
                    r[j] = cut ? 0.0f : keep[i][j] * g;
                }
                c.store(df + i * a.lddf, f_out);
                c.store(dx + i * a.lddx, x_out);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) carry[j] = leaves[j];
        }
    }
    if constexpr (ONLY_MAP) {
        if (wave == 0) {
            float A[N], S[N];
#pragma unroll
            for (int j = 0; j < N; ++j) { A[j] = whole[j].A; S[j] = whole[j].S; }
            float *m = a.maps + (b * a.spans + span) * 2 * a.D;
            c.store_wide(m, A);
            c.store_wide(m + a.D, S);
        }
    } else if (a.dh0 && begin == 0 && wave == 0) {
        c.store_wide(a.dh0 + b * a.D, carry);
    }
}

// No steps: the state passes through.
__global__ __launch_bounds__(256) void pass_kernel(const float *from, float *to, int64_t n)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

struct Split {
    int spans;
    int64_t span_steps, bytes;
};

// Fewer workgroups than this leave CUs idle for longer than a second reading takes.
constexpr int64_t kSplitBelow = 128, kSplitTo = 512;

Split split_of(int64_t B, int64_t T, int32_t D, int slab)
{
    const int64_t groups = B * ceil_div(D, slab), tiles = ceil_div(T, kTile);
    int64_t spans = groups < kSplitBelow ? ceil_div(kSplitTo, groups) : 1;
    spans = spans < tiles ? spans : tiles;
    spans = spans < kMaxSpans ? spans : kMaxSpans;
    if (spans <= 1) return {1, round_up(T, kTile), 0};
    const int64_t span_tiles = ceil_div(tiles, spans);
    spans = ceil_div(tiles, span_tiles);
    return {static_cast<int>(spans), span_tiles * kTile, spans > 1 ? (B * spans * 2 + B) * D * 4 : 0};
}

// Whether two matrices of the same number of rows share an element.  Halves of the rows of one wider matrix do not.
template <class E>
bool share(const typename E::T *a, int64_t lda, const typename E::T *b, int64_t ldb, int64_t rows, int64_t columns)
{
    constexpr int kElem = sizeof(typename E::T);
    if (!a || !b || !overlap(a, span(rows, lda, columns, kElem), b, span(rows, ldb, columns, kElem))) return false;
    if (lda != ldb) return true;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(a < b ? a : b), hi = reinterpret_cast<uintptr_t>(a < b ? b : a);
    const uint64_t off = (hi - lo) % (static_cast<uint64_t>(lda) * kElem), width = static_cast<uint64_t>(columns) * kElem;
    return off < width || off + width > static_cast<uint64_t>(lda) * kElem;
}

int check_sizes(int64_t B, int64_t T, int32_t D)
{
    return B < 0 || B > CX_MAX_SEQUENCES || T < 0 || T > kMaxSeq || D < 1 || D > kMaxColumns ? CX_ERR_SHAPE : CX_OK;
}

template <class E>
int scan(const typename E::T *f, int64_t ldf, const typename E::T *x, int64_t ldx, typename E::T *y, int64_t ldy, int64_t B, int64_t T,
         int32_t D, const uint8_t *reset, const float *h0, float *h_last, float *states, void *workspace, int64_t workspace_bytes, void *stream)
{
    int rc = check_sizes(B, T, D);
    if (rc != CX_OK) return rc;
    if (B == 0) return CX_OK;
    constexpr int kElem = sizeof(typename E::T);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const uint64_t state_bytes = B * D * 4;
    if (misaligned_to(h0, 4) || misaligned_to(h_last, 4)) return CX_ERR_ALIGN;
    if (h0 != h_last && overlap(h0, state_bytes, h_last, state_bytes)) return CX_ERR_ALIAS;
    if (T == 0) {
        if (!h_last || h_last == h0) return CX_OK;
        hipLaunchKernelGGL(pass_kernel, dim3(static_cast<unsigned>(ceil_div(B * D, 256))), dim3(256), 0, st, h0, h_last, B * D);
        return launched();
    }
    if (!f || !x || !y) return CX_ERR_NULL;
    if (bad_matrix(B * T, ldf, D) || bad_matrix(B * T, ldx, D) || bad_matrix(B * T, ldy, D)) return CX_ERR_SHAPE;
    const Split split = split_of(B, T, D, Cols<E>::kSlab);
    if (split.bytes > 0 && !workspace) return CX_ERR_NULL;
    if (split.bytes > 0 && workspace_bytes < split.bytes) return CX_ERR_SHAPE;
    if (misaligned_to(f, kElem) || misaligned_to(x, kElem) || misaligned_to(y, kElem) || misaligned_to(states, 4) ||
        misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const uint64_t y_bytes = span(B * T, ldy, D, kElem), states_bytes = B * ceil_div(T, kSteps) * D * 4;
    if (share<E>(y, ldy, f, ldf, B * T, D) || share<E>(y, ldy, x, ldx, B * T, D) || overlap(y, y_bytes, reset, B * T) ||
        overlap(y, y_bytes, h0, state_bytes) || overlap(y, y_bytes, h_last, state_bytes) || overlap(y, y_bytes, states, states_bytes) ||
        overlap(states, states_bytes, h0, state_bytes) || overlap(states, states_bytes, h_last, state_bytes)) return CX_ERR_ALIAS;
    ScanArgs<E> a{};
    a.f = f; a.ldf = ldf; a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy;
    a.reset = reset; a.h0 = h0; a.h_last = h_last; a.states = states;
    a.maps = static_cast<float *>(workspace);
    a.T_ = T; a.D = D; a.spans = split.spans; a.span_steps = split.span_steps;
    const int64_t pieces = ceil_div(T, kSteps);
    const dim3 grid(static_cast<unsigned>(B), split.spans, static_cast<unsigned>(ceil_div(D, Cols<E>::kSlab)));
    const dim3 block(static_cast<unsigned>(pieces < kMaxWaves ? pieces : kMaxWaves) * kWave);
    if (split.spans > 1) {
        hipLaunchKernelGGL((scan_kernel<E, true>), grid, block, 0, st, a);
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    hipLaunchKernelGGL((scan_kernel<E, false>), grid, block, 0, st, a);
    return launched();
}

template <class E>
int scan_grad(const typename E::T *f, int64_t ldf, const typename E::T *x, int64_t ldx, const typename E::T *dy, int64_t lddy,
              typename E::T *df, int64_t lddf, typename E::T *dx, int64_t lddx, int64_t B, int64_t T, int32_t D, const uint8_t *reset,
              const float *states, const float *dh_last, float *dh0, void *workspace, int64_t workspace_bytes, void *stream)
{
    int rc = check_sizes(B, T, D);
    if (rc != CX_OK) return rc;
    if (B == 0) return CX_OK;
    constexpr int kElem = sizeof(typename E::T);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const uint64_t state_bytes = B * D * 4;
    if (misaligned_to(dh_last, 4) || misaligned_to(dh0, 4)) return CX_ERR_ALIGN;
    if (dh0 != dh_last && overlap(dh0, state_bytes, dh_last, state_bytes)) return CX_ERR_ALIAS;
    if (T == 0) {
        if (!dh0 || dh0 == dh_last) return CX_OK;
        hipLaunchKernelGGL(pass_kernel, dim3(static_cast<unsigned>(ceil_div(B * D, 256))), dim3(256), 0, st, dh_last, dh0, B * D);
        return launched();
    }
    if (!f || !x || !dy || !df || !dx || !states) return CX_ERR_NULL;
    if (bad_matrix(B * T, ldf, D) || bad_matrix(B * T, ldx, D) || bad_matrix(B * T, lddy, D) || bad_matrix(B * T, lddf, D) ||
        bad_matrix(B * T, lddx, D)) return CX_ERR_SHAPE;
    const Split split = split_of(B, T, D, Cols<E>::kSlab);
    if (split.bytes > 0 && !workspace) return CX_ERR_NULL;
    if (split.bytes > 0 && workspace_bytes < split.bytes) return CX_ERR_SHAPE;
    if (misaligned_to(f, kElem) || misaligned_to(x, kElem) || misaligned_to(dy, kElem) || misaligned_to(df, kElem) ||
        misaligned_to(dx, kElem) || misaligned_to(states, 4) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const uint64_t states_bytes = B * ceil_div(T, kSteps) * D * 4;
    const typename E::T *outs[2] = {df, dx};
    const int64_t lds[2] = {lddf, lddx};
    for (int k = 0; k < 2; ++k) {
        const uint64_t bytes = span(B * T, lds[k], D, kElem);
        if (share<E>(outs[k], lds[k], f, ldf, B * T, D) || share<E>(outs[k], lds[k], x, ldx, B * T, D) ||
            share<E>(outs[k], lds[k], dy, lddy, B * T, D) || overlap(outs[k], bytes, reset, B * T) || overlap(outs[k], bytes, states, states_bytes) ||
            overlap(outs[k], bytes, dh_last, state_bytes) || overlap(outs[k], bytes, dh0, state_bytes)) return CX_ERR_ALIAS;
    }
    if (share<E>(df, lddf, dx, lddx, B * T, D) || overlap(dh0, state_bytes, states, states_bytes)) return CX_ERR_ALIAS;
    ScanArgs<E> a{};
    a.f = f; a.ldf = ldf; a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.df = df; a.lddf = lddf; a.dx = dx; a.lddx = lddx;
    a.reset = reset; a.states_in = states; a.dh_last = dh_last; a.dh0 = dh0;
    a.maps = static_cast<float *>(workspace);
    a.T_ = T; a.D = D; a.spans = split.spans; a.span_steps = split.span_steps;
    const int64_t pieces = ceil_div(T, kSteps);
    const dim3 grid(static_cast<unsigned>(B), split.spans, static_cast<unsigned>(ceil_div(D, Cols<E>::kSlab)));
    const dim3 block(static_cast<unsigned>(pieces < kMaxWaves ? pieces : kMaxWaves) * kWave);
    if (split.spans > 1) {
        hipLaunchKernelGGL((scan_grad_kernel<E, true>), grid, block, 0, st, a);
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    hipLaunchKernelGGL((scan_grad_kernel<E, false>), grid, block, 0, st, a);
    return launched();
}

}  // namespace

extern "C" {

#define CX_LM_SCAN(SUFFIX, E)                                                                                                         \
    int cx_gated_scan##SUFFIX(const E::T *f, int64_t ldf, const E::T *x, int64_t ldx, E::T *y, int64_t ldy, int64_t B, int64_t T,     \
                              int32_t D, const uint8_t *reset, const float *h0, float *h_last, float *states, void *workspace,        \
                              int64_t workspace_bytes, void *stream)                                                                  \
    {                                                                                                                                 \
        return scan<E>(f, ldf, x, ldx, y, ldy, B, T, D, reset, h0, h_last, states, workspace, workspace_bytes, stream);               \
    }                                                                                                                                 \
    int cx_gated_scan_grad##SUFFIX(const E::T *f, int64_t ldf, const E::T *x, int64_t ldx, const E::T *dy, int64_t lddy, E::T *df,    \
                                   int64_t lddf, E::T *dx, int64_t lddx, int64_t B, int64_t T, int32_t D, const uint8_t *reset,       \
                                   const float *states, const float *dh_last, float *dh0, void *workspace, int64_t workspace_bytes,   \
                                   void *stream)                                                                                      \
    {                                                                                                                                 \
        return scan_grad<E>(f, ldf, x, ldx, dy, lddy, df, lddf, dx, lddx, B, T, D, reset, states, dh_last, dh0, workspace,            \
                            workspace_bytes, stream);                                                                                 \
    }
CX_LM_SCAN(, F32)
CX_LM_SCAN(_bf16, Bf16)
CX_LM_SCAN(_f16, F16)
#undef CX_LM_SCAN

int cx_scan_workspace(int64_t B, int64_t T, int32_t D, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_sizes(B, T, D);
    if (rc != CX_OK || B == 0 || T == 0) return rc;
    const int64_t wide = split_of(B, T, D, Cols<F32>::kSlab).bytes, narrow = split_of(B, T, D, Cols<Bf16>::kSlab).bytes;
    *bytes = wide > narrow ? wide : narrow;
    return CX_OK;
}

}  // extern "C"
