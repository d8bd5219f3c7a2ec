// C-ABI entry points cx_gated_scan*, cx_gated_scan_grad*, cx_scan_workspace: the gated linear recurrence (see include/cx_lm.h)
//
//   a = sigmoid(f)    h_t = a_t * (reset_t ? 0 : h_{t-1}) + (1 - a_t) * x_t    y = round(h)
//   r_t = dL/dh_t = dy_t + keep_{t+1} a_{t+1} r_{t+1}    dx = (1 - a) r    df = r (keep h_{t-1} - x) a (1 - a)
//
// One column's steps are a composition of affine maps h -> A h + S, and compositions associate: the steps are cut into pieces,
// a lane composes the maps of its piece in registers, the pieces' maps are joined through LDS, and the lane then walks its
// piece once more with the state that enters it.  So the data are read once, whatever the length.
//
//   lane       a column of every row (16-bit rows: two where there are enough) and 16 consecutive steps: 64 lanes read whole lines of a
//              row, and a walk needs no exchange between lanes
//   workgroup  8 wavefronts, one piece each = a tile of 128 steps, tile after tile; the loads of the next tile are
//              issued before the present one is computed, into a second set of registers
//   split      where columns are few (workgroups < kSplitBelow) the steps are also split over workgroups: a first launch composes
//              the map of each span (it reads what the second reads again, from the last-level cache where the call fits there)
//
// Bound by memory in long calls (32 sequences of 2,048 x 1,024 in bfloat16: 86 to 90 us, 4.5 TB/s; gradient 139 us, 4.8 TB/s; the forward pass's
// two transcendental instructions an element take half as long as its loads), by the launches' latency and by the second reading where few
// columns are split (one sequence of 16,381 x 1,024: 40 us, 2.5 TB/s), and by the launch for single steps.
//
// States, maps and gates are fp32 throughout; y, df and dx are rounded once.  1 - a comes as exp(-f) a, which keeps its
// relative accuracy where a is near one.  A reset makes a map forget its input: such a map's A carries a sign bit (a
// product of gates has none), and what enters is dropped rather than multiplied by zero, so no NaN or infinity crosses it.
#include "lm_common.hpp"

namespace {

constexpr int kTile = 128;                              // steps of a full tile
constexpr int kSteps = CX_SCAN_CHUNK;                   // steps of a piece: one begins where a state is kept
constexpr int kWaves = kTile / kSteps;
constexpr int kMaxSpans = 64;                           // workgroups that the steps of one column are split over
constexpr int64_t kMaxColumns = CX_MAX_WIDTH, kMaxSeq = CX_MAX_TOKENS;

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

// A lane's columns: one, or of 16-bit rows two, loaded as one pair.  The pair of the last lane of an odd row begins one column
// earlier, at its neighbour's, whose results it does not store.  32-bit offsets: rows have uniform addresses, lanes a place in them.
template <class T>
__device__ __forceinline__ const T &at_byte(const void *row, uint32_t byte) { return *reinterpret_cast<const T *>(static_cast<const char *>(row) + byte); }
template <class T>
__device__ __forceinline__ T &at_byte(void *row, uint32_t byte) { return *reinterpret_cast<T *>(static_cast<char *>(row) + byte); }

// LAST: nothing of the call reads it again.  It then need not stay in the caches, which the results can have.
template <bool LAST, class T>
__device__ __forceinline__ T read(const T &v) { if constexpr (LAST) return __builtin_nontemporal_load(&v); else return v; }

template <class E, int N>
struct LaneColumns;
template <class E>
struct LaneColumns<E, 1> {
    using T = typename E::T;
    uint32_t byte, wide;                                // of the first column in rows of T and of float
    bool any;
    __device__ __forceinline__ LaneColumns(int column, int D)
        : byte((column < D ? column : D - 1) * sizeof(T)), wide((column < D ? column : D - 1) * 4), any(column < D) {}
    __device__ __forceinline__ bool whole() const { return any; }
    template <bool LAST>
    __device__ __forceinline__ T load(const T *row) const { return read<LAST>(at_byte<T>(row, byte)); }
    static __device__ __forceinline__ float value(T w, int) { return E::widen(w); }
    __device__ __forceinline__ void store_whole(T *row, const float (&v)[1]) const { at_byte<T>(row, byte) = E::narrow(v[0]); }
    __device__ __forceinline__ void store(T *row, const float (&v)[1]) const { if (any) store_whole(row, v); }
    __device__ __forceinline__ void load_wide(const float *row, float (&v)[1]) const { v[0] = at_byte<float>(row, wide); }
    __device__ __forceinline__ void store_wide(float *row, const float (&v)[1]) const { if (any) at_byte<float>(row, wide) = v[0]; }
};
template <class E>
struct LaneColumns<E, 2> {                              // at least two columns
    using T = typename E::T;
    uint32_t byte, wide;
    bool any, both;
    __device__ __forceinline__ LaneColumns(int column, int D)
        : byte((column + 2 <= D ? column : D - 2) * 2), wide((column + 2 <= D ? column : D - 2) * 4), any(column < D), both(column + 2 <= D) {}
    __device__ __forceinline__ bool whole() const { return both; }
    template <bool LAST>
    __device__ __forceinline__ unsigned load(const T *row) const { return read<LAST>(at_byte<u1_at2>(row, byte)); }
    static __device__ __forceinline__ float value(unsigned w, int j) { return j ? E::high(w) : E::low(w); }
    __device__ __forceinline__ void store_whole(T *row, const float (&v)[2]) const { at_byte<u1_at2>(row, byte) = E::two(v[0], v[1]); }
    __device__ __forceinline__ void store(T *row, const float (&v)[2]) const
    {
        if (both) store_whole(row, v);
        else if (any) at_byte<T>(row, byte + 2) = E::narrow(v[1]);
    }
    __device__ __forceinline__ void load_wide(const float *row, float (&v)[2]) const
    {
        v[0] = at_byte<float>(row, both ? wide : wide + 4);             // another workgroup may own the column before the last
        v[1] = at_byte<float>(row, wide + 4);
    }
    __device__ __forceinline__ void store_wide(float *row, const float (&v)[2]) const
    {
        if (both) at_byte<float>(row, wide) = v[0];
        if (any) at_byte<float>(row, wide + 4) = v[1];
    }
};
template <class E, int N>
using Word = std::conditional_t<N == 2, unsigned, typename E::T>;      // what a lane loads of a row

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
    int64_t B, T_;
    int32_t D, spans, slabs;
    int64_t span_steps;                                 // a multiple of kTile; the steps of one workgroup
};

// Bit i: step i of the piece forgets; the same for the wavefront.
template <bool RESETS>
__device__ __forceinline__ unsigned reset_bits(const uint8_t *reset, int64_t row, int steps)
{
    if (!RESETS) return 0;
    const int lane = threadIdx.x & (kWave - 1);
    const bool here = lane < steps && reset[row + lane] != 0;
    return static_cast<unsigned>(__ballot(here));
}

template <int N>
struct alignas(8 * N) Maps {                            // of a lane's columns
    Map of[N];
};

template <int N>
struct Exchange {                                       // the maps of the pieces of a tile, two tiles in turn
    Maps<N> map[2][kWaves][kWave];
};

// What enters this wavefront's piece, and what leaves the tile, in the order of the walk.  One barrier.
template <bool RESETS, int N>
__device__ __forceinline__ void join_pieces(Exchange<N> &lds, int turn, int place, int pieces, const Map (&mine)[N], float (&carry)[N],
                                            float (&enters)[N])
{
    const int lane = threadIdx.x & (kWave - 1);
    const auto pass = [&](int k) {
        const Maps<N> m = lds.map[turn][k][lane];
#pragma unroll
        for (int j = 0; j < N; ++j) carry[j] = RESETS ? apply(m.of[j], carry[j]) : __builtin_fmaf(m.of[j].A, carry[j], m.of[j].S);
    };
    if (pieces > 1) {
        Maps<N> m;
#pragma unroll
        for (int j = 0; j < N; ++j) m.of[j] = mine[j];
        lds.map[turn][place][lane] = m;
        __syncthreads();
        for (int k = 0; k < place; ++k) pass(k);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) enters[j] = carry[j];
    if (pieces > 1)
        for (int k = place; k < pieces; ++k) pass(k);
    else
#pragma unroll
        for (int j = 0; j < N; ++j) carry[j] = apply(mine[j], carry[j]);
}

// The map of a tile behind those of the tiles before it (in the order of the walk).  One barrier.
template <int N>
__device__ __forceinline__ void compose_pieces(Exchange<N> &lds, int turn, int place, int pieces, const Map (&mine)[N], Map (&whole)[N])
{
    const int lane = threadIdx.x & (kWave - 1);
    if (pieces > 1) {
        Maps<N> m;
#pragma unroll
        for (int j = 0; j < N; ++j) m.of[j] = mine[j];
        lds.map[turn][place][lane] = m;
        __syncthreads();
        for (int k = 0; k < pieces; ++k) {
            m = lds.map[turn][k][lane];
#pragma unroll
            for (int j = 0; j < N; ++j) whole[j] = then(whole[j], m.of[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) whole[j] = then(whole[j], mine[j]);
    }
}

// What enters this workgroup's span: the maps of the spans on the way to it, applied to what enters the first.  The wavefronts
// compose a part of them each.  Nothing is left in LDS that a later tile's first exchange could meet: a barrier ends it.
template <class E, int N>
__device__ __forceinline__ void entering(const ScanArgs<E> &a, Exchange<N> &lds, const LaneColumns<E, N> &c, int64_t b, int span, bool backwards,
                                         const float *first, float (&h)[N])
{
    if (a.spans == 1) {
        if (first) c.load_wide(first + b * a.D, h);
        else
#pragma unroll
            for (int j = 0; j < N; ++j) h[j] = 0.0f;
        return;
    }
    constexpr int kEach = kMaxSpans / kWaves;    // a split call has all its wavefronts
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x & (kWave - 1);
    const float *maps = a.maps + b * a.spans * 2 * a.D;
    c.load_wide(a.maps + (a.B * a.spans * 2 + b) * a.D, h);
    const int before = backwards ? a.spans - 1 - span : span;
    float A[kEach][N], S[kEach][N];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = wave * kEach + i;
        if (at < before) {
            const float *m = maps + static_cast<int64_t>(backwards ? a.spans - 1 - at : at) * 2 * a.D;
            c.load_wide(m, A[i]);
            c.load_wide(m + a.D, S[i]);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) { A[i][j] = 1.0f; S[i][j] = 0.0f; }
        }
    }
    Maps<N> part;
#pragma unroll
    for (int j = 0; j < N; ++j) part.of[j] = {A[0][j], S[0][j]};
#pragma unroll
    for (int i = 1; i < kEach; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) part.of[j] = then(part.of[j], Map{A[i][j], S[i][j]});
    lds.map[0][wave][lane] = part;
    __syncthreads();
    for (int k = 0; k * kEach < before; ++k) {
        const Maps<N> m = lds.map[0][k][lane];
#pragma unroll
        for (int j = 0; j < N; ++j) h[j] = apply(m.of[j], h[j]);
    }
    __syncthreads();
}

__device__ __forceinline__ int steps_at(int64_t t, int64_t end)
{
    const int64_t left = end - t;
    return left >= kSteps ? kSteps : left > 0 ? static_cast<int>(left) : 0;
}

// The first `steps` rows of a piece, at row `row` of the matrix.
template <bool LAST, class E, int N>
__device__ __forceinline__ void load_piece(const LaneColumns<E, N> &c, const typename E::T *m, int64_t ld, int64_t row, int steps, Word<E, N> (&v)[kSteps])
{
    const typename E::T *p = m + row * ld;
    if (steps >= kSteps) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) v[i] = c.template load<LAST>(p + i * ld);
    } else {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) v[i] = i < steps ? c.template load<LAST>(p + i * ld) : 0;
    }
}

template <class E, int N>
__device__ __forceinline__ void store_map(const ScanArgs<E> &a, const LaneColumns<E, N> &c, int64_t b, int span, const Map (&whole)[N])
{
    float A[N], S[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { A[j] = whole[j].A; S[j] = whole[j].S; }
    float *m = a.maps + (b * a.spans + span) * 2 * a.D;
    c.store_wide(m, A);
    c.store_wide(m + a.D, S);
}

// What enters the first span of a split call goes to the workspace: the second launch may replace it (h_last may be h0).
template <class E, int N>
__device__ __forceinline__ void keep_first(const ScanArgs<E> &a, const LaneColumns<E, N> &c, int64_t b, const float *first)
{
    float h[N] = {};
    if (first) c.load_wide(first + b * a.D, h);
    c.store_wide(a.maps + (a.B * a.spans * 2 + b) * a.D, h);
}

template <bool V>
using Flag = std::integral_constant<bool, V>;

// What a launch does: a whole call, or of a split one the spans' maps or the spans.  Reading past the caches is for the whole call: 32 sequences of
// 2,048 x 1,024 take 86 us in bfloat16 against 99, their gradient 139 against 150 (float32 164 and 171, 276 and 279); in a split one, whose
// two launches read the same, one sequence of 16,381 x 1,024 would take 47 against 40.
enum Pass { kWhole, kMaps, kSpans };

// Grid (slabs of columns of sequences, spans): workgroups that run together read whole rows.  kMaps: the first launch of a split call,
// over the spans that another one follows.
template <class E, int N, bool RESETS, Pass PASS>
__global__ __launch_bounds__(kWaves *kWave, N == 1 ? 4 : 2) void scan_kernel(const ScanArgs<E> a)
{
    constexpr bool ONLY_MAP = PASS == kMaps, LAST = PASS == kWhole;
    __shared__ Exchange<N> lds;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int64_t b = blockIdx.x / a.slabs;
    const int span = blockIdx.y, slab = static_cast<int>(blockIdx.x) % a.slabs;
    const LaneColumns<E, N> c((slab * kWave + lane) * N, a.D);
    const bool whole_lanes = __ballot(c.whole()) == ~0ull;
    const int64_t row0 = b * a.T_, begin = span * a.span_steps, end = begin + a.span_steps < a.T_ ? begin + a.span_steps : a.T_;
    const int tile = waves * kSteps;
    Word<E, N> fw[2][kSteps], xw[2][kSteps];
    int64_t t = begin + wave * kSteps;                   // of the piece whose rows were loaded last
    int steps = steps_at(t, end);
    load_piece<LAST>(c, a.f, a.ldf, row0 + t, steps, fw[0]);
    load_piece<LAST>(c, a.x, a.ldx, row0 + t, steps, xw[0]);
    float carry[N];
    Map whole[N];
    if constexpr (ONLY_MAP) {
        if (blockIdx.y == 0 && wave == 0) keep_first<E, N>(a, c, b, a.h0);
#pragma unroll
        for (int j = 0; j < N; ++j) whole[j] = {1.0f, 0.0f};
    } else {
        entering<E>(a, lds, c, b, span, false, a.h0, carry);
    }
    const auto one_tile = [&](auto turn_flag) {
        constexpr int turn = decltype(turn_flag)::value;
        const int64_t t_now = t;
        const int steps_now = steps;
        const unsigned resets = reset_bits<RESETS>(a.reset, row0 + t_now, steps_now);
        t += tile;
        steps = steps_at(t, end);
        load_piece<LAST>(c, a.f, a.ldf, row0 + t, steps, fw[!turn]);
        load_piece<LAST>(c, a.x, a.ldx, row0 + t, steps, xw[!turn]);
        float keep[kSteps][N], in[kSteps][N];
        Map mine[N];
#pragma unroll
        for (int j = 0; j < N; ++j) mine[j] = {1.0f, 0.0f};
        const auto maps = [&](auto full) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (!decltype(full)::value && i >= steps_now) break;
                const bool cut = RESETS && ((resets >> i) & 1u);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const Gate g = gate(c.value(fw[turn][i], j));
                    keep[i][j] = g.a;
                    in[i][j] = g.b * c.value(xw[turn][i], j);
                    mine[j].S = cut ? in[i][j] : __builtin_fmaf(g.a, mine[j].S, in[i][j]);
                    mine[j].A = cut ? -1.0f : g.a * mine[j].A;
                }
            }
        };
        if (steps_now == kSteps) maps(Flag<true>{}); else maps(Flag<false>{});
        if constexpr (ONLY_MAP) {
            compose_pieces(lds, turn, wave, waves, mine, whole);
        } else {
            float h[N];
            join_pieces<RESETS>(lds, turn, wave, waves, mine, carry, h);
            if (a.states && steps_now > 0)
                c.store_wide(a.states + (b * ceil_div(a.T_, kSteps) + t_now / kSteps) * a.D, h);
            typename E::T *out = a.y + (row0 + t_now) * a.ldy;
            const auto walk = [&](auto full) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    if (!decltype(full)::value && i >= steps_now) break;
                    const bool cut = RESETS && ((resets >> i) & 1u);
#pragma unroll
                    for (int j = 0; j < N; ++j) h[j] = cut ? in[i][j] : __builtin_fmaf(keep[i][j], h[j], in[i][j]);
                    if (decltype(full)::value) c.store_whole(out + i * a.ldy, h); else c.store(out + i * a.ldy, h);
                }
            };
            if (steps_now == kSteps && whole_lanes) walk(Flag<true>{}); else walk(Flag<false>{});
        }
    };
    for (int64_t tile0 = begin; tile0 < end; tile0 += 2 * tile) {
        one_tile(Flag<false>{});
        if (tile0 + tile < end) one_tile(Flag<true>{});
    }
    if constexpr (ONLY_MAP) {
        if (wave == 0) store_map<E>(a, c, b, span, whole);
    } else if (a.h_last && end == a.T_ && wave == waves - 1) {
        c.store_wide(a.h_last + b * a.D, carry);
    }
}

// The gradient, from the last step to the first.  What a piece hands to the one before it is keep a r of its first step.
template <class E, int N, bool RESETS, Pass PASS>
__global__ __launch_bounds__(kWaves *kWave) void scan_grad_kernel(const ScanArgs<E> a)
{
    constexpr bool ONLY_MAP = PASS == kMaps, LAST = PASS == kWhole;
    __shared__ Exchange<N> lds;
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int64_t b = blockIdx.x / a.slabs;
    const int span = blockIdx.y + (ONLY_MAP ? 1 : 0), slab = static_cast<int>(blockIdx.x) % a.slabs;
    const LaneColumns<E, N> c((slab * kWave + lane) * N, a.D);
    const bool whole_lanes = __ballot(c.whole()) == ~0ull;
    const int64_t row0 = b * a.T_, begin = span * a.span_steps, end = begin + a.span_steps < a.T_ ? begin + a.span_steps : a.T_;
    const int tile = waves * kSteps;
    Word<E, N> fw[2][kSteps], xw[2][kSteps], gw[2][kSteps];
    int64_t tile0 = begin + (end - 1 - begin) / tile * tile;
    int64_t t = tile0 + wave * kSteps;
    int steps = steps_at(t, end);
    float entered[2][N];                                // the state before the piece
    const auto load = [&](auto turn_flag) {
        constexpr int turn = decltype(turn_flag)::value;
        load_piece<LAST>(c, a.f, a.ldf, row0 + t, steps, fw[turn]);
        load_piece<LAST>(c, a.dy, a.lddy, row0 + t, steps, gw[turn]);
        if constexpr (!ONLY_MAP) {
            load_piece<LAST>(c, a.x, a.ldx, row0 + t, steps, xw[turn]);
            if (steps > 0) c.load_wide(a.states_in + (b * ceil_div(a.T_, kSteps) + t / kSteps) * a.D, entered[turn]);
        }
    };
    load(Flag<false>{});
    float carry[N];
    Map whole[N];
    if constexpr (ONLY_MAP) {
        if (blockIdx.y == 0 && wave == 0) keep_first<E, N>(a, c, b, a.dh_last);
#pragma unroll
        for (int j = 0; j < N; ++j) whole[j] = {1.0f, 0.0f};
    } else {
        entering<E>(a, lds, c, b, span, true, a.dh_last, carry);
    }
    const auto one_tile = [&](auto turn_flag) {
        constexpr int turn = decltype(turn_flag)::value;
        const int64_t t_now = t;
        const int steps_now = steps;
        const unsigned resets = reset_bits<RESETS>(a.reset, row0 + t_now, steps_now);
        t -= tile;
        steps = tile0 > begin ? kSteps : 0;
        load(Flag<!turn>{});
        float keep[kSteps][N], open[kSteps][N], pull[kSteps][N];     // pull: a (keep h - x)
        Map mine[N];
#pragma unroll
        for (int j = 0; j < N; ++j) mine[j] = {1.0f, 0.0f};
        const auto maps = [&](auto full) {
            float h[N];
#pragma unroll
            for (int j = 0; j < N; ++j) h[j] = ONLY_MAP ? 0.0f : entered[turn][j];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (!decltype(full)::value && i >= steps_now) break;
                const bool cut = RESETS && ((resets >> i) & 1u);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const Gate g = gate(c.value(fw[turn][i], j));
                    keep[i][j] = g.a;
                    if constexpr (!ONLY_MAP) {
                        const float x = c.value(xw[turn][i], j), in = g.b * x;
                        open[i][j] = g.b;
                        pull[i][j] = ((cut ? 0.0f : h[j]) - x) * g.a;
                        h[j] = cut ? in : __builtin_fmaf(g.a, h[j], in);
                    }
                }
            }
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                if (!decltype(full)::value && i >= steps_now) continue;
                const bool cut = RESETS && ((resets >> i) & 1u);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    mine[j].S = cut ? 0.0f : keep[i][j] * (c.value(gw[turn][i], j) + mine[j].S);
                    mine[j].A = cut ? -1.0f : keep[i][j] * mine[j].A;
                }
            }
        };
        if (steps_now == kSteps) maps(Flag<true>{}); else maps(Flag<false>{});
        if constexpr (ONLY_MAP) {
            compose_pieces(lds, turn, waves - 1 - wave, waves, mine, whole);
        } else {
            float r[N];
            join_pieces<RESETS>(lds, turn, waves - 1 - wave, waves, mine, carry, r);
            typename E::T *df = a.df + (row0 + t_now) * a.lddf, *dx = a.dx + (row0 + t_now) * a.lddx;
            const auto walk = [&](auto full) {
#pragma unroll
                for (int i = kSteps - 1; i >= 0; --i) {
                    if (!decltype(full)::value && i >= steps_now) continue;
                    const bool cut = RESETS && ((resets >> i) & 1u);
                    float f_out[N], x_out[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float g = c.value(gw[turn][i], j) + r[j];
                        x_out[j] = open[i][j] * g;
                        f_out[j] = pull[i][j] * x_out[j];
                        r[j] = cut ? 0.0f : keep[i][j] * g;
                    }
                    if (decltype(full)::value) {
                        c.store_whole(df + i * a.lddf, f_out);
                        c.store_whole(dx + i * a.lddx, x_out);
                    } else {
                        c.store(df + i * a.lddf, f_out);
                        c.store(dx + i * a.lddx, x_out);
                    }
                }
            };
            if (steps_now == kSteps && whole_lanes) walk(Flag<true>{}); else walk(Flag<false>{});
        }
        tile0 -= tile;
    };
    while (tile0 >= begin) {
        one_tile(Flag<false>{});
        if (tile0 >= begin) one_tile(Flag<true>{});
    }
    if constexpr (ONLY_MAP) {
        if (wave == 0) store_map<E>(a, c, b, span, whole);
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

// One step, as decoding takes them: an element to a thread, all loads at once, where a walk waits for the state that enters and then steps
// over 15 absent ones.  64 sequences of 2,048 columns take 2.5 us in bfloat16 against a walk's 4.3, 4,096 of 4,096 56 to 63 against 212 (4 TB/s).
template <class E>
__global__ __launch_bounds__(256) void step_kernel(const ScanArgs<E> a)
{
    const int64_t b = blockIdx.x / a.slabs;
    const int64_t d = static_cast<int64_t>(blockIdx.x % a.slabs) * blockDim.x + threadIdx.x;
    if (d >= a.D) return;
    const Gate g = gate(E::widen(a.f[b * a.ldf + d]));
    const float enters = a.h0 ? a.h0[b * a.D + d] : 0.0f, in = g.b * E::widen(a.x[b * a.ldx + d]);
    const float h = a.reset && a.reset[b] != 0 ? in : __builtin_fmaf(g.a, enters, in);
    if (a.states) a.states[b * a.D + d] = enters;
    a.y[b * a.ldy + d] = E::narrow(h);
    if (a.h_last) a.h_last[b * a.D + d] = h;
}

// Workgroups from which the steps are not split: fewer leave CUs idle for longer than a second reading takes.
constexpr int64_t kSplitBelow = 128, kUnits = 256;

// Columns of a lane.  Two of 16 bits halve the loads.  One makes twice the workgroups, which is more where even those do not fill the card:
// forward 16 sequences of 2,048 x 1,024 take 56 us in bfloat16 against 74 with two, 6 of 1,111 x 515 19 against 25; more than kUnits gain
// nothing (18 sequences: 76 and 75).  The gradient's split costs less, so that it gains only where one column fills the card without a
// split (16 sequences 90 us against 103, 12: 83 against 87, but 10: 83 against 69).  Up to 64 columns two would leave half the lanes idle
// (64 sequences of 1,024 x 64: 16 us against 22, gradient 21 against 26).
template <class E>
int columns_of_lane(int64_t B, int32_t D, bool forward)
{
    if (sizeof(typename E::T) == 4 || D <= kWave) return 1;
    const int64_t groups = B * ceil_div(D, kWave);
    return groups > kUnits || (!forward && groups < kUnits * 3 / 4) ? 2 : 1;
}

struct Split {
    int spans;
    int64_t span_steps, bytes;
};

// Split calls become as many workgroups as the CUs take at once, one each, or two of the forward pass on single columns: one sequence of
// 16,381 x 1,024 takes 40 us forward in bfloat16 with 512 and 49 with 256, in float32 63 and 68.
template <class E>
Split split_of(int64_t B, int64_t T, int32_t D, bool forward)
{
    const int lane_columns = columns_of_lane<E>(B, D, forward);
    const bool two = forward && lane_columns == 1;
    const int64_t groups = B * ceil_div(D, kWave * lane_columns), tiles = ceil_div(T, kTile);
    int64_t spans = groups < kSplitBelow || (two && groups == kSplitBelow) ? (two ? 2 * kUnits : kUnits) / groups : 1;
    spans = spans < tiles ? spans : tiles;
    spans = spans < kMaxSpans ? spans : kMaxSpans;
    if (spans <= 1) return {1, round_up(T, kTile), 0};
    const int64_t span_tiles = ceil_div(tiles, spans);
    spans = ceil_div(tiles, span_tiles);
    return {static_cast<int>(spans), span_tiles * kTile, spans > 1 ? (B * spans * 2 + B) * D * 4 : 0};
}

int check_sizes(int64_t B, int64_t T, int32_t D)
{
    return B < 0 || B > CX_MAX_SEQUENCES || B * D > (int64_t(1) << 31) || T < 0 || T > kMaxSeq || D < 1 || D > kMaxColumns ? CX_ERR_SHAPE : CX_OK;
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
    const Split split = split_of<E>(B, T, D, true);
    if (split.bytes > 0 && !workspace) return CX_ERR_NULL;
    if (split.bytes > 0 && workspace_bytes < split.bytes) return CX_ERR_SHAPE;
    if (misaligned_to(f, kElem) || misaligned_to(x, kElem) || misaligned_to(y, kElem) || misaligned_to(states, 4) ||
        misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const Extent in[4] = {matrix_of(f, B * T, ldf, D, kElem), matrix_of(x, B * T, ldx, D, kElem), dense_of(reset, B * T), dense_of(h0, state_bytes)};
    const Extent out[4] = {matrix_of(y, B * T, ldy, D, kElem), dense_of(h_last, state_bytes), dense_of(states, B * ceil_div(T, kSteps) * D * 4),
                           dense_of(workspace, split.bytes)};
    if (outputs_share(in, out, 1, 3)) return CX_ERR_ALIAS;
    ScanArgs<E> a{};
    a.f = f; a.ldf = ldf; a.x = x; a.ldx = ldx; a.y = y; a.ldy = ldy;
    a.reset = reset; a.h0 = h0; a.h_last = h_last; a.states = states;
    a.maps = static_cast<float *>(workspace);
    a.B = B; a.T_ = T; a.D = D; a.spans = split.spans; a.span_steps = split.span_steps;
    if (T == 1) {
        const int threads = D < 256 ? static_cast<int>(round_up(D, kWave)) : 256;
        a.slabs = static_cast<int32_t>(ceil_div(D, threads));
        hipLaunchKernelGGL((step_kernel<E>), dim3(static_cast<unsigned>(B * a.slabs)), dim3(threads), 0, st, a);
        return launched();
    }
    a.slabs = static_cast<int32_t>(ceil_div(D, kWave * columns_of_lane<E>(B, D, true)));
    const int64_t pieces = ceil_div(T, kSteps);
    const dim3 grid(static_cast<unsigned>(B * a.slabs), split.spans), maps(grid.x, split.spans - 1);
    const dim3 block(static_cast<unsigned>(pieces < kWaves ? pieces : kWaves) * kWave);
    const auto launch = [&](auto lane_columns) -> int {
        constexpr int N = decltype(lane_columns)::value;
        if constexpr (N == 1) {                         // two columns are taken by calls of too many workgroups for a split
            if (split.spans > 1) {
                if (reset) hipLaunchKernelGGL((scan_kernel<E, N, true, kMaps>), maps, block, 0, st, a);
                else hipLaunchKernelGGL((scan_kernel<E, N, false, kMaps>), maps, block, 0, st, a);
                if (launched() != CX_OK) return CX_ERR_HIP;
                if (reset) hipLaunchKernelGGL((scan_kernel<E, N, true, kSpans>), grid, block, 0, st, a);
                else hipLaunchKernelGGL((scan_kernel<E, N, false, kSpans>), grid, block, 0, st, a);
                return launched();
            }
        }
        if (reset) hipLaunchKernelGGL((scan_kernel<E, N, true, kWhole>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((scan_kernel<E, N, false, kWhole>), grid, block, 0, st, a);
        return launched();
    };
    if constexpr (sizeof(typename E::T) == 2)
        if (columns_of_lane<E>(B, D, true) == 2) return launch(std::integral_constant<int, 2>{});
    return launch(std::integral_constant<int, 1>{});
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
    const Split split = split_of<E>(B, T, D, false);
    if (split.bytes > 0 && !workspace) return CX_ERR_NULL;
    if (split.bytes > 0 && workspace_bytes < split.bytes) return CX_ERR_SHAPE;
    if (misaligned_to(f, kElem) || misaligned_to(x, kElem) || misaligned_to(dy, kElem) || misaligned_to(df, kElem) ||
        misaligned_to(dx, kElem) || misaligned_to(states, 4) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const Extent in[6] = {matrix_of(f, B * T, ldf, D, kElem), matrix_of(x, B * T, ldx, D, kElem), matrix_of(dy, B * T, lddy, D, kElem), dense_of(reset, B * T),
                          dense_of(states, B * ceil_div(T, kSteps) * D * 4), dense_of(dh_last, state_bytes)};
    const Extent out[4] = {matrix_of(df, B * T, lddf, D, kElem), matrix_of(dx, B * T, lddx, D, kElem), dense_of(dh0, state_bytes),
                           dense_of(workspace, split.bytes)};
    if (outputs_share(in, out, 2, 5)) return CX_ERR_ALIAS;
    ScanArgs<E> a{};
    a.f = f; a.ldf = ldf; a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.df = df; a.lddf = lddf; a.dx = dx; a.lddx = lddx;
    a.reset = reset; a.states_in = states; a.dh_last = dh_last; a.dh0 = dh0;
    a.maps = static_cast<float *>(workspace);
    a.B = B; a.T_ = T; a.D = D; a.spans = split.spans; a.span_steps = split.span_steps;
    a.slabs = static_cast<int32_t>(ceil_div(D, kWave * columns_of_lane<E>(B, D, false)));
    const int64_t pieces = ceil_div(T, kSteps);
    const dim3 grid(static_cast<unsigned>(B * a.slabs), split.spans), maps(grid.x, split.spans - 1);
    const dim3 block(static_cast<unsigned>(pieces < kWaves ? pieces : kWaves) * kWave);
    const auto launch = [&](auto lane_columns) -> int {
        constexpr int N = decltype(lane_columns)::value;
        if (split.spans > 1) {
            if (reset) hipLaunchKernelGGL((scan_grad_kernel<E, N, true, kMaps>), maps, block, 0, st, a);
            else hipLaunchKernelGGL((scan_grad_kernel<E, N, false, kMaps>), maps, block, 0, st, a);
            if (launched() != CX_OK) return CX_ERR_HIP;
            if (reset) hipLaunchKernelGGL((scan_grad_kernel<E, N, true, kSpans>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((scan_grad_kernel<E, N, false, kSpans>), grid, block, 0, st, a);
            return launched();
        }
        if (reset) hipLaunchKernelGGL((scan_grad_kernel<E, N, true, kWhole>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((scan_grad_kernel<E, N, false, kWhole>), grid, block, 0, st, a);
        return launched();
    };
    if constexpr (sizeof(typename E::T) == 2)
        if (columns_of_lane<E>(B, D, false) == 2) return launch(std::integral_constant<int, 2>{});
    return launch(std::integral_constant<int, 1>{});
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
    for (const int64_t n : {split_of<F32>(B, T, D, true).bytes, split_of<F32>(B, T, D, false).bytes, split_of<Bf16>(B, T, D, true).bytes,
                            split_of<Bf16>(B, T, D, false).bytes})
        *bytes = n > *bytes ? n : *bytes;
    return CX_OK;
}

}  // extern "C"
