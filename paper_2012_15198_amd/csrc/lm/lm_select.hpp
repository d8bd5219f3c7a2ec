// What the selective scan and its gradient share (internal header).
//
//   delta_t = softplus(dt_t + bias)    a_t[n] = exp(-delta_t exp(A_log[n]))
//   h_t[n] = a_t[n] (reset_t ? 0 : h_{t-1}[n]) + delta_t B_t[n] u_t    y_t = (sum_n C_t[n] h_t[n] + skip u_t) silu(z_t)
//
// A workgroup takes 64 columns of one sequence and walks its steps in tiles of kTile.  Between barriers it works in two shapes:
//
//   elements   a thread has four columns of one step: it reads them in one piece, computes what belongs to a column alone (delta,
//              the gates) and leaves it in LDS
//   states     four lanes share a column, each with a quarter of its states in registers; they walk the tile's steps, and four steps'
//              sums over states take three exchanges of rows of lanes
//
// The states' map over a span of steps is h -> exp(-exp(A_log) sum of delta) h + S: one number and the N of S.
#ifndef CX_LM_SELECT_HPP
#define CX_LM_SELECT_HPP
#include "lm_block.hpp"

namespace {

constexpr int kTile = CX_SCAN_CHUNK;                    // steps: a state is kept where a tile begins
constexpr int kThreads = 256, kColumns = 64, kQuarters = 4, kEach = 4;     // kEach: columns of a thread in the shape of elements
constexpr int kMaxStates = CX_MAX_STATES;
constexpr int64_t kMaxSeq = CX_MAX_TOKENS;
static_assert(kTile * kColumns == kThreads * kEach && kColumns * kQuarters == kThreads && kMaxStates == 16, "the two shapes");

// log(1 + e^v) within (3 |v| + 24) 2^-24 of itself: with e = exp(-|v|) <= 1 it is max(v, 0) + log1p(e), and log1p(e) = s P(s^2) with
// s = e / (2 + e) <= 1/3 and P(q) = 2 artanh(sqrt q) / sqrt q.  The coefficients are the polynomial of the least largest relative error on
// [0, 1/9] (Remez exchange), 8e-9 after their rounding.  What grows with |v| is the rounding of the exponent.  -inf gives 0.
__device__ __forceinline__ float softplus(float v)
{
    const float e = exp2_fast(-kLog2e * __builtin_fabsf(v)), s = e * rcp_fast(2.0f + e), q = s * s;
    float p = 0x1.208bdp-2f;
    p = __builtin_fmaf(p, q, 0x1.1e510ap-2f);
    p = __builtin_fmaf(p, q, 0x1.99dae6p-2f);
    p = __builtin_fmaf(p, q, 0x1.5554ep-1f);
    p = __builtin_fmaf(p, q, 2.0f);
    return __builtin_fmaf(p, s, __builtin_fmaxf(v, 0.0f));  // a NaN is in s
}

// log2 of what a step of delta = 1 leaves of a state.  Finite where exp(A_log) leaves float32's range, so that its product with a delta of 0 is 0.
__device__ __forceinline__ float rate_of(float a_log) { return finite_below(-kLog2e * exp2_fast(kLog2e * a_log)); }

template <class E>
struct SelectArgs {
    using T = typename E::T;
    const T *u, *dt, *bm, *cm, *z, *params, *dy;
    T *y, *du, *ddt, *dbm, *dcm, *dz;
    int64_t ldu, lddt, ldb, ldc, ldz, ldp, ldy, lddy, lddu, ldddt, lddb, lddc, lddz;
    const uint8_t *reset;
    const float *h0, *states_in, *dh_last;
    float *h_last, *states, *dh0;
    float *maps;                                        // split: [B][pieces][D][N] what a piece of a span makes of zeros, then what enters it
    float *sums;                                        // [B][pieces][D] sum of delta; below zero: the piece forgets what enters
    float *shared_parts, *parts;                        // gradient: [slabs][B][T][2][N] of B and C; [W][parts][D (N + 2)] of the parameters
    int64_t B, T_;
    uint32_t per_worker;                                // sequences of a worker
    int32_t D, N, slabs, spans, pieces;                 // pieces of all spans, as many of each
    int64_t span_steps, piece_steps;                    // multiples of kTile
};

// Rows of a tile have uniform addresses, threads a place in them: 32 bits of bytes, which rows of at most kMaxPitch elements leave room for.
constexpr int64_t kMaxPitch = int64_t(1) << 24;
template <class T>
__device__ __forceinline__ T *at_byte(T *base, uint32_t byte)
{
    using Byte = std::conditional_t<std::is_const_v<T>, const char, char>;
    return reinterpret_cast<T *>(reinterpret_cast<Byte *>(base) + byte);
}
template <class T>
__device__ __forceinline__ uint32_t place_in(int64_t ld, int step, int column) { return (static_cast<uint32_t>(step) * static_cast<uint32_t>(ld) + column) * sizeof(T); }
[[maybe_unused]] bool bad_strip(int64_t rows, int64_t ld, int64_t columns) { return bad_matrix(rows, ld, columns) || ld > kMaxPitch; }

// Where a row of 16-bit elements ends inside a thread's four, they are read as the row's last four and moved into place where they are used: element by
// element the halves would be waited for to be put together.
template <class E>
__device__ __forceinline__ int back_of(int left, int D) { return sizeof(typename E::T) == 2 && left > 0 && left < kEach && D >= kEach ? kEach - left : 0; }
template <class E>
__device__ __forceinline__ Columns<E, 4> load_back(const typename E::T *p, int left, int back)
{
    return load_columns<E, 4>(p, left > 0 ? left + back : 0);
}
template <class E>
__device__ __forceinline__ void settle(Columns<E, 4> &r, int back)
{
    if constexpr (sizeof(typename E::T) == 2) {
        const uint64_t v = (static_cast<uint64_t>(r.w[1]) << 32 | r.w[0]) >> (16 * back);
        r.w[0] = static_cast<unsigned>(v);
        r.w[1] = static_cast<unsigned>(v >> 32);
    }
}

template <class E>
__device__ __forceinline__ void load_four(const typename E::T *p, int left, float (&v)[4]) { widen<E, 4>(load_columns<E, 4>(p, left), v); }

// Four neighbours in LDS in one piece: four writes of one would meet in the same banks.
typedef float f4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void put_four(float *p, const float (&v)[4]) { *reinterpret_cast<f4 *>(p) = f4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void get_four(const float *p, float (&v)[4])
{
    const f4 w = *reinterpret_cast<const f4 *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = w[j];
}
__device__ __forceinline__ void put_pairs(float2 *p, const float (&x)[4], const float (&y)[4])
{
    f4 *to = reinterpret_cast<f4 *>(p);
    to[0] = f4{x[0], y[0], x[1], y[1]};
    to[1] = f4{x[2], y[2], x[3], y[3]};
}

// In LDS the states of a quarter take four places, NQ of them used: whatever NQ is, a lane reads its own in one piece.
template <int NQ>
__device__ __forceinline__ int state_of(int place) { return place % 4 < NQ ? place / 4 * NQ + place % 4 : kMaxStates; }

// Lane 16 q + c of a wavefront has quarter q of the states of its column c.  Sums over quarters cross its four rows of 16 lanes.
// Four steps' sums over the quarters: the one of step quarter_step(q) in quarter q's lanes.
__device__ __forceinline__ float quarters_sum(const float (&v)[4]) { return add16(add32(v[0], v[1]), add32(v[2], v[3])); }
__device__ __forceinline__ int quarter_step(int q) { return (q & 1) * 2 + q / 2; }

// A row of 16 lanes has the elements of one step, and that step's B and C: whether something holds in all of them.  Steps without a delta (padding: dt of
// -inf) take their u and B as 0, the gradient steps without a dy their C, z and u, so that what padding holds does not get out of it.  The rows are
// folded by the scalar unit: over lanes it would take a dozen of the vector unit's slots.
static_assert(kColumns / kEach == 16 && kMaxStates == 16, "a step's threads in either shape");
__device__ __forceinline__ bool all_of_step(bool v)
{
    uint64_t rows = __ballot(v);
#pragma unroll
    for (int k = 1; k < 16; k *= 2) rows &= rows >> k;      // a row's first bit: all of its bits
    rows &= 0x0001000100010001u;
    return __builtin_amdgcn_inverse_ballot_w64((rows << 16) - rows);
}
// Of a step's four deltas or sizes, none below zero: a NaN is not nothing.
__device__ __forceinline__ bool nothing_of(const float (&v)[4]) { return (v[0] + v[1]) + (v[2] + v[3]) == 0.0f; }
// Columns behind D make no steps.
__device__ __forceinline__ void close_behind(float (&bias)[4], int left)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) bias[j] = j < left ? bias[j] : -__builtin_inff();
}

// Bit i: step i of the tile that begins at `row` forgets.
template <bool RESETS>
__device__ __forceinline__ unsigned resets_of(const uint8_t *reset, int64_t row, int steps)
{
    if (!RESETS) return 0;
    const int lane = threadIdx.x & (kWave - 1);
    const bool here = lane < steps && reset[row + lane] != 0;
    return static_cast<unsigned>(__ballot(here));
}

// A lane's states in float [..][D][N] at p, the column's first: what is beyond N or D is zero and not stored.
template <int NQ>
__device__ __forceinline__ void load_states(const float *p, int n0, int N, bool any, float (&h)[NQ])
{
    if (NQ == 4 && any && n0 + 4 <= N) {
        const u4 w = *reinterpret_cast<const u4_at4 *>(p + n0);
#pragma unroll
        for (int i = 0; i < NQ; ++i) h[i] = __uint_as_float(w[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) h[i] = any && n0 + i < N ? p[n0 + i] : 0.0f;
}
template <int NQ>
__device__ __forceinline__ void store_states(float *p, int n0, int N, bool any, const float (&h)[NQ])
{
    if (!any) return;
    if (NQ == 4 && n0 + 4 <= N) {
        *reinterpret_cast<u4_at4 *>(p + n0) = u4{__float_as_uint(h[0]), __float_as_uint(h[1 % NQ]), __float_as_uint(h[2 % NQ]), __float_as_uint(h[3 % NQ])};
        return;
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i)
        if (n0 + i < N) p[n0 + i] = h[i];
}

// What enters each piece, in the place of what the piece makes of zeros.  `backwards`: the adjoint, from the last piece on.  `needed` pieces have
// been composed, in the order of the walk.  A lane has a state of a column; the wavefronts of a workgroup compose a stretch of the pieces each, pass the
// stretches' maps on through LDS and walk theirs again: one after the other 64 pieces of 16,384 states take 13 us.
constexpr int kStretches = 8;
template <class E>
__global__ __launch_bounds__(kWave *kStretches) void enter_kernel(const SelectArgs<E> a, const float *first, bool backwards, int needed)
{
    __shared__ float2 maps_of[kStretches][kWave];       // sum of delta (below zero: forgets), S
    const int lane = threadIdx.x % kWave, stretch = threadIdx.x / kWave, stretches = blockDim.x / kWave;
    const int64_t of = static_cast<int64_t>(a.D) * a.N, at0 = static_cast<int64_t>(blockIdx.x) * kWave + lane, all = a.B * of;
    const int64_t i = at0 < all ? at0 : all - 1;
    const int64_t b = i / of, at = i - b * of;
    const int d = static_cast<int>(at / a.N), n = static_cast<int>(at - static_cast<int64_t>(d) * a.N);
    const float rate = rate_of(E::widen(a.params[(static_cast<uint32_t>(b) / a.per_worker) * a.ldp + static_cast<int64_t>(d) * a.N + n]));
    float *maps = a.maps + b * a.pieces * of + at;
    const float *sums = a.sums + b * a.pieces * a.D + d;
    const int each = (needed + stretches) / stretches, begin = stretch * each;         // of needed + 1 places, the last of which only receives
    const int end = begin + each < needed + 1 ? begin + each : needed + 1;
    const auto place = [&](int k) -> int64_t { return backwards ? a.pieces - 1 - k : k; };
    constexpr int kBatch = 8;                           // loads in flight
    const auto walk = [&](auto &&step) {
        for (int k0 = begin; k0 < end; k0 += kBatch) {
            float S[kBatch], sum[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                S[k] = sum[k] = 0.0f;
                if (k0 + k < end && k0 + k < needed) {
                    S[k] = maps[place(k0 + k) * of];
                    sum[k] = sums[place(k0 + k) * a.D];
                }
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (k0 + k < end) step(k0 + k, S[k], sum[k]);
        }
    };
    const auto apply = [&](float sum, float S, float h) { return sum < 0.0f ? S : __builtin_fmaf(exp2_fast(rate * sum), h, S); };
    float h = 0.0f, total = 0.0f;
    walk([&](int, float S, float sum) {
        h = apply(sum, S, h);
        total = sum < 0.0f || total < 0.0f ? -1.0f : total + sum;
    });
    maps_of[stretch][lane] = float2{total, h};
    __syncthreads();
    h = first ? first[i] : 0.0f;
    for (int k = 0; k < stretch; ++k) h = apply(maps_of[k][lane].x, maps_of[k][lane].y, h);
    if (at0 >= all) return;
    walk([&](int k, float S, float sum) {
        maps[place(k) * of] = h;
        h = apply(sum, S, h);
    });
}
template <class E>
[[maybe_unused]] int enter(const SelectArgs<E> &a, const float *first, bool backwards, int needed, hipStream_t st)
{
    const int stretches = needed < 8 * kStretches ? needed / 8 + 1 : kStretches;             // short ones only wait for each other
    hipLaunchKernelGGL(enter_kernel<E>, dim3(static_cast<unsigned>(ceil_div(a.B * a.D * a.N, kWave))), dim3(kWave * stretches), 0, st, a, first, backwards, needed);
    return launched();
}

[[maybe_unused]] int check_select(int32_t W, int64_t B, int64_t T, int32_t D, int32_t N)
{
    return W < 1 || W > CX_MAX_ROWS || B < 0 || B > CX_MAX_SEQUENCES || B % W != 0 || T < 0 || T > kMaxSeq || D < 1 || D > CX_MAX_WIDTH || N < 1 ||
                   N > kMaxStates || B * D > (int64_t(1) << 29)        // a launch has fewer than 2^32 threads, four to a column
               ? CX_ERR_SHAPE
               : CX_OK;
}

struct Spans {
    int32_t slabs, spans, pieces;
    int64_t steps, piece_steps;
};

// Into how many spans the steps are split: as many as make the rounds of `at_once` workgroups take least, in tiles, with a quarter for the maps' launch
// where there is one.  Spans have at least kLeastTiles tiles.
constexpr int64_t kLeastTiles = 2, kMostSpans = 256, kMapsAtOnce = 1536;
[[maybe_unused]] Spans spans_of(int64_t B, int64_t T, int32_t D, int64_t at_once)
{
    const int64_t slabs = ceil_div(D, kColumns), groups = B * slabs, tiles = ceil_div(T, kTile);
    int64_t best = 1, least = 4 * ceil_div(groups, at_once) * tiles;
    for (int64_t spans = 2; spans <= kMostSpans && spans * kLeastTiles <= tiles && groups < 8 * at_once; ++spans) {
        const int64_t each = ceil_div(tiles, spans), cost = 4 * ceil_div(groups * spans, at_once) * each + ceil_div(groups * (spans - 1), at_once) * each + spans / 4;
        if (cost < least) {
            least = cost;
            best = spans;
        }
    }
    // a span's map is composed of pieces of it, where spans alone would leave the maps' launch short of workgroups
    const int64_t each = ceil_div(tiles, best), spans = ceil_div(tiles, each), others = groups * (spans - 1);
    int64_t parts = spans > 1 ? kMapsAtOnce / others : 1;
    parts = parts < each / kLeastTiles ? parts : each / kLeastTiles;
    if (parts < 1) parts = 1;
    const int64_t piece = ceil_div(each, parts);
    parts = ceil_div(each, piece);
    return {static_cast<int32_t>(slabs), static_cast<int32_t>(spans), static_cast<int32_t>(spans * parts), each * kTile, piece * kTile};
}

template <class F>
[[maybe_unused]] int by_states(int32_t N, bool resets, const F &launch)
{
    const auto with = [&](auto nq) {
        if (resets) launch(nq, std::true_type{});
        else launch(nq, std::false_type{});
    };
    if (N <= 4) with(std::integral_constant<int, 1>{});
    else if (N <= 8) with(std::integral_constant<int, 2>{});
    else if (N <= 12) with(std::integral_constant<int, 3>{});
    else with(std::integral_constant<int, 4>{});
    return launched();
}

}  // namespace

#endif  // CX_LM_SELECT_HPP
