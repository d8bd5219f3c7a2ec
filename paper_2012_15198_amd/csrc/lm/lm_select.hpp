// What the selective scan and its gradient share (internal header).
//
//   delta_t = softplus(dt_t + bias)    a_t[n] = exp(-delta_t exp(A_log[n]))
//   h_t[n] = a_t[n] (reset_t ? 0 : h_{t-1}[n]) + delta_t B_t[n] u_t    y_t = (sum_n C_t[n] h_t[n] + skip u_t) silu(z_t)
//
// A workgroup takes 64 columns of one sequence and walks its steps in tiles of kTile.  Between barriers it works in two shapes:
//
//   elements   a thread has four columns of one step: it reads them in one piece, computes what belongs to a column alone (delta,
//              the gates) and leaves it in LDS
//   states     four lanes share a column, each with a quarter of its states in registers; they walk the tile's steps, and their
//              sums over states are two additions across lanes
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

// 1 / (1 + e^-v) and log(1 + e^v), both to a few units in the last place at either end: with e = exp(-|v|) <= 1,
// softplus = max(v, 0) + log1p(e), log1p(e) = 2 artanh(e / (2 + e)) by its series (argument at most 1/3).  -inf: 0 and 0.
__device__ __forceinline__ float softplus(float v)
{
    const float e = exp2_fast(-kLog2e * __builtin_fabsf(v)), s = e * rcp_fast(2.0f + e), q = s * s;
    float p = 2.0f / 17;
    p = __builtin_fmaf(p, q, 2.0f / 15);
    p = __builtin_fmaf(p, q, 2.0f / 13);
    p = __builtin_fmaf(p, q, 2.0f / 11);
    p = __builtin_fmaf(p, q, 2.0f / 9);
    p = __builtin_fmaf(p, q, 2.0f / 7);
    p = __builtin_fmaf(p, q, 2.0f / 5);
    p = __builtin_fmaf(p, q, 2.0f / 3);
    p = __builtin_fmaf(p, q, 2.0f);
    return __builtin_fmaf(p, s, v > 0.0f ? v : v != v ? v : 0.0f);
}

template <class E>
struct SelectArgs {
    using T = typename E::T;
    const T *u, *dt, *bm, *cm, *z, *params, *dy;
    T *y, *du, *ddt, *dbm, *dcm, *dz;
    int64_t ldu, lddt, ldb, ldc, ldz, ldp, ldy, lddy, lddu, ldddt, lddb, lddc, lddz;
    const uint8_t *reset;
    const float *h0, *states_in, *dh_last;
    float *h_last, *states, *dh0;
    float *maps;                                        // split: [B][spans][D][N] what a span makes of zeros, then what enters it
    float *sums;                                        // [B][spans][D] sum of delta; below zero: the span forgets what enters
    float *shared_parts, *parts;                        // gradient: [slabs][B][T][2][N] of B and C; [W][parts][D (N + 2)] of the parameters
    int64_t B, T_, per_worker;
    int32_t D, N, slabs, spans;
    int64_t span_steps;                                 // a multiple of kTile
};

// Four columns of a row; `left`: columns from p to the row's end, zeros behind them.
template <class E>
__device__ __forceinline__ void load_four(const typename E::T *p, int left, float (&v)[4])
{
    if constexpr (sizeof(typename E::T) == 4) {
        if (left >= 4) {
            const u4 w = load16<E>(p);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(w[j]);
            return;
        }
    } else {
        if (left >= 4) {
            typedef unsigned u2 __attribute__((ext_vector_type(2)));
            typedef u2 u2_at2 __attribute__((aligned(2)));
            const u2 w = *reinterpret_cast<const u2_at2 *>(p);
            v[0] = E::low(w[0]); v[1] = E::high(w[0]); v[2] = E::low(w[1]); v[3] = E::high(w[1]);
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = j < left ? E::widen(p[j]) : 0.0f;
}
template <class E>
__device__ __forceinline__ void store_four(typename E::T *p, int left, const float (&v)[4])
{
    if (left >= 4) {
        if constexpr (sizeof(typename E::T) == 4) {
            store16<E>(p, u4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
        } else {
            typedef unsigned u2 __attribute__((ext_vector_type(2)));
            typedef u2 u2_at2 __attribute__((aligned(2)));
            *reinterpret_cast<u2_at2 *>(p) = u2{E::two(v[0], v[1]), E::two(v[2], v[3])};
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) p[j] = E::narrow(v[j]);
}

// Sum over the four lanes of a column, in all of them.
template <int PATTERN>
__device__ __forceinline__ float from_quad(float v)
{
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), PATTERN, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_sum(float v)
{
    v += from_quad<0xb1>(v);                            // lanes 1 0 3 2
    return v + from_quad<0x4e>(v);                      // lanes 2 3 0 1
}

// Four steps' sums, one to each of a column's lanes.
__device__ __forceinline__ float one_of(int q, float a, float b, float c, float d)
{
    const float low = (q & 1) ? b : a, high = (q & 1) ? d : c;
    return (q & 2) ? high : low;
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

// What enters each span, in the place of what the span makes of zeros: a thread a state of a column.  `backwards`: the adjoint, from the last
// span on.  What the span at the end makes is not needed.
template <class E>
__global__ __launch_bounds__(256) void enter_kernel(const SelectArgs<E> a, const float *first, bool backwards)
{
    const int64_t of = static_cast<int64_t>(a.D) * a.N, i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= a.B * of) return;
    const int64_t b = i / of, at = i - b * of;
    const int d = static_cast<int>(at / a.N), n = static_cast<int>(at - static_cast<int64_t>(d) * a.N);
    const float rate = -kLog2e * exp2_fast(kLog2e * E::widen(a.params[(b / a.per_worker) * a.ldp + static_cast<int64_t>(d) * a.N + n]));
    float *maps = a.maps + b * a.spans * of + at;
    const float *sums = a.sums + b * a.spans * a.D + d;
    float h = first ? first[i] : 0.0f;
    constexpr int kBatch = 8;                           // loads in flight
    for (int k0 = 0; k0 < a.spans; k0 += kBatch) {
        float S[kBatch], sum[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int step = k0 + k, span = backwards ? a.spans - 1 - step : step;
            if (step + 1 < a.spans) {
                S[k] = maps[span * of];
                sum[k] = sums[static_cast<int64_t>(span) * a.D];
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int step = k0 + k, span = backwards ? a.spans - 1 - step : step;
            if (step < a.spans) maps[span * of] = h;
            if (step + 1 < a.spans) h = sum[k] < 0.0f ? S[k] : __builtin_fmaf(exp2_fast(rate * sum[k]), h, S[k]);
        }
    }
}

// No steps: the state passes through.
__global__ __launch_bounds__(256) void pass_states_kernel(const float *from, float *to, int64_t n)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

[[maybe_unused]] int check_select(int32_t W, int64_t B, int64_t T, int32_t D, int32_t N)
{
    return W < 1 || W > CX_MAX_ROWS || B < 0 || B > CX_MAX_SEQUENCES || B % W != 0 || T < 0 || T > kMaxSeq || D < 1 || D > CX_MAX_WIDTH || N < 1 ||
                   N > kMaxStates || B * D > (int64_t(1) << 31)
               ? CX_ERR_SHAPE
               : CX_OK;
}

struct Spans {
    int32_t slabs, spans;
    int64_t steps;
};

// Workgroups that a call is to have; spans hold at least `least` tiles.
[[maybe_unused]] Spans spans_of(int64_t B, int64_t T, int32_t D, int64_t wanted, int64_t least)
{
    Spans s{};
    s.slabs = static_cast<int32_t>(ceil_div(D, kColumns));
    const int64_t groups = B * s.slabs, tiles = ceil_div(T, kTile);
    int64_t spans = groups >= wanted ? 1 : ceil_div(wanted, groups);
    const int64_t most = tiles / least;
    spans = spans < most ? spans : most;
    if (spans < 1) spans = 1;
    const int64_t span_tiles = ceil_div(tiles, spans);
    s.spans = static_cast<int32_t>(ceil_div(tiles, span_tiles));
    s.steps = span_tiles * kTile;
    return s;
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
    else with(std::integral_constant<int, 4>{});
    return launched();
}

}  // namespace

#endif  // CX_LM_SELECT_HPP
