// C-ABI entry points cx_select_scan*, cx_select_workspace: the selective state space scan (see include/cx_lm.h, lm_select.hpp)
//
// Bound by the vector units: a state's step takes an exponential, which counts as two, and four products and sums, 96 issue slots with 16 states (80 without
// results), and a quarter as many again go to what the states share; 94 % of the busy cycles issue one (16 sequences of 2,048 x 1,024 in bfloat16: 87 us
// the maps of three spans in four, 7 what enters, 160 the walk).  Without a split they took 257 us, one wavefront to a SIMD, and 245 with it, before
// padding was kept out of the states (2 %).
#include "lm_select.hpp"

namespace {

enum Pass { kMaps, kWalk };

constexpr int kOutPitch = kColumns + 16;                // the four steps that a column's lanes write lie in different banks

template <class E, int NQ, bool RESETS, Pass PASS>
__global__ __launch_bounds__(kThreads) void select_kernel(const SelectArgs<E> a)
{
    using T = typename E::T;
    constexpr bool MAPS = PASS == kMaps;
    // two tiles in turn: while one is walked the other's elements are computed
    __shared__ alignas(16) float2 step[2][kTile][kColumns];            // delta, delta u
    __shared__ alignas(16) float both[2][kTile][2][kMaxStates];        // B, C
    __shared__ alignas(16) float out[MAPS ? 1 : 2][MAPS ? 1 : kTile][kOutPitch];
    const int64_t b = blockIdx.x / a.slabs, w = static_cast<uint32_t>(b) / a.per_worker, row0 = b * a.T_;
    const int column0 = static_cast<int>(blockIdx.x % a.slabs) * kColumns;
    // maps: piece i of each span; spans may have fewer steps than their pieces' together
    const int parts = a.pieces / a.spans, span = MAPS ? blockIdx.y / parts : blockIdx.y;
    const int64_t span_begin = span * a.span_steps, span_end = span_begin + a.span_steps < a.T_ ? span_begin + a.span_steps : a.T_;
    const int64_t begin = MAPS ? span_begin + (blockIdx.y % parts) * a.piece_steps : span_begin;
    const int64_t end = MAPS && begin + a.piece_steps < span_end ? begin + a.piece_steps : span_end;
    const T *params = a.params + w * a.ldp;
    // elements
    const int es = threadIdx.x / (kColumns / kEach), ec = threadIdx.x % (kColumns / kEach) * kEach, left = a.D - column0 - ec;
    float bias[4], skip[4];
    load_four<E>(params + static_cast<int64_t>(a.D) * a.N + column0 + ec, left, bias);
    load_four<E>(params + static_cast<int64_t>(a.D) * (a.N + 1) + column0 + ec, left, skip);
    close_behind(bias, left);
    // states
    const int q = threadIdx.x / 16 % kQuarters, c = threadIdx.x / kWave * 16 + threadIdx.x % 16, n0 = q * NQ;
    const bool any = column0 + c < a.D;
    const int64_t state = (static_cast<int64_t>(column0) + c) * a.N;   // of a column in [D][N]
    const int64_t of = static_cast<int64_t>(a.D) * a.N, chunks = ceil_div(a.T_, kTile);
    float rate[NQ], h[NQ], sum = 0.0f;
    bool gone = false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        rate[i] = any && n0 + i < a.N ? rate_of(E::widen(params[state + n0 + i])) : 0.0f;
        h[i] = 0.0f;
    }
    if constexpr (!MAPS) {
        if (a.spans > 1) load_states<NQ>(a.maps + (b * a.pieces + span * parts) * of + state, n0, a.N, any, h);
        else if (a.h0) load_states<NQ>(a.h0 + b * of + state, n0, a.N, any, h);
    }
    const int back = back_of<E>(left, a.D), first = ec - back + kEach;      // of loads, from kEach columns before the slab's on
    const uint32_t u_at = place_in<T>(a.ldu, es, first), dt_at = place_in<T>(a.lddt, es, first), z_at = place_in<T>(a.ldz, es, first), y_at = place_in<T>(a.ldy, es, ec);
    const int bs = threadIdx.x / kMaxStates, bp = threadIdx.x % kMaxStates, bn = state_of<NQ>(bp);           // a thread's element of B and of C
    const uint32_t b_at = place_in<T>(a.ldb, bs, bn), c_at = place_in<T>(a.ldc, bs, bn), state_at = (c * a.N) * 4;
    const auto steps_from = [&](int64_t t0) { return end - t0 >= kTile ? kTile : end > t0 ? static_cast<int>(end - t0) : 0; };
    Columns<E, 4> u, dt, z{};
    T b_next, c_next;
    const auto load = [&](int64_t t0) {
        const int64_t row = row0 + t0;
        const int steps = steps_from(t0), there = es < steps ? left : 0;
        const bool has = bn < a.N && bs < steps;
        u = load_back<E>(at_byte(a.u + row * a.ldu + column0 - kEach, u_at), there, back);
        dt = load_back<E>(at_byte(a.dt + row * a.lddt + column0 - kEach, dt_at), there, back);
        b_next = has ? *at_byte(a.bm + row * a.ldb, b_at) : 0;
        if constexpr (!MAPS) {
            if (a.z) z = load_back<E>(at_byte(a.z + row * a.ldz + column0 - kEach, z_at), there, back);
            c_next = has ? *at_byte(a.cm + row * a.ldc, c_at) : 0;
        }
    };
    float gate[4], direct[4];
    const auto elements = [&](int64_t t0, int turn, float (&gates)[4], float (&directs)[4]) {
        const bool there = es < steps_from(t0);
        settle<E>(u, back);
        settle<E>(dt, back);
        if constexpr (!MAPS) settle<E>(z, back);
        float delta[4], enters[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float uj = value_of<E, 4>(u, j), zj = finite_below(value_of<E, 4>(z, j)), soft = softplus(value_of<E, 4>(dt, j) + bias[j]);
            delta[j] = there ? soft : 0.0f;                             // behind the end: a step that changes nothing
            enters[j] = delta[j] == 0.0f ? 0.0f : delta[j] * uj;
            if constexpr (!MAPS) {
                const float open = zj * sigmoid(zj);
                directs[j] = skip[j] * uj;
                gates[j] = a.z ? open : 1.0f;
            }
        }
        put_pairs(&step[turn][es][ec], delta, enters);
        both[turn][bs][0][bp] = E::widen(all_of_step(nothing_of(delta)) ? T(0) : b_next);
        if constexpr (!MAPS) both[turn][bs][1][bp] = E::widen(c_next);
    };
    const auto tile = [&](int64_t t0, auto turn_of) {
        constexpr int turn = decltype(turn_of)::value;
        const int steps = steps_from(t0);
        const unsigned resets = resets_of<RESETS>(a.reset, row0 + t0, steps);
        if constexpr (!MAPS)
            if (a.states) store_states<NQ>(at_byte(a.states + (b * chunks + t0 / kTile) * of + static_cast<int64_t>(column0) * a.N, state_at), n0, a.N, any, h);
        float next_gate[4], next_direct[4], four[4];
        elements(t0 + kTile, !turn, next_gate, next_direct);
        load(t0 + 2 * kTile);
#pragma unroll
        for (int i = 0; i < kTile; ++i) {
            const float2 s = step[turn][i][c];
            const bool cut = RESETS && ((resets >> i) & 1u);
            float y = 0.0f;
#pragma unroll
            for (int j = 0; j < NQ; ++j) {
                const float in = s.y * both[turn][i][0][q * 4 + j], keep = exp2_fast(rate[j] * s.x);
                h[j] = cut ? in : __builtin_fmaf(keep, h[j], in);
                if constexpr (!MAPS) y = __builtin_fmaf(both[turn][i][1][q * 4 + j], h[j], y);
            }
            if constexpr (MAPS) {
                sum += s.x;
            } else {
                four[i % 4] = y;
                if (i % 4 == 3) out[turn][i - 3 + quarter_step(q)][c] = quarters_sum(four);
            }
        }
        if (RESETS) gone = gone || resets != 0;
        __syncthreads();
        if constexpr (!MAPS) {
            float v[4];
            get_four(&out[turn][es][ec], v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = (v[j] + direct[j]) * gate[j];
                gate[j] = next_gate[j];
                direct[j] = next_direct[j];
            }
            if (es < steps) store_columns<E, 4>(at_byte(a.y + (row0 + t0) * a.ldy + column0, y_at), left, v);
        }
    };
    if (begin < end) {
        load(begin);
        elements(begin, 0, gate, direct);
        load(begin + kTile);
        __syncthreads();
    }
    for (int64_t t0 = begin; t0 < end; t0 += 2 * kTile) {
        tile(t0, std::integral_constant<int, 0>{});
        if (t0 + kTile < end) tile(t0 + kTile, std::integral_constant<int, 1>{});
    }
    if constexpr (MAPS) {
        store_states<NQ>(a.maps + (b * a.pieces + blockIdx.y) * of + state, n0, a.N, any, h);
        if (any && q == 0) a.sums[(b * a.pieces + blockIdx.y) * a.D + column0 + c] = gone ? -1.0f : sum;
    } else if (a.h_last && end == a.T_) {
        store_states<NQ>(a.h_last + b * of + state, n0, a.N, any, h);
    }
}

// One step, as decoding takes them: four lanes a column, its states read and written once, nothing shared.
template <class E, int NQ>
__global__ __launch_bounds__(kThreads) void select_step_kernel(const SelectArgs<E> a)
{
    const int64_t b = blockIdx.x / a.slabs, w = static_cast<uint32_t>(b) / a.per_worker;
    const int q = threadIdx.x / 16 % kQuarters, n0 = q * NQ;
    const int d = static_cast<int>(blockIdx.x % a.slabs) * kColumns + threadIdx.x / kWave * 16 + threadIdx.x % 16;
    const bool any = d < a.D;
    const int at = any ? d : 0;
    const int64_t of = static_cast<int64_t>(a.D) * a.N, state = static_cast<int64_t>(at) * a.N;
    const typename E::T *params = a.params + w * a.ldp;
    float h[NQ] = {};
    if (a.h0) load_states<NQ>(a.h0 + b * of + state, n0, a.N, any, h);
    const float u = E::widen(a.u[b * a.ldu + at]), delta = softplus(E::widen(a.dt[b * a.lddt + at]) + E::widen(params[of + at]));
    const float skip = E::widen(params[of + a.D + at]), z = a.z ? E::widen(a.z[b * a.ldz + at]) : 0.0f;
    const bool cut = a.reset && a.reset[b] != 0;
    if (a.states) store_states<NQ>(a.states + b * of + state, n0, a.N, any, h);
    const int here = any ? a.N - n0 : 0;
    const Columns<E, 4> logs = load_columns<E, 4>(params + state + n0, here), bs = load_columns<E, 4>(a.bm + b * a.ldb + n0, here),
                        cs = load_columns<E, 4>(a.cm + b * a.ldc + n0, here);
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const float rate = i < here ? rate_of(value_of<E, 4>(logs, i)) : 0.0f, in = i < here && delta != 0.0f ? delta * u * value_of<E, 4>(bs, i) : 0.0f;
        h[i] = cut ? in : __builtin_fmaf(exp2_fast(rate * delta), h[i], in);
        y = __builtin_fmaf(i < here ? value_of<E, 4>(cs, i) : 0.0f, h[i], y);
    }
    if (a.h_last) store_states<NQ>(a.h_last + b * of + state, n0, a.N, any, h);
    y = add32(y, y);
    y = add16(y, y) + skip * u;
    if (a.z) y *= finite_below(z) * sigmoid(z);
    if (any && q == 0) a.y[b * a.ldy + d] = E::narrow(y);
}

constexpr int64_t kAtOnce = 1024;                       // workgroups that run at a time: four to a CU

Spans forward_spans(int64_t B, int64_t T, int32_t D) { return spans_of(B, T, D, kAtOnce); }

int64_t maps_bytes(int64_t B, int32_t D, int32_t N, const Spans &s) { return s.spans > 1 ? B * s.pieces * D * (N + 1) * 4 : 0; }

template <class E>
int select_scan(const typename E::T *u, int64_t ldu, const typename E::T *dt, int64_t lddt, const typename E::T *bm, int64_t ldb, const typename E::T *cm,
                int64_t ldc, const typename E::T *z, int64_t ldz, const typename E::T *params, int64_t ldp, int32_t W, int64_t offset, typename E::T *y,
                int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t N, const uint8_t *reset, const float *h0, float *h_last, float *states,
                void *workspace, int64_t workspace_bytes, void *stream)
{
    const int rc = check_select(W, B, T, D, N);
    const int64_t count = static_cast<int64_t>(D) * (N + 2), state_bytes = B * D * N * 4;
    if (rc != CX_OK || bad_rows(W, ldp, offset, count)) return CX_ERR_SHAPE;
    if (B == 0) return CX_OK;
    constexpr int kElem = sizeof(typename E::T);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (misaligned_to(h0, 4) || misaligned_to(h_last, 4)) return CX_ERR_ALIGN;
    if (h0 != h_last && overlap(h0, state_bytes, h_last, state_bytes)) return CX_ERR_ALIAS;
    if (T == 0) return pass_through(h0, h_last, state_bytes / 4, st);
    if (!u || !dt || !bm || !cm || !params || !y) return CX_ERR_NULL;
    const int64_t rows = B * T;
    if (bad_strip(rows, ldu, D) || bad_strip(rows, lddt, D) || bad_strip(rows, ldb, N) || bad_strip(rows, ldc, N) || (z && bad_strip(rows, ldz, D)) ||
        bad_strip(rows, ldy, D)) return CX_ERR_SHAPE;
    const Spans s = forward_spans(B, T, D);
    const int64_t bytes = maps_bytes(B, D, N, s);
    if (bytes > 0 && !workspace) return CX_ERR_NULL;
    if (bytes > 0 && workspace_bytes < bytes) return CX_ERR_SHAPE;
    if (misaligned_to(u, kElem) || misaligned_to(dt, kElem) || misaligned_to(bm, kElem) || misaligned_to(cm, kElem) || misaligned_to(z, kElem) ||
        misaligned_to(params, kElem) || misaligned_to(y, kElem) || misaligned_to(states, 4) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const Extent in[8] = {matrix_of(u, rows, ldu, D, kElem), matrix_of(dt, rows, lddt, D, kElem), matrix_of(bm, rows, ldb, N, kElem),
                          matrix_of(cm, rows, ldc, N, kElem), matrix_of(z, rows, ldz, D, kElem), matrix_of(params, W, ldp, offset + count, kElem),
                          dense_of(reset, rows), dense_of(h0, state_bytes)};
    const Extent out[4] = {matrix_of(y, rows, ldy, D, kElem), dense_of(h_last, state_bytes), dense_of(states, B * ceil_div(T, kTile) * D * N * 4),
                           dense_of(workspace, bytes)};
    const Same same[1] = {{1, 7}};
    if (outputs_share_but(in, out, same)) return CX_ERR_ALIAS;
    SelectArgs<E> a{};
    a.u = u; a.ldu = ldu; a.dt = dt; a.lddt = lddt; a.bm = bm; a.ldb = ldb; a.cm = cm; a.ldc = ldc; a.z = z; a.ldz = ldz; a.params = params + offset;
    a.ldp = ldp; a.y = y; a.ldy = ldy; a.reset = reset; a.h0 = h0; a.h_last = h_last; a.states = states; a.B = B; a.T_ = T; a.per_worker = static_cast<uint32_t>(B / W);
    a.D = D; a.N = N; a.slabs = s.slabs; a.spans = s.spans; a.span_steps = s.steps; a.pieces = s.pieces; a.piece_steps = s.piece_steps;
    a.maps = static_cast<float *>(workspace);
    a.sums = a.maps + B * s.pieces * D * N;
    const unsigned groups = static_cast<unsigned>(B * s.slabs);
    if (T == 1)
        return by_states(N, false, [&](auto nq, auto) {
            hipLaunchKernelGGL((select_step_kernel<E, decltype(nq)::value>), dim3(groups), dim3(kThreads), 0, st, a);
        });
    if (s.spans > 1) {
        const int composed = s.pieces - s.pieces / s.spans;     // all but the last span's
        const int rc2 = by_states(N, reset != nullptr, [&](auto nq, auto resets) {
            hipLaunchKernelGGL((select_kernel<E, decltype(nq)::value, decltype(resets)::value, kMaps>), dim3(groups, composed), dim3(kThreads), 0, st, a);
        });
        if (rc2 != CX_OK) return rc2;
        if (enter<E>(a, h0, false, composed, st) != CX_OK) return CX_ERR_HIP;
    }
    return by_states(N, reset != nullptr, [&](auto nq, auto resets) {
        hipLaunchKernelGGL((select_kernel<E, decltype(nq)::value, decltype(resets)::value, kWalk>), dim3(groups, s.spans), dim3(kThreads), 0, st, a);
    });
}

}  // namespace

extern "C" {

#define CX_LM_SELECT(SUFFIX, E)                                                                                                       \
    int cx_select_scan##SUFFIX(const E::T *u, int64_t ldu, const E::T *dt, int64_t lddt, const E::T *bm, int64_t ldb, const E::T *cm, \
                               int64_t ldc, const E::T *z, int64_t ldz, const E::T *params, int64_t ldp, int32_t W, int64_t offset,   \
                               E::T *y, int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t N, const uint8_t *reset,                \
                               const float *h0, float *h_last, float *states, void *workspace, int64_t workspace_bytes, void *stream) \
    {                                                                                                                                 \
        return select_scan<E>(u, ldu, dt, lddt, bm, ldb, cm, ldc, z, ldz, params, ldp, W, offset, y, ldy, B, T, D, N, reset, h0,      \
                              h_last, states, workspace, workspace_bytes, stream);                                                    \
    }
CX_LM_SELECT(, F32)
CX_LM_SELECT(_bf16, Bf16)
CX_LM_SELECT(_f16, F16)
#undef CX_LM_SELECT

int cx_select_workspace(int64_t B, int64_t T, int32_t D, int32_t N, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_select(1, B, T, D, N);
    if (rc == CX_OK && B > 0 && T > 1) *bytes = maps_bytes(B, D, N, forward_spans(B, T, D));
    return rc;
}

}  // extern "C"
