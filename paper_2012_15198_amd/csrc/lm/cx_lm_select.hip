// C-ABI entry points cx_select_scan*, cx_select_workspace: the selective state space scan (see include/cx_lm.h, lm_select.hpp)
#include "lm_select.hpp"

namespace {

enum Pass { kMaps, kWalk };

constexpr int kOutPitch = kColumns + 16;                // the four steps that a column's lanes write lie in different banks

template <class E, int NQ, bool RESETS, Pass PASS>
__global__ __launch_bounds__(kThreads) void select_kernel(const SelectArgs<E> a)
{
    using T = typename E::T;
    constexpr bool MAPS = PASS == kMaps;
    __shared__ alignas(16) float2 step[kTile][kColumns];               // delta, delta u
    __shared__ alignas(16) float both[kTile][2][kMaxStates];           // B, C
    __shared__ alignas(16) float out[MAPS ? 1 : kTile][kOutPitch];
    const int64_t b = blockIdx.x / a.slabs, w = b / a.per_worker, row0 = b * a.T_;
    const int column0 = static_cast<int>(blockIdx.x % a.slabs) * kColumns, span = blockIdx.y;
    const int64_t begin = span * a.span_steps, end = begin + a.span_steps < a.T_ ? begin + a.span_steps : a.T_;
    const T *params = a.params + w * a.ldp;
    // elements
    const int es = threadIdx.x / (kColumns / kEach), ec = threadIdx.x % (kColumns / kEach) * kEach, left = a.D - column0 - ec;
    float bias[4], skip[4];
    load_four<E>(params + static_cast<int64_t>(a.D) * a.N + column0 + ec, left, bias);
    load_four<E>(params + static_cast<int64_t>(a.D) * (a.N + 1) + column0 + ec, left, skip);
    // states
    const int q = threadIdx.x % kQuarters, c = threadIdx.x / kQuarters, n0 = q * NQ;
    const bool any = column0 + c < a.D;
    const int64_t state = (static_cast<int64_t>(column0) + c) * a.N;   // of a column in [D][N]
    float rate[NQ], h[NQ], sum = 0.0f;
    bool gone = false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        rate[i] = any && n0 + i < a.N ? -kLog2e * exp2_fast(kLog2e * E::widen(params[state + n0 + i])) : 0.0f;
        h[i] = 0.0f;
    }
    const int64_t of = static_cast<int64_t>(a.D) * a.N;
    if constexpr (!MAPS) {
        if (a.spans > 1) load_states<NQ>(a.maps + (b * a.spans + span) * of + state, n0, a.N, any, h);
        else if (a.h0) load_states<NQ>(a.h0 + b * of + state, n0, a.N, any, h);
    }
    float u[4], dt[4], z[4], shared_[2];
    const auto load = [&](int64_t t0) {
        const int64_t t = t0 + es;
        const int there = t < end ? left : 0;
        load_four<E>(a.u + (row0 + t) * a.ldu + column0 + ec, there, u);
        load_four<E>(a.dt + (row0 + t) * a.lddt + column0 + ec, there, dt);
        if constexpr (!MAPS)
            if (a.z) load_four<E>(a.z + (row0 + t) * a.ldz + column0 + ec, there, z);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = threadIdx.x + k * kThreads, n = at % kMaxStates, which = at / kMaxStates % 2;
            const int64_t s = t0 + at / (2 * kMaxStates);
            shared_[k] = 0.0f;
            if (n < a.N && s < end && !(MAPS && which)) shared_[k] = E::widen(which ? a.cm[(row0 + s) * a.ldc + n] : a.bm[(row0 + s) * a.ldb + n]);
        }
    };
    load(begin);
    for (int64_t t0 = begin; t0 < end; t0 += kTile) {
        const unsigned resets = resets_of<RESETS>(a.reset, row0 + t0, end - t0 < kTile ? static_cast<int>(end - t0) : kTile);
        const bool there = t0 + es < end;
        float gate[4], direct[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float delta = there ? softplus(dt[j] + bias[j]) : 0.0f;            // behind the end: a step that changes nothing
            step[es][ec + j] = float2{delta, delta * u[j]};
            if constexpr (!MAPS) {
                direct[j] = skip[j] * u[j];
                gate[j] = a.z ? finite_below(z[j]) * sigmoid(z[j]) : 1.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) (&both[0][0][0])[threadIdx.x + k * kThreads] = shared_[k];
        if (t0 + kTile < end) load(t0 + kTile);
        __syncthreads();
        if constexpr (!MAPS)
            if (a.states) store_states<NQ>(a.states + (b * ceil_div(a.T_, kTile) + t0 / kTile) * of + state, n0, a.N, any, h);
        float four[4];
#pragma unroll
        for (int i = 0; i < kTile; ++i) {
            const float2 s = step[i][c];
            const bool cut = RESETS && ((resets >> i) & 1u);
            float y = 0.0f;
#pragma unroll
            for (int j = 0; j < NQ; ++j) {
                const float in = s.y * both[i][0][n0 + j], keep = exp2_fast(rate[j] * s.x);
                h[j] = cut ? in : __builtin_fmaf(keep, h[j], in);
                if constexpr (!MAPS) y = __builtin_fmaf(both[i][1][n0 + j], h[j], y);
            }
            if constexpr (MAPS) {
                sum += s.x;
            } else {
                four[i % 4] = quad_sum(y);
                if (i % 4 == 3) out[i - 3 + q][c] = one_of(q, four[0], four[1], four[2], four[3]);
            }
        }
        if (RESETS) gone = gone || resets != 0;
        __syncthreads();
        if constexpr (!MAPS) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (out[es][ec + j] + direct[j]) * gate[j];
            if (there) store_four<E>(a.y + (row0 + t0 + es) * a.ldy + column0 + ec, left, v);
        }
    }
    if constexpr (MAPS) {
        store_states<NQ>(a.maps + (b * a.spans + span) * of + state, n0, a.N, any, h);
        if (any && q == 0) a.sums[(b * a.spans + span) * a.D + column0 + c] = gone ? -1.0f : sum;
    } else if (a.h_last && end == a.T_) {
        store_states<NQ>(a.h_last + b * of + state, n0, a.N, any, h);
    }
}

// One step, as decoding takes them: four lanes a column, its states read and written once, nothing shared.
template <class E, int NQ>
__global__ __launch_bounds__(kThreads) void select_step_kernel(const SelectArgs<E> a)
{
    const int64_t b = blockIdx.x / a.slabs, w = b / a.per_worker;
    const int d = static_cast<int>(blockIdx.x % a.slabs) * kColumns + threadIdx.x / kQuarters, q = threadIdx.x % kQuarters, n0 = q * NQ;
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
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const bool has = n0 + i < a.N;
        const float rate = has ? -kLog2e * exp2_fast(kLog2e * E::widen(params[state + n0 + i])) : 0.0f;
        const float in = has ? delta * u * E::widen(a.bm[b * a.ldb + n0 + i]) : 0.0f, read = has ? E::widen(a.cm[b * a.ldc + n0 + i]) : 0.0f;
        h[i] = cut ? in : __builtin_fmaf(exp2_fast(rate * delta), h[i], in);
        y = __builtin_fmaf(read, h[i], y);
    }
    if (a.h_last) store_states<NQ>(a.h_last + b * of + state, n0, a.N, any, h);
    y = quad_sum(y) + skip * u;
    if (a.z) y *= finite_below(z) * sigmoid(z);
    if (any && q == 0) a.y[b * a.ldy + d] = E::narrow(y);
}

constexpr int64_t kWanted = 1024, kLeastTiles = 4;      // workgroups of a call; tiles of a span

Spans forward_spans(int64_t B, int64_t T, int32_t D) { return spans_of(B, T, D, kWanted, kLeastTiles); }

int64_t maps_bytes(int64_t B, int32_t D, int32_t N, const Spans &s) { return s.spans > 1 ? B * s.spans * D * (N + 1) * 4 : 0; }

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
    if (T == 0) {
        if (!h_last || h_last == h0) return CX_OK;
        hipLaunchKernelGGL(pass_states_kernel, dim3(static_cast<unsigned>(ceil_div(state_bytes / 4, 256))), dim3(256), 0, st, h0, h_last, state_bytes / 4);
        return launched();
    }
    if (!u || !dt || !bm || !cm || !params || !y) return CX_ERR_NULL;
    const int64_t rows = B * T;
    if (bad_matrix(rows, ldu, D) || bad_matrix(rows, lddt, D) || bad_matrix(rows, ldb, N) || bad_matrix(rows, ldc, N) || (z && bad_matrix(rows, ldz, D)) ||
        bad_matrix(rows, ldy, D)) return CX_ERR_SHAPE;
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
    a.ldp = ldp; a.y = y; a.ldy = ldy; a.reset = reset; a.h0 = h0; a.h_last = h_last; a.states = states; a.B = B; a.T_ = T; a.per_worker = B / W;
    a.D = D; a.N = N; a.slabs = s.slabs; a.spans = s.spans; a.span_steps = s.steps;
    a.maps = static_cast<float *>(workspace);
    a.sums = a.maps + B * s.spans * D * N;
    const unsigned groups = static_cast<unsigned>(B * s.slabs);
    if (T == 1)
        return by_states(N, false, [&](auto nq, auto) {
            hipLaunchKernelGGL((select_step_kernel<E, decltype(nq)::value>), dim3(groups), dim3(kThreads), 0, st, a);
        });
    if (s.spans > 1) {
        const int rc2 = by_states(N, reset != nullptr, [&](auto nq, auto resets) {
            hipLaunchKernelGGL((select_kernel<E, decltype(nq)::value, decltype(resets)::value, kMaps>), dim3(groups, s.spans - 1), dim3(kThreads), 0, st, a);
        });
        if (rc2 != CX_OK) return rc2;
        hipLaunchKernelGGL(enter_kernel<E>, dim3(static_cast<unsigned>(ceil_div(B * D * N, 256))), dim3(256), 0, st, a, h0, false);
        if (launched() != CX_OK) return CX_ERR_HIP;
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
