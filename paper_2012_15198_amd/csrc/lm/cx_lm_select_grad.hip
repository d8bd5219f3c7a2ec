// C-ABI entry points cx_select_scan_grad*, cx_select_grad_workspace: the gradient of the selective scan (see include/cx_lm.h, lm_select.hpp)
//
// With g_t = dy_t silu(z_t), r_t[n] = dL/dh_t[n], keep_t = (reset_t ? 0 : a_t) and A = -exp(A_log):
//
//   r_t = C_t g_t + keep_{t+1} r_{t+1}    into_t = sum_n r_t B_t    across_t = sum_n r_t A keep_t h_{t-1}
//   du = delta into + skip g    ddt = (across + u into) sigmoid(dt + bias)    dz = dy y' silu'(z), y' the result before its gate
//   dB_t = sum over columns of r_t delta_t u_t    dC_t = sum over columns of h_t g_t
//   dA_log = A sum_t r_t delta_t keep_t h_{t-1}    dbias = sum_t ddt    dskip = sum_t g u
//
// A tile's states are computed again from the one kept where it begins and stay in registers; the walk back meets them there.
#include "lm_select.hpp"

namespace {

enum Pass { kMaps, kWalk };

constexpr int kOutPitch = kColumns + 16;                // the four steps that a column's lanes write lie in different banks
constexpr int kWaves = kThreads / kWave;

// The sums of 2 NQ values over the 16 columns of a wavefront (lanes of equal q), each value's in some lanes: two exchanges leave a lane half of
// the values each, rotations of rows the rest.  `which`: B or C; `j`: the state; `holds`: this lane is the one to write it.
template <int NQ>
struct Reduced {
    float v;
    int which, j;
    bool holds;
};
__device__ __forceinline__ float add32(float x, float y)               // lanes 0 to 31: x of both halves, 32 to 63: y
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add16(float x, float y)               // even rows of 16 lanes: x of the row and the next, odd ones: y
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int BY>
__device__ __forceinline__ float add_turned(float v)                   // with the lane BY places on in its row of 16
{
    return v + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x120 + BY, 0xf, 0xf, true));
}
template <int NQ>
__device__ __forceinline__ Reduced<NQ> reduce_columns(const float (&pb)[NQ], const float (&pc)[NQ])
{
    const int lane = threadIdx.x & (kWave - 1);
    Reduced<NQ> r;
    r.which = lane >> 5;
    if constexpr (NQ == 4) {
        const float first = add_turned<4>(add_turned<8>(add16(add32(pb[0], pc[0]), add32(pb[1], pc[1]))));
        const float second = add_turned<4>(add_turned<8>(add16(add32(pb[2], pc[2]), add32(pb[3], pc[3]))));
        r.v = (lane & 8) ? second : first;
        r.j = ((lane >> 4) & 1) + ((lane >> 2) & 2);
        r.holds = (lane & 4) == 0;
    } else if constexpr (NQ == 2) {
        r.v = add_turned<4>(add_turned<8>(add16(add32(pb[0], pc[0]), add32(pb[1], pc[1]))));
        r.j = (lane >> 4) & 1;
        r.holds = (lane & 12) == 0;
    } else {
        const float t = add32(pb[0], pc[0]);
        r.v = add_turned<4>(add_turned<8>(add16(t, t)));
        r.j = 0;
        r.holds = (lane & 28) == 0;
    }
    return r;
}

template <class E, int NQ, bool RESETS, Pass PASS>
__global__ __launch_bounds__(kThreads, 2) void select_grad_kernel(const SelectArgs<E> a)
{
    using T = typename E::T;
    constexpr bool MAPS = PASS == kMaps;
    __shared__ alignas(16) float2 step[kTile][kColumns];               // delta, delta u
    __shared__ alignas(16) float pull[kTile][kColumns];                // g
    __shared__ alignas(16) float both[kTile][2][kMaxStates];           // B, C
    __shared__ alignas(16) float out[MAPS ? 1 : 3][MAPS ? 1 : kTile][kOutPitch];       // y', into, across
    __shared__ alignas(16) float shares[MAPS ? 1 : kWaves][kTile][2][kMaxStates];      // dB, dC of a wavefront's columns
    const int64_t b = blockIdx.x / a.slabs, w = b / a.per_worker, row0 = b * a.T_;
    const int slab = static_cast<int>(blockIdx.x % a.slabs), column0 = slab * kColumns, span = blockIdx.y + (MAPS ? 1 : 0);
    const int64_t begin = span * a.span_steps, end = begin + a.span_steps < a.T_ ? begin + a.span_steps : a.T_;
    const T *params = a.params + w * a.ldp;
    const int es = threadIdx.x / (kColumns / kEach), ec = threadIdx.x % (kColumns / kEach) * kEach, left = a.D - column0 - ec;
    float bias[4], skip[4], dbias[4] = {}, dskip[4] = {};
    load_four<E>(params + static_cast<int64_t>(a.D) * a.N + column0 + ec, left, bias);
    load_four<E>(params + static_cast<int64_t>(a.D) * (a.N + 1) + column0 + ec, left, skip);
    const int q = threadIdx.x % kQuarters, c = threadIdx.x / kQuarters, n0 = q * NQ, wave = threadIdx.x / kWave;
    const bool any = column0 + c < a.D;
    const int64_t state = (static_cast<int64_t>(column0) + c) * a.N, of = static_cast<int64_t>(a.D) * a.N, chunks = ceil_div(a.T_, kTile);
    float rate[NQ], carry[NQ], drate[NQ] = {}, sum = 0.0f;
    bool gone = false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        rate[i] = any && n0 + i < a.N ? -kLog2e * exp2_fast(kLog2e * E::widen(params[state + n0 + i])) : 0.0f;
        carry[i] = 0.0f;
    }
    if constexpr (!MAPS) {
        if (a.spans > 1) load_states<NQ>(a.maps + (b * a.spans + span) * of + state, n0, a.N, any, carry);
        else if (a.dh_last) load_states<NQ>(a.dh_last + b * of + state, n0, a.N, any, carry);
    }
    float u[4], dt[4], z[4] = {}, dy[4], shared_[2], entering[NQ];
    const auto load = [&](int64_t t0) {
        const int64_t t = t0 + es;
        const int there = t < end ? left : 0;
        load_four<E>(a.dt + (row0 + t) * a.lddt + column0 + ec, there, dt);
        load_four<E>(a.dy + (row0 + t) * a.lddy + column0 + ec, there, dy);
        if (a.z) load_four<E>(a.z + (row0 + t) * a.ldz + column0 + ec, there, z);
        if constexpr (!MAPS) {
            load_four<E>(a.u + (row0 + t) * a.ldu + column0 + ec, there, u);
            load_states<NQ>(a.states_in + (b * chunks + t0 / kTile) * of + state, n0, a.N, any, entering);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = threadIdx.x + k * kThreads, n = at % kMaxStates, which = at / kMaxStates % 2;
            const int64_t s = t0 + at / (2 * kMaxStates);
            shared_[k] = 0.0f;
            if (n < a.N && s < end && !(MAPS && !which)) shared_[k] = E::widen(which ? a.cm[(row0 + s) * a.ldc + n] : a.bm[(row0 + s) * a.ldb + n]);
        }
    };
    int64_t t0 = begin + (end - 1 - begin) / kTile * kTile;
    load(t0);
    for (; t0 >= begin; t0 -= kTile) {
        const unsigned resets = resets_of<RESETS>(a.reset, row0 + t0, end - t0 < kTile ? static_cast<int>(end - t0) : kTile);
        const bool there = t0 + es < end;
        float own_u[4], delta[4], opens[4], g[4], dgate[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = dt[j] + bias[j], zj = finite_below(z[j]), e = sigmoid(zj);
            delta[j] = there ? softplus(v) : 0.0f;
            g[j] = a.z ? dy[j] * (zj * e) : dy[j];
            if constexpr (!MAPS) {
                own_u[j] = u[j];
                opens[j] = sigmoid(v);
                dgate[j] = dy[j] * silu_slope(zj, e);
            }
            step[es][ec + j] = float2{delta[j], MAPS ? 0.0f : delta[j] * u[j]};
            pull[es][ec + j] = g[j];
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) (&both[0][0][0])[threadIdx.x + k * kThreads] = shared_[k];
        float h[MAPS ? 1 : kTile + 1][NQ];
        if constexpr (!MAPS)
#pragma unroll
            for (int j = 0; j < NQ; ++j) h[0][j] = entering[j];
        if (t0 > begin) load(t0 - kTile);
        __syncthreads();
        if constexpr (MAPS) {
#pragma unroll
            for (int i = kTile - 1; i >= 0; --i) {
                const float delta_i = step[i][c].x, g_i = pull[i][c];
                const bool cut = RESETS && ((resets >> i) & 1u);
#pragma unroll
                for (int j = 0; j < NQ; ++j) {
                    const float r = __builtin_fmaf(both[i][1][n0 + j], g_i, carry[j]);
                    carry[j] = cut ? 0.0f : exp2_fast(rate[j] * delta_i) * r;
                }
                sum += delta_i;
            }
            if (RESETS) gone = gone || resets != 0;
        } else {
            float four[4], other[4];
#pragma unroll
            for (int i = 0; i < kTile; ++i) {
                if (i % 4 == 0) asm volatile("" ::: "memory");         // LDS is read where it is used rather than all at once
                const float2 s = step[i][c];
                const bool cut = RESETS && ((resets >> i) & 1u);
                float y = 0.0f;
#pragma unroll
                for (int j = 0; j < NQ; ++j) {
                    const float in = s.y * both[i][0][n0 + j];
                    h[i + 1][j] = cut ? in : __builtin_fmaf(exp2_fast(rate[j] * s.x), h[i][j], in);
                    y = __builtin_fmaf(both[i][1][n0 + j], h[i + 1][j], y);
                }
                four[i % 4] = quad_sum(y);
                if (i % 4 == 3) out[0][i - 3 + q][c] = one_of(q, four[0], four[1], four[2], four[3]);
            }
#pragma unroll
            for (int i = kTile - 1; i >= 0; --i) {
                if (i % 4 == 3) asm volatile("" ::: "memory");         // LDS is read again rather than kept in registers over the walks
                const float2 s = step[i][c];
                const float g_i = pull[i][c];
                const bool cut = RESETS && ((resets >> i) & 1u);
                float into = 0.0f, across = 0.0f, pb[NQ], pc[NQ];
#pragma unroll
                for (int j = 0; j < NQ; ++j) {
                    const float r = __builtin_fmaf(both[i][1][n0 + j], g_i, carry[j]);
                    into = __builtin_fmaf(r, both[i][0][n0 + j], into);
                    const float keep = exp2_fast(rate[j] * s.x), moved = cut ? 0.0f : r * (keep * h[i][j]);
                    across = __builtin_fmaf(rate[j], moved, across);
                    drate[j] = __builtin_fmaf(s.x, moved, drate[j]);
                    carry[j] = cut ? 0.0f : keep * r;
                    pb[j] = r * s.y;
                    pc[j] = h[i + 1][j] * g_i;
                }
                four[i % 4] = quad_sum(into);
                other[i % 4] = quad_sum(across);
                if (i % 4 == 0) {
                    out[1][i + q][c] = one_of(q, four[0], four[1], four[2], four[3]);
                    out[2][i + q][c] = one_of(q, other[0], other[1], other[2], other[3]);
                }
                const Reduced<NQ> sums = reduce_columns<NQ>(pb, pc);
                if (sums.holds) shares[wave][i][sums.which][n0 + sums.j] = sums.v;
            }
        }
        __syncthreads();
        if constexpr (!MAPS) {
            float du[4], ddt[4], dz[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float y = out[0][es][ec + j] + skip[j] * own_u[j], into = out[1][es][ec + j], across = kLn2 * out[2][es][ec + j];
                du[j] = __builtin_fmaf(delta[j], into, skip[j] * g[j]);
                ddt[j] = __builtin_fmaf(own_u[j], into, across) * opens[j];
                dz[j] = dgate[j] * y;
                if (there) {
                    dbias[j] += ddt[j];
                    dskip[j] = __builtin_fmaf(g[j], own_u[j], dskip[j]);
                }
            }
            if (there) {
                const int64_t row = row0 + t0 + es;
                store_four<E>(a.du + row * a.lddu + column0 + ec, left, du);
                store_four<E>(a.ddt + row * a.ldddt + column0 + ec, left, ddt);
                if (a.dz) store_four<E>(a.dz + row * a.lddz + column0 + ec, left, dz);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = threadIdx.x + k * kThreads, n = at % kMaxStates, which = at / kMaxStates % 2, i = at / (2 * kMaxStates);
                if (n >= a.N || t0 + i >= end) continue;
                float v = 0.0f;
#pragma unroll
                for (int k2 = 0; k2 < kWaves; ++k2) v += shares[k2][i][which][n];
                a.shared_parts[((slab * a.B * a.T_ + row0 + t0 + i) * 2 + which) * a.N + n] = v;
            }
        }
    }
    if constexpr (MAPS) {
        store_states<NQ>(a.maps + (b * a.spans + span) * of + state, n0, a.N, any, carry);
        if (any && q == 0) a.sums[(b * a.spans + span) * a.D + column0 + c] = gone ? -1.0f : sum;
    } else {
        if (a.dh0 && begin == 0) store_states<NQ>(a.dh0 + b * of + state, n0, a.N, any, carry);
        const int64_t count = static_cast<int64_t>(a.D) * (a.N + 2);
        float *part = a.parts + (b * a.spans + span) * count;          // a worker's sequences lie together
#pragma unroll
        for (int j = 0; j < NQ; ++j) drate[j] *= kLn2 * rate[j];
        store_states<NQ>(part + state, n0, a.N, any, drate);
        const auto over_steps = [&](const float(&v)[4], int64_t at) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 4; ++j) out[0][es][ec + j] = v[j];
            __syncthreads();
            if (threadIdx.x < kColumns && column0 + static_cast<int>(threadIdx.x) < a.D) {
                float all = 0.0f;
#pragma unroll
                for (int i = 0; i < kTile; ++i) all += out[0][i][threadIdx.x];
                part[at + column0 + threadIdx.x] = all;
            }
        };
        over_steps(dbias, of);
        over_steps(dskip, of + a.D);
    }
}

// dB and dC of a row: the slabs' shares in their order.
template <class E>
__global__ __launch_bounds__(256) void share_kernel(const SelectArgs<E> a)
{
    const int64_t of = 2 * static_cast<int64_t>(a.N), all = a.B * a.T_ * of, i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= all) return;
    float v = 0.0f;
#pragma unroll 4
    for (int k = 0; k < a.slabs; ++k) v += a.shared_parts[k * all + i];
    const int64_t row = i / of;
    const int at = static_cast<int>(i - row * of);
    if (at < a.N) a.dbm[row * a.lddb + at] = E::narrow(v);
    else a.dcm[row * a.lddc + at - a.N] = E::narrow(v);
}

constexpr int64_t kWanted = 768, kLeastTiles = 4;       // workgroups of a call; tiles of a span

struct Space {
    Spans s;
    int64_t sums, shared, parts, bytes;
};
Space space_of(int64_t B, int64_t T, int32_t D, int32_t N)
{
    Space p{};
    p.s = spans_of(B, T, D, kWanted, kLeastTiles);
    const bool split = p.s.spans > 1;
    p.sums = split ? round_up(B * p.s.spans * D * N * 4, 16) : 0;
    p.shared = p.sums + (split ? round_up(B * p.s.spans * D * 4, 16) : 0);
    p.parts = p.shared + round_up(p.s.slabs * B * T * 2 * N * 4, 16);
    p.bytes = p.parts + B * p.s.spans * D * (N + 2) * 4;
    return p;
}

template <class E>
int select_scan_grad(const typename E::T *u, int64_t ldu, const typename E::T *dt, int64_t lddt, const typename E::T *bm, int64_t ldb,
                     const typename E::T *cm, int64_t ldc, const typename E::T *z, int64_t ldz, const typename E::T *params, int64_t ldp, int32_t W,
                     int64_t offset, const typename E::T *dy, int64_t lddy, typename E::T *du, int64_t lddu, typename E::T *ddt, int64_t ldddt,
                     typename E::T *dbm, int64_t lddb, typename E::T *dcm, int64_t lddc, typename E::T *dz, int64_t lddz, const typename E::T *g_in,
                     typename E::T *g_out, int64_t ld, int64_t B, int64_t T, int32_t D, int32_t N, const uint8_t *reset, const float *states,
                     const float *dh_last, float *dh0, void *workspace, int64_t workspace_bytes, void *stream)
{
    const int rc = check_select(W, B, T, D, N);
    const int64_t count = static_cast<int64_t>(D) * (N + 2), state_bytes = B * D * N * 4, rows = B * T;
    if (rc != CX_OK || bad_rows(W, ldp, offset, count) || bad_rows(W, ld, offset, count)) return CX_ERR_SHAPE;
    if (!g_out) return CX_ERR_NULL;
    constexpr int kElem = sizeof(typename E::T);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool none = B == 0 || T == 0;
    Space space{};
    if (!none) {
        if (!u || !dt || !bm || !cm || !params || !dy || !du || !ddt || !dbm || !dcm || !states || !workspace || (z && !dz) || (!z && dz)) return CX_ERR_NULL;
        if (bad_matrix(rows, ldu, D) || bad_matrix(rows, lddt, D) || bad_matrix(rows, ldb, N) || bad_matrix(rows, ldc, N) || (z && bad_matrix(rows, ldz, D)) ||
            bad_matrix(rows, lddy, D) || bad_matrix(rows, lddu, D) || bad_matrix(rows, ldddt, D) || bad_matrix(rows, lddb, N) || bad_matrix(rows, lddc, N) ||
            (dz && bad_matrix(rows, lddz, D))) return CX_ERR_SHAPE;
        space = space_of(B, T, D, N);
        if (workspace_bytes < space.bytes) return CX_ERR_SHAPE;
    }
    for (const void *p : {static_cast<const void *>(u), static_cast<const void *>(dt), static_cast<const void *>(bm), static_cast<const void *>(cm),
                          static_cast<const void *>(z), static_cast<const void *>(params), static_cast<const void *>(dy), static_cast<const void *>(du),
                          static_cast<const void *>(ddt), static_cast<const void *>(dbm), static_cast<const void *>(dcm), static_cast<const void *>(dz),
                          static_cast<const void *>(g_in), static_cast<const void *>(g_out)})
        if (misaligned_to(p, kElem)) return CX_ERR_ALIGN;
    if (misaligned_to(states, 4) || misaligned_to(dh_last, 4) || misaligned_to(dh0, 4) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const Extent in[11] = {matrix_of(u, rows, ldu, D, kElem), matrix_of(dt, rows, lddt, D, kElem), matrix_of(bm, rows, ldb, N, kElem), matrix_of(cm, rows, ldc, N, kElem),
                           matrix_of(z, rows, ldz, D, kElem), matrix_of(params, W, ldp, offset + count, kElem), matrix_of(dy, rows, lddy, D, kElem),
                           dense_of(reset, rows), dense_of(states, B * ceil_div(T, kTile) * D * N * 4), dense_of(dh_last, state_bytes),
                           matrix_of(g_in, W, ld, offset + count, kElem)};
    const Extent out[8] = {matrix_of(du, rows, lddu, D, kElem), matrix_of(ddt, rows, ldddt, D, kElem), matrix_of(dbm, rows, lddb, N, kElem),
                           matrix_of(dcm, rows, lddc, N, kElem), matrix_of(dz, rows, lddz, D, kElem), matrix_of(g_out, W, ld, offset + count, kElem),
                           dense_of(dh0, state_bytes), dense_of(workspace, space.bytes)};
    const Same same[2] = {{5, 10}, {6, 9}};
    if (outputs_share_but(in, out, same)) return CX_ERR_ALIAS;
    char *base = static_cast<char *>(workspace);
    SelectArgs<E> a{};
    a.dh_last = dh_last; a.dh0 = dh0; a.B = B; a.T_ = T; a.D = D; a.N = N;
    if (!none) {
        a.u = u; a.ldu = ldu; a.dt = dt; a.lddt = lddt; a.bm = bm; a.ldb = ldb; a.cm = cm; a.ldc = ldc; a.z = z; a.ldz = ldz; a.params = params + offset;
        a.ldp = ldp; a.dy = dy; a.lddy = lddy; a.du = du; a.lddu = lddu; a.ddt = ddt; a.ldddt = ldddt; a.dbm = dbm; a.lddb = lddb; a.dcm = dcm; a.lddc = lddc;
        a.dz = dz; a.lddz = lddz; a.reset = reset; a.states_in = states; a.per_worker = B / W; a.slabs = space.s.slabs; a.spans = space.s.spans;
        a.span_steps = space.s.steps;
        a.maps = reinterpret_cast<float *>(base);
        a.sums = reinterpret_cast<float *>(base + space.sums);
        a.shared_parts = reinterpret_cast<float *>(base + space.shared);
        a.parts = reinterpret_cast<float *>(base + space.parts);
        const unsigned groups = static_cast<unsigned>(B * a.slabs);
        int rc2 = CX_OK;
        if (a.spans > 1) {
            rc2 = by_states(N, reset != nullptr, [&](auto nq, auto resets) {
                hipLaunchKernelGGL((select_grad_kernel<E, decltype(nq)::value, decltype(resets)::value, kMaps>), dim3(groups, a.spans - 1), dim3(kThreads), 0, st, a);
            });
            if (rc2 != CX_OK) return rc2;
            hipLaunchKernelGGL(enter_kernel<E>, dim3(static_cast<unsigned>(ceil_div(B * D * N, 256))), dim3(256), 0, st, a, dh_last, true);
            if (launched() != CX_OK) return CX_ERR_HIP;
        }
        rc2 = by_states(N, reset != nullptr, [&](auto nq, auto resets) {
            hipLaunchKernelGGL((select_grad_kernel<E, decltype(nq)::value, decltype(resets)::value, kWalk>), dim3(groups, a.spans), dim3(kThreads), 0, st, a);
        });
        if (rc2 != CX_OK) return rc2;
        hipLaunchKernelGGL(share_kernel<E>, dim3(static_cast<unsigned>(ceil_div(rows * 2 * N, 256))), dim3(256), 0, st, a);
        if (launched() != CX_OK) return CX_ERR_HIP;
    } else if (dh0 && dh0 != dh_last && B > 0) {
        hipLaunchKernelGGL(pass_states_kernel, dim3(static_cast<unsigned>(ceil_div(state_bytes / 4, 256))), dim3(256), 0, st, dh_last, dh0, state_bytes / 4);
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    if (none && g_in == g_out) return CX_OK;
    return sum_parts<E>(a.parts, none ? 0 : B / W * a.spans, count, g_in ? g_in + offset : nullptr, g_out + offset, ld, W, st);
}

}  // namespace

extern "C" {

#define CX_LM_SELECT_GRAD(SUFFIX, E)                                                                                                  \
    int cx_select_scan_grad##SUFFIX(const E::T *u, int64_t ldu, const E::T *dt, int64_t lddt, const E::T *bm, int64_t ldb,            \
                                    const E::T *cm, int64_t ldc, const E::T *z, int64_t ldz, const E::T *params, int64_t ldp,         \
                                    int32_t W, int64_t offset, const E::T *dy, int64_t lddy, E::T *du, int64_t lddu, E::T *ddt,       \
                                    int64_t ldddt, E::T *dbm, int64_t lddb, E::T *dcm, int64_t lddc, E::T *dz, int64_t lddz,          \
                                    const E::T *g_in, E::T *g_out, int64_t ldg, int64_t B, int64_t T, int32_t D, int32_t N,           \
                                    const uint8_t *reset, const float *states, const float *dh_last, float *dh0, void *workspace,     \
                                    int64_t workspace_bytes, void *stream)                                                            \
    {                                                                                                                                 \
        return select_scan_grad<E>(u, ldu, dt, lddt, bm, ldb, cm, ldc, z, ldz, params, ldp, W, offset, dy, lddy, du, lddu, ddt,       \
                                   ldddt, dbm, lddb, dcm, lddc, dz, lddz, g_in, g_out, ldg, B, T, D, N, reset, states, dh_last, dh0,  \
                                   workspace, workspace_bytes, stream);                                                               \
    }
CX_LM_SELECT_GRAD(, F32)
CX_LM_SELECT_GRAD(_bf16, Bf16)
CX_LM_SELECT_GRAD(_f16, F16)
#undef CX_LM_SELECT_GRAD

int cx_select_grad_workspace(int64_t B, int64_t T, int32_t D, int32_t N, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_select(1, B, T, D, N);
    if (rc == CX_OK && B > 0 && T > 0) *bytes = space_of(B, T, D, N).bytes;
    return rc;
}

}  // extern "C"
