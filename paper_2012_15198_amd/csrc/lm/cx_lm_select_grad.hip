// C-ABI entry points cx_select_scan_grad*, cx_select_grad_workspace: the gradient of the selective scan (see include/cx_lm.h, lm_select.hpp)
//
// With g_t = dy_t silu(z_t), r_t[n] = dL/dh_t[n], keep_t = (reset_t ? 0 : a_t) and A = -exp(A_log):
//
//   r_t = C_t g_t + keep_{t+1} r_{t+1}    into_t = sum_n r_t B_t    across_t = sum_n r_t A keep_t h_{t-1}
//   du = delta into + skip g    ddt = (across + u into) sigmoid(dt + bias)    dz = dy y' silu'(z), y' the result before its gate
//   dB_t = sum over columns of r_t delta_t u_t    dC_t = sum over columns of h_t g_t
//   dA_log = A sum_t r_t delta_t keep_t h_{t-1}    dbias = sum_t ddt    dskip = sum_t g u
//
// A tile's states are computed again from the one kept where it begins and stay in registers with their gates; the walk back meets them there.
// That takes 246 to 256 registers with 16 states, so two wavefronts to a SIMD, which issue vector instructions in 80 % of the busy cycles (16 sequences of
// 2,048 x 1,024 in bfloat16: 63 us the maps, 7 what enters, 480 to 499 the walks, 13 and 6 the sums over columns and parts).  The workspace has a float of
// dB and of dC for each step, state and 64 columns: 268 MB for 16 sequences of 2,048 x 4,096 with 16 states.
#include "lm_select.hpp"

namespace {

enum Pass { kMaps, kWalk };

constexpr int kOutPitch = kColumns + 16;                // the four steps that a column's lanes write lie in different banks
constexpr int kWaves = kThreads / kWave;

// The sums of 2 NQ values over the 16 columns of a row of lanes, each in some of its lanes: `which` (B or C) and `j` (the state); `holds`: this lane
// is the one to write it.  Each stage leaves a lane half of the values, its own and its partner's: partners lie opposite each other in the
// row, in half of it, in a group of four, beside each other.
struct Reduced {
    float v;
    int which, j;
    bool holds;
};
// Every lane adds both, then keeps one.
template <int PATTERN>
__device__ __forceinline__ float half_of(int second, float x, float y)
{
    const float a = add_partner<PATTERN>(x), b = add_partner<PATTERN>(y);
    return second ? b : a;
}
template <int NQ>
__device__ __forceinline__ Reduced reduce_columns(const float (&pb)[NQ], const float (&pc)[NQ])
{
    const int lane = threadIdx.x & 15;
    Reduced r;
    r.which = lane >> 3;
    if constexpr (NQ >= 3) {
        // Two additions a pair: the second value's in all lanes, then the first one's over it in the half of the lanes (banks of four) that keep it.
        // A value is read across lanes two instructions after it was written at the earliest.
        const float b0 = pb[0], b1 = pb[1], b2 = pb[2], b3 = NQ > 3 ? pb[NQ - 1] : 0.0f;
        float c0 = pc[0], c1 = pc[1], c2 = pc[2], c3 = NQ > 3 ? pc[NQ - 1] : 0.0f;
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %2, %2 row_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %3, %3, %3 row_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %6, %6 row_mirror row_mask:0xf bank_mask:0x3\n\t"
            "v_add_f32_dpp %3, %7, %7 row_mirror row_mask:0xf bank_mask:0x3\n\t"
            "v_add_f32_dpp %0, %4, %4 row_mirror row_mask:0xf bank_mask:0x3\n\t"
            "v_add_f32_dpp %1, %5, %5 row_mirror row_mask:0xf bank_mask:0x3\n\t"
            "v_add_f32_dpp %2, %2, %2 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %3, %3, %3 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %0, %0 row_half_mirror row_mask:0xf bank_mask:0x5\n\t"
            "v_add_f32_dpp %3, %1, %1 row_half_mirror row_mask:0xf bank_mask:0x5\n\t"
            "s_nop 0\n\t"
            "v_add_f32_dpp %2, %2, %2 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %3, %3, %3 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf"
            : "+&v"(c0), "+&v"(c1), "+&v"(c2), "+&v"(c3)        // written before b0 to b3 are read
            : "v"(b0), "v"(b1), "v"(b2), "v"(b3));
        r.v = add_partner<kBeside>((lane & 2) ? c3 : c2);
        r.j = ((lane >> 1) & 1) + ((lane >> 1) & 2);
        r.holds = (lane & 1) == 0;
    } else if constexpr (NQ == 2) {
        const float first = half_of<kMirror>(lane & 8, pb[0], pc[0]), second = half_of<kMirror>(lane & 8, pb[1], pc[1]);
        const float v = half_of<kHalfMirror>(lane & 4, first, second);
        r.v = add_partner<kBeside>(add_partner<kOppositePair>(v));
        r.j = (lane >> 2) & 1;
        r.holds = (lane & 3) == 0;
    } else {
        const float v = half_of<kMirror>(lane & 8, pb[0], pc[0]);
        r.v = add_partner<kBeside>(add_partner<kOppositePair>(add_partner<kHalfMirror>(v)));
        r.j = 0;
        r.holds = (lane & 7) == 0;
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
    const int64_t b = blockIdx.x / a.slabs, w = static_cast<uint32_t>(b) / a.per_worker, row0 = b * a.T_;
    const int slab = static_cast<int>(blockIdx.x % a.slabs), column0 = slab * kColumns;
    const int parts = a.pieces / a.spans, piece = blockIdx.y + parts, span = MAPS ? piece / parts : blockIdx.y;       // maps: all but the first span's
    const int64_t span_begin = span * a.span_steps, span_end = span_begin + a.span_steps < a.T_ ? span_begin + a.span_steps : a.T_;
    const int64_t begin = MAPS ? span_begin + (piece % parts) * a.piece_steps : span_begin;
    const int64_t end = MAPS && begin + a.piece_steps < span_end ? begin + a.piece_steps : span_end;
    const T *params = a.params + w * a.ldp;
    const int es = threadIdx.x / (kColumns / kEach), ec = threadIdx.x % (kColumns / kEach) * kEach, left = a.D - column0 - ec;
    float bias[4], skip[4], dbias[4] = {}, dskip[4] = {};
    __shared__ alignas(16) float parked[MAPS ? 1 : 3][MAPS ? 1 : kTile][kColumns];     // u, sigmoid(dt + bias), dy silu'(z): a thread's own, over the walks
    load_four<E>(params + static_cast<int64_t>(a.D) * a.N + column0 + ec, left, bias);
    load_four<E>(params + static_cast<int64_t>(a.D) * (a.N + 1) + column0 + ec, left, skip);
    close_behind(bias, left);
    const int wave = threadIdx.x / kWave, q = threadIdx.x / 16 % kQuarters, c = wave * 16 + threadIdx.x % 16, n0 = q * NQ;
    const bool any = column0 + c < a.D;
    const int64_t state = (static_cast<int64_t>(column0) + c) * a.N, of = static_cast<int64_t>(a.D) * a.N, chunks = ceil_div(a.T_, kTile);
    float rate[NQ], carry[NQ], drate[NQ] = {}, sum = 0.0f;
    bool gone = false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        rate[i] = any && n0 + i < a.N ? rate_of(E::widen(params[state + n0 + i])) : 0.0f;
        carry[i] = 0.0f;
    }
    if constexpr (!MAPS) {
        if (a.spans > 1) load_states<NQ>(a.maps + (b * a.pieces + span * parts + parts - 1) * of + state, n0, a.N, any, carry);
        else if (a.dh_last) load_states<NQ>(a.dh_last + b * of + state, n0, a.N, any, carry);
    }
    const int back = back_of<E>(left, a.D), first = ec - back + kEach;      // of loads, from kEach columns before the slab's on
    const uint32_t u_at = place_in<T>(a.ldu, es, first), dt_at = place_in<T>(a.lddt, es, first), z_at = place_in<T>(a.ldz, es, first), dy_at = place_in<T>(a.lddy, es, first);
    const int bs = threadIdx.x / kMaxStates, bp = threadIdx.x % kMaxStates, bn = state_of<NQ>(bp);           // a thread's element of B and of C
    const uint32_t b_at = place_in<T>(a.ldb, bs, bn), c_at = place_in<T>(a.ldc, bs, bn), state_at = (c * a.N) * 4;
    Columns<E, 4> u, dt, z{}, dy;
    T b_next, c_next;
    float entering[NQ];
    const auto load = [&](int64_t t0) {
        const int64_t row = row0 + t0;
        const int steps = end - t0 < kTile ? static_cast<int>(end - t0) : kTile, there = es < steps ? left : 0;
        const bool has = bn < a.N && bs < steps;
        dt = load_back<E>(at_byte(a.dt + row * a.lddt + column0 - kEach, dt_at), there, back);
        dy = load_back<E>(at_byte(a.dy + row * a.lddy + column0 - kEach, dy_at), there, back);
        if (a.z) z = load_back<E>(at_byte(a.z + row * a.ldz + column0 - kEach, z_at), there, back);
        c_next = has ? *at_byte(a.cm + row * a.ldc, c_at) : 0;
        if constexpr (!MAPS) {
            u = load_back<E>(at_byte(a.u + row * a.ldu + column0 - kEach, u_at), there, back);
            b_next = has ? *at_byte(a.bm + row * a.ldb, b_at) : 0;
            load_states<NQ>(at_byte(a.states_in + (b * chunks + t0 / kTile) * of + static_cast<int64_t>(column0) * a.N, state_at), n0, a.N, any, entering);
        }
    };
    int64_t t0 = begin < end ? begin + (end - 1 - begin) / kTile * kTile : begin - kTile;        // a last span may leave its last pieces empty
    if (begin < end) load(t0);
    for (; t0 >= begin; t0 -= kTile) {
        const int steps = end - t0 < kTile ? static_cast<int>(end - t0) : kTile;
        const unsigned resets = resets_of<RESETS>(a.reset, row0 + t0, steps);
        const bool there = es < steps;
        settle<E>(dt, back);
        settle<E>(dy, back);
        settle<E>(z, back);
        if constexpr (!MAPS) settle<E>(u, back);
        float delta[4], enters[4], g[4], own[3][4], pulls = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = value_of<E, 4>(dt, j) + bias[j], zj = finite_below(value_of<E, 4>(z, j)), e = sigmoid(zj), dyj = value_of<E, 4>(dy, j), soft = softplus(v);
            delta[j] = there ? soft : 0.0f;                             // behind the end: a step that changes nothing
            g[j] = a.z && dyj != 0.0f ? dyj * (zj * e) : dyj;
            pulls += __builtin_fabsf(dyj);
            enters[j] = 0.0f;
            if constexpr (!MAPS) {
                own[0][j] = value_of<E, 4>(u, j);
                own[1][j] = sigmoid(v);
                own[2][j] = dyj == 0.0f ? 0.0f : dyj * silu_slope(zj, e);
                enters[j] = delta[j] == 0.0f ? 0.0f : delta[j] * own[0][j];
            }
        }
        put_pairs(&step[es][ec], delta, enters);
        put_four(&pull[es][ec], g);
        if constexpr (!MAPS)
#pragma unroll
            for (int k = 0; k < 3; ++k) put_four(&parked[k][es][ec], own[k]);
        if constexpr (!MAPS) both[bs][0][bp] = E::widen(all_of_step(nothing_of(delta)) ? T(0) : b_next);
        both[bs][1][bp] = E::widen(all_of_step(pulls == 0.0f) ? T(0) : c_next);
        float h[MAPS ? 1 : kTile + 1][NQ], keep[MAPS ? 1 : kTile][NQ];
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
                    const float r = __builtin_fmaf(both[i][1][q * 4 + j], g_i, carry[j]);
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
                    const float in = s.y * both[i][0][q * 4 + j];
                    keep[i][j] = exp2_fast(rate[j] * s.x);
                    h[i + 1][j] = cut ? in : __builtin_fmaf(keep[i][j], h[i][j], in);
                    y = __builtin_fmaf(both[i][1][q * 4 + j], h[i + 1][j], y);
                }
                four[i % 4] = y;
                if (i % 4 == 3) out[0][i - 3 + quarter_step(q)][c] = quarters_sum(four);
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
                    const float r = __builtin_fmaf(both[i][1][q * 4 + j], g_i, carry[j]);
                    into = __builtin_fmaf(r, both[i][0][q * 4 + j], into);
                    const float moved = cut ? 0.0f : r * (keep[i][j] * h[i][j]);
                    across = __builtin_fmaf(rate[j], moved, across);
                    drate[j] = __builtin_fmaf(s.x, moved, drate[j]);
                    carry[j] = cut ? 0.0f : keep[i][j] * r;
                    pb[j] = r * s.y;
                    pc[j] = h[i + 1][j] * g_i;
                }
                four[i % 4] = into;
                other[i % 4] = across;
                if (i % 4 == 0) {
                    out[1][i + quarter_step(q)][c] = quarters_sum(four);
                    out[2][i + quarter_step(q)][c] = quarters_sum(other);
                }
#pragma unroll
                for (int j = 0; j < NQ; ++j) asm volatile("" : "+v"(drate[j]));       // summed here: 64 products waiting for it would cost as many registers
                const Reduced sums = reduce_columns<NQ>(pb, pc);
                if (sums.holds) shares[wave][i][sums.which][q * 4 + sums.j] = sums.v;
            }
        }
        __syncthreads();
        if constexpr (!MAPS) {
            float du[4], ddt[4], dz[4], own_u[4], opens[4], slopes[4], g_[4], y[4], into[4], across[4];
            get_four(&parked[0][es][ec], own_u);
            get_four(&parked[1][es][ec], opens);
            get_four(&parked[2][es][ec], slopes);
            get_four(&pull[es][ec], g_);
            get_four(&out[0][es][ec], y);
            get_four(&out[1][es][ec], into);
            get_four(&out[2][es][ec], across);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                du[j] = __builtin_fmaf(step[es][ec + j].x, into[j], skip[j] * g_[j]);
                ddt[j] = opens[j] == 0.0f ? 0.0f : __builtin_fmaf(own_u[j], into[j], kLn2 * across[j]) * opens[j];       // closed: rates may be as large as numbers are
                dz[j] = slopes[j] == 0.0f ? 0.0f : slopes[j] * __builtin_fmaf(skip[j], own_u[j], y[j]);
                if (there) {
                    dbias[j] += ddt[j];
                    if (g_[j] != 0.0f) dskip[j] = __builtin_fmaf(g_[j], own_u[j], dskip[j]);
                }
            }
            const int64_t row = row0 + t0;
            if (there) {
                store_columns<E, 4>(at_byte(a.du + row * a.lddu + column0, place_in<T>(a.lddu, es, ec)), left, du);
                store_columns<E, 4>(at_byte(a.ddt + row * a.ldddt + column0, place_in<T>(a.ldddt, es, ec)), left, ddt);
                if (a.dz) store_columns<E, 4>(at_byte(a.dz + row * a.lddz + column0, place_in<T>(a.lddz, es, ec)), left, dz);
            }
            if (bn < a.N && bs < steps) {
                float *share = at_byte(a.shared_parts + (slab * a.B * a.T_ + row) * 2 * a.N, (bs * 2 * a.N + bn) * 4);
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    float v = 0.0f;
#pragma unroll
                    for (int k = 0; k < kWaves; ++k) v += shares[k][bs][which][bp];
                    share[which * a.N] = v;
                }
            }
        }
    }
    if constexpr (MAPS) {
        store_states<NQ>(a.maps + (b * a.pieces + piece) * of + state, n0, a.N, any, carry);
        if (any && q == 0) a.sums[(b * a.pieces + piece) * a.D + column0 + c] = gone ? -1.0f : sum;
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
    const int64_t of = 2 * static_cast<int64_t>(a.N), all = a.B * a.T_ * of;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * 256) {
        float v = 0.0f;
#pragma unroll 4
        for (int k = 0; k < a.slabs; ++k) v += a.shared_parts[k * all + i];
        const int64_t row = i / of;
        const int at = static_cast<int>(i - row * of);
        if (at < a.N) a.dbm[row * a.lddb + at] = E::narrow(v);
        else a.dcm[row * a.lddc + at - a.N] = E::narrow(v);
    }
}

constexpr int64_t kAtOnce = 512;                        // workgroups that run at a time: two to a CU, by their registers

struct Space {
    Spans s;
    int64_t sums, shared, parts, bytes;
};
Space space_of(int64_t B, int64_t T, int32_t D, int32_t N)
{
    Space p{};
    p.s = spans_of(B, T, D, kAtOnce);
    const bool split = p.s.spans > 1;
    p.sums = split ? round_up(B * p.s.pieces * D * N * 4, 16) : 0;
    p.shared = p.sums + (split ? round_up(B * p.s.pieces * D * 4, 16) : 0);
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
        if (bad_strip(rows, ldu, D) || bad_strip(rows, lddt, D) || bad_strip(rows, ldb, N) || bad_strip(rows, ldc, N) || (z && bad_strip(rows, ldz, D)) ||
            bad_strip(rows, lddy, D) || bad_strip(rows, lddu, D) || bad_strip(rows, ldddt, D) || bad_strip(rows, lddb, N) || bad_strip(rows, lddc, N) ||
            (dz && bad_strip(rows, lddz, D))) return CX_ERR_SHAPE;
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
        a.dz = dz; a.lddz = lddz; a.reset = reset; a.states_in = states; a.per_worker = static_cast<uint32_t>(B / W); a.slabs = space.s.slabs; a.spans = space.s.spans;
        a.span_steps = space.s.steps; a.pieces = space.s.pieces; a.piece_steps = space.s.piece_steps;
        a.maps = reinterpret_cast<float *>(base);
        a.sums = reinterpret_cast<float *>(base + space.sums);
        a.shared_parts = reinterpret_cast<float *>(base + space.shared);
        a.parts = reinterpret_cast<float *>(base + space.parts);
        const unsigned groups = static_cast<unsigned>(B * a.slabs);
        int rc2 = CX_OK;
        if (a.spans > 1) {
            const int composed = a.pieces - a.pieces / a.spans;
            rc2 = by_states(N, reset != nullptr, [&](auto nq, auto resets) {
                hipLaunchKernelGGL((select_grad_kernel<E, decltype(nq)::value, decltype(resets)::value, kMaps>), dim3(groups, composed), dim3(kThreads), 0, st, a);
            });
            if (rc2 != CX_OK) return rc2;
            if (enter<E>(a, dh_last, true, composed, st) != CX_OK) return CX_ERR_HIP;
        }
        rc2 = by_states(N, reset != nullptr, [&](auto nq, auto resets) {
            hipLaunchKernelGGL((select_grad_kernel<E, decltype(nq)::value, decltype(resets)::value, kWalk>), dim3(groups, a.spans), dim3(kThreads), 0, st, a);
        });
        if (rc2 != CX_OK) return rc2;
        const int64_t blocks = ceil_div(rows * 2 * N, 256);
        hipLaunchKernelGGL(share_kernel<E>, dim3(static_cast<unsigned>(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0, st, a);
        if (launched() != CX_OK) return CX_ERR_HIP;
    } else if (pass_through(dh_last, dh0, state_bytes / 4, st) != CX_OK) {
        return CX_ERR_HIP;
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
