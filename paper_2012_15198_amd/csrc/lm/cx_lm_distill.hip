// C-ABI entry points cx_distill_loss*, cx_distill_grad*, cx_distill_step*, cx_distill_workspace: distillation from a teacher's
// top logits with the label's cross entropy beside it (see include/cx_lm.h).
//
//   q = softmax(t / tau) over the teacher's valid ids      p = softmax(z / tau)      p1 = softmax(z)
//   loss = w_kl tau^2 sum_k q_k (log q_k - log p[id_k])  -  w_ce log p1[label]
//   dz   = gout (w_kl tau (p - q) + w_ce (p1 - onehot(label)))
//
// Bound by memory where the exponentials allow it: loss and gradient together read a row of logits once, into registers, as long as it
// fits there.  q and the label touch K + 1 elements: every element is written with its share of p and p1, and behind a
// barrier those few are written again with their targets.
// 8,192 bfloat16 rows of 65,536 take 419 us at tau = 2 (5.1 TB/s, what a copy of the logits takes), 431 in rows of twenty calls and up to 490
// there under the profiler; 4,096 float32 rows of 50,257 330 us (5.0 TB/s).
// Where rows are few, several workgroups share one: part_kernel leaves the parts' statistics in the workspace, and each
// workgroup of the second launch joins them for itself.
#include "lm_vocab.hpp"

namespace {

constexpr int kMaxTeacher = CX_MAX_TEACHER;
static_assert(kMaxTeacher < kRowThreads, "a thread for every target");
constexpr int kMostThreads = 1024;

template <class E>
struct DistillArgs {
    const typename E::T *z;
    typename E::T *dz;                                  // NULL: the loss alone
    const int32_t *ids, *labels;
    const float *t, *gout;
    float *loss, *stats;                                // stats: [N][4]: maximum, sum at tau, sum at 1
    int64_t ld, ld_dz, V;
    int K, parts;
    float tau, w_kl, w_ce;
    Stats *part_stats;                                  // [N][parts]
};

// Both sums at their factors of log2(e) z: one sum where tau = 1 or only one of the two terms counts.
template <class E>
__device__ __forceinline__ float soft_factor(const DistillArgs<E> &a) { return a.w_kl != 0.0f ? kLog2e / a.tau : kLog2e; }

template <class E, Extra X>
__device__ __forceinline__ Stats slice_stats(const Slice<E> &slice, float c, Stats (&lds)[kRowWaves])
{
    Stats own{kLowest, 0.0f, 0.0f};
    const int rounds = slice.rounds();
    for (int round = 0; round < rounds; ++round) {
        float v[kAhead * E::kPer16];
        slice.load(round, v);
        accumulate<X>(own, v, c, kLog2e);
    }
    if (slice.has_tail()) {
        const float v[1] = {E::widen(slice.z[slice.tail_at()])};
        accumulate<X>(own, v, c, kLog2e);
    }
    return join_workgroup<X>(own, lds, c, kLog2e);
}

// Grid (parts, N).
template <class E, Extra X>
__global__ __launch_bounds__(kRowThreads) void part_kernel(const DistillArgs<E> a)
{
    __shared__ Stats lds[kRowWaves];
    const int64_t n = blockIdx.y;
    const Slice<E> slice(a.z + n * a.ld, part_begin(a.V, a.parts, blockIdx.x, E::kPer16), part_begin(a.V, a.parts, blockIdx.x + 1, E::kPer16));
    const Stats all = slice_stats<E, X>(slice, soft_factor(a), lds);
    if (threadIdx.x == 0) a.part_stats[n * a.parts + blockIdx.x] = all;
}

struct Targets {                                        // of a row: the teacher's tokens, then the label
    int id[kMaxTeacher + 1];                            // -1: none
    float t[kMaxTeacher + 1];                           // the teacher's logits (-inf: none)
    float z[kMaxTeacher + 1];                           // their logits
    float q[kMaxTeacher + 1];                           // weight of the gradient's target, without gout: w_kl tau q, w_ce
    float soft, hard, loss;                             // w_kl tau, w_ce if these terms count in this row; the row's loss
};

struct Target {
    int id;
    float t;
};

// The k-th of a row's targets, k <= K, from memory.
template <class E>
__device__ __forceinline__ Target load_target(const DistillArgs<E> &a, int64_t n, int k)
{
    if (k < a.K) return {a.ids[n * a.K + k], a.t[n * a.K + k]};
    return {k == a.K && a.labels && a.w_ce != 0.0f ? a.labels[n] : -1, 0.0f};
}
template <class E>
__device__ __forceinline__ void keep_target(const DistillArgs<E> &a, int64_t n, int k, Target own, Targets &to)
{
    if (k > a.K) return;
    const bool valid = own.id >= 0 && own.id < a.V;
    to.id[k] = valid ? own.id : -1;
    to.t[k] = valid && k < a.K ? own.t : -__builtin_inff();
    to.z[k] = valid ? E::widen(a.z[n * a.ld + own.id]) : 0.0f;
}
template <class E>
__device__ __forceinline__ void keep_others(const DistillArgs<E> &a, int64_t n, Targets &to)
{
    for (int k = threadIdx.x + blockDim.x; k <= a.K; k += blockDim.x) keep_target(a, n, k, load_target(a, n, k), to);
}

// Wavefront 0, behind a barrier: the teacher's distribution, and the loss from the row's statistics.  The row's own logits at
// the targets count for the loss alone.  Only differences of logits are divided by tau, and the loss is taken as
//   w_kl tau sum_k q_k ((t_k - max t) - (z_k - m) + tau (log s - log sum_t)):
// a quotient such as the lowest value / 0.5 is infinite, and tau^2 times an infinite log p would be no loss where tau^2 log p is one.
template <class E>
__device__ __forceinline__ void settle(const DistillArgs<E> &a, const Stats &all, Targets &to)
{
    const float lowest = -__builtin_inff();
    float high = lowest, sum = 0.0f, loss = 0.0f;
    for (int k = threadIdx.x; k < a.K; k += kWave) high = fmaxf(high, to.t[k]);
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) high = fmaxf(high, __shfl_xor(high, d));
    for (int k = threadIdx.x; k < a.K; k += kWave) sum += to.t[k] == lowest ? 0.0f : expf((to.t[k] - high) / a.tau);
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    const bool row = all.s != 0.0f;                     // a row of -inf alone has no distribution: it counts for nothing
    const bool soft = row && a.w_kl != 0.0f && sum != 0.0f;
    const float log_sum = logf(sum), sums = a.tau * (logf(all.s) - log_sum);
    for (int k = threadIdx.x; k < a.K; k += kWave) {
        const float below = to.t[k] - high;
        const float q = soft && to.t[k] != lowest ? expf(below / a.tau - log_sum) : 0.0f;
        if (q != 0.0f) loss += q * (below - (to.z[k] - all.m) + sums);
        to.q[k] = a.w_kl * a.tau * q;
    }
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2) loss += __shfl_xor(loss, d);
    if (threadIdx.x == 0) {
        const bool hard = row && to.id[a.K] >= 0;
        loss = soft ? a.w_kl * a.tau * loss : 0.0f;
        if (hard) loss -= a.w_ce * ((to.z[a.K] - all.m) - logf(all.u));
        to.q[a.K] = hard ? a.w_ce : 0.0f;
        to.soft = soft ? a.w_kl * a.tau : 0.0f;
        to.hard = hard ? a.w_ce : 0.0f;
        to.loss = loss;
    }
}

// What a row's gradient is made of once its targets are settled: every element's share of p and p1, and the targets'.
template <class E, Extra X>
struct RowGradient {
    float m, c, soft, hard, gout;
    bool idle;                                          // a row without targets has no gradient, whatever its logits are
    __device__ __forceinline__ RowGradient(const DistillArgs<E> &a, int64_t n, const Stats &all, const Targets &to)
        : m(all.m), c(soft_factor(a)), gout(a.gout[n]), idle(to.soft == 0.0f && to.hard == 0.0f)
    {
        soft = to.soft == 0.0f ? 0.0f : gout * to.soft / all.s;
        hard = to.hard == 0.0f ? 0.0f : gout * to.hard / all.u;
    }
    __device__ __forceinline__ float share(float z) const
    {
        const float d = z - m, e = exp2_fast(d * c);
        if (X == kDual) return __builtin_fmaf(soft, e, hard * second<X>(d, e, kLog2e));
        if (X == kSquare) return e * __builtin_fmaf(hard, e, soft);
        if (X == kCube) return e * __builtin_fmaf(hard * e, e, soft);
        if (X == kFourth) return e * __builtin_fmaf(hard * e, e * e, soft);
        return (soft + hard) * e;
    }
    __device__ __forceinline__ u4 share_of(const u4 &w) const
    {
        float v[E::kPer16];
        E::unpack(w, v);
#pragma unroll
        for (int j = 0; j < E::kPer16; ++j) v[j] = share(v[j]);
        return E::pack(v);
    }
    // the targets in [lo, hi), behind a barrier that orders their second writing
    __device__ __forceinline__ void write_targets(const DistillArgs<E> &a, int64_t n, int64_t lo, int64_t hi, const Targets &to) const
    {
        for (int k = threadIdx.x; k <= a.K; k += blockDim.x) {
            const int id = to.id[k];
            if (id < lo || id >= hi) continue;
            float q = 0.0f;
            for (int i = 0; i <= a.K; ++i) q += to.id[i] == id ? to.q[i] : 0.0f;        // an id may be there twice, and be the label
            a.dz[n * a.ld_dz + id] = E::narrow(__builtin_fmaf(-gout, q, share(to.z[k])));
        }
    }
};

template <class E>
__device__ __forceinline__ void write_loss(const DistillArgs<E> &a, int64_t n, const Stats &all, const Targets &to)
{
    if (!a.loss) return;
    a.loss[n] = to.loss;
    if (a.stats) {
        a.stats[n * 4] = all.m; a.stats[n * 4 + 1] = all.s; a.stats[n * 4 + 2] = all.u; a.stats[n * 4 + 3] = 0.0f;
    }
}

// Keeps the compiler from holding a row's widened values between the passes over it: they would take twice the registers.
__device__ __forceinline__ void forget_widened(u4 &w) { asm volatile("" : "+v"(w)); }

// Loss and, if it is wanted, gradient of a row that fits the registers of one workgroup, KV vectors to a thread: it is read once.  The caches do
// not hold the rows of all workgroups, so a second reading would cross the same path as the first and the writing.  SAVED: the gradient alone,
// from the statistics that the loss left.
template <class E, Extra X, int KV, bool SAVED = false>
__global__ __launch_bounds__(kMostThreads, KV > 8 ? 4 : 8) void row_kernel(const DistillArgs<E> a)
{
    __shared__ Stats lds[kMostThreads / kWave];
    __shared__ Targets to;
    const int64_t n = blockIdx.x;
    const typename E::T *z = a.z + n * a.ld;
    const int vectors = static_cast<int>(a.V / E::kPer16), tail = static_cast<int>(a.V % E::kPer16), threads = blockDim.x;
    const Target own = load_target(a, n, threadIdx.x);
    // a thread's vector of those that begin at vector `first`: a uniform address and a 32-bit offset
    const uint32_t mine = threadIdx.x * 16u;
    const auto place = [&](auto *row, int first) {
        using P = decltype(row);
        return reinterpret_cast<P>(reinterpret_cast<std::conditional_t<std::is_const_v<std::remove_pointer_t<P>>, const char, char> *>(row) +
                                   static_cast<int64_t>(first) * 16 + mine);
    };
    u4 w[KV];
#pragma unroll
    for (int k = 0; k < KV; ++k) {
        w[k] = u4{E::kNothing, E::kNothing, E::kNothing, E::kNothing};
        if (k * threads + static_cast<int>(threadIdx.x) < vectors) w[k] = load16<E>(place(z, k * threads));
    }
    const bool has_tail = static_cast<int>(threadIdx.x) < tail;
    const float z_tail = has_tail ? E::widen(z[static_cast<int64_t>(vectors) * E::kPer16 + threadIdx.x]) : -__builtin_inff();
    keep_target(a, n, threadIdx.x, own, to);
    keep_others(a, n, to);
    const float c = soft_factor(a);
    Stats all{kLowest, 0.0f, 0.0f};
    if constexpr (SAVED) {
        all = {a.stats[n * 4], a.stats[n * 4 + 1], a.stats[n * 4 + 2]};
        __syncthreads();
    } else {
        {
            float high[2] = {z_tail, z_tail};
    #pragma unroll
            for (int k = 0; k < KV; ++k) {
                float v[E::kPer16];
                E::unpack(w[k], v);
    #pragma unroll
                for (int j = 0; j < E::kPer16; ++j) high[j & 1] = fmaxf(high[j & 1], v[j]);
            }
            all.m = fmaxf(all.m, fmaxf(high[0], high[1]));
        }
    #pragma unroll
        for (int k = 0; k < KV; ++k) {
            float v[E::kPer16];
            forget_widened(w[k]);
            E::unpack(w[k], v);
            add_terms<X>(all, v, c, kLog2e);
        }
        const float last[1] = {z_tail};
        add_terms<X>(all, last, c, kLog2e);
        all = join_workgroup<X>(all, lds, c, kLog2e, threads / kWave);
        if (!two_sums(X)) all.u = all.s;                    // one sum serves both
    }
    if (threadIdx.x < kWave) settle(a, all, to);
    __syncthreads();
    if (!SAVED && threadIdx.x == 0) write_loss(a, n, all, to);
    if (!a.dz) return;
    const RowGradient<E, X> gradient(a, n, all, to);
    typename E::T *dz = a.dz + n * a.ld_dz;
#pragma unroll
    for (int k = 0; k < KV; ++k) {
        forget_widened(w[k]);
        if (k * threads + static_cast<int>(threadIdx.x) < vectors) store16<E>(place(dz, k * threads), gradient.idle ? u4{} : gradient.share_of(w[k]));
    }
    if (has_tail) dz[static_cast<int64_t>(vectors) * E::kPer16 + threadIdx.x] = gradient.idle ? E::narrow(0.0f) : E::narrow(gradient.share(z_tail));
    __syncthreads();
    if (!gradient.idle) gradient.write_targets(a, n, 0, a.V, to);
}

enum Source { kHere, kParts, kSaved };                  // where a row's statistics come from

// Grid (parts, N).  kHere: one part, read a second time for the gradient, its end first: what the caches still hold.
template <class E, Extra X, Source FROM>
__global__ __launch_bounds__(kRowThreads) void distill_kernel(const DistillArgs<E> a)
{
    __shared__ Stats lds[kRowWaves];
    __shared__ Targets to;
    const int part = FROM == kHere ? 0 : blockIdx.x, parts = FROM == kHere ? 1 : a.parts;
    const int64_t n = blockIdx.y, lo = part_begin(a.V, parts, part, E::kPer16), hi = part_begin(a.V, parts, part + 1, E::kPer16);
    const Slice<E> slice(a.z + n * a.ld, lo, hi);
    keep_target(a, n, threadIdx.x, load_target(a, n, threadIdx.x), to);
    Stats all;
    if constexpr (FROM == kHere) {
        all = slice_stats<E, X>(slice, soft_factor(a), lds);
    } else if constexpr (FROM == kParts) {
        all = a.part_stats[n * parts];
        for (int k = 1; k < parts; ++k) all = join<X>(all, a.part_stats[n * parts + k], soft_factor(a), kLog2e);
    } else {
        all = {a.stats[n * 4], a.stats[n * 4 + 1], a.stats[n * 4 + 2]};
    }
    if (FROM != kSaved && !two_sums(X)) all.u = all.s;
    __syncthreads();
    if (threadIdx.x < kWave) settle(a, all, to);
    __syncthreads();
    if (FROM != kSaved && part == 0 && threadIdx.x == 0) write_loss(a, n, all, to);
    if (!a.dz) return;
    const RowGradient<E, X> gradient(a, n, all, to);
    typename E::T *dz = a.dz + n * a.ld_dz + lo;
    if (slice.has_tail()) dz[slice.tail_at()] = gradient.idle ? E::narrow(0.0f) : E::narrow(gradient.share(E::widen(slice.z[slice.tail_at()])));
    for (int round = slice.rounds() - 1; round >= 0; --round) {
        u4 w[kAhead];
        slice.load(round, w);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int at = slice.vector_of(round, i);
            if (at < slice.vectors) store16<E>(dz + static_cast<int64_t>(at) * E::kPer16, gradient.idle ? u4{} : gradient.share_of(w[i]));
        }
    }
    __syncthreads();
    if (!gradient.idle) gradient.write_targets(a, n, lo, hi, to);
}

struct DistillSpace {
    int parts;
    int64_t bytes;
};

// From so many rows on the gradient alone takes a row in registers too, if it fits 4 vectors of a thread: workgroups as large as the row is long take
// 11 us for 8,192 rows of 500 bfloat16 logits against 40 with the others' 256 threads, 50 against 58 for 4,096 of 16,000.
constexpr int64_t kManyRows = 512;

// The gradient alone needs nothing of a row but its statistics: as many workgroups to a row as give a CU two.
int grad_parts(int64_t N, int64_t V, int per16)
{
    const int64_t fit = ceil_div(V, static_cast<int64_t>(kRowThreads) * per16 * 2), wanted = ceil_div(512, N);
    return static_cast<int>(N >= kManyRows ? 1 : fit < wanted ? fit : wanted);
}

constexpr int64_t kRegisterVectors = 16 * kMostThreads;         // of a row that one workgroup's registers hold
// Up to so many rows the long ones are split even if they would fit, as a workgroup to a row leaves CUs idle: loss and gradient of 4 rows of 131,072
// bfloat16 logits take 14 us against 25, of 128 rows 26 against 31, but of 200 36 against 33.
constexpr int64_t kFewRows = 128;

DistillSpace distill_space(int64_t N, int64_t V, int per16)
{
    const int parts = V / per16 > kRegisterVectors || N <= kFewRows ? parts_of(N, V, per16) : 1;
    return {parts, parts > 1 ? N * parts * static_cast<int64_t>(sizeof(Stats)) : 0};
}

int check_sizes(int64_t N, int32_t V, int32_t K)
{
    return N < 0 || N > CX_MAX_TOKENS || V < 1 || V > CX_MAX_VOCAB || K < 0 || K > kMaxTeacher ? CX_ERR_SHAPE : CX_OK;
}

// from_saved: the gradient alone, from the statistics that the loss left.
template <class E>
int distill(DistillArgs<E> a, int64_t N, bool from_saved, bool want_dz, void *workspace, int64_t workspace_bytes, void *stream)
{
    const int rc = check_sizes(N, static_cast<int32_t>(a.V), a.K);
    if (rc != CX_OK) return rc;
    if (!(a.tau > 0.0f) || !(a.tau <= 3.0e38f) || !(a.w_kl >= 0.0f) || !(a.w_ce >= 0.0f) || !(a.w_kl <= 3.0e38f) || !(a.w_ce <= 3.0e38f)) return CX_ERR_SHAPE;
    if (!(kLog2e / a.tau <= kLargest) || !(a.w_kl * a.tau <= kLargest)) return CX_ERR_SHAPE;        // factors of every element
    if (N == 0) return CX_OK;
    if (!a.z || (a.K > 0 && (!a.ids || !a.t)) || (want_dz && (!a.dz || !a.gout)) || (!from_saved && !a.loss) || (from_saved && !a.stats)) return CX_ERR_NULL;
    if (bad_matrix(N, a.ld, a.V) || (want_dz && bad_matrix(N, a.ld_dz, a.V))) return CX_ERR_SHAPE;
    DistillSpace space = distill_space(N, a.V, E::kPer16);
    if (from_saved) space.parts = grad_parts(N, a.V, E::kPer16);
    const int64_t need = from_saved ? 0 : space.bytes;
    if (need > 0 && !workspace) return CX_ERR_NULL;
    if (need > 0 && workspace_bytes < need) return CX_ERR_SHAPE;
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(a.z, kElem) || misaligned_to(a.dz, kElem) || misaligned_to(a.ids, 4) || misaligned_to(a.labels, 4) || misaligned_to(a.t, 4) ||
        misaligned_to(a.gout, 4) || misaligned_to(a.loss, 4) || misaligned_to(a.stats, 4) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const uint64_t row_bytes = N * 4, top_bytes = N * a.K * 4;
    const Extent in[5] = {matrix_of(a.z, N, a.ld, a.V, kElem), dense_of(a.ids, top_bytes), dense_of(a.t, top_bytes), dense_of(a.labels, row_bytes),
                          dense_of(a.gout, row_bytes)};
    const Extent out[4] = {matrix_of(a.dz, want_dz ? N : 0, a.ld_dz, a.V, kElem), dense_of(a.loss, from_saved ? 0 : row_bytes),
                           dense_of(a.stats, row_bytes * 4), dense_of(workspace, need)};
    if (outputs_share(in, out, 0, 0)) return CX_ERR_ALIAS;
    if (!want_dz) a.dz = nullptr;
    a.parts = space.parts;
    a.part_stats = static_cast<Stats *>(workspace);
    const bool dual = a.w_kl != 0.0f && a.w_ce != 0.0f && a.tau != 1.0f;
    const Extra sums = !dual ? kNone : a.tau == 2.0f ? kSquare : a.tau == 3.0f ? kCube : a.tau == 4.0f ? kFourth : kDual;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    for (int64_t n0 = 0; n0 < N; n0 += 65535) {         // rows in slices of a grid's second dimension
        const unsigned rows = static_cast<unsigned>(N - n0 < 65535 ? N - n0 : 65535);
        DistillArgs<E> b = a;
        b.z += n0 * a.ld;
        if (b.dz) b.dz += n0 * a.ld_dz;
        if (b.ids) b.ids += n0 * a.K;
        if (b.t) b.t += n0 * a.K;
        if (b.labels) b.labels += n0;
        if (b.gout) b.gout += n0;
        if (b.loss) b.loss += n0;
        if (b.stats) b.stats += n0 * 4;
        const dim3 whole(1, rows), parted(space.parts, rows), block(kRowThreads);
        const auto launch = [&](auto kind) {
            constexpr Extra X = decltype(kind)::value;
            const int64_t vectors = a.V / E::kPer16;
            const auto threads = [&](int64_t each) { return dim3(static_cast<unsigned>(vectors < each ? kWave : round_up(ceil_div(vectors, each), kWave))); };
            if (from_saved && N >= kManyRows && vectors <= 4 * kMostThreads) {
                hipLaunchKernelGGL((row_kernel<E, X, 4, true>), dim3(rows), threads(4), 0, st, b);
            } else if (from_saved) {
                hipLaunchKernelGGL((distill_kernel<E, X, kSaved>), parted, block, 0, st, b);
            } else if (space.parts == 1) {
                if (vectors > kRegisterVectors) hipLaunchKernelGGL((distill_kernel<E, X, kHere>), whole, block, 0, st, b);
                else if (vectors > 8 * kMostThreads) hipLaunchKernelGGL((row_kernel<E, X, 16>), dim3(rows), threads(16), 0, st, b);
                else if (vectors > 4 * kMostThreads) hipLaunchKernelGGL((row_kernel<E, X, 8>), dim3(rows), threads(8), 0, st, b);
                else hipLaunchKernelGGL((row_kernel<E, X, 4>), dim3(rows), threads(4), 0, st, b);
            } else {                                    // few rows: one slice of them
                hipLaunchKernelGGL((part_kernel<E, X>), parted, block, 0, st, b);
                if (want_dz && static_cast<const void *>(a.dz) == a.z) {
                    // the loss reads logits of all parts: where gradients replace them, it comes first, in a launch of its own
                    DistillArgs<E> first = b;
                    first.dz = nullptr;
                    hipLaunchKernelGGL((distill_kernel<E, X, kParts>), whole, block, 0, st, first);
                    b.loss = nullptr;
                }
                hipLaunchKernelGGL((distill_kernel<E, X, kParts>), want_dz ? parted : whole, block, 0, st, b);
            }
        };
        switch (sums) {
        case kDual: launch(std::integral_constant<Extra, kDual>{}); break;
        case kSquare: launch(std::integral_constant<Extra, kSquare>{}); break;
        case kCube: launch(std::integral_constant<Extra, kCube>{}); break;
        case kFourth: launch(std::integral_constant<Extra, kFourth>{}); break;
        default: launch(std::integral_constant<Extra, kNone>{});
        }
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    return CX_OK;
}

}  // namespace

extern "C" {

#define CX_LM_DISTILL(SUFFIX, E)                                                                                                      \
    int cx_distill_loss##SUFFIX(const E::T *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,       \
                                const int32_t *labels, float tau, float w_kl, float w_ce, float *loss, float *stats,                  \
                                void *workspace, int64_t workspace_bytes, void *stream)                                               \
    {                                                                                                                                 \
        DistillArgs<E> a{};                                                                                                           \
        a.z = z; a.ids = ids; a.labels = labels; a.t = t; a.loss = loss; a.stats = stats; a.ld = ld; a.V = V; a.K = K;                \
        a.tau = tau; a.w_kl = w_kl; a.w_ce = w_ce;                                                                                    \
        return distill<E>(a, N, false, false, workspace, workspace_bytes, stream);                                                    \
    }                                                                                                                                 \
    int cx_distill_grad##SUFFIX(const E::T *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,       \
                                const int32_t *labels, float tau, float w_kl, float w_ce, const float *stats, const float *gout,      \
                                E::T *dz, int64_t ld_dz, void *stream)                                                                \
    {                                                                                                                                 \
        DistillArgs<E> a{};                                                                                                           \
        a.z = z; a.ids = ids; a.labels = labels; a.t = t; a.stats = const_cast<float *>(stats); a.gout = gout; a.dz = dz; a.ld = ld;  \
        a.ld_dz = ld_dz; a.V = V; a.K = K; a.tau = tau; a.w_kl = w_kl; a.w_ce = w_ce;                                                 \
        return distill<E>(a, N, true, true, nullptr, 0, stream);                                                                      \
    }                                                                                                                                 \
    int cx_distill_step##SUFFIX(const E::T *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,       \
                                const int32_t *labels, float tau, float w_kl, float w_ce, const float *gout, float *loss,             \
                                E::T *dz, int64_t ld_dz, void *workspace, int64_t workspace_bytes, void *stream)                      \
    {                                                                                                                                 \
        DistillArgs<E> a{};                                                                                                           \
        a.z = z; a.ids = ids; a.labels = labels; a.t = t; a.loss = loss; a.gout = gout; a.dz = dz; a.ld = ld; a.ld_dz = ld_dz;        \
        a.V = V; a.K = K; a.tau = tau; a.w_kl = w_kl; a.w_ce = w_ce;                                                                  \
        return distill<E>(a, N, false, true, workspace, workspace_bytes, stream);                                                     \
    }
CX_LM_DISTILL(, F32)
CX_LM_DISTILL(_bf16, Bf16)
CX_LM_DISTILL(_f16, F16)
#undef CX_LM_DISTILL

int cx_distill_workspace(int64_t N, int32_t V, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_sizes(N, V, 0);
    if (rc != CX_OK || N == 0) return rc;
    const int64_t wide = distill_space(N, V, F32::kPer16).bytes, narrow = distill_space(N, V, Bf16::kPer16).bytes;
    *bytes = wide > narrow ? wide : narrow;
    return CX_OK;
}

}  // extern "C"
