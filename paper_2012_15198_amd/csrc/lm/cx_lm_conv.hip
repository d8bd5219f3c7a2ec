// C-ABI entry points cx_short_conv*, cx_short_conv_grad*, cx_conv_workspace: the short causal convolution (see include/cx_lm.h)
//
//   z_t = bias + sum_k w_k x_{t-K+1+k}    y = silu(z) or z    nothing is seen across a reset
//   d_t = dy_t silu'(z_t)    dx_t = sum_j w_{K-1-j} d_{t+j}    dw_k = sum_t d_t x_{t-K+1+k}    dbias = sum_t d_t
//
// A lane holds 16 bytes of columns (the gradient: four columns), their K taps and the last K - 1 inputs in registers and walks a span of steps, so that a
// row is read once, but for the K - 1 rows in front of a span (the gradient: also behind it).
//
// Bound by memory: 32 sequences of 2,048 x 1,024 in bfloat16 take 54 us (5.0 TB/s), the gradient 92 and 5 for the sums of its parts (4.4 TB/s): its
// spans of 64 steps read 9 % more, and vector instructions issue in two thirds of the time, so that neither bounds it alone.  Short spans hide what few lanes wait for: 6 sequences of
// 5,519 x 23 take 16 us in the gradient with 8 steps, 60 with 32.  A step of 64 x 2,048 takes 3.6.  Tried and not kept for the gradient: eight columns of a lane
// (230 registers, 115 us), four rows ahead (99), results past the caches (96; 83 where the forward pass's go past them too, which takes 58 then).
#include "lm_block.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4, kGradAhead = 2;               // rows whose loads are in flight; spans are whole multiples
constexpr int64_t kMaxSeq = CX_MAX_TOKENS;

template <class E>
struct ConvArgs {
    using T = typename E::T;
    const T *x, *dy, *weights, *before;
    T *y, *dx, *after;
    int64_t ldx, ldy, lddy, lddx, ldw;
    const uint8_t *reset;
    float *parts;
    int64_t B, T_;
    uint32_t per_worker;                                // sequences of a worker
    int64_t span, spans;                                // steps of a lane's walk; spans of a sequence, rounded up to whole workgroups
    int32_t D, shift, slabs;                            // 1 << shift lanes beside each other
    bool silu;
    bool shared_ends;                                   // the last lane begins C columns before the end of the row: what it has in common with the one before both compute
};

template <class E, int C, int K>
__device__ __forceinline__ void load_taps(const ConvArgs<E> &a, int64_t w, int column, int left, float (&tap)[K][C], float (&bias)[C])
{
    const typename E::T *p = a.weights + w * a.ldw;
    widen<E, C>(load_columns<E, C>(p + static_cast<int64_t>(a.D) * K + column, left), bias);
    float flat[K][C];                                   // C K elements in a row: column j, tap k at j K + k
#pragma unroll
    for (int i = 0; i < K; ++i) widen<E, C>(load_columns<E, C>(p + static_cast<int64_t>(column) * K + i * C, left * K - i * C), flat[i]);
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int k = 0; k < K; ++k) tap[k][j] = flat[(j * K + k) / C][(j * K + k) % C];
}

// seen[0 .. K - 2] before a step, the oldest first, its input behind them; a reset clears what is before it.
template <int C, int K>
__device__ __forceinline__ void clear(float (&seen)[K][C], int count = K - 1)
{
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (k < count) seen[k][j] = 0.0f;
}
template <int C, int K>
__device__ __forceinline__ void shift_out(float (&seen)[K][C])
{
#pragma unroll
    for (int k = 0; k + 1 < K; ++k)
#pragma unroll
        for (int j = 0; j < C; ++j) seen[k][j] = seen[k + 1][j];
}

// The inputs before step t: of this sequence's earlier rows or of `before`; zeros from before a reset.
template <class E, int C, int K>
__device__ __forceinline__ void enter(const ConvArgs<E> &a, int64_t b, int64_t t, int column, int left, float (&seen)[K][C])
{
#pragma unroll
    for (int k = 0; k < K - 1; ++k) {
        const int64_t s = t - (K - 1) + k;
        if (s >= 0) {
            if (a.reset && a.reset[b * a.T_ + s] != 0) clear<C, K>(seen, k);
            widen<E, C>(load_columns<E, C>(a.x + (b * a.T_ + s) * a.ldx + column, left), seen[k]);
        } else if (a.before) {
            widen<E, C>(load_columns<E, C>(a.before + (b * (K - 1) + (K - 1 + s)) * a.D + column, left), seen[k]);
        } else {
#pragma unroll
            for (int j = 0; j < C; ++j) seen[k][j] = 0.0f;
        }
    }
}

template <int C, int K>
__device__ __forceinline__ void convolve(const float (&seen)[K][C], const float (&tap)[K][C], const float (&bias)[C], float (&z)[C])
{
#pragma unroll
    for (int j = 0; j < C; ++j) {
        z[j] = bias[j];
#pragma unroll
        for (int k = 0; k < K; ++k) z[j] = __builtin_fmaf(tap[k][j], seen[k][j], z[j]);
    }
}

struct Place {
    int64_t b, begin, end, span;
    int column;
    bool any;
};
// Grid: (slabs of columns of groups of spans, sequences in two dimensions).
template <class E, int C>
__device__ __forceinline__ Place place_of(const ConvArgs<E> &a)
{
    const int lane = threadIdx.x & ((1 << a.shift) - 1), together = blockDim.x >> a.shift;
    const int slab = static_cast<int>(blockIdx.x % a.slabs);
    Place p;
    p.b = blockIdx.y + static_cast<int64_t>(blockIdx.z) * gridDim.y;
    p.span = static_cast<int64_t>(blockIdx.x / a.slabs) * together + (threadIdx.x >> a.shift);
    p.begin = p.span * a.span;
    p.end = p.begin + a.span < a.T_ ? p.begin + a.span : a.T_;
    p.column = ((slab << a.shift) + lane) * C;
    p.any = p.begin < a.T_ && p.column < a.D && p.b < a.B;
    if (a.shared_ends && p.column < a.D && p.column > a.D - C) p.column = a.D - C;
    return p;
}

template <class E, int C, int K, bool RESETS>
__global__ __launch_bounds__(kThreads) void conv_kernel(const ConvArgs<E> a)
{
    const Place p = place_of<E, C>(a);
    if (!p.any) return;
    const int left = a.D - p.column;
    float tap[K][C], bias[C], seen[K][C];
    load_taps<E, C, K>(a, static_cast<uint32_t>(p.b) / a.per_worker, p.column, left, tap, bias);
    enter<E, C, K>(a, p.b, p.begin, p.column, left, seen);
    if (K > 1 && p.begin == 0 && a.after) {             // by the lanes that have read `before`, which may be the same
        float last[K][C];
        enter<E, C, K>(a, p.b, a.T_, p.column, left, last);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) store_columns<E, C>(a.after + (p.b * (K - 1) + k) * a.D + p.column, left, last[k]);
    }
    const int64_t row0 = p.b * a.T_ + p.begin;
    const typename E::T *x = a.x + row0 * a.ldx + p.column;
    typename E::T *y = a.y + row0 * a.ldy + p.column;
    const int steps = static_cast<int>(p.end - p.begin);
    const auto some = [&](auto whole, int t0) {         // whole: kAhead steps, all columns
        constexpr bool WHOLE = decltype(whole)::value;
        const int columns = WHOLE ? C : left;
        Columns<E, C> ahead[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ahead[i] = load_columns<E, C>(x + i * a.ldx, WHOLE || t0 + i < steps ? columns : 0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (!WHOLE && t0 + i >= steps) break;
            if (RESETS && a.reset[row0 + t0 + i] != 0) clear<C, K>(seen);
            widen<E, C>(ahead[i], seen[K - 1]);
            float z[C];
            convolve<C, K>(seen, tap, bias, z);
            if (a.silu)
#pragma unroll
                for (int j = 0; j < C; ++j) z[j] = finite_below(z[j]) * sigmoid(z[j]);
            store_columns<E, C>(y + i * a.ldy, columns, z);
            shift_out<C, K>(seen);
        }
        x += kAhead * a.ldx;
        y += kAhead * a.ldy;
    };
    for (int t0 = 0; t0 < steps; t0 += kAhead) {
        if (t0 + kAhead <= steps && left >= C) some(std::true_type{}, t0);
        else some(std::false_type{}, t0);
    }
}

// One step, as decoding takes them: everything is loaded before anything is stored, and no step waits for another.
template <class E, int C, int K>
__global__ __launch_bounds__(kWave) void conv_step_kernel(const ConvArgs<E> a)
{
    const int column = (static_cast<int>(blockIdx.x % a.slabs) * kWave + threadIdx.x) * C, left = a.D - column;
    const int64_t b = blockIdx.x / a.slabs;
    if (left <= 0) return;
    Columns<E, C> inputs[K];
    const bool fresh = a.reset && a.reset[b] != 0;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) inputs[k] = load_columns<E, C>(a.before + (b * (K - 1) + k) * a.D + column, a.before && !fresh ? left : 0);
    inputs[K - 1] = load_columns<E, C>(a.x + b * a.ldx + column, left);
    float tap[K][C], bias[C], seen[K][C], z[C];
    load_taps<E, C, K>(a, static_cast<uint32_t>(b) / a.per_worker, column, left, tap, bias);
#pragma unroll
    for (int k = 0; k < K; ++k) widen<E, C>(inputs[k], seen[k]);
    convolve<C, K>(seen, tap, bias, z);
    if (a.silu)
#pragma unroll
        for (int j = 0; j < C; ++j) z[j] = finite_below(z[j]) * sigmoid(z[j]);
    store_columns<E, C>(a.y + b * a.ldy + column, left, z);
    if (a.after)
#pragma unroll
        for (int k = 0; k < K - 1; ++k) store_columns<E, C>(a.after + (b * (K - 1) + k) * a.D + column, left, seen[k + 1]);
}

template <class E, int C, int K, bool RESETS>
__global__ __launch_bounds__(kThreads) void conv_grad_kernel(const ConvArgs<E> a)
{
    __shared__ float sums[kThreads][C + 1];
    const Place p = place_of<E, C>(a);
    const int lane = threadIdx.x & ((1 << a.shift) - 1), group = threadIdx.x >> a.shift, together = blockDim.x >> a.shift;
    const int left = p.any ? a.D - p.column : 0;
    float dw[K + 1][C] = {};                            // the bias's behind the taps'
    if (p.any) {
        float tap[K][C], bias[C], seen[K][C];
        load_taps<E, C, K>(a, static_cast<uint32_t>(p.b) / a.per_worker, p.column, left, tap, bias);
        enter<E, C, K>(a, p.b, p.begin, p.column, left, seen);
        float open[K][C] = {};                          // gradients of the inputs of steps t - K + 1 .. t, oldest first
        int visible = 0;                                // steps behind that step t's taps see and that belong to this span
        const int64_t row0 = p.b * a.T_ + p.begin;
        const typename E::T *x = a.x + row0 * a.ldx + p.column, *dy = a.dy + row0 * a.lddy + p.column;
        typename E::T *dx = a.dx + (row0 - (K - 1)) * a.lddx + p.column;            // of the step that nothing later reaches
        // K - 1 steps more than the span's: what later steps add to its inputs
        const int own = static_cast<int>(p.end - p.begin), stop = own + K - 1;
        const int there = a.T_ - p.begin < stop ? static_cast<int>(a.T_ - p.begin) : stop;
        const auto some = [&](auto whole, int t0) {     // whole: kGradAhead steps of the span whose results are all its own, all columns
            constexpr bool WHOLE = decltype(whole)::value;
            const int columns = WHOLE ? C : left;
            Columns<E, C> xs[kGradAhead], gs[kGradAhead];
#pragma unroll
            for (int i = 0; i < kGradAhead; ++i) {
                xs[i] = load_columns<E, C>(x + i * a.ldx, WHOLE || t0 + i < there ? columns : 0);
                gs[i] = load_columns<E, C>(dy + i * a.lddy, WHOLE || t0 + i < there ? columns : 0);
            }
#pragma unroll
            for (int i = 0; i < kGradAhead; ++i) {
                const int t = t0 + i;
                if (!WHOLE && t >= stop) break;
                if (RESETS && (WHOLE || t < there) && a.reset[row0 + t] != 0) {
                    clear<C, K>(seen);
                    visible = 0;
                }
                widen<E, C>(xs[i], seen[K - 1]);
                float d[C], z[C];
                widen<E, C>(gs[i], d);
                if (a.silu) {
                    convolve<C, K>(seen, tap, bias, z);
#pragma unroll
                    for (int j = 0; j < C; ++j) {
                        z[j] = finite_below(z[j]);
                        d[j] *= silu_slope(z[j], sigmoid(z[j]));
                    }
                }
                if (WHOLE || t < there) {
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const bool reaches = !RESETS || K - 1 - k <= visible;
#pragma unroll
                        for (int j = 0; j < C; ++j)
                            if (reaches) open[k][j] = __builtin_fmaf(tap[k][j], d[j], open[k][j]);
                    }
                    if (WHOLE || t < own)
#pragma unroll
                        for (int k = 0; k <= K; ++k)
#pragma unroll
                            for (int j = 0; j < C; ++j) dw[k][j] = k < K ? __builtin_fmaf(d[j], seen[k < K ? k : 0][j], dw[k][j]) : dw[k][j] + d[j];
                }
                if (WHOLE || t >= K - 1) store_columns<E, C>(dx + i * a.lddx, columns, open[0]);
                shift_out<C, K>(open);
#pragma unroll
                for (int j = 0; j < C; ++j) open[K - 1][j] = 0.0f;
                shift_out<C, K>(seen);
                visible = visible < K - 1 ? visible + 1 : K - 1;
            }
            x += kGradAhead * a.ldx;
            dy += kGradAhead * a.lddy;
            dx += kGradAhead * a.lddx;
        };
        for (int t0 = 0; t0 < stop; t0 += kGradAhead) {
            if (t0 >= K - 1 && t0 + kGradAhead <= own && left >= C) some(std::true_type{}, t0);
            else some(std::false_type{}, t0);
        }
    }
    // the sums of the workgroup's spans, of columns [D][K] and then [D]
    const int64_t columns = static_cast<int64_t>(a.D) * (K + 1), groups = a.spans / together;
    float *part = a.parts + (p.b * groups + blockIdx.x / a.slabs) * columns;
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < C; ++j) sums[threadIdx.x][j] = dw[k][j];
        __syncthreads();
        if (group > 0 || p.b >= a.B) continue;
        for (int g = 1; g < together; ++g)
#pragma unroll
            for (int j = 0; j < C; ++j) dw[k][j] += sums[(g << a.shift) + lane][j];
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (p.column + j < a.D) part[k < K ? (p.column + j) * static_cast<int64_t>(K) + k : static_cast<int64_t>(a.D) * K + p.column + j] = dw[k][j];
    }
}

struct Walk {
    int shift, slabs, together;
    int64_t span, spans, groups;                        // groups of spans that share a workgroup
};

constexpr int64_t kWalks = 1 << 18;                     // lanes that fill the card

constexpr int64_t kLeastSteps = 8, kLeastGradSteps = 32, kFewWalks = 1 << 15;

Walk walk_of(int64_t B, int64_t T, int32_t D, int columns, int64_t least)
{
    Walk w{};
    const int64_t lanes = ceil_div(D, columns);
    while ((1 << w.shift) < lanes && (1 << w.shift) < kWave) ++w.shift;
    w.slabs = static_cast<int>(ceil_div(lanes, 1 << w.shift));
    const int64_t wanted = ceil_div(kWalks, B * lanes);
    const int64_t span = ceil_div(T, wanted);
    if (B * lanes * ceil_div(T, least) < kFewWalks) least = kLeastSteps;       // too few to hide a step's loads
    w.span = round_up(span < least ? (T < least ? T : least) : span, kAhead);
    const int64_t spans = ceil_div(T, w.span);
    w.together = kThreads >> w.shift;
    while (w.together > 1 && w.together / 2 >= spans && (w.together / 2) << w.shift >= kWave) w.together /= 2;
    w.groups = ceil_div(spans, w.together);
    w.spans = w.groups * w.together;
    return w;
}
constexpr int kGradColumns = 4;                         // columns of a lane

int check_conv(int32_t W, int64_t B, int64_t T, int32_t D, int32_t K)
{
    return W < 1 || W > CX_MAX_ROWS || B < 0 || B > CX_MAX_SEQUENCES || B % W != 0 || T < 0 || T > kMaxSeq || D < 1 || D > CX_MAX_WIDTH || K < 1 ||
                   K > CX_MAX_TAPS || B * D > (int64_t(1) << 31)
               ? CX_ERR_SHAPE
               : CX_OK;
}

int64_t parts_bytes(int64_t B, int64_t T, int32_t D, int32_t K)
{
    if (B == 0 || T == 0) return 0;
    return B * walk_of(B, T, D, kGradColumns, kLeastGradSteps).groups * D * (K + 1) * 4;
}

template <class E>
void set_walk(ConvArgs<E> &a, const Walk &w)
{
    a.shift = w.shift; a.slabs = w.slabs; a.span = w.span; a.spans = w.spans;
}

template <class F>
int by_taps(int K, const F &launch)
{
    switch (K) {
    case 1: launch(std::integral_constant<int, 1>{}); break;
    case 2: launch(std::integral_constant<int, 2>{}); break;
    case 3: launch(std::integral_constant<int, 3>{}); break;
    default: launch(std::integral_constant<int, 4>{}); break;
    }
    return launched();
}

dim3 grid_of(const Walk &w, int64_t B)
{
    const int64_t y = B < 32768 ? B : 32768;
    return dim3(static_cast<unsigned>(w.groups * w.slabs), static_cast<unsigned>(y), static_cast<unsigned>(ceil_div(B, y)));
}

template <class E>
int conv(const typename E::T *x, int64_t ldx, const typename E::T *weights, int64_t ld, int32_t W, int64_t offset, typename E::T *y, int64_t ldy, int64_t B,
         int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const typename E::T *before, typename E::T *after, void *stream)
{
    const int rc = check_conv(W, B, T, D, K);
    if (rc != CX_OK || bad_rows(W, ld, offset, static_cast<int64_t>(D) * (K + 1))) return CX_ERR_SHAPE;
    if (B == 0) return CX_OK;
    constexpr int kElem = sizeof(typename E::T);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t ends = B * (K - 1) * D;
    if (misaligned_to(before, kElem) || misaligned_to(after, kElem)) return CX_ERR_ALIGN;
    if (before != after && overlap(before, ends * kElem, after, ends * kElem)) return CX_ERR_ALIAS;
    if (T == 0) return pass_through(before, after, ends, st);
    if (!x || !y || !weights) return CX_ERR_NULL;
    if (bad_matrix(B * T, ldx, D) || bad_matrix(B * T, ldy, D)) return CX_ERR_SHAPE;
    if (misaligned_to(x, kElem) || misaligned_to(weights, kElem) || misaligned_to(y, kElem)) return CX_ERR_ALIGN;
    const Extent in[4] = {matrix_of(x, B * T, ldx, D, kElem), matrix_of(weights, W, ld, offset + static_cast<int64_t>(D) * (K + 1), kElem), dense_of(reset, B * T),
                          dense_of(before, ends * kElem)};
    const Extent out[2] = {matrix_of(y, B * T, ldy, D, kElem), dense_of(after, ends * kElem)};
    const Same same[1] = {{1, 3}};
    if (outputs_share_but(in, out, same)) return CX_ERR_ALIAS;
    constexpr int kForward = sizeof(typename E::T) == 4 ? 4 : 8;         // 16 bytes
    const Walk w = walk_of(B, T, D, kForward, kLeastSteps);
    if (w.groups * w.slabs > 0x7fffffff) return CX_ERR_SHAPE;
    ConvArgs<E> a{};
    a.x = x; a.ldx = ldx; a.weights = weights + offset; a.ldw = ld; a.y = y; a.ldy = ldy; a.before = before; a.after = after; a.reset = reset;
    a.B = B; a.T_ = T; a.per_worker = static_cast<uint32_t>(B / W); a.D = D; a.silu = silu != 0;
    set_walk(a, w);
    a.shared_ends = D >= kForward && !(before && before == after);      // a state in place has one reader and writer
    if (T == 1) {
        a.slabs = static_cast<int32_t>(ceil_div(ceil_div(D, kForward), kWave));
        return by_taps(K, [&](auto k) {
            hipLaunchKernelGGL((conv_step_kernel<E, kForward, decltype(k)::value>), dim3(static_cast<unsigned>(B * a.slabs)), dim3(kWave), 0, st, a);
        });
    }
    return by_taps(K, [&](auto k) {
        if (reset) hipLaunchKernelGGL((conv_kernel<E, kForward, decltype(k)::value, true>), grid_of(w, B), dim3(w.together << w.shift), 0, st, a);
        else hipLaunchKernelGGL((conv_kernel<E, kForward, decltype(k)::value, false>), grid_of(w, B), dim3(w.together << w.shift), 0, st, a);
    });
}

template <class E>
int conv_grad(const typename E::T *x, int64_t ldx, const typename E::T *dy, int64_t lddy, const typename E::T *weights, int64_t ldw, int32_t W,
              int64_t offset, typename E::T *dx, int64_t lddx, const typename E::T *g_in, typename E::T *g_out, int64_t ld, int64_t B, int64_t T,
              int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const typename E::T *before, void *workspace, int64_t workspace_bytes, void *stream)
{
    const int rc = check_conv(W, B, T, D, K);
    const int64_t columns = static_cast<int64_t>(D) * (K + 1);
    if (rc != CX_OK || bad_rows(W, ldw, offset, columns) || bad_rows(W, ld, offset, columns)) return CX_ERR_SHAPE;
    if (!g_out) return CX_ERR_NULL;
    constexpr int kElem = sizeof(typename E::T);
    const bool none = B == 0 || T == 0;
    const int64_t ends = B * (K - 1) * D, bytes = parts_bytes(B, T, D, K);
    if (!none) {
        if (!x || !dy || !weights || !dx || !workspace) return CX_ERR_NULL;
        if (bad_matrix(B * T, ldx, D) || bad_matrix(B * T, lddy, D) || bad_matrix(B * T, lddx, D) || workspace_bytes < bytes) return CX_ERR_SHAPE;
    }
    if (misaligned_to(x, kElem) || misaligned_to(dy, kElem) || misaligned_to(weights, kElem) || misaligned_to(dx, kElem) || misaligned_to(g_in, kElem) ||
        misaligned_to(g_out, kElem) || misaligned_to(before, kElem) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const Extent in[6] = {matrix_of(x, B * T, ldx, D, kElem), matrix_of(dy, B * T, lddy, D, kElem), matrix_of(weights, W, ldw, offset + columns, kElem),
                          dense_of(reset, B * T), dense_of(before, ends * kElem), matrix_of(g_in, W, ld, offset + columns, kElem)};
    const Extent out[3] = {matrix_of(dx, B * T, lddx, D, kElem), matrix_of(g_out, W, ld, offset + columns, kElem), dense_of(workspace, bytes)};
    const Same same[1] = {{1, 5}};
    if (outputs_share_but(in, out, same)) return CX_ERR_ALIAS;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    float *parts = static_cast<float *>(workspace);
    int64_t count = 0;
    if (!none) {
        const Walk w = walk_of(B, T, D, kGradColumns, kLeastGradSteps);
        if (w.groups * w.slabs > 0x7fffffff) return CX_ERR_SHAPE;
        ConvArgs<E> a{};
        a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.weights = weights + offset; a.ldw = ldw; a.dx = dx; a.lddx = lddx; a.before = before;
        a.reset = reset; a.parts = parts; a.B = B; a.T_ = T; a.per_worker = static_cast<uint32_t>(B / W); a.D = D; a.silu = silu != 0;
        set_walk(a, w);
        a.shared_ends = D >= kGradColumns;
        const int rc2 = by_taps(K, [&](auto k) {
            if (reset) hipLaunchKernelGGL((conv_grad_kernel<E, kGradColumns, decltype(k)::value, true>), grid_of(w, B), dim3(w.together << w.shift), 0, st, a);
            else hipLaunchKernelGGL((conv_grad_kernel<E, kGradColumns, decltype(k)::value, false>), grid_of(w, B), dim3(w.together << w.shift), 0, st, a);
        });
        if (rc2 != CX_OK) return rc2;
        count = B / W * w.groups;
    }
    if (none && g_in == g_out) return CX_OK;
    return sum_parts<E>(parts, count, columns, g_in ? g_in + offset : nullptr, g_out + offset, ld, W, st);
}

}  // namespace

extern "C" {

#define CX_LM_CONV(SUFFIX, E)                                                                                                         \
    int cx_short_conv##SUFFIX(const E::T *x, int64_t ldx, const E::T *weights, int64_t ldw, int32_t W, int64_t offset, E::T *y,       \
                              int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset,            \
                              const E::T *before, E::T *after, void *stream)                                                          \
    {                                                                                                                                 \
        return conv<E>(x, ldx, weights, ldw, W, offset, y, ldy, B, T, D, K, silu, reset, before, after, stream);                      \
    }                                                                                                                                 \
    int cx_short_conv_grad##SUFFIX(const E::T *x, int64_t ldx, const E::T *dy, int64_t lddy, const E::T *weights, int64_t ldw,        \
                                   int32_t W, int64_t offset, E::T *dx, int64_t lddx, const E::T *g_in, E::T *g_out, int64_t ldg,     \
                                   int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset,                    \
                                   const E::T *before, void *workspace, int64_t workspace_bytes, void *stream)                        \
    {                                                                                                                                 \
        return conv_grad<E>(x, ldx, dy, lddy, weights, ldw, W, offset, dx, lddx, g_in, g_out, ldg, B, T, D, K, silu, reset, before,   \
                            workspace, workspace_bytes, stream);                                                                      \
    }
CX_LM_CONV(, F32)
CX_LM_CONV(_bf16, Bf16)
CX_LM_CONV(_f16, F16)
#undef CX_LM_CONV

int cx_conv_workspace(int32_t W, int64_t B, int64_t T, int32_t D, int32_t K, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_conv(W, B, T, D, K);
    if (rc == CX_OK) *bytes = parts_bytes(B, T, D, K);
    return rc;
}

}  // extern "C"
