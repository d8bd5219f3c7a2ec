// C-ABI entry points cx_dropout*, cx_add_norm*, cx_add_norm_grad*, cx_norm_workspace (see include/cx_lm.h)
//
//   drop(x) = keep ? x / (1 - p) : 0       keep from a counter-based generator: key, draw, row and column
//   s = residual + drop(x)    inv = 1 / sqrt(mean(s^2) + eps)    y = s inv w        (8 bits: y / scale, scale = max |y| / 448)
//   g = dy w    ds = inv (g - s inv mean(g s inv)) + ds_in    dx = drop(ds)    dw = sum over a worker's rows of dy s inv
//
// A row stays in the registers of a group of lanes between its statistics and its results, so that each matrix is read and
// written once.  A lane holds up to four times eight columns; groups are a power of two of lanes.
//
// Bound by memory: 65,536 rows of 768 in bfloat16 take 72 us with dropout (5.6 TB/s), their gradient 103 to 119, by how warm the card is, and 5 for the
// sums of its parts (4.9 to 4.2 TB/s), dropout alone 48 (6.3 TB/s); 8,192 rows of 2,048 to 8 bits 22 to 23 (two sets of operands by turns, 234 MB, of which the
// last level of the caches keeps a part).  Tried for the gradient and not kept: the next row's loads ahead (103 to 133), rows widened twice to that end
// (spills), results past the caches (110).
#include "lm_block.hpp"

namespace {

constexpr int kThreads = 256, kMaxLanes = 512, kMaxEights = 4;
constexpr int64_t kMaxRows = int64_t(1) << 31, kMaxGroups = int64_t(1) << 24;       // a launch has fewer than 2^32 threads
constexpr float kLargest8 = 448.0f, kLeastScale = 0x1p-126f;

// What is read once goes past the caches, of 16-bit rows: a lane's eight float32 columns are two reads of half of each line.
template <class E>
constexpr bool kPast = sizeof(typename E::T) == 2;

// ---------------------------------------------------------------------------------
// Dropout alone
// ---------------------------------------------------------------------------------
template <class E>
struct DropArgs {
    const typename E::T *x, *residual;
    typename E::T *out;
    int64_t ldx, ldr, ldo, rows;
    int32_t D, eights;                                  // eights: ceil(D / 8)
    uint32_t per;                                       // ceil(2^32 / eights)
    Drop d;
};

constexpr int kDropEach = 2;                            // eights of a thread

template <class E>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const DropArgs<E> a)
{
    const int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads * kDropEach);
    const int64_t row0 = first / a.eights;
    const uint32_t at0 = static_cast<uint32_t>(first - row0 * a.eights) + threadIdx.x;
    const uint64_t key = a.d.rng[0], draw = a.d.rng[1];
    Columns<E, 8> x[kDropEach], r[kDropEach];
    int64_t row[kDropEach];
    int column[kDropEach];
#pragma unroll
    for (int k = 0; k < kDropEach; ++k) {
        const uint32_t at = at0 + k * kThreads;
        // at / eights: the product's error is below one, upwards
        uint32_t q = a.eights == 1 ? at : __umulhi(at, a.per);
        q -= q * static_cast<uint32_t>(a.eights) > at;
        row[k] = row0 + q;
        column[k] = static_cast<int>(at - q * a.eights) * 8;
        if (row[k] < a.rows) {
            x[k] = load_columns<E, 8, kPast<E>>(a.x + row[k] * a.ldx + column[k], a.D - column[k]);
            if (a.residual) r[k] = load_columns<E, 8, kPast<E>>(a.residual + row[k] * a.ldr + column[k], a.D - column[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kDropEach; ++k) {
        if (row[k] >= a.rows) continue;
        float v[8];
        widen<E, 8>(x[k], v);
        if (a.d.border) drop(random_block(key, draw, static_cast<uint64_t>(row[k]) * a.eights + column[k] / 8), a.d.border, a.d.scale, v);
        if (a.residual) {
            float f[8];
            widen<E, 8>(r[k], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = f[j] + v[j];
        }
        store_columns<E, 8>(a.out + row[k] * a.ldo + column[k], a.D - column[k], v);
    }
}

template <class E>
int dropout(const typename E::T *x, int64_t ldx, const typename E::T *residual, int64_t ldr, typename E::T *out, int64_t ldo, int64_t N, int32_t D,
            const int64_t *rng, float p, void *stream)
{
    DropArgs<E> a{};
    if (N < 0 || N > kMaxRows || D < 1 || D > CX_MAX_WIDTH || !drop_of(p, rng, a.d)) return CX_ERR_SHAPE;
    if (N == 0) return CX_OK;
    if (!x || !out || !rng) return CX_ERR_NULL;
    a.eights = static_cast<int32_t>(ceil_div(D, 8));
    const int64_t groups = ceil_div(N * a.eights, kThreads * kDropEach);
    if (bad_matrix(N, ldx, D) || (residual && bad_matrix(N, ldr, D)) || bad_matrix(N, ldo, D) || groups >= kMaxGroups) return CX_ERR_SHAPE;
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(x, kElem) || misaligned_to(residual, kElem) || misaligned_to(out, kElem) || misaligned_to(rng, 8)) return CX_ERR_ALIGN;
    const Extent in[3] = {matrix_of(x, N, ldx, D, kElem), matrix_of(residual, N, ldr, D, kElem), dense_of(rng, 16)};
    const Extent outs[1] = {matrix_of(out, N, ldo, D, kElem)};
    const Same same[2] = {{0, 0}, {0, 1}};
    if (outputs_share_but(in, outs, same)) return CX_ERR_ALIAS;
    a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.out = out; a.ldo = ldo; a.rows = N; a.D = D;
    a.per = static_cast<uint32_t>(ceil_div(int64_t(1) << 32, a.eights));
    hipLaunchKernelGGL(dropout_kernel<E>, dim3(static_cast<unsigned>(groups)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
    return launched();
}

// ---------------------------------------------------------------------------------
// Residual and norm
// ---------------------------------------------------------------------------------
template <class E>
struct NormArgs {
    using T = typename E::T;
    const T *x, *residual, *weights, *dy, *ds_in;
    T *s, *y, *ds, *dx;
    const T *s_in;
    int64_t ldx, ldr, ldw, lds, ldy, ldq, lddy, ldi, ldds, lddx;
    uint8_t *q;
    float *scale, *inv, *parts;
    const float *inv_in;
    int64_t N, part_rows;                               // rows of a worker, of a part
    int32_t D, eights, shift;                           // 1 << shift lanes a row
    float eps;
    Drop d;
};

// A row's sum over its lanes, in every lane.  `turn`: two buffers, so that one barrier does.
__device__ __forceinline__ float row_sum(float v, int shift, float (&lds)[2][kMaxLanes / kWave], int turn)
{
    v = sum_lanes(v, shift < 6 ? shift : 6);
    if (shift <= 6) return v;
    const int wave = threadIdx.x / kWave, waves = 1 << (shift - 6), first = wave & ~(waves - 1);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[turn][wave] = v;
    __syncthreads();
    v = 0.0f;
    for (int k = 0; k < waves; ++k) v += lds[turn][first + k];
    return v;
}
__device__ __forceinline__ unsigned row_max(unsigned v, int shift, float (&lds)[2][kMaxLanes / kWave], int turn)
{
    v = max_lanes(v, shift < 6 ? shift : 6);
    if (shift <= 6) return v;
    const int wave = threadIdx.x / kWave, waves = 1 << (shift - 6), first = wave & ~(waves - 1);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[turn][wave] = __uint_as_float(v);
    __syncthreads();
    v = 0;
    for (int k = 0; k < waves; ++k) {
        const unsigned u = __float_as_uint(lds[turn][first + k]);
        v = u > v ? u : v;
    }
    return v;
}

// LARGE: the matrices are beyond the caches, which are passed by.
template <class E, int V, bool DROP, bool LARGE>
__global__ __launch_bounds__(kMaxLanes) void norm_kernel(const NormArgs<E> a)
{
    __shared__ float lds[2][kMaxLanes / kWave];
    const int lanes = 1 << a.shift, lane = threadIdx.x & (lanes - 1);
    const int64_t w = blockIdx.y, block = static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x;
    const int64_t r = block * (blockDim.x >> a.shift) + (threadIdx.x >> a.shift), row = w * a.N + r;
    const bool here = r < a.N;
    float s[V][8];
    float squares = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int column = (v * lanes + lane) * 8, left = here ? a.D - column : 0;
        const Columns<E, 8> xs = load_columns<E, 8, LARGE>(a.x + row * a.ldx + column, left);
        Columns<E, 8> rs;
        if (a.residual) rs = load_columns<E, 8, LARGE>(a.residual + row * a.ldr + column, left);
        widen<E, 8>(xs, s[v]);
        if constexpr (DROP)
            if (left > 0) drop(random_block(a.d.rng[0], a.d.rng[1], static_cast<uint64_t>(row) * a.eights + column / 8), a.d.border, a.d.scale, s[v]);
        if (a.residual) {
            float f[8];
            widen<E, 8>(rs, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[v][j] = f[j] + s[v][j];
        }
        if (a.s && left > 0) store_columns<E, 8, LARGE>(a.s + row * a.lds + column, left, s[v]);
#pragma unroll
        for (int j = 0; j < 8; ++j) squares = __builtin_fmaf(s[v][j], s[v][j], squares);
    }
    squares = row_sum(squares, a.shift, lds, 0);
    const float inv = 1.0f / __builtin_sqrtf(squares / static_cast<float>(a.D) + a.eps);
    if (a.inv && here && lane == 0) a.inv[row] = inv;
    unsigned high = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int column = (v * lanes + lane) * 8, left = here ? a.D - column : 0;
        float f[8];
        widen<E, 8>(load_columns<E, 8>(a.weights + w * a.ldw + column, left), f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[v][j] = s[v][j] * inv * f[j];
            const unsigned u = __float_as_uint(s[v][j]) & 0x7fffffffu;        // ordered like the magnitudes, NaN above infinity
            if (j < left) high = u > high ? u : high;
        }
        if (a.y && left > 0) store_columns<E, 8, LARGE>(a.y + row * a.ldy + column, left, s[v]);
    }
    if (!a.q) return;
    const float most = __uint_as_float(row_max(high, a.shift, lds, 1)), whole = most / kLargest8;
    const float scale = whole < kLeastScale ? kLeastScale : whole;
    if (here && lane == 0) a.scale[row] = scale;
    // The float32 quotients by the scale, correctly rounded: with the rounded reciprocal, the product and what it leaves of the dividend give them wherever
    // that remainder is normal (Markstein 1990).  A division each takes 23 us instead of 22 for 8,192 rows of 2,048, the product alone 21, but it is off
    // by one and moves results next to a midpoint of e4m3 by a step.
    if (scale > 0x1p-80f && scale < 0x1p+120f) {
        const float factor = 1.0f / scale;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float near = s[v][j] * factor;
                s[v][j] = __builtin_fmaf(__builtin_fmaf(-near, scale, s[v][j]), factor, near);
            }
    } else {                                            // an infinite scale and a NaN too
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[v][j] /= scale;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int column = (v * lanes + lane) * 8, left = here ? a.D - column : 0;
        if (left <= 0) continue;
        unsigned q[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            q[k] = __builtin_amdgcn_cvt_pk_fp8_f32(s[v][4 * k], s[v][4 * k + 1], 0, false);
            q[k] = __builtin_amdgcn_cvt_pk_fp8_f32(s[v][4 * k + 2], s[v][4 * k + 3], q[k], true);
        }
        uint8_t *p = a.q + row * a.ldq + column;
        if (left >= 8) {
            typedef unsigned u2 __attribute__((ext_vector_type(2)));
            typedef u2 u2_at1 __attribute__((aligned(1)));
            *reinterpret_cast<u2_at1 *>(p) = u2{q[0], q[1]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) p[j] = static_cast<uint8_t>(q[j / 4] >> (8 * (j % 4)));
        }
    }
}

// A workgroup takes the rows of a part one after the other (several at a time where a row has fewer lanes) and keeps its columns' share of dw.
// s is the forward pass's sum rounded to the rows' type, inv that of the sum before: of 4,096 rows of 768 in bfloat16 dw is off by 0.0023 of itself, 0.0017
// from the sum as it was; in binary16 3.0e-4 and 2.1e-4.  A float32 copy of s for it would
// add 4 bytes to the 8 that an element moves forward and 2 to the 10 back.
template <class E, int V, bool DROP>
__global__ __launch_bounds__(kMaxLanes) void norm_grad_kernel(const NormArgs<E> a)
{
    __shared__ float lds[2][kMaxLanes / kWave];
    __shared__ float sums[kThreads][9];                 // 9: lanes of a wavefront in different banks
    const int lanes = 1 << a.shift, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.shift, groups = blockDim.x >> a.shift;
    const int64_t w = blockIdx.y, begin = blockIdx.x * a.part_rows, end = begin + a.part_rows < a.N ? begin + a.part_rows : a.N;
    float dw[V][8] = {};
    int turn = 0;
    for (int64_t r0 = begin; r0 < end; r0 += groups) {
        const bool here = r0 + group < end;
        const int64_t row = w * a.N + (here ? r0 + group : begin);
        const float inv = a.inv_in[row];
        float unit[V][8], g[V][8];
        Columns<E, 8> more[V];
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int column = (v * lanes + lane) * 8, left = here ? a.D - column : 0;
            const Columns<E, 8> ss = load_columns<E, 8, kPast<E>>(a.s_in + row * a.lds + column, left), ds = load_columns<E, 8, kPast<E>>(a.dy + row * a.lddy + column, left);
            if (a.ds_in) more[v] = load_columns<E, 8, kPast<E>>(a.ds_in + row * a.ldi + column, left);
            float f[8];
            widen<E, 8>(ss, unit[v]);
            widen<E, 8>(ds, g[v]);
            widen<E, 8>(load_columns<E, 8>(a.weights + w * a.ldw + column, left), f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                unit[v][j] *= inv;
                dw[v][j] = __builtin_fmaf(g[v][j], unit[v][j], dw[v][j]);
                g[v][j] *= f[j];
                dot = __builtin_fmaf(g[v][j], unit[v][j], dot);
            }
        }
        dot = row_sum(dot, a.shift, lds, turn);
        turn ^= 1;
        const float mean = dot / static_cast<float>(a.D);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int column = (v * lanes + lane) * 8, left = here ? a.D - column : 0;
            if (left <= 0) continue;
            float f[8];
            if (a.ds_in) widen<E, 8>(more[v], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float own = __builtin_fmaf(-unit[v][j], mean, g[v][j]);
                g[v][j] = a.ds_in ? __builtin_fmaf(inv, own, f[j]) : inv * own;
            }
            if (a.ds) store_columns<E, 8>(a.ds + row * a.ldds + column, left, g[v]);
            if (a.dx) {
                if constexpr (DROP) drop(random_block(a.d.rng[0], a.d.rng[1], static_cast<uint64_t>(row) * a.eights + column / 8), a.d.border, a.d.scale, g[v]);
                store_columns<E, 8>(a.dx + row * a.lddx + column, left, g[v]);
            }
        }
    }
    float *part = a.parts + (w * gridDim.x + blockIdx.x) * a.D;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int column = (v * lanes + lane) * 8;
        if (groups > 1) {                               // of kThreads threads
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[threadIdx.x][j] = dw[v][j];
            __syncthreads();
            if (group > 0) continue;
            for (int k = 1; k < groups; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) dw[v][j] += sums[(k << a.shift) + lane][j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (column + j < a.D) part[column + j] = dw[v][j];
    }
}

struct Layout {
    int shift, eights, threads;                         // lanes of a row as a power of two, eights of a lane
};

// Two layouts: one eight of columns to a lane where a row has no more than 4,096, and the fewest idle places.  The first is the forward pass's: 32 rows
// of 1,024 take 3.4 us in bfloat16 against 4.9, 4,000 float32 rows of 515 9.4 against 10.6.  The gradient keeps sums of its columns over rows and takes the
// second: 65,536 rows of 768 in bfloat16 107 us with three eights of 32 lanes, 120 with one of 128.  So does a forward pass of matrices beyond the caches, with
// its reads and results past them: the same rows 73 us against 81, 34,080 rows of 1,266 70 against 87, but 8,192 rows of 2,048 to 8 bits, 117 MB, 26.6 against 21.8.
Layout layout_of(int32_t D, bool fewest)
{
    const int n = static_cast<int>(ceil_div(D, 8));
    Layout best{};
    int least = 1 << 30;
    for (int shift = 1; (1 << shift) <= kMaxLanes; ++shift) {
        const int each = static_cast<int>(ceil_div(n, 1 << shift));
        if (each > (!fewest && n <= kMaxLanes ? 1 : kMaxEights)) continue;
        if ((each << shift) < least) {
            least = each << shift;
            best = {shift, each, (1 << shift) > kThreads ? 1 << shift : kThreads};
        }
    }
    return best;
}

constexpr int64_t kCaches = 256 << 20;                  // bytes
// Workgroups of a gradient, by the eights alone: two wavefronts to a SIMD of three or four (34,080 rows of 1,266 101 us with 512, 115 with 1,024), four of
// fewer.  Not all variants fill them: three eights of 16 bits without dropout have 160 registers, which three wavefronts would have room for, two of
// float32 with dropout 131, which leave room for three, and one has at most 89, for five.
constexpr int64_t kParts = 512, kPartsOfFew = 1024;

int64_t parts_of(int32_t W, int64_t N, int32_t D)
{
    const Layout l = layout_of(D, true);
    const int64_t groups = l.threads >> l.shift, most = ceil_div(N, groups), wanted = ceil_div(l.eights > 2 ? kParts : kPartsOfFew, W);
    const int64_t rows = ceil_div(ceil_div(N, wanted < most ? wanted : most), groups) * groups;
    return ceil_div(N, rows);
}

int check_norm(int32_t W, int64_t N, int32_t D)
{
    return W < 1 || W > CX_MAX_ROWS || N < 0 || N > CX_MAX_TOKENS || D < 1 || D > CX_MAX_NORM_WIDTH ? CX_ERR_SHAPE : CX_OK;
}

template <class E, class F>
int by_layout(const Layout &l, bool drops, const F &launch)
{
    const auto with = [&](auto v) {
        if (drops) launch(v, std::true_type{});
        else launch(v, std::false_type{});
    };
    switch (l.eights) {
    case 1: with(std::integral_constant<int, 1>{}); break;
    case 2: with(std::integral_constant<int, 2>{}); break;
    case 3: with(std::integral_constant<int, 3>{}); break;
    default: with(std::integral_constant<int, 4>{}); break;
    }
    return launched();
}

template <class E>
int add_norm(const typename E::T *x, int64_t ldx, const typename E::T *residual, int64_t ldr, const typename E::T *weights, int64_t ld, int32_t W,
             int64_t offset, int64_t N, int32_t D, float eps, const int64_t *rng, float p, typename E::T *s, int64_t lds, typename E::T *y, int64_t ldy,
             float *inv, uint8_t *q, int64_t ldq, float *scale, void *stream)
{
    NormArgs<E> a{};
    const int rc = check_norm(W, N, D);
    if (rc != CX_OK || !(eps >= 0.0f && eps < INFINITY) || !drop_of(p, rng, a.d)) return CX_ERR_SHAPE;
    if (bad_rows(W, ld, offset, D)) return CX_ERR_SHAPE;
    if (N == 0) return CX_OK;
    const int64_t rows = W * N;
    if (!x || !weights || (!s && !y && !q) || (a.d.border && !rng) || (q && !scale)) return CX_ERR_NULL;
    if (bad_matrix(rows, ldx, D) || (residual && bad_matrix(rows, ldr, D)) || (s && bad_matrix(rows, lds, D)) || (y && bad_matrix(rows, ldy, D)) ||
        (q && bad_matrix(rows, ldq, D))) return CX_ERR_SHAPE;
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(x, kElem) || misaligned_to(residual, kElem) || misaligned_to(weights, kElem) || misaligned_to(s, kElem) || misaligned_to(y, kElem) ||
        misaligned_to(rng, 8) || misaligned_to(inv, 4) || misaligned_to(scale, 4)) return CX_ERR_ALIGN;
    const Extent in[4] = {matrix_of(x, rows, ldx, D, kElem), matrix_of(residual, rows, ldr, D, kElem), matrix_of(weights, W, ld, offset + D, kElem), dense_of(rng, 16)};
    const Extent out[5] = {matrix_of(s, rows, lds, D, kElem), matrix_of(y, rows, ldy, D, kElem), dense_of(inv, rows * 4), matrix_of(q, rows, ldq, D, 1),
                           dense_of(q ? scale : nullptr, rows * 4)};
    const Same same[3] = {{0, 0}, {0, 1}, {1, 0}};
    if (outputs_share_but(in, out, same)) return CX_ERR_ALIAS;
    const int64_t bytes = rows * D * (kElem * (1 + (residual != nullptr) + (s != nullptr) + (y != nullptr)) + (q != nullptr));
    const bool large = kElem == 2 && bytes >= kCaches;
    const Layout l = layout_of(D, large);
    a.x = x; a.ldx = ldx; a.residual = residual; a.ldr = ldr; a.weights = weights + offset; a.ldw = ld; a.s = s; a.lds = lds; a.y = y; a.ldy = ldy;
    a.inv = inv; a.q = q; a.ldq = ldq; a.scale = scale; a.N = N; a.D = D; a.eights = static_cast<int32_t>(ceil_div(D, 8)); a.shift = l.shift; a.eps = eps;
    const int64_t blocks = ceil_div(N, l.threads >> l.shift), wide = blocks < (1 << 22) ? blocks : 1 << 22;
    const dim3 grid(static_cast<unsigned>(wide), W, static_cast<unsigned>(ceil_div(blocks, wide)));
    return by_layout<E>(l, a.d.border != 0, [&](auto v, auto drops) {
        constexpr bool kMayBe = kElem == 2;
        if (kMayBe && large)
            hipLaunchKernelGGL((norm_kernel<E, decltype(v)::value, decltype(drops)::value, kMayBe>), grid, dim3(l.threads), 0, static_cast<hipStream_t>(stream), a);
        else
            hipLaunchKernelGGL((norm_kernel<E, decltype(v)::value, decltype(drops)::value, false>), grid, dim3(l.threads), 0, static_cast<hipStream_t>(stream), a);
    });
}

template <class E>
int add_norm_grad(const typename E::T *dy, int64_t lddy, const typename E::T *s, int64_t lds, const float *inv, const typename E::T *weights, int64_t ldw,
                  int32_t W, int64_t offset, int64_t N, int32_t D, const typename E::T *ds_in, int64_t ldi, const int64_t *rng, float p,
                  typename E::T *ds, int64_t ldds, typename E::T *dx, int64_t lddx, const typename E::T *g_in, typename E::T *g_out, int64_t ld,
                  void *workspace, int64_t workspace_bytes, void *stream)
{
    NormArgs<E> a{};
    const int rc = check_norm(W, N, D);
    if (rc != CX_OK || !drop_of(p, rng, a.d)) return CX_ERR_SHAPE;
    if (bad_rows(W, ldw, offset, D) || bad_rows(W, ld, offset, D)) return CX_ERR_SHAPE;
    if (!g_out) return CX_ERR_NULL;
    const int64_t rows = W * N, parts = N > 0 ? parts_of(W, N, D) : 0, bytes = W * parts * D * 4;
    if (N > 0) {
        if (!dy || !s || !inv || !weights || (!ds && !dx) || (a.d.border && !rng) || !workspace) return CX_ERR_NULL;
        if (bad_matrix(rows, lddy, D) || bad_matrix(rows, lds, D) || (ds_in && bad_matrix(rows, ldi, D)) || (ds && bad_matrix(rows, ldds, D)) ||
            (dx && bad_matrix(rows, lddx, D)) || workspace_bytes < bytes) return CX_ERR_SHAPE;
    }
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(dy, kElem) || misaligned_to(s, kElem) || misaligned_to(inv, 4) || misaligned_to(weights, kElem) || misaligned_to(ds_in, kElem) ||
        misaligned_to(rng, 8) || misaligned_to(ds, kElem) || misaligned_to(dx, kElem) || misaligned_to(g_in, kElem) || misaligned_to(g_out, kElem) ||
        misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const Extent in[7] = {matrix_of(dy, rows, lddy, D, kElem), matrix_of(s, rows, lds, D, kElem), dense_of(inv, rows * 4), matrix_of(weights, W, ldw, offset + D, kElem),
                          matrix_of(ds_in, rows, ldi, D, kElem), dense_of(rng, 16), matrix_of(g_in, W, ld, offset + D, kElem)};
    const Extent out[4] = {matrix_of(ds, rows, ldds, D, kElem), matrix_of(dx, rows, lddx, D, kElem), matrix_of(g_out, W, ld, offset + D, kElem),
                           dense_of(workspace, bytes)};
    const Same same[5] = {{0, 0}, {0, 4}, {1, 0}, {1, 4}, {2, 6}};
    if (outputs_share_but(in, out, same)) return CX_ERR_ALIAS;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    float *sums = static_cast<float *>(workspace);
    if (N > 0) {
        const Layout l = layout_of(D, true);
        a.dy = dy; a.lddy = lddy; a.s_in = s; a.lds = lds; a.inv_in = inv; a.weights = weights + offset; a.ldw = ldw; a.ds_in = ds_in; a.ldi = ldi;
        a.ds = ds; a.ldds = ldds; a.dx = dx; a.lddx = lddx; a.parts = sums; a.N = N; a.part_rows = 0;
        a.D = D; a.eights = static_cast<int32_t>(ceil_div(D, 8)); a.shift = l.shift;
        const int64_t groups = l.threads >> l.shift;
        a.part_rows = ceil_div(ceil_div(N, parts), groups) * groups;
        const dim3 grid(static_cast<unsigned>(parts), W);
        const int rc2 = by_layout<E>(l, a.d.border != 0, [&](auto v, auto drops) {
            hipLaunchKernelGGL((norm_grad_kernel<E, decltype(v)::value, decltype(drops)::value>), grid, dim3(l.threads), 0, st, a);
        });
        if (rc2 != CX_OK) return rc2;
    }
    if (N == 0 && g_in == g_out) return CX_OK;
    return sum_parts<E>(sums, parts, D, g_in ? g_in + offset : nullptr, g_out + offset, ld, W, st);
}

}  // namespace

extern "C" {

#define CX_LM_NORM(SUFFIX, E)                                                                                                         \
    int cx_dropout##SUFFIX(const E::T *x, int64_t ldx, const E::T *residual, int64_t ldr, E::T *out, int64_t ldo, int64_t N,          \
                           int32_t D, const int64_t *rng, float p, void *stream)                                                      \
    {                                                                                                                                 \
        return dropout<E>(x, ldx, residual, ldr, out, ldo, N, D, rng, p, stream);                                                     \
    }                                                                                                                                 \
    int cx_add_norm##SUFFIX(const E::T *x, int64_t ldx, const E::T *residual, int64_t ldr, const E::T *weights, int64_t ldw,          \
                            int32_t W, int64_t offset, int64_t N, int32_t D, float eps, const int64_t *rng, float p, E::T *s,         \
                            int64_t lds, E::T *y, int64_t ldy, float *inv, uint8_t *q, int64_t ldq, float *scale, void *stream)       \
    {                                                                                                                                 \
        return add_norm<E>(x, ldx, residual, ldr, weights, ldw, W, offset, N, D, eps, rng, p, s, lds, y, ldy, inv, q, ldq, scale,     \
                           stream);                                                                                                   \
    }                                                                                                                                 \
    int cx_add_norm_grad##SUFFIX(const E::T *dy, int64_t lddy, const E::T *s, int64_t lds, const float *inv, const E::T *weights,     \
                                 int64_t ldw, int32_t W, int64_t offset, int64_t N, int32_t D, const E::T *ds_in, int64_t ldi,        \
                                 const int64_t *rng, float p, E::T *ds, int64_t ldds, E::T *dx, int64_t lddx, const E::T *g_in,       \
                                 E::T *g_out, int64_t ldg, void *workspace, int64_t workspace_bytes, void *stream)                    \
    {                                                                                                                                 \
        return add_norm_grad<E>(dy, lddy, s, lds, inv, weights, ldw, W, offset, N, D, ds_in, ldi, rng, p, ds, ldds, dx, lddx, g_in,   \
                                g_out, ldg, workspace, workspace_bytes, stream);                                                      \
    }
CX_LM_NORM(, F32)
CX_LM_NORM(_bf16, Bf16)
CX_LM_NORM(_f16, F16)
#undef CX_LM_NORM

int cx_norm_workspace(int32_t W, int64_t N, int32_t D, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_norm(W, N, D);
    if (rc == CX_OK && N > 0) *bytes = W * parts_of(W, N, D) * D * 4;
    return rc;
}

}  // extern "C"
