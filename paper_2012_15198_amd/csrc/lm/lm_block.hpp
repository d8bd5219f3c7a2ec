// What the operators of a residual block share (internal header): a few columns of a row at a time, random bits of a counter,
// and sums of a worker's parameter gradients over the parts that workgroups leave.
#ifndef CX_LM_BLOCK_HPP
#define CX_LM_BLOCK_HPP
#include "lm_common.hpp"

#include <cmath>

namespace {

// ---------------------------------------------------------------------------------
// C = 4 or 8 columns of a row as they lie in memory, widened where they are used: what is loaded ahead is then not waited for.
// ---------------------------------------------------------------------------------
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef u2 u2_at2 __attribute__((aligned(2)));

template <class E, int C>
struct Columns {
    static constexpr int kWords = C * sizeof(typename E::T) / 4;
    unsigned w[kWords];
};

// `left`: columns from p to the row's end; those behind it are zeros.  LAST: nothing of the call reads it again.
template <class E, int C, bool LAST = false>
__device__ __forceinline__ Columns<E, C> load_columns(const typename E::T *p, int left)
{
    constexpr int kWords = Columns<E, C>::kWords;
    Columns<E, C> r;
    if (left >= C) {
        if constexpr (kWords == 2) {
            const u2 v = LAST ? __builtin_nontemporal_load(reinterpret_cast<const u2_at2 *>(p)) : *reinterpret_cast<const u2_at2 *>(p);
            r.w[0] = v[0];
            r.w[1] = v[1];
        } else {
#pragma unroll
            for (int k = 0; k < kWords / 4; ++k) {
                const u4 v = LAST ? load16_last<E>(p + k * E::kPer16) : load16<E>(p + k * E::kPer16);
#pragma unroll
                for (int j = 0; j < 4; ++j) r.w[4 * k + j] = v[j];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < kWords; ++j) r.w[j] = 0;
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (j < left) {
                if constexpr (sizeof(typename E::T) == 4) r.w[j] = __float_as_uint(p[j]);
                else r.w[j / 2] |= static_cast<unsigned>(p[j]) << (16 * (j & 1));
            }
    }
    return r;
}
template <class E, int C>
__device__ __forceinline__ float value_of(const Columns<E, C> &r, int j)
{
    if constexpr (sizeof(typename E::T) == 4) return __uint_as_float(r.w[j]);
    else return (j & 1) ? E::high(r.w[j / 2]) : E::low(r.w[j / 2]);
}
template <class E, int C>
__device__ __forceinline__ void widen(const Columns<E, C> &r, float (&v)[C])
{
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = value_of<E, C>(r, j);
}
// THROUGH: past the caches, for results so large that none keeps them for their reader.
template <class E, int C, bool THROUGH = false>
__device__ __forceinline__ void store_columns(typename E::T *p, int left, const float (&v)[C])
{
    const auto put = [](typename E::T *to, const u4 &w) {
        if constexpr (THROUGH) store16_through<E>(to, w);
        else store16<E>(to, w);
    };
    if (left >= C) {
        if constexpr (sizeof(typename E::T) == 4) {
#pragma unroll
            for (int k = 0; k < C / 4; ++k)
                put(p + 4 * k, u4{__float_as_uint(v[4 * k]), __float_as_uint(v[4 * k + 1]), __float_as_uint(v[4 * k + 2]), __float_as_uint(v[4 * k + 3])});
        } else if constexpr (C == 4) {
            const u2 w{E::two(v[0], v[1]), E::two(v[2], v[3])};
            if constexpr (THROUGH) __builtin_nontemporal_store(w, reinterpret_cast<u2_at2 *>(p));
            else *reinterpret_cast<u2_at2 *>(p) = w;
        } else {
            put(p, E::pack(v));
        }
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (j < left) p[j] = E::narrow(v[j]);
    }
}

// ---------------------------------------------------------------------------------
// Dropout's bits: Philox4x32 of ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011),
// eight times 16 bits a block.  The counter names the place, so nothing is stored and every pass finds the same bits.
// ---------------------------------------------------------------------------------
struct Drop {
    const int64_t *rng;                                 // device: key, draw
    uint32_t border;                                    // bits below it are dropped: share * 2^16
    float scale;                                        // 2^16 / (2^16 - border)
};

__device__ __forceinline__ u4 random_block(uint64_t key, uint64_t draw, uint64_t block)
{
    uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32), c2 = static_cast<uint32_t>(draw), c3 = static_cast<uint32_t>(draw >> 32);
    uint32_t k0 = static_cast<uint32_t>(key), k1 = static_cast<uint32_t>(key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        // one multiplication each: both halves of the products
        const uint64_t m0 = static_cast<uint64_t>(c0) * 0xD2511F53u, m1 = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(m1 >> 32) ^ c1 ^ k0;
        c1 = static_cast<uint32_t>(m1);
        c2 = static_cast<uint32_t>(m0 >> 32) ^ c3 ^ k1;
        c3 = static_cast<uint32_t>(m0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u4{c0, c1, c2, c3};
}

// A dropped element is 0 whatever it held.
__device__ __forceinline__ void drop(const u4 &bits, uint32_t border, float scale, float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = (j & 1) ? bits[j / 2] >> 16 : bits[j / 2] & 0xffffu;
        v[j] = b >= border ? v[j] * scale : 0.0f;
    }
}

// The share p in [0, 1) to a multiple of 2^-16; false if it has none.
[[maybe_unused]] bool drop_of(float p, const int64_t *rng, Drop &d)
{
    if (!(p >= 0.0f && p < 1.0f)) return false;
    d.border = static_cast<uint32_t>(std::nearbyint(static_cast<double>(p) * 65536.0));
    if (d.border > 65535u) return false;
    d.scale = 65536.0f / static_cast<float>(65536u - d.border);
    d.rng = rng;
    return true;
}

// 0 and 1 far out, to the last bit.
__device__ __forceinline__ float sigmoid(float v) { return rcp_fast(1.0f + exp2_fast(v * -kLog2e)); }
// -inf as the lowest number: its product with a sigmoid of 0 is 0.  A NaN passes the comparison.
__device__ __forceinline__ float finite_below(float v) { return v < -3.0e38f ? -3.0e38f : v; }
// e = sigmoid(v), v from finite_below(); +inf as the largest number, whose product with 1 - e is 0.  A NaN is in e.
__device__ __forceinline__ float silu_slope(float v, float e) { return e * __builtin_fmaf(__builtin_fminf(v, 3.0e38f), 1.0f - e, 1.0f); }

// ---------------------------------------------------------------------------------
// Sums over lanes.  A value is read from the partner's lane by the addition itself within a row of 16 lanes, rows are exchanged whole; all lanes
// that are to take part have to be active.
// ---------------------------------------------------------------------------------
constexpr int kBeside = 0xb1, kOppositePair = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;      // lanes 1 0 3 2; 2 3 0 1; 7 .. 0 of eight; 15 .. 0 of a row
template <int PATTERN>
__device__ __forceinline__ unsigned partner(unsigned v) { return __builtin_amdgcn_mov_dpp(v, PATTERN, 0xf, 0xf, true); }
template <int PATTERN>
__device__ __forceinline__ float add_partner(float v) { return v + __uint_as_float(partner<PATTERN>(__float_as_uint(v))); }
__device__ __forceinline__ float add32(float x, float y)               // rows 0 and 1: x of both halves of the wavefront; rows 2 and 3: y
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add16(float x, float y)               // even rows: x of the row and the next; odd rows: y of the row and the one before
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Over groups of 1 << shift <= 64 lanes, in every lane.  Each stage doubles the lanes that hold the same sum.
__device__ __forceinline__ float sum_lanes(float v, int shift)
{
    if (shift > 0) v = add_partner<kBeside>(v);
    if (shift > 1) v = add_partner<kOppositePair>(v);
    if (shift > 2) v = add_partner<kHalfMirror>(v);
    if (shift > 3) v = add_partner<kMirror>(v);
    if (shift > 4) v = add16(v, v);
    if (shift > 5) v = add32(v, v);
    return v;
}
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
__device__ __forceinline__ unsigned max_lanes(unsigned v, int shift)
{
    if (shift > 0) v = larger(v, partner<kBeside>(v));
    if (shift > 1) v = larger(v, partner<kOppositePair>(v));
    if (shift > 2) v = larger(v, partner<kHalfMirror>(v));
    if (shift > 3) v = larger(v, partner<kMirror>(v));
    if (shift > 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = larger(r[0], r[1]);
    }
    if (shift > 5) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = larger(r[0], r[1]);
    }
    return v;
}

// ---------------------------------------------------------------------------------
// Parameter gradients: parts float [W][parts][columns] added in a fixed order, to g_in where there is one, into columns of flat rows.
// ---------------------------------------------------------------------------------
constexpr int kSumSlices = 16;

template <class E>
__global__ __launch_bounds__(kWave *kSumSlices) void sum_parts_kernel(const float *parts, int64_t count, int64_t columns, const typename E::T *g_in,
                                                                      typename E::T *g_out, int64_t ld)
{
    __shared__ float sums[kSumSlices][kWave];
    const int lane = threadIdx.x & (kWave - 1), slice = threadIdx.x / kWave;
    const int64_t column = static_cast<int64_t>(blockIdx.x) * kWave + lane, w = blockIdx.y;
    float v = 0.0f;
    if (column < columns) {
        const float *p = parts + w * count * columns + column;
#pragma unroll 4
        for (int64_t k = slice; k < count; k += kSumSlices) v += p[k * columns];
    }
    sums[slice][lane] = v;
    __syncthreads();
    if (slice > 0 || column >= columns) return;
#pragma unroll
    for (int k = 1; k < kSumSlices; ++k) v += sums[k][lane];
    if (g_in) v += E::widen(g_in[w * ld + column]);
    g_out[w * ld + column] = E::narrow(v);
}

template <class E>
[[maybe_unused]] int sum_parts(const float *parts, int64_t count, int64_t columns, const typename E::T *g_in, typename E::T *g_out, int64_t ld, int32_t W,
                               hipStream_t st)
{
    hipLaunchKernelGGL(sum_parts_kernel<E>, dim3(static_cast<unsigned>(ceil_div(columns, kWave)), W), dim3(kWave * kSumSlices), 0, st, parts, count, columns,
                       g_in, g_out, ld);
    return launched();
}

// No steps: the state passes through.
constexpr int64_t kPassBlocks = 1 << 16;
template <class T>
__global__ __launch_bounds__(256) void pass_through_kernel(const T *from, T *to, int64_t n)
{
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<int64_t>(gridDim.x) * 256) to[i] = from ? from[i] : static_cast<T>(0);
}
template <class T>
[[maybe_unused]] int pass_through(const T *from, T *to, int64_t n, hipStream_t st)
{
    if (!to || to == from || n == 0) return CX_OK;
    const int64_t blocks = ceil_div(n, 256);
    hipLaunchKernelGGL(pass_through_kernel<T>, dim3(static_cast<unsigned>(blocks < kPassBlocks ? blocks : kPassBlocks)), dim3(256), 0, st, from, to, n);
    return launched();
}

// Pairs of an output and an input that may be the same array, element for element.
struct Same {
    int out, in;
};
template <int INS, int OUTS, int PAIRS>
[[maybe_unused]] bool outputs_share_but(const Extent (&in)[INS], const Extent (&out)[OUTS], const Same (&same)[PAIRS])
{
    for (int i = 0; i < OUTS; ++i) {
        for (int k = 0; k < INS; ++k) {
            bool may = false;
            for (const Same &s : same) may = may || (s.out == i && s.in == k && out[i].first == in[k].first && out[i].pitch == in[k].pitch);
            if (!may && share(out[i], in[k])) return true;
        }
        for (int k = i + 1; k < OUTS; ++k)
            if (share(out[i], out[k])) return true;
    }
    return false;
}

// Flat rows of W workers with `columns` parameters from `offset` on.
[[maybe_unused]] bool bad_rows(int32_t W, int64_t ld, int64_t offset, int64_t columns)
{
    return W < 1 || W > CX_MAX_ROWS || offset < 0 || offset > kMaxExtent || bad_matrix(W, ld, offset + columns);
}

}  // namespace

#endif  // CX_LM_BLOCK_HPP
