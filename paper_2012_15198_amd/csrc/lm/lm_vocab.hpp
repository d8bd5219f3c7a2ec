// One pass over a row of logits (internal header): running maximum and sums of exponentials of what a workgroup reads, and the
// joining of such statistics over lanes, wavefronts and the parts of a split row.
//
// Logits count as differences to the running maximum, so that rows of a type's lowest value are a uniform distribution
// rather than an overflow.  The maximum starts at the lowest finite value: a row of -inf alone ends with s = 0, +inf and NaN
// make s NaN.
#ifndef CX_LM_VOCAB_HPP
#define CX_LM_VOCAB_HPP
#include "lm_common.hpp"

namespace {

constexpr int kRowThreads = 512, kRowWaves = kRowThreads / kWave;
constexpr int kAhead = 4;                               // 16-byte loads a thread has in flight
constexpr float kLargest = 3.40282346638528859812e38f, kLowest = -kLargest;
constexpr float kVanish = -200.0f;                      // exponents (base 2) from here on give 0; keeps 0 * inf out of the sums

// With e = 2^((z - m) c), s is the sum of e, and u
//   kEntropy          the sum of e * log2(e)
//   kDual             the sum of 2^((z - m) c2);  kSquare, kCube, kFourth: the same where c2 is 2, 3 or 4 times c: a power of e by
//                     multiplications.  Two exponentials an element bound the loop before memory does: loss and gradient of
//                     8,192 x 65,536 bfloat16 logits take 405 us with one, 419 with one and its square, 458 with its third or fourth
//                     power, 503 with two, in turn with each other and with a copy of as many bytes, which takes 417.
enum Extra { kNone, kEntropy, kDual, kSquare, kCube, kFourth };
__host__ __device__ constexpr bool two_sums(Extra x) { return x == kDual || x == kSquare || x == kCube || x == kFourth; }

// 2^((z - m) c2), d = z - m, e = 2^(d c)
template <Extra X>
__device__ __forceinline__ float second(float d, float e, float c2)
{
    if (X == kDual) return __builtin_amdgcn_exp2f(d * c2);
    return X == kFourth ? (e * e) * (e * e) : X == kCube ? e * e * e : e * e;
}

struct Stats {
    float m, s, u;
};

__device__ __forceinline__ float not_below(float v, float lowest) { return v < lowest ? lowest : v; }

template <Extra X>
__device__ __forceinline__ void rebase(Stats &a, float m, float c, float c2)
{
    const float d = not_below((a.m - m) * c, kVanish), f = exp2_fast(d);
    if (X == kEntropy) a.u = f * __builtin_fmaf(a.s, d, a.u);
    if (two_sums(X)) a.u *= second<X>(not_below(a.m - m, kLowest), f, c2);
    a.s *= f;
    a.m = m;
}

template <Extra X>
__device__ __forceinline__ Stats join(Stats a, Stats b, float c, float c2)
{
    const float m = fmaxf(a.m, b.m);
    rebase<X>(a, m, c, c2);
    rebase<X>(b, m, c, c2);
    return {m, a.s + b.s, a.u + b.u};
}

// Terms of elements that a.m is the maximum of already.
template <Extra X, int N>
__device__ __forceinline__ void add_terms(Stats &a, const float (&z)[N], float c, float c2)
{
    float s[2] = {}, u[2] = {};
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float d = z[j] - a.m, t = d * c, e = exp2_fast(t);
        s[j & 1] += e;
        if (X == kEntropy) u[j & 1] = __builtin_fmaf(e, fmaxf(t, kVanish), u[j & 1]);
        if (two_sums(X)) u[j & 1] += second<X>(d, e, c2);
    }
    a.s += s[0] + s[1];
    a.u += u[0] + u[1];
}

template <Extra X, int N>
__device__ __forceinline__ float accumulate(Stats &a, const float (&z)[N], float c, float c2)
{
    float top = z[0];
#pragma unroll
    for (int j = 1; j < N; ++j) top = fmaxf(top, z[j]);
    rebase<X>(a, fmaxf(a.m, top), c, c2);
    add_terms<X>(a, z, c, c2);
    return top;
}

// The statistics of all threads of the workgroup, in every thread.
template <Extra X, int WAVES>
__device__ __forceinline__ Stats join_workgroup(Stats a, Stats (&lds)[WAVES], float c, float c2, int waves = WAVES)
{
#pragma unroll
    for (int d = kWave / 2; d > 0; d /= 2)
        a = join<X>(a, {__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.u, d)}, c, c2);
    if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = a;
    __syncthreads();
    a = lds[0];
    for (int k = 1; k < waves; ++k) a = join<X>(a, lds[k], c, c2);
    return a;
}

// A slice of a row: `vectors` whole 16-byte vectors from its first element on (which need not be aligned to more than an
// element), then `tail` elements.  LAST: nothing of the call reads (most of) it again.
template <class E, int THREADS = kRowThreads, bool LAST = false>
struct Slice {
    const typename E::T *z;
    int vectors, tail;
    __device__ __forceinline__ Slice(const typename E::T *row, int64_t lo, int64_t hi)
        : z(row + lo), vectors(static_cast<int>((hi - lo) / E::kPer16)), tail(static_cast<int>((hi - lo) % E::kPer16)) {}
    static __device__ __forceinline__ u4 read(const typename E::T *p) { return LAST ? load16_last<E>(p) : load16<E>(p); }
    __device__ __forceinline__ int rounds() const { return (vectors + THREADS * kAhead - 1) / (THREADS * kAhead); }
    static __device__ __forceinline__ int vector_of(int round, int k) { return (round * kAhead + k) * THREADS + static_cast<int>(threadIdx.x); }
    // the thread's kAhead vectors of a round; what lies beyond the slice counts as -inf
    __device__ __forceinline__ void load(int round, u4 (&w)[kAhead]) const
    {
        if ((round + 1) * kAhead * THREADS <= vectors) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) w[k] = read(z + static_cast<int64_t>(vector_of(round, k)) * E::kPer16);
        } else {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                w[k] = u4{E::kNothing, E::kNothing, E::kNothing, E::kNothing};
                if (vector_of(round, k) < vectors) w[k] = read(z + static_cast<int64_t>(vector_of(round, k)) * E::kPer16);
            }
        }
    }
    __device__ __forceinline__ void load(int round, float (&v)[kAhead * E::kPer16]) const
    {
        u4 w[kAhead];
        load(round, w);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) unpack(w[k], v, k);
    }
    static __device__ __forceinline__ void unpack(const u4 &w, float (&v)[kAhead * E::kPer16], int k)
    {
        float one[E::kPer16];
        E::unpack(w, one);
#pragma unroll
        for (int j = 0; j < E::kPer16; ++j) v[k * E::kPer16 + j] = one[j];
    }
    __device__ __forceinline__ bool has_tail() const { return static_cast<int>(threadIdx.x) < tail; }
    __device__ __forceinline__ int64_t tail_at() const { return static_cast<int64_t>(vectors) * E::kPer16 + threadIdx.x; }
};

// How many workgroups share a row.  One, up to 8,192 vectors (128 KB): 128 rows of 65,536 bfloat16 logits take 13 us whole and 15 in
// four parts with their join, one row of 32,768 9 and 10.  Longer ones are cut where rows are few, into parts of 2,048 vectors and
// no more than give a CU two: one row of 131,072 12.6 us in eight parts, 18 whole; 64 such rows 15 in four parts, 20 whole.
[[maybe_unused]] int parts_of(int64_t N, int64_t V, int per16)
{
    constexpr int64_t kWhole = 8192, kPart = 2048, kMost = 16, kWanted = 512;
    const int64_t vectors = V / per16;
    if (vectors <= kWhole || 2 * N > kWanted) return 1;
    int64_t parts = ceil_div(vectors, kPart);
    parts = parts < kWanted / N ? parts : kWanted / N;
    return static_cast<int>(parts < kMost ? parts : kMost);
}

// Columns of part `part`: whole vectors but for the last part's end.
__host__ __device__ __forceinline__ int64_t part_begin(int64_t V, int parts, int part, int per16)
{
    const int64_t each = (V / per16 + parts - 1) / parts * per16, at = each * part;
    return part >= parts || at > V ? V : at;
}

}  // namespace

#endif  // CX_LM_VOCAB_HPP
