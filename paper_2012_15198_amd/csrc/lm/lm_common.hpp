// Building blocks of the language-model operators (internal header): the three element types with their 16-byte
// vectors, wavefront and workgroup reductions, and the argument checks shared by the entry points.  Each cx_lm_*.hip
// includes this header and defines its entry points; everything has internal linkage.
#ifndef CX_LM_COMMON_HPP
#define CX_LM_COMMON_HPP
#include "cx_lm.h"

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#pragma clang fp contract(off)          // fused multiply-adds are written where they are meant

namespace {

constexpr int kWave = 64;

typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef u4 u4_at4 __attribute__((aligned(4)));             // rows may begin at any element: a vector access needs the
typedef u4 u4_at2 __attribute__((aligned(2)));             // alignment of one element, no more
typedef unsigned u1_at2 __attribute__((aligned(2)));

// ---------------------------------------------------------------------------------
// Element types.  Every value is widened exactly; every result is rounded once, to the nearest (ties to even).
// ---------------------------------------------------------------------------------
struct F32 {
    using T = float;
    using Vec = u4_at4;
    static constexpr int kPer16 = 4;
    static constexpr int kBits = 32;                       // of a value widened to fp32, from the top: the others are zero
    static constexpr unsigned kNothing = 0xff800000u;      // -inf, as often as a word holds it
    static __device__ __forceinline__ float widen(T v) { return v; }
    static __device__ __forceinline__ T narrow(float v) { return v; }
    static __device__ __forceinline__ void unpack(const u4 &w, float (&out)[4])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = __uint_as_float(w[j]);
    }
    static __device__ __forceinline__ u4 pack(const float (&in)[4])
    {
        return u4{__float_as_uint(in[0]), __float_as_uint(in[1]), __float_as_uint(in[2]), __float_as_uint(in[3])};
    }
};

struct Bf16 {
    using T = uint16_t;
    using Vec = u4_at2;
    static constexpr int kPer16 = 8;
    static constexpr int kBits = 16;
    static constexpr unsigned kNothing = 0xff80ff80u;
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ float widen(T v) { return __uint_as_float(static_cast<unsigned>(v) << 16); }
    static __device__ __forceinline__ float low(unsigned w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float high(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ unsigned two(float a, float b)
    {
        return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{a, b}), pair));
    }
    static __device__ __forceinline__ T narrow(float v) { return static_cast<T>(two(v, 0.0f)); }
    static __device__ __forceinline__ void unpack(const u4 &w, float (&out)[8])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) { out[2 * j] = low(w[j]); out[2 * j + 1] = high(w[j]); }
    }
    static __device__ __forceinline__ u4 pack(const float (&in)[8])
    {
        return u4{two(in[0], in[1]), two(in[2], in[3]), two(in[4], in[5]), two(in[6], in[7])};
    }
};

struct F16 {
    using T = uint16_t;
    using Vec = u4_at2;
    static constexpr int kPer16 = 8;
    static constexpr int kBits = 19;
    static constexpr unsigned kNothing = 0xfc00fc00u;
    static __device__ __forceinline__ float widen(T v) { return static_cast<float>(__builtin_bit_cast(_Float16, v)); }
    static __device__ __forceinline__ float low(unsigned w) { return widen(static_cast<T>(w)); }
    static __device__ __forceinline__ float high(unsigned w) { return widen(static_cast<T>(w >> 16)); }
    static __device__ __forceinline__ T narrow(float v) { return __builtin_bit_cast(T, static_cast<_Float16>(v)); }
    static __device__ __forceinline__ unsigned two(float a, float b)
    {
        return static_cast<unsigned>(narrow(a)) | static_cast<unsigned>(narrow(b)) << 16;
    }
    static __device__ __forceinline__ void unpack(const u4 &w, float (&out)[8])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) { out[2 * j] = low(w[j]); out[2 * j + 1] = high(w[j]); }
    }
    static __device__ __forceinline__ u4 pack(const float (&in)[8])
    {
        return u4{two(in[0], in[1]), two(in[2], in[3]), two(in[4], in[5]), two(in[6], in[7])};
    }
};

template <class E>
__device__ __forceinline__ u4 load16(const typename E::T *p) { return *reinterpret_cast<const typename E::Vec *>(p); }
// What nothing of the call reads again need not stay in the caches.
template <class E>
__device__ __forceinline__ u4 load16_last(const typename E::T *p) { return __builtin_nontemporal_load(reinterpret_cast<const typename E::Vec *>(p)); }
template <class E>
__device__ __forceinline__ void store16(typename E::T *p, const u4 &v) { *reinterpret_cast<typename E::Vec *>(p) = v; }

// For results so large that no cache keeps them for their reader: they do not push out what is being read.
template <class E>
__device__ __forceinline__ void store16_through(typename E::T *p, const u4 &v) { __builtin_nontemporal_store(v, reinterpret_cast<typename E::Vec *>(p)); }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }     // one instruction, 1 ulp
__device__ __forceinline__ float rcp_fast(float v) { return __builtin_amdgcn_rcpf(v); }       // likewise

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// ---------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------
[[maybe_unused]] int launched() { return hipGetLastError() == hipSuccess ? CX_OK : CX_ERR_HIP; }

// Whether two byte ranges share a byte.
[[maybe_unused]] bool overlap(const void *a, uint64_t a_bytes, const void *b, uint64_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && a_bytes && b_bytes && x < y + b_bytes && y < x + a_bytes;
}

// An array of a call for the question whether two of them share an element: rows of `width` bytes, `pitch` bytes from row to row.
struct Extent {
    const void *first;
    uint64_t rows, width, pitch;
};
[[maybe_unused]] Extent matrix_of(const void *first, int64_t rows, int64_t ld, int64_t columns, int elem)
{
    const uint64_t width = static_cast<uint64_t>(columns) * elem;
    return {first, static_cast<uint64_t>(rows), width, rows > 1 ? static_cast<uint64_t>(ld) * elem : width};
}
[[maybe_unused]] Extent dense_of(const void *first, uint64_t bytes) { return {first, 1, bytes, bytes}; }

// Exact where the pitches are equal or one of them is a single row: parts of the rows of one wider matrix share nothing.  Of other pitches
// whatever lies between the first and the last element counts.
[[maybe_unused]] bool share(const Extent &a, const Extent &b)
{
    if (a.rows < 1 || b.rows < 1 || !overlap(a.first, (a.rows - 1) * a.pitch + a.width, b.first, (b.rows - 1) * b.pitch + b.width)) return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) return true;
    const bool in_order = a.first <= b.first;
    const Extent &lo = in_order ? a : b, &hi = in_order ? b : a;
    if (lo.rows == 1) return true;                       // the other one begins inside it
    const uint64_t off = (reinterpret_cast<uintptr_t>(hi.first) - reinterpret_cast<uintptr_t>(lo.first)) % lo.pitch;
    return off < lo.width || off + hi.width > lo.pitch;
}

// Whether an output shares an element with an input or with another output.  may_out may be may_in, element for element (-1: none may).
template <int INS, int OUTS>
[[maybe_unused]] bool outputs_share(const Extent (&in)[INS], const Extent (&out)[OUTS], int may_out, int may_in)
{
    for (int i = 0; i < OUTS; ++i) {
        for (int k = 0; k < INS; ++k) {
            if (i == may_out && k == may_in && out[i].first == in[k].first && out[i].pitch == in[k].pitch) continue;
            if (share(out[i], in[k])) return true;
        }
        for (int k = i + 1; k < OUTS; ++k)
            if (share(out[i], out[k])) return true;
    }
    return false;
}

// Sizes whose products stay far inside 64 bits.
constexpr int64_t kMaxExtent = int64_t(1) << 40;
[[maybe_unused]] bool bad_matrix(int64_t rows, int64_t ld, int64_t columns)
{
    return rows < 1 || columns < 1 || ld < columns || ld > kMaxExtent || rows > kMaxExtent / ld;
}

[[maybe_unused]] bool misaligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

constexpr int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
constexpr int64_t ceil_div(int64_t v, int64_t by) { return (v + by - 1) / by; }

}  // namespace

#endif  // CX_LM_COMMON_HPP
