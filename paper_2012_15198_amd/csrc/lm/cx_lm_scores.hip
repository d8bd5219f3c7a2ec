// C-ABI entry points cx_token_scores*, cx_scores_workspace: log probabilities of given tokens, entropy and the K largest
// logits of each row (see include/cx_lm.h).
//
//   lse = log sum_v exp(c z_v)    logp = c z_token - lse    H = lse - sum_v p_v c z_v = ln s - ln2 u / s
//
// One pass over the logits keeps maximum, sum and entropy sum in registers.  The K largest come almost for free from the maxima
// that this pass needs anyway: each thread notes the maximum of every few vectors it read (its subsets); the K-th largest of
// the threads' maxima is a threshold that at least K elements reach, and few more than K do; only the subsets whose maximum
// reaches it are read again.  Elements are compared by a 64-bit key (value, then lower id first), so ties are decided and the
// result does not depend on the order in which threads find them.
// Bound by memory: 4,096 float32 rows of 50,003 with 5 tokens take 139 us (5.9 TB/s).  Few rows are bound by the chain of waits: 16 bfloat16 rows of
// 131,072 with 20 tokens take 8 us, and 5 for joining the parts.
// Rows are split over workgroups where there are few; join_kernel then joins statistics and keys of the parts.
#include "lm_vocab.hpp"

namespace {

constexpr int kMaxTop = CX_MAX_TOP;
constexpr int kGroups = 4;                              // subsets of a thread
constexpr int kTurnKeys = 1024;                         // elements looked at between two checks of the list's length, at most
constexpr int kRankable = 256;                      // a list of this length is ranked by counting, a longer one cut to K first
constexpr unsigned kRankStep = 4;                       // keys of the list compared at once: eight take the kernel from 52 to 80 registers (4,096 float32 rows of 50,003: 145 to 160 us)

typedef unsigned long long Key;

// Ascending with the value (NaN apart); zeros of both signs are equal.
__device__ __forceinline__ unsigned ordered(float v)
{
    const unsigned b = __float_as_uint(v + 0.0f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
template <class E>
constexpr unsigned kValueMask = 0xffffffffu << (32 - E::kBits);
template <class E>
__device__ __forceinline__ float value_of(Key key)
{
    const unsigned o = static_cast<unsigned>(key >> 32);
    return __uint_as_float((o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)) & kValueMask<E>);
}
template <class E>
__device__ __forceinline__ Key key_of(float v, int64_t id)
{
    return static_cast<Key>(ordered(v) & kValueMask<E>) << 32 | (0xffffffffu - static_cast<unsigned>(id));
}
__device__ __forceinline__ int id_of(Key key) { return static_cast<int>(0xffffffffu - static_cast<unsigned>(key)); }

template <int THREADS>
struct TopSpace {
    static constexpr int kTurn = THREADS * 8 < kTurnKeys ? THREADS * 8 : kTurnKeys, kList = 2 * kTurn + kMaxTop;
    union {
        float maxima[kGroups][THREADS];                 // first pass
        Key list[kList];                                // second
    };
    uint16_t subsets[kGroups * THREADS];
    Key kept[kMaxTop];
    int reach[2][THREADS / kWave];
    Key least;                                          // keys below it are out
    unsigned count, subset_count;
};

// A key that exactly K of the list reach: as much of the K-th largest as tells it from the next, bit after bit from the top.  Only the bits that
// keys of this type and of ids below V differ in are tried.  The list stays in LDS, as held in registers it takes code that costs calls
// which never come here (8,192 rows of 1,000 with 64 tokens 63 us instead of 56).  All threads.
template <class E, int THREADS>
__device__ Key reached_by(TopSpace<THREADS> &s, unsigned count, int K, int64_t V)
{
    constexpr int kWaves = THREADS / kWave;
    const int id_bits = V > 1 ? 64 - __clzll(V - 1) : 0;
    Key kth = 0;
    int turn = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
        if (bit == 63 - E::kBits) {                     // the same in all keys: the zeros below the value, the ones above the id
            bit = id_bits - 1;
            kth |= 0xffffffffull >> id_bits << id_bits;
            if (bit < 0) break;
        }
        const Key probe = kth | (1ull << bit);
        int reach = 0;
#pragma unroll 1
        for (unsigned i = threadIdx.x; i - threadIdx.x < count; i += THREADS) reach += __popcll(__ballot(i < count && s.list[i] >= probe));
        if (kWaves > 1) {
            if ((threadIdx.x & (kWave - 1)) == 0) s.reach[turn & 1][threadIdx.x / kWave] = reach;
            ++turn;
            __syncthreads();
            reach = 0;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) reach += s.reach[(turn & 1) ^ 1][k];
        }
        if (reach >= K) kth = probe;
        if (reach == K) break;
    }
    return kth;
}

// Cuts the list to its K largest keys and raises `least`.  All threads, after a barrier; count > K.
template <class E, int THREADS>
__device__ void cut_list(TopSpace<THREADS> &s, int K, int64_t V)
{
    constexpr int kEach = (TopSpace<THREADS>::kList + THREADS - 1) / THREADS;
    const unsigned count = s.count;
    const Key kth = reached_by<E>(s, count, K, V);
    Key own[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) own[i] = i * THREADS + threadIdx.x < count ? s.list[i * THREADS + threadIdx.x] : 0;
    __syncthreads();                                    // everyone has the list in registers and the count read
    if (threadIdx.x == 0) { s.least = kth; s.count = 0; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (own[i] >= kth && own[i]) s.list[atomicAdd(&s.count, 1u)] = own[i];
    __syncthreads();
}

// The K largest keys of the list to kept[], the largest first; absent ones are 0.  All threads.
template <class E, int THREADS>
__device__ void rank_list(TopSpace<THREADS> &s, int K, int64_t V)
{
    __syncthreads();
    if (s.count > kRankable) cut_list<E>(s, K, V);
    const unsigned count = s.count;
    if (static_cast<int>(threadIdx.x) < K) s.kept[threadIdx.x] = 0;
    if (threadIdx.x < kRankStep) s.list[count + threadIdx.x] = 0;       // so that whole steps are compared
    __syncthreads();
    for (unsigned at = threadIdx.x; at < count; at += THREADS) {
        const Key mine = s.list[at];
        int rank = 0;
        for (unsigned i = 0; i < count; i += kRankStep)
#pragma unroll
            for (unsigned k = 0; k < kRankStep; ++k) rank += s.list[i + k] > mine;
        if (rank < K) s.kept[rank] = mine;
    }
    __syncthreads();
}

// The K largest keys of a slice, after the first pass has noted the maxima.  `rounds_each` rounds make a subset.
template <class E, int THREADS>
__device__ void top_of_slice(TopSpace<THREADS> &s, const Slice<E, THREADS, true> &slice, int64_t lo, int rounds_each, int K, int64_t V)
{
    __syncthreads();
    // wavefront 0: the largest 16-bit prefix of a value that the maxima of K threads reach
    if (threadIdx.x < kWave) {
        unsigned own[THREADS / kWave];
#pragma unroll
        for (int k = 0; k < THREADS / kWave; ++k) {
            float top = s.maxima[0][k * kWave + threadIdx.x];
#pragma unroll
            for (int g = 1; g < kGroups; ++g) top = fmaxf(top, s.maxima[g][k * kWave + threadIdx.x]);
            own[k] = ordered(top) >> 16;
        }
        unsigned prefix = 0;
#pragma unroll 1
        for (int bit = 15; bit >= 0; --bit) {
            const unsigned probe = prefix | (1u << bit);
            int reach = 0;
#pragma unroll
            for (int k = 0; k < THREADS / kWave; ++k) reach += __popcll(__ballot(own[k] >= probe));
            if (reach >= K) prefix = probe;             // to the last bit: the sharper, the fewer are read again
        }
        if (threadIdx.x == 0) { s.least = static_cast<Key>(prefix) << 48; s.subset_count = 0; }
    }
    __syncthreads();
    const unsigned prefix = static_cast<unsigned>(s.least >> 48);
    const int each = rounds_each * kAhead;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
        if (g * each * THREADS + static_cast<int>(threadIdx.x) < slice.vectors && ordered(s.maxima[g][threadIdx.x]) >> 16 >= prefix)
            s.subsets[atomicAdd(&s.subset_count, 1u)] = static_cast<uint16_t>(g * THREADS + threadIdx.x);
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();                                    // the maxima are dead from here on: their place is the list's
    const auto offer = [&](float v, int64_t at, Key least) {
        const Key key = key_of<E>(v, lo + at);
        if (v == v && key >= least) s.list[atomicAdd(&s.count, 1u)] = key;
    };
    if (slice.has_tail()) offer(E::widen(slice.z[slice.tail_at()]), slice.tail_at(), s.least);
    const int pieces = static_cast<int>(s.subset_count) * each;
    constexpr int kTurn = TopSpace<THREADS>::kTurn, kPieces = kTurn / E::kPer16 < THREADS ? kTurn / E::kPer16 : THREADS;      // vectors looked at in a turn
    for (int p0 = 0; p0 < pieces; p0 += kPieces) {
        __syncthreads();
        if (s.count + kTurn > TopSpace<THREADS>::kList) cut_list<E>(s, K, V);
        __syncthreads();
        const Key least = s.least;
        const int p = p0 + static_cast<int>(threadIdx.x);
        if (static_cast<int>(threadIdx.x) < kPieces && p < pieces) {
            const unsigned subset = s.subsets[p / each];
            const int in = p % each, group = subset / THREADS, thread = subset % THREADS;
            const int q = (group * each + in) * THREADS + thread;
            if (q < slice.vectors) {
                float v[E::kPer16];
                E::unpack(load16<E>(slice.z + static_cast<int64_t>(q) * E::kPer16), v);
#pragma unroll
                for (int j = 0; j < E::kPer16; ++j) offer(v[j], static_cast<int64_t>(q) * E::kPer16 + j, least);
            }
        }
    }
    rank_list<E>(s, K, V);
}

template <class E>
struct ScoreArgs {
    const typename E::T *z;
    const int32_t *tokens;
    float *logp, *entropy, *top_logp;
    int32_t *top_ids;
    int64_t ld, V;
    int K, parts;
    float scale;
    Stats *part_stats;                                  // [N][parts]
    Key *part_keys;                                     // [N][parts][K]
};

// What a row's statistics say; kept[] holds its K largest keys.
template <class E>
__device__ __forceinline__ void write_row(const ScoreArgs<E> &a, int64_t n, const Stats &all, const Key *kept)
{
    const float log_s = logf(all.s);
    const auto log_probability = [&](float z) { return all.s == 0.0f ? -__builtin_inff() : (z - all.m) * a.scale - log_s; };
    if (threadIdx.x == 0) {
        if (a.logp) {
            const int token = a.tokens[n];
            a.logp[n] = token >= 0 && token < a.V ? log_probability(E::widen(a.z[n * a.ld + token])) : 0.0f;
        }
        if (a.entropy) {
            const float h = log_s - kLn2 * all.u / all.s;
            a.entropy[n] = all.s == 0.0f || h < 0.0f ? 0.0f : h;
        }
    }
    if (static_cast<int>(threadIdx.x) < a.K) {
        const Key key = kept[threadIdx.x];
        a.top_ids[n * a.K + threadIdx.x] = key ? id_of(key) : -1;
        a.top_logp[n * a.K + threadIdx.x] = key ? log_probability(value_of<E>(key)) : __builtin_nanf("");
    }
}

// Grid (parts, N): one part of one row.  The first pass reads past the caches (4,096 float32 rows of 50,003: 139 us against 149).
template <class E, bool TOP, int THREADS>
__global__ __launch_bounds__(THREADS) void scores_kernel(const ScoreArgs<E> a)
{
    __shared__ Stats lds[THREADS / kWave];
    __shared__ TopSpace<THREADS> top;
    const int part = blockIdx.x;
    const int64_t n = blockIdx.y, lo = part_begin(a.V, a.parts, part, E::kPer16), hi = part_begin(a.V, a.parts, part + 1, E::kPer16);
    const Slice<E, THREADS, true> slice(a.z + n * a.ld, lo, hi);
    const float c = a.scale * kLog2e;
    const int rounds = slice.rounds(), rounds_each = (rounds + kGroups - 1) / kGroups;
    Stats own{kLowest, 0.0f, 0.0f};
    for (int g = 0, round = 0; g < kGroups; ++g) {
        float highest = -__builtin_inff();
        for (int r = 0; r < rounds_each && round < rounds; ++r, ++round) {
            float v[kAhead * E::kPer16];
            slice.load(round, v);
            highest = fmaxf(highest, accumulate<kEntropy>(own, v, c, 0.0f));
        }
        if (TOP) top.maxima[g][threadIdx.x] = highest;
    }
    if (slice.has_tail()) {
        const float v[1] = {E::widen(slice.z[slice.tail_at()])};
        accumulate<kEntropy>(own, v, c, 0.0f);
    }
    const Stats all = join_workgroup<kEntropy>(own, lds, c, 0.0f);
    if (TOP) top_of_slice<E, THREADS>(top, slice, lo, rounds_each, a.K, a.V);
    if (a.parts == 1) {
        write_row<E>(a, n, all, top.kept);
    } else {
        if (threadIdx.x == 0) a.part_stats[n * a.parts + part] = all;
        if (TOP && static_cast<int>(threadIdx.x) < a.K) a.part_keys[(n * a.parts + part) * a.K + threadIdx.x] = top.kept[threadIdx.x];
    }
}

template <class E, bool TOP>
__global__ __launch_bounds__(kRowThreads) void join_kernel(const ScoreArgs<E> a)
{
    __shared__ TopSpace<kRowThreads> top;
    const int64_t n = blockIdx.x;
    const float c = a.scale * kLog2e;
    Stats all = a.part_stats[n * a.parts];
    for (int k = 1; k < a.parts; ++k) all = join<kEntropy>(all, a.part_stats[n * a.parts + k], c, 0.0f);
    if (TOP) {
        // K keys reach a part's K-th one, and K keys reach the least of all parts' (K / parts)-th ones: the larger bound leaves little more than K
        const Key *keys = a.part_keys + n * a.parts * a.K;
        if (threadIdx.x == 0) top.count = 0;
        if (threadIdx.x < kWave) {
            const bool here = static_cast<int>(threadIdx.x) < a.parts;
            const int share = (a.K + a.parts - 1) / a.parts;
            Key most = here ? keys[(threadIdx.x + 1) * a.K - 1] : 0, least = here ? keys[threadIdx.x * a.K + share - 1] : ~0ull;
#pragma unroll
            for (int d = kWave / 2; d > 0; d /= 2) {
                const Key m = __shfl_xor(most, d), l = __shfl_xor(least, d);
                most = m > most ? m : most;
                least = l < least ? l : least;
            }
            if (threadIdx.x == 0) top.least = most > least ? most : least;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.parts * a.K; i += kRowThreads) {
            const Key key = keys[i];
            if (key && key >= top.least) top.list[atomicAdd(&top.count, 1u)] = key;
        }
        rank_list<E>(top, a.K, a.V);
    }
    write_row<E>(a, n, all, top.kept);
}

struct ScoreSpace {
    int parts;
    int64_t keys, bytes;
};

ScoreSpace score_space(int64_t N, int64_t V, int32_t K, int per16)
{
    ScoreSpace s{};
    s.parts = parts_of(N, V, per16);
    if (s.parts <= 1) return s;
    s.keys = round_up(N * s.parts * static_cast<int64_t>(sizeof(Stats)), 16);
    s.bytes = s.keys + N * s.parts * K * 8;
    return s;
}

int check_sizes(int64_t N, int32_t V, int32_t K)
{
    return N < 0 || N > CX_MAX_TOKENS || V < 1 || V > CX_MAX_VOCAB || K < 0 || K > kMaxTop || K > V ? CX_ERR_SHAPE : CX_OK;
}

template <class E>
int scores(const typename E::T *z, int64_t ld, int64_t N, int32_t V, const int32_t *tokens, float scale, float *logp, float *entropy,
           int32_t K, int32_t *top_ids, float *top_logp, void *workspace, int64_t workspace_bytes, void *stream)
{
    const int rc = check_sizes(N, V, K);
    if (rc != CX_OK) return rc;
    if (!(scale > 0.0f) || !(scale * kLog2e <= kLargest)) return CX_ERR_SHAPE;      // an infinite factor would make the maximum's term 0 * inf
    if (N == 0) return CX_OK;
    if (!z || (logp && !tokens) || (K > 0 && (!top_ids || !top_logp))) return CX_ERR_NULL;
    if (bad_matrix(N, ld, V)) return CX_ERR_SHAPE;
    const ScoreSpace space = score_space(N, V, K, E::kPer16);
    if (space.bytes > 0 && !workspace) return CX_ERR_NULL;
    if (space.bytes > 0 && workspace_bytes < space.bytes) return CX_ERR_SHAPE;
    constexpr int kElem = sizeof(typename E::T);
    if (misaligned_to(z, kElem) || misaligned_to(tokens, 4) || misaligned_to(logp, 4) || misaligned_to(entropy, 4) || misaligned_to(top_ids, 4) ||
        misaligned_to(top_logp, 4) || misaligned_to(workspace, 16)) return CX_ERR_ALIGN;
    const uint64_t row_bytes = N * 4, top_bytes = N * K * 4;
    const Extent in[2] = {matrix_of(z, N, ld, V, kElem), dense_of(tokens, row_bytes)};
    const Extent out[5] = {dense_of(logp, row_bytes), dense_of(entropy, row_bytes), dense_of(top_ids, top_bytes), dense_of(top_logp, top_bytes),
                           dense_of(workspace, space.bytes)};
    if (outputs_share(in, out, -1, -1)) return CX_ERR_ALIAS;
    char *base = static_cast<char *>(workspace);
    const ScoreArgs<E> a{z, tokens, logp, entropy, top_logp, top_ids, ld, V, K, space.parts, scale, reinterpret_cast<Stats *>(base),
                         reinterpret_cast<Key *>(base + space.keys)};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    // rows in slices of a grid's second dimension
    for (int64_t n0 = 0; n0 < N; n0 += 65535) {
        const unsigned rows = static_cast<unsigned>(N - n0 < 65535 ? N - n0 : 65535);
        ScoreArgs<E> b = a;
        b.z += n0 * ld;
        if (b.tokens) b.tokens += n0;
        if (b.logp) b.logp += n0;
        if (b.entropy) b.entropy += n0;
        if (K > 0) { b.top_ids += n0 * K; b.top_logp += n0 * K; }
        const auto launch = [&](auto size) {
            constexpr int THREADS = decltype(size)::value;
            if (K > 0) hipLaunchKernelGGL((scores_kernel<E, true, THREADS>), dim3(space.parts, rows), dim3(THREADS), 0, st, b);
            else hipLaunchKernelGGL((scores_kernel<E, false, THREADS>), dim3(space.parts, rows), dim3(THREADS), 0, st, b);
        };
        // threads of a row by its length: 8,192 rows of 1,000 bfloat16 logits take 37 us with 256 each and 75 with 512, 4,096 rows of 50,003
        // 106 and 109, 2,048 rows of 262,144 219 and 204; with 1,024 all but the longest rows take twice as long.  The K-th largest of
        // as many maxima as threads is a sharp threshold only where K is well below their number: with 64 threads 8,192 rows of 1,000 take
        // 16 us for 5 tokens against 37 with 256, 22 against 44 for 32, but 70 against 53 for 64, and 5 rows of 3,557 27 against 9
        const int64_t vectors = ceil_div(V / space.parts, E::kPer16);
        if (vectors <= 512 && K <= kWave / 2) launch(std::integral_constant<int, 64>{});
        else if (vectors <= 8192) launch(std::integral_constant<int, 256>{});
        else launch(std::integral_constant<int, 512>{});
        if (launched() != CX_OK) return CX_ERR_HIP;
    }
    if (space.parts == 1) return CX_OK;                 // split rows are few: one slice
    if (K > 0) hipLaunchKernelGGL((join_kernel<E, true>), dim3(static_cast<unsigned>(N)), dim3(kRowThreads), 0, st, a);
    else hipLaunchKernelGGL((join_kernel<E, false>), dim3(static_cast<unsigned>(N)), dim3(kRowThreads), 0, st, a);
    return launched();
}

}  // namespace

extern "C" {

#define CX_LM_SCORES(SUFFIX, E)                                                                                                       \
    int cx_token_scores##SUFFIX(const E::T *z, int64_t ld, int64_t N, int32_t V, const int32_t *tokens, float scale, float *logp,     \
                                float *entropy, int32_t K, int32_t *top_ids, float *top_logp, void *workspace,                        \
                                int64_t workspace_bytes, void *stream)                                                                \
    {                                                                                                                                 \
        return scores<E>(z, ld, N, V, tokens, scale, logp, entropy, K, top_ids, top_logp, workspace, workspace_bytes, stream);        \
    }
CX_LM_SCORES(, F32)
CX_LM_SCORES(_bf16, Bf16)
CX_LM_SCORES(_f16, F16)
#undef CX_LM_SCORES

int cx_scores_workspace(int64_t N, int32_t V, int32_t K, int64_t *bytes)
{
    if (!bytes) return CX_ERR_NULL;
    *bytes = 0;
    const int rc = check_sizes(N, V, K);
    if (rc != CX_OK || N == 0) return rc;
    const int64_t wide = score_space(N, V, K, F32::kPer16).bytes, narrow = score_space(N, V, K, Bf16::kPer16).bytes;
    *bytes = wide > narrow ? wide : narrow;
    return CX_OK;
}

}  // extern "C"
