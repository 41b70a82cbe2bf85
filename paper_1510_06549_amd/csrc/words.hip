// words.hip -- scores under rules, the best words of a row, and words drawn from a
// row's law (gfx950).
#include "words.hpp"

namespace spdp {
namespace {

typedef unsigned long long u64;

// One workgroup per (row, chunk).  Scores are read once and written once, and nothing else
// takes as long: 1 000 x 100 000 in bf16 with all rules, 200 MB each way, take 81 us (4.9 TB/s;
// 94 where a vector's bias and mask are requested only when the listed words are counted).
// fp32 scores, twice as many bytes, take 138 us (5.8 TB/s).
constexpr int kAdjustThreads = 512;

template <typename T, bool STREAM>
__global__ void __launch_bounds__(kAdjustThreads) k_adjust(const T *x, int64_t ldx, T *y,
                                                           int64_t ldy, int64_t V, int32_t chunks,
                                                           spdp_rules rules)
{
    using C = Chunk<T, kAdjustThreads, 16, STREAM>;
    __shared__ typename C::Listed listed;
    const int64_t row = blockIdx.x / (uint32_t)chunks;
    const int64_t w0 = (int64_t)(blockIdx.x % (uint32_t)chunks) * C::kWords;
    C c;
    c.request(x + row * ldx, w0, V);
    const RowRules r = row_rules(rules, row);
    typename C::Held held[C::U];
#pragma unroll
    for (int u = 0; u < C::U; ++u) C::hold(r, w0, V, u, held[u]);
    if (r.n_words > 0) C::count(r, w0, listed);
    T *out = y + row * ldy + w0;
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
        float v[C::N];
        c.scores(r, w0, V, listed, u, v, &held[u]);
        Vec<T> k;
#pragma unroll
        for (int i = 0; i < C::N; ++i) k.v[i] = (T)v[i];
        const int a = C::at(u);
        if (w0 + a + C::N <= V) {
            store_vec<STREAM>(out + a, k);
        } else {
#pragma unroll
            for (int i = 0; i < C::N; ++i)
                if (w0 + a + i < V) out[a + i] = k.v[i];
        }
    }
}

// ---------------------------------------------------------------------------
// The best words.  A word of a row is a 64-bit key, its score's order above the
// complement of the word, so that keys are distinct and the k largest keys are
// the k best words with ties to the lowest word.  Key 0: no word.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t order_of(float x)
{
    x = x + 0.f;  // -0 and 0 are a tie
    const uint32_t b = __float_as_uint(x);
    const uint32_t order = b & 0x80000000u ? ~b : b | 0x80000000u;
    return x > -__builtin_inff() ? order : 0;  // neither -inf nor NaN
}

// The least score with this order; the lowest finite one for 0.
__device__ __forceinline__ float score_of_order(uint32_t order)
{
    const uint32_t b = order & 0x80000000u ? order & 0x7FFFFFFFu : ~order;
    return order ? __uint_as_float(b) : -3.402823466e+38f;
}

__device__ __forceinline__ u64 key_of(float x, int64_t w)
{
    const uint32_t order = order_of(x);
    return order ? (u64)order << 32 | (uint32_t)~(uint32_t)w : 0;
}

constexpr int kTopThreads = 256;
constexpr int kTopWaves = kTopThreads / 64;
constexpr int kKeys = 2048;  // kept at a time in LDS
constexpr int kKeysEach = kKeys / kTopThreads;

struct Kept {  // LDS
    u64 key[kKeys];
    int in_wave[2][3][kTopWaves];
};

// The value of another lane: lane ^ 1, lane ^ 2, a lane of the other half of eight, of the
// other half of sixteen (D = 1, 2, 4, 8).
template <int D>
__device__ __forceinline__ int other(int v)
{
    constexpr int ctrl = D == 1 ? 0xB1 : D == 2 ? 0x4E : D == 4 ? 0x141 : 0x140;
    return __builtin_amdgcn_update_dpp(v, v, ctrl, 0xF, 0xF, false);
}

__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, __int_as_float(other<1>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(other<2>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(other<4>(__float_as_int(v))));
    v = fmaxf(v, __int_as_float(other<8>(__float_as_int(v))));
    float m = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0));
    for (int row = 16; row < 64; row += 16)
        m = fmaxf(m, __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), row)));
    return m;
}

__device__ __forceinline__ uint32_t wave_or(uint32_t v)
{
    v |= (uint32_t)other<1>((int)v);
    v |= (uint32_t)other<2>((int)v);
    v |= (uint32_t)other<4>((int)v);
    v |= (uint32_t)other<8>((int)v);
    uint32_t m = 0;
    for (int row = 0; row < 64; row += 16) m |= (uint32_t)__builtin_amdgcn_readlane((int)v, row);
    return m;
}

__device__ __forceinline__ u64 wave_or(u64 v)
{
    return (u64)wave_or((uint32_t)(v >> 32)) << 32 | wave_or((uint32_t)v);
}

// Sum over the lanes up to and with each.
__device__ __forceinline__ int prefix(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // shift right by 1, 2, 4,
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // 8 in rows of 16 lanes,
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // lane 15 to the next row,
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to the upper half
    return v;
}

// A bound that at least k (<= kTopThreads) of the threads' values reach, and not many more:
// found a bit at a time, over the bits that not all values have alike, until it is reached by
// at most k / 8 more.  All threads call it, with a barrier between two calls; there is
// one in it.  Every wavefront counts for itself, so that no barrier is needed for a bit.
__device__ __forceinline__ uint32_t reached(uint32_t mine, int k, uint32_t (&value)[kTopThreads])
{
    static_assert(kTopThreads == 256, "four values a lane");
    typedef uint32_t quad __attribute__((ext_vector_type(4)));
    value[threadIdx.x] = mine;
    __syncthreads();
    const quad v = reinterpret_cast<const quad *>(value)[threadIdx.x & 63];
    uint32_t bound = ~wave_or(~(v[0] & v[1] & v[2] & v[3]));
    uint32_t differ = wave_or(v[0] | v[1] | v[2] | v[3]) ^ bound;
    while (differ) {
        const uint32_t high = 1u << (31 - __builtin_clz(differ)), t = bound | high;
        int reach = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) reach += __builtin_popcountll(__ballot(v[i] >= t));
        if (reach >= k) {
            bound = t;
            if (reach <= k + k / 8) break;
        }
        differ ^= high;
    }
    return bound;
}

// Places for `mine` keys of each thread, in the threads' order: the thread's first place
// behind `before`, and in total how many places there are.  All threads call it, and meet
// a barrier; `slot` may be used again behind the next one.
__device__ __forceinline__ int places(int mine, int before, int (&slot)[kTopWaves], int &total)
{
    const int upto = prefix(mine), wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) slot[wave] = upto;
    __syncthreads();
    total = 0;
    for (int i = 0; i < kTopWaves; ++i) {
        if (i < wave) before += slot[i];
        total += slot[i];
    }
    return before + upto - mine;
}

// The keys of each thread, of n; 0 for none.
__device__ __forceinline__ void for_keys(const Kept &kept, int n, u64 (&key)[kKeysEach])
{
#pragma unroll
    for (int i = 0; i < kKeysEach; ++i) {
        const int at = threadIdx.x + i * kTopThreads;
        key[i] = at < n ? kept.key[at] : 0;
    }
}

// Keeps of the keys that each thread holds those that reach the bound (> 0), and returns how
// many there are.  All threads call it; there is a barrier before the keys are written and
// one before it returns.
__device__ __forceinline__ int keep_keys(Kept &kept, const u64 (&key)[kKeysEach], u64 bound)
{
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kKeysEach; ++i) mine += key[i] >= bound;
    __syncthreads();
    int total, to = places(mine, 0, kept.in_wave[0][0], total);
#pragma unroll
    for (int i = 0; i < kKeysEach; ++i)
        if (key[i] >= bound) kept.key[to++] = key[i];
    __syncthreads();
    return total;
}

// So many keys for the k best are ranked rather than brought further down.
__device__ __forceinline__ int enough_keys(int k)
{
    const int n = k + k / 4 < 64 ? 64 : k + k / 4;
    return n < kTopThreads ? n : kTopThreads;
}

// Cuts the n keys (kTopThreads < n <= kKeys, none 0) down to at least k and no more than are
// enough, the k largest among them, in any order, and returns how many; least is a bound
// that only they reach, found two bits at a time, over the bits that not all keys have
// alike.  All threads call it, behind a barrier; there is one before it returns.
__device__ __forceinline__ int cut_keys(Kept &kept, int n, int k, u64 &least)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 key[kKeysEach];
    for_keys(kept, n, key);
    u64 any = 0, all = ~0ull;
#pragma unroll
    for (int i = 0; i < kKeysEach; ++i)
        if ((int)threadIdx.x + i * kTopThreads < n) {
            any |= key[i];
            all &= key[i];
        }
    any = wave_or(any);
    all = ~wave_or(~all);
    __syncthreads();
    if (lane == 0) {
        kept.key[2 * wave] = any;
        kept.key[2 * wave + 1] = all;
    }
    __syncthreads();
    for (int i = 0; i < kTopWaves; ++i) {
        any |= kept.key[2 * i];
        all &= kept.key[2 * i + 1];
    }
    u64 differ = any ^ all, bound = all;
    for (int turn = 0; differ; turn ^= 1) {
        const u64 high = 1ull << (63 - __builtin_clzll(differ)), rest = differ ^ high;
        const u64 low = rest ? 1ull << (63 - __builtin_clzll(rest)) : 0;
        const u64 t[3] = {bound | high | low, bound | high, bound | low};
        int reach[3] = {0, 0, 0};
#pragma unroll
        for (int i = 0; i < kKeysEach; ++i) {
            if (i * kTopThreads >= n) break;
#pragma unroll
            for (int j = 0; j < 3; ++j) reach[j] += __builtin_popcountll(__ballot(key[i] >= t[j]));
        }
        if (lane == 0)
            for (int j = 0; j < 3; ++j) kept.in_wave[turn][j][wave] = reach[j];
        __syncthreads();
        for (int j = 0; j < 3; ++j) {
            reach[j] = 0;
            for (int i = 0; i < kTopWaves; ++i) reach[j] += kept.in_wave[turn][j][i];
        }
        const int j = reach[0] >= k ? 0 : reach[1] >= k ? 1 : low && reach[2] >= k ? 2 : 3;
        if (j < 3) bound = t[j];
        if (j < 3 && reach[j] <= enough_keys(k)) break;
        differ = rest ^ low;
    }
    least = bound;
    return keep_keys(kept, key, bound);
}

// Calls put(rank, key) for the k largest of the n keys, n <= kTopThreads: a key's rank is
// the number of larger ones.  All threads call it, behind a barrier.
template <typename F>
__device__ __forceinline__ void rank_keys(Kept &kept, int n, int k, F put)
{
    constexpr int kAtOnce = 8;  // keys read at a time
    if ((int)threadIdx.x < kAtOnce) kept.key[n + threadIdx.x] = 0;
    __syncthreads();
    if ((int)threadIdx.x >= n) return;
    const u64 key = kept.key[threadIdx.x];
    int rank = 0;
    for (int i = 0; i < n; i += kAtOnce) {
        u64 o[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) o[j] = kept.key[i + j];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) rank += o[j] > key;
    }
    if (rank < k) put(rank, key);
}

__device__ __forceinline__ void put_top(u64 key, int32_t *word, float *value)
{
    *word = key ? (int32_t)~(uint32_t)key : -1;
    *value = key ? score_of_order((uint32_t)(key >> 32)) : -__builtin_inff();
}

// One workgroup per part of a row: `words` words, a chunk at a time.  What could be among
// the k best is collected in LDS: scores at or above a bound that at least k of those seen
// so far reach, namely the largest scores that k of the threads have seen.  Of 256 threads
// that have seen m scores each about k (1 + k / 512) reach the bound; it rises each time that
// the threads have seen twice as many, so that few scores pass.  Where the collection would
// overflow (many ties), it is cut down to little more than its k best, again and again.
//
// 400 x 50 000 in fp32 (80 MB), 50 best: 47 us with rules, of which the join takes 5, and 33
// without (2.4 TB/s); the single best 24.  The scores' bytes would take 16: a chunk is waited
// for four times over (its scores, counts, places and, in turn, the bound), and four
// workgroups a compute unit are all that the LDS holds to hide it.  512 threads: as long
// there, 30 us and not 19 for 1 000 x 20 000 in bf16.
template <typename T>
__global__ void __launch_bounds__(kTopThreads, 4) k_top_part(const T *__restrict__ x, int64_t ld,
                                                             int64_t V, int32_t parts, int64_t words,
                                                          spdp_rules rules, int32_t k,
                                                          u64 *__restrict__ best,
                                                          int32_t *__restrict__ word,
                                                          float *__restrict__ value)
{
    using C = Chunk<T, kTopThreads, 16>;
    __shared__ typename C::Listed listed;
    __shared__ Kept kept;
    __shared__ alignas(16) uint32_t largest[kTopThreads];
    __shared__ int wave_pass[2][kTopWaves];
    const int64_t row = blockIdx.x / (uint32_t)parts;
    const int64_t first = (int64_t)(blockIdx.x % (uint32_t)parts) * words;
    const int64_t end = first + words < V ? first + words : V;
    x += row * ld;
    C c;
    c.request(x, first, end);
    const RowRules r = row_rules(rules, row);
    int n = 0;           // keys kept
    float mine = -__builtin_inff();  // largest score that this thread has seen
    u64 bound = 1;       // keys below are not among the k best
    int chunk = 0;
    for (int64_t w0 = first; w0 < end; w0 += C::kWords, ++chunk) {
        if (r.n_words > 0) C::count(r, w0, listed);
        float v[C::U][C::N];
#pragma unroll
        for (int u = 0; u < C::U; ++u) {
            c.scores(r, w0, end, listed, u, v[u]);
#pragma unroll
            for (int i = 0; i < C::N; ++i) mine = fmaxf(mine, v[u][i]);
        }
        if (w0 + C::kWords < end) c.request(x, w0 + C::kWords, end);
        if ((chunk & (chunk + 1)) == 0) {  // chunks 0, 1, 3, 7, ..: twice as much seen
            const u64 b = (u64)reached(order_of(mine), k, largest) << 32;
            bound = b > bound ? b : bound;
        }
        // (at least the lowest finite score, so that neither -inf nor NaN passes)
        const float low = score_of_order((uint32_t)(bound >> 32));
        int pass = 0;
#pragma unroll
        for (int u = 0; u < C::U; ++u)
#pragma unroll
            for (int i = 0; i < C::N; ++i) pass += v[u][i] >= low;
        int passing, to = places(pass, n, wave_pass[chunk & 1], passing);
        if (__builtin_expect(n + passing <= kKeys, 1)) {
            if (pass) {
#pragma unroll
                for (int u = 0; u < C::U; ++u)
#pragma unroll
                    for (int i = 0; i < C::N; ++i)
                        if (v[u][i] >= low)
                            kept.key[to++] = key_of(v[u][i], w0 + C::at(u) + i);
            }
            n += passing;  // (the counts are free again: all have passed a barrier behind them)
            continue;
        }
        // kKeys / 2 scores at a time, so that there is room after every cut, from LDS (the
        // counts are not needed any more)
        float *score = reinterpret_cast<float *>(listed.count);
#pragma unroll
        for (int u = 0; u < C::U; ++u)
#pragma unroll
            for (int i = 0; i < C::N; ++i) score[C::at(u) + i] = v[u][i];
        constexpr int kEach = kKeys / 2 / kTopThreads;
        for (int from = 0; from < C::kWords; from += kEach * kTopThreads) {
            __syncthreads();
            if (n > kKeys / 2) {
                u64 least;
                n = cut_keys(kept, n, k, least);
                bound = least > bound ? least : bound;
            }
            u64 key[kEach];
            int more = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int at = from + e * kTopThreads + threadIdx.x;
                key[e] = key_of(score[at], w0 + at);
                more += key[e] >= bound;
            }
            int at = places(more, n, wave_pass[0], passing);
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                if (key[e] >= bound) kept.key[at++] = key[e];
            n += passing;
        }
        __syncthreads();
    }
    __syncthreads();
    // the bound by all scores, for the keys from before it rose (ranks of few keys cost less)
    if (chunk > 1 && n > enough_keys(k)) {
        const u64 b = (u64)reached(order_of(mine), k, largest) << 32;
        u64 key[kKeysEach];
        for_keys(kept, n, key);
        n = keep_keys(kept, key, b > 1 ? b : 1);
    }
    if (n > kTopThreads) {
        u64 least;
        n = cut_keys(kept, n, k, least);
    }
    word += row * k;
    value += row * k;
    best += (int64_t)blockIdx.x * k;
    rank_keys(kept, n, k, [&](int rank, u64 key) {
        if (parts == 1) put_top(key, word + rank, value + rank);
        else best[rank] = key;
    });
    for (int t = n + threadIdx.x; t < k; t += kTopThreads) {
        if (parts == 1) put_top(0, word + t, value + t);
        else best[t] = 0;
    }
}

// One workgroup per row: the k best of its parts' keys, k of each part in order.  Where four
// keys a thread are all, what k of the threads' largest reach bounds the k best.  Of more, the
// last of a run of four is reached by all four, so that what (k + 3) / 4 of the threads'
// runs reach does; the keys that reach it are few beside all (k and less than four of each
// part's, where no thread has more than one run).
__global__ void __launch_bounds__(kTopThreads) k_top_join(const u64 *__restrict__ best,
                                                          int32_t parts, int32_t k,
                                                          int32_t *__restrict__ word,
                                                          float *__restrict__ value)
{
    constexpr int kEach = 4, kAtOnce = kEach * kTopThreads;
    static_assert(kAtOnce <= kKeys / 2, "room after every cut");
    __shared__ Kept kept;
    __shared__ alignas(16) uint32_t largest[kTopThreads];
    const int64_t row = blockIdx.x;
    const int n = parts * k;
    best += row * n;
    u64 key[kEach];
    auto request = [&](int from) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int at = from + i * kTopThreads + threadIdx.x;
            key[i] = at < n ? best[at] : 0;
        }
    };
    request(0);
    u64 most = 0;
    int reach = k;
    if (n <= kAtOnce) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) most = key[i] > most ? key[i] : most;
    } else {
        const int run = k < 4 ? 1 : 4, runs = k / run;  // (of a part; keys behind are in none)
        reach = (k + run - 1) / run;
        for (int i = threadIdx.x; i < parts * runs; i += kTopThreads) {
            const int part = i / runs;
            const u64 last = best[part * k + (i - part * runs) * run + run - 1];
            most = last > most ? last : most;
        }
    }
    u64 bound = (u64)reached((uint32_t)(most >> 32), reach, largest) << 32;
    bound = bound ? bound : 1;
    int have = 0;
    for (int from = 0; from < n; from += kAtOnce) {
        if (from) request(from);
        int more = 0, total;
#pragma unroll
        for (int i = 0; i < kEach; ++i) more += key[i] >= bound;
        int to = places(more, have, kept.in_wave[0][0], total);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (key[i] >= bound) kept.key[to++] = key[i];
        have += total;
        __syncthreads();
        if (have > kKeys / 2) {
            u64 least;
            have = cut_keys(kept, have, k, least);
            bound = least > bound ? least : bound;
        }
    }
    if (have > kTopThreads) {
        u64 least;
        have = cut_keys(kept, have, k, least);
    }
    word += row * k;
    value += row * k;
    rank_keys(kept, have, k, [&](int rank, u64 key) {
        put_top(key, word + rank, value + rank);
    });
    for (int t = have + threadIdx.x; t < k; t += kTopThreads) put_top(0, word + t, value + t);
}

// ---------------------------------------------------------------------------
// Draws.  Word w of a row has the weight exp((x[w] - max x) / T); a draw with
// uniform u is the first word whose prefix of the weights exceeds u times their
// sum.  Two words' border is a sum of up to V weights, and a draw is decided by
// where u falls between borders that lie 1/V apart, so everything is in fp64.
//
// One pass over the scores leaves of every chunk its largest score, the sum of its
// weights relative to that (the largest is then 1 in every chunk, and they do not
// vanish beside the row's largest), the sums up to the end of each of its blocks of 64
// words, and of each block's quarters the sum of 16 weights.  A wavefront then makes up to
// 64 draws: the chunk among the chunks, each lane for its draw; the block among the
// chunk's 128, all lanes for one draw after another; the quarter, each lane for its draw;
// the word among the quarter's 16 scores, 16 lanes for a draw; each by where the target
// falls between the sums up to one and up to the next.
// ---------------------------------------------------------------------------
constexpr int kDrawThreads = 512, kDrawPer = 16;
constexpr int kDrawChunk = kDrawThreads * kDrawPer;
constexpr int kBlockWords = 64, kBlocks = kDrawChunk / kBlockWords;  // two blocks a lane
constexpr int kQuarterWords = 16, kQuarters = kDrawChunk / kQuarterWords;
constexpr int kSums = kBlocks + kQuarters;  // of a chunk: up to each block, of each quarter

struct Part {
    double top, sum;  // top: NaN where the chunk holds NaN or +inf
};

// Weights: exp((x - top) / T) = 2^(n / 128) 2^(f / 128), where (x - top) (128 / (T log 2)) = n
// + f with n whole and |f| <= 1/2.  The first factor is a table's entry for n mod 128 times a
// power of two, the second the series of exp(f log 2 / 128) up to f^4 (the rest is below
// 2^-49 of it; 32 entries, on which no two lanes of a bank meet, need f^5 for 2^-48).
// The product's rounding adds 2^-53 |n| / 128 log 2: 2^-49 for weights of exp(-20), 2^-43
// for the least fp64 weights.
constexpr int kLogPowers = 7, kPowers = 1 << kLogPowers;
constexpr double kLogStep = 0.693147180559945309417 / kPowers;  // of one step of n

struct Powers {  // LDS
    double of[kPowers];
};

__device__ __forceinline__ void make_powers(Powers &p)  // (a barrier has to follow)
{
    if (threadIdx.x < kPowers) p.of[threadIdx.x] = exp2((double)threadIdx.x / kPowers);
}

// scale = 1 / (T kLogStep)
__device__ __forceinline__ double power_of(double z, const Powers &p)
{
    // z <= 0: its magnitude is cut to 137 760 and a little, whose weight rounds to 0 (a comparison
    // of the high words as they are, one instruction; -inf and -0 come out right)
    const u64 bits = __builtin_bit_cast(u64, z);
    const uint32_t high = min((uint32_t)(bits >> 32), 0xC100D100u);
    z = __builtin_bit_cast(double, (u64)high << 32 | (uint32_t)bits);
    const double n = rint(z), f = z - n;
    const int i = (int)n;
    constexpr double a = kLogStep;
    double q = a * a * a * a / 24.0;
    q = fma(q, f, a * a * a / 6.0);
    q = fma(q, f, a * a / 2.0);
    q = fma(q, f, a);
    const double t = p.of[i & (kPowers - 1)];
    return ldexp(fma(q * f, t, t), i >> kLogPowers);
}

__device__ __forceinline__ double weight_of(float x, double top, double scale, const Powers &p)
{
    return power_of(((double)x - top) * scale, p);
}

// The value that DPP control CTRL brings to a lane; 0 where it brings none, and in the rows
// of 16 lanes that are not among ROWS.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ double moved(double v)
{
    const u64 b = __builtin_bit_cast(u64, v);
    const int l = (int)(uint32_t)b, h = (int)(uint32_t)(b >> 32);
    uint32_t lo, hi;
    if constexpr (ROWS == 0xF) {
        lo = __builtin_amdgcn_mov_dpp(l, CTRL, 0xF, 0xF, true);
        hi = __builtin_amdgcn_mov_dpp(h, CTRL, 0xF, 0xF, true);
    } else {
        lo = __builtin_amdgcn_update_dpp(0, l, CTRL, ROWS, 0xF, false);
        hi = __builtin_amdgcn_update_dpp(0, h, CTRL, ROWS, 0xF, false);
    }
    return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}

__device__ __forceinline__ double of_lane(double v, int lane)  // (the same lane for all)
{
    const u64 b = __builtin_bit_cast(u64, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (u64)hi << 32 | lo);
}

// Sum over the lanes up to and with each, in its row of 16 lanes.
__device__ __forceinline__ double row_prefix(double v)
{
    v += moved<0x111>(v);  // shift right by 1, 2, 4, 8 in the row
    v += moved<0x112>(v);
    v += moved<0x114>(v);
    v += moved<0x118>(v);
    return v;
}

// Sum over the lanes up to and with each: within rows of 16 lanes, then a row's last lane
// to the next row, then the lower half's last to the upper half.
__device__ __forceinline__ double prefix(double v)
{
    v = row_prefix(v);
    v += moved<0x142, 0xA>(v);  // lane 15 of a row to the next
    v += moved<0x143, 0xC>(v);  // lane 31 to the upper half
    return v;
}

// Sums over a quarter's lanes (2 or 4, each with its part) in each of them; of those, over a
// block's lanes (8 or 16).
template <int LANES>
__device__ __forceinline__ double quarter_sum(double v)
{
    v += moved<0xB1>(v);                         // lane ^ 1
    if constexpr (LANES == 4) v += moved<0x4E>(v);  // lane ^ 2
    return v;
}

template <int LANES>
__device__ __forceinline__ double block_sum(double v)
{
    if constexpr (LANES == 8) v += moved<0x4E>(v);
    v += moved<0x141>(v);                            // the other four of eight
    if constexpr (LANES == 16) v += moved<0x140>(v);  // the other eight of sixteen
    return v;
}

// The largest of the lanes up to and with each, of values >= 0.
__device__ __forceinline__ double largest_upto(double v)
{
    v = fmax(v, moved<0x111>(v));
    v = fmax(v, moved<0x112>(v));
    v = fmax(v, moved<0x114>(v));
    v = fmax(v, moved<0x118>(v));
    v = fmax(v, moved<0x142, 0xA>(v));
    return fmax(v, moved<0x143, 0xC>(v));
}

__device__ __forceinline__ double lane_before(double v)  // (0 for the first)
{
    const double o = __shfl_up(v, 1);
    return (threadIdx.x & 63) ? o : 0.0;
}

// Two shares a lane, in order: upto[i] the sum up to and with share i.  The sums of different
// lanes are rounded differently, so they are made to rise: never below the one before,
// and above it only where there is a share.
__device__ __forceinline__ void rising(const double (&share)[2], double (&upto)[2])
{
    const double all = prefix(share[0] + share[1]);
    // (all lanes hand theirs on: one that a branch leaves out would give 0)
    const double to_here = lane_before(all);
    const double a = share[0] > 0.0 ? to_here + share[0] : 0.0;
    const double b = share[1] > 0.0 ? all : 0.0;
    const double before = lane_before(largest_upto(fmax(a, b)));
    upto[0] = fmax(before, a);
    upto[1] = fmax(upto[0], b);
}

// Of 64 rising sums, one a lane, with `last` the last: the first that exceeds this lane's
// goal, else (rounding) the first that reaches the last one.
__device__ __forceinline__ int first_past(double upto, double last, double goal)
{
    const bool past = last > goal;
    int at = 0;
#pragma unroll
    for (int step = 32; step; step >>= 1) {
        const double v = __shfl(upto, at + step - 1);
        at += past ? (v > goal ? 0 : step) : (v < last ? step : 0);
    }
    return at;  // (<= 63)
}

// What a row's draws share.
struct Law {
    double top, total;    // largest score; sum of the weights
    double upto;          // sum of the weights up to and with this lane's chunk;
    double own, inverse;  // its largest score, and 2^-100 of what its own weights are times theirs
    bool some;            // whether it holds some weight
    int32_t last;         // first of the last 64 chunks that hold some weight
    bool is;
};

// This lane's chunk.
__device__ __forceinline__ void lane_chunk(Law &law, const Part *part, int32_t c, int32_t chunks,
                                           double scale, const Powers &powers)
{
    double share = 0.0;
    law.own = law.top;
    law.inverse = 0x1p-100;
    if (c < chunks) {
        const Part p = part[c];
        if (p.sum > 0.0) {
            const double w = power_of((p.top - law.top) * scale, powers);
            share = p.sum * w;
            law.own = p.top;
            law.inverse = 1.0 / (w * 0x1p+100);  // (finite for the least weights)
        }
    }
    law.some = share > 0.0;
    const double upto = prefix(share);
    law.upto = largest_upto(law.some ? upto : 0.0);
}

__device__ __forceinline__ Law law_of(const Part *part, int32_t chunks, double scale,
                                      const Powers &powers)
{
    const int lane = threadIdx.x & 63;
    Law law{};
    float top = -__builtin_inff();
    bool is = true;
    for (int32_t c0 = 0; c0 < chunks; c0 += 64) {
        const float t = c0 + lane < chunks ? (float)part[c0 + lane].top : -__builtin_inff();
        is = is && t == t;
        top = fmaxf(top, t);
    }
    top = wave_max(top);
    law.top = top;
    law.is = !__any(!is) && top > -__builtin_inff();
    if (law.is)
        for (int32_t c0 = 0; c0 < chunks; c0 += 64) {
            lane_chunk(law, part, c0 + lane, chunks, scale, powers);
            law.total += of_lane(law.upto, 63);
            if (of_lane(law.upto, 63) > 0.0) law.last = c0;
        }
    return law;
}

// How often words are among a document's, which is looked up for a few words only.
struct Times {  // LDS: a table by hash, of which a quarter stays empty
    static constexpr int kSlots = 2048, kLogSlots = 11;
    int32_t word[kSlots], count[kSlots];

    // (longer documents are gone through, every wavefront with counts of its own)
    static __device__ __forceinline__ bool fits(const RowRules &r)
    {
        return r.n_words <= kSlots / 4 * 3;
    }

    static __device__ __forceinline__ int slot(int32_t w)
    {
        return (int)((uint32_t)w * 0x9E3779B1u >> (32 - kLogSlots));
    }

    // The workgroup makes it; a barrier has to follow.
    __device__ __forceinline__ void make(const RowRules &r)
    {
        if (!fits(r)) return;
        for (int i = threadIdx.x; i < kSlots; i += blockDim.x) {
            word[i] = -1;
            count[i] = 0;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < (int)r.n_words; i += blockDim.x) {
            const int32_t w = r.words[i];
            if (w < 0) continue;
            int at = slot(w);
            for (;; at = (at + 1) % kSlots) {
                const int32_t was = atomicCAS(&word[at], -1, w);
                if (was == -1 || was == w) break;
            }
            atomicAdd(&count[at], 1);
        }
    }

    // For the lane's word, where each row of 16 lanes has 16 words from base on.  All lanes
    // call it.
    __device__ __forceinline__ int of(const RowRules &r, int32_t base)
    {
        const int lane = threadIdx.x & 63;
        if (fits(r)) {
            const int32_t w = (int32_t)((uint32_t)base + (lane & 15));
            int at = slot(w);
            while (word[at] != w && word[at] != -1) at = (at + 1) % kSlots;
            return word[at] == w ? count[at] : 0;
        }
        int32_t *own = count + (threadIdx.x & ~63u);
        own[lane] = 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        constexpr int kEach = 4;
        for (int64_t i = 0; i < r.n_words; i += 64 * kEach) {
            int32_t entry[kEach];
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                entry[e] = i + 64 * e + lane < r.n_words ? r.words[i + 64 * e + lane] : -1;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t from = (uint32_t)__builtin_amdgcn_readlane(base, 16 * j);
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const uint32_t a = (uint32_t)entry[e] - from;
                    if (a < (uint32_t)kQuarterWords && entry[e] >= 0) atomicAdd(&own[16 * j + a], 1);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        return own[lane];
    }
};

// `count` draws from d0 on of a row by one wavefront.  times(base) is how often a lane's word
// is listed, where rows of 16 lanes have 16 words each from base on.
template <typename T, typename F>
__device__ __forceinline__ void draw_words(const T *__restrict__ x, int64_t V, const RowRules &r,
                                           double scale, int32_t chunks, const Part *part,
                                           const double *sums, const Powers &powers, int64_t d0,
                                           int32_t count, const double *__restrict__ u,
                                           uint64_t seed, uint32_t step, int64_t draw0,
                                           int32_t *__restrict__ word, float *__restrict__ logp,
                                           F times)
{
    const int lane = threadIdx.x & 63;
    double given = u && lane < count ? u[d0 + lane] : 0.0;
    Law law = law_of(part, chunks, scale, powers);
    if (!law.is) {
        for (int32_t t = lane; t < count; t += 64) {
            word[d0 + t] = -1;
            logp[d0 + t] = __builtin_nanf("");
        }
        return;
    }
    const double log_total = log(law.total);
    for (int32_t t0 = 0; t0 < count; t0 += 64) {
        const int64_t d = d0 + t0 + lane;
        const int32_t many = count - t0 < 64 ? count - t0 : 64;
        if (u && t0 && lane < many) given = u[d];
        const double uniform =
            lane >= many ? 0.0
            : u          ? given
                         : (double)philox_x0(seed, (uint64_t)(draw0 + d), step, kPurposeWord) * 0x1p-32;
        // (NaN, and 1 or more: the last word with weight, however little it adds)
        const bool end = !(uniform * law.total < law.total);
        double goal = end ? 0.0 : fmax(uniform * law.total, 0.0);
        // the chunk: 64 at a time, the first whose sum exceeds what is left
        int32_t chunk = 0;
        double own = 0.0;
        bool found = false;
        for (int32_t c0 = 0;; c0 += 64) {
            if (chunks > 64) lane_chunk(law, part, c0 + lane, chunks, scale, powers);
            const double sum = of_lane(law.upto, 63);
            const bool last = c0 >= law.last;
            const u64 some = __ballot(law.some);
            // (by all lanes: draws at the end hand their chunks' sums to the others)
            const int past = chunks == 1 ? 0 : first_past(law.upto, sum, goal);
            const int at = chunks > 1 && end ? 63 - __builtin_clzll(some | 1) : past;
            const double before = __shfl(law.upto, at ? at - 1 : 0);
            const double its = __shfl(law.own, at), inverse = __shfl(law.inverse, at);
            if (!found && (last || (!end && sum > goal))) {
                found = true;
                chunk = min(c0 + at, chunks - 1);
                own = its;
                goal = at ? goal - before : goal;
                goal = goal > 0.0 ? goal * 0x1p+100 * inverse : 0.0;
            } else if (!found) {
                goal -= sum;
            }
            if (last || !__any(!found)) break;
        }
        // A word has weight where it is above 2^-1075 beside the row's largest, which fp64 rounds to
        // 0: beside its chunk's largest, above `least` (0 where that is the row's).
        double least = 0.0;
        int way = 0;  // from where the first (1) or last (-1) such word is looked for, if by itself
        if (chunks > 1 && __any(lane < many && !(goal > 0.0))) {
            least = power_of(-1075.0 * kPowers - (own - law.top) * scale, powers);
            if (lane < many && least > 0.0) way = end ? -1 : !(goal > 0.0) ? 1 : 0;
            if (!end) goal = fmax(goal, least);
        }
        const bool ends = chunks > 1 && __any(way != 0);
        // the block (four draws' sums requested at a time)
        int32_t block = 0;
        for (int32_t t4 = 0; t4 < many; t4 += 4) {
            double2 upto[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                upto[j] = reinterpret_cast<const double2 *>(
                    sums + (int64_t)__builtin_amdgcn_readlane(chunk, t4 + j) * kSums)[lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double g = of_lane(goal, t4 + j);
                int b = __builtin_popcountll(__ballot(!(upto[j].x > g))) +
                        __builtin_popcountll(__ballot(!(upto[j].y > g)));
                if (b == kBlocks) {  // (rounding: the first that reaches the last)
                    const double end_sum = of_lane(upto[j].y, 63);
                    b = __builtin_popcountll(__ballot(upto[j].x < end_sum)) +
                        __builtin_popcountll(__ballot(upto[j].y < end_sum));
                }
                const double before =
                    b ? of_lane(b & 1 ? upto[j].x : upto[j].y, (b - 1) >> 1) : 0.0;
                if (lane == t4 + j) {
                    block = b;
                    goal = fmax(g - before, 0.0);
                }
            }
        }
        // the quarter
        const double *of_quarter = sums + (int64_t)chunk * kSums + kBlocks;
        int32_t quarter = kQuarters - 1;
        if (end) {
            while (quarter > 0 && !(of_quarter[quarter] > least)) --quarter;
            goal = __builtin_inf();
        } else {
            const double2 a = reinterpret_cast<const double2 *>(of_quarter)[2 * block];
            const double2 b = reinterpret_cast<const double2 *>(of_quarter)[2 * block + 1];
            const double s1 = a.x + a.y, s2 = s1 + b.x, s3 = s2 + b.y;
            const int q = a.x > goal   ? 0
                          : s1 > goal  ? 1
                          : s2 > goal  ? 2
                          : s3 > goal  ? 3
                          : b.y > 0.0  ? 3  // (rounding: the last with weight)
                          : b.x > 0.0  ? 2
                          : a.y > 0.0  ? 1
                                       : 0;
            goal = fmax(goal - (q == 0 ? 0.0 : q == 1 ? a.x : q == 2 ? s1 : s2), 0.0);
            quarter = 4 * block + q;
        }
        const int32_t first = chunk * kDrawChunk + quarter * kQuarterWords;
        // the word: 16 lanes for a draw, four draws at a time, the scores of 16 requested
        const int place = lane & 15, group = lane >> 4;
        for (int32_t t16 = 0; t16 < many; t16 += 16) {
            int32_t base[4];
            float score[4], bias[4];
            uint32_t allowed[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                base[j] = __shfl(first, t16 + 4 * j + group);
                const int64_t w = (int64_t)base[j] + place;
                score[j] = bias[j] = 0.f;
                allowed[j] = 0;
                if (w < V && t16 + 4 * j < many) {
                    score[j] = (float)x[w];
                    if (r.bias) bias[j] = r.bias[w];
                    allowed[j] = r.mask ? r.mask[w >> 5] >> (w & 31) : 1;
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t t = t16 + 4 * j + group;
                if (t16 + 4 * j >= many) break;
                const double g = __shfl(goal, t), top = __shfl(own, t);
                float s = score[j];
                if (r.n_words > 0) {
                    const int n = times(base[j]);
                    if (n > 0) s = penalised(r, s, n);
                }
                if (r.bias) s = s + bias[j];
                s = allowed[j] & 1u ? s : -__builtin_inff();
                const double weight = weight_of(s, top, scale, powers);
                const double upto = row_prefix(weight);
                const u64 positive = __ballot(weight > 0.0), past = __ballot(upto > g) & positive;
                uint32_t in_row = (uint32_t)(past >> (lane & 48)) & 0xFFFFu;
                uint32_t have = (uint32_t)(positive >> (lane & 48)) & 0xFFFFu;
                if (ends) {
                    // quarter by quarter, whose sums say only that their words together may have
                    // weight, until a word has, the chunk's largest at the latest
                    const double floor = __shfl(least, t);
                    const int by = __shfl(way, t);
                    double at_base = weight;
                    uint32_t its = 0;
                    for (int left = kQuarters; left > 0; --left) {
                        const u64 above = __ballot(at_base > floor);
                        its = (uint32_t)(above >> (lane & 48)) & 0xFFFFu;
                        const bool more = by != 0 && its == 0;
                        if (!__any(more)) break;
                        if (more) base[j] += by * kQuarterWords;
                        const int64_t w = (int64_t)base[j] + place;
                        s = -__builtin_inff();
                        const int n = r.n_words > 0 ? times(base[j]) : 0;
                        if (w >= 0 && w < V) s = ruled(r, (float)x[w], w, n);
                        at_base = weight_of(s, top, scale, powers);
                    }
                    in_row = by == 0 ? in_row : by > 0 ? its : 0;
                    have = by < 0 ? its : have;
                }
                const int l = in_row ? __builtin_ctz(in_row) : 31 - __builtin_clz(have | 1u);
                if (place == l && t < many) {
                    word[d0 + t0 + t] = base[j] + place;
                    logp[d0 + t0 + t] = (float)(((double)s - law.top) * scale * kLogStep - log_total);
                }
            }
        }
    }
}

// One workgroup per (row, chunk): its largest score and its sums.  From rows of one chunk the
// workgroup draws at once (ONE).
//
// 500 x 100 000 in bf16 (100 MB): 53 us, 65 with rules.  The scores' bytes would take 22:
// what bounds it are 30 vector instructions for each score, 13 of them in fp64, which issue
// without a pause for 41 us.
template <typename T, bool ONE>
__global__ void __launch_bounds__(kDrawThreads, ONE ? 4 : 8) k_draw_parts(
    const T *__restrict__ x, int64_t ld, int64_t V, int32_t chunks, spdp_rules rules, double scale,
    Part *__restrict__ part, double *__restrict__ sums, int32_t draws,
    const double *__restrict__ u, uint64_t seed, uint32_t step, int64_t draw0,
    int32_t *__restrict__ word, float *__restrict__ logp)
{
    using C = Chunk<T, kDrawThreads, kDrawPer>;
    constexpr int kLanes = kBlockWords / C::N;  // lanes whose vectors make a block
    constexpr int kQuarterLanes = kQuarterWords / C::N;
    __shared__ typename C::Listed listed;
    __shared__ float wave_top[kDrawThreads / 64];
    __shared__ alignas(16) double sum_of[kSums];
    __shared__ Part own;
    __shared__ Powers powers;
    make_powers(powers);
    const int64_t row = blockIdx.x / (uint32_t)chunks;
    const int32_t chunk = blockIdx.x % (uint32_t)chunks;
    const int64_t w0 = (int64_t)chunk * C::kWords;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    C c;
    c.request(x + row * ld, w0, V);
    const RowRules r = row_rules(rules, row);
    typename C::Held held[C::U];
#pragma unroll
    for (int u = 0; u < C::U; ++u) C::hold(r, w0, V, u, held[u]);
    if (r.n_words > 0) C::count(r, w0, listed);
    float v[C::U][C::N];
    float top = -__builtin_inff();
    bool law = true;  // no NaN (two scores a comparison)
#pragma unroll
    for (int k = 0; k < C::U; ++k) {
        c.scores(r, w0, V, listed, k, v[k], &held[k]);
#pragma unroll
        for (int i = 0; i < C::N; ++i) {
            if (i % 2) law = law && !__builtin_isunordered(v[k][i - 1], v[k][i]);
            top = fmaxf(top, v[k][i]);
        }
    }
    top = wave_max(top);
    if (lane == 0) wave_top[wave] = top;
    law = !__syncthreads_or(!law);
    for (int i = 0; i < kDrawThreads / 64; ++i) top = fmaxf(top, wave_top[i]);
    law = law && top < __builtin_inff();
    const bool some = top > -__builtin_inff() && top < __builtin_inff();
    double *to = ONE ? sum_of : sums + (int64_t)blockIdx.x * kSums;
#pragma unroll
    for (int k = 0; k < C::U; ++k) {
        double s = 0.0;
        if (some) {
#pragma unroll
            for (int i = 0; i < C::N; ++i) s += weight_of(v[k][i], top, scale, powers);
        }
        s = quarter_sum<kQuarterLanes>(s);
        if (lane % kQuarterLanes == 0) to[kBlocks + C::at(k) / kQuarterWords] = s;
        s = block_sum<kLanes>(s);
        if (lane % kLanes == 0) sum_of[C::at(k) / kBlockWords] = s;
    }
    __syncthreads();
    if (wave == 0) {
        const double share[2] = {sum_of[2 * lane], sum_of[2 * lane + 1]};
        double upto[2];
        rising(share, upto);
        const Part p{law ? (double)top : __builtin_nan(""), of_lane(upto[1], 63)};
        to[2 * lane] = upto[0];
        to[2 * lane + 1] = upto[1];
        if (lane == 0) {
            own = p;
            if (!ONE) part[blockIdx.x] = p;
        }
    }
    if constexpr (ONE) {
        __syncthreads();
        constexpr int kWaves = kDrawThreads / 64;
        const int32_t each = (draws + kWaves - 1) / kWaves, t0 = wave * each;
        if (t0 < draws)
            draw_words(x + row * ld, V, r, scale, 1, &own, sum_of, powers, row * draws + t0,
                       draws - t0 < each ? draws - t0 : each, u, seed, step, draw0, word, logp,
                       [&](int32_t base) { return listed.count[base + (lane & 15)]; });
    }
}

// `share` workgroups of four wavefronts per row, `each` draws a wavefront.  250 draws of each
// of 500 rows: 28 us, 38 with rules, mostly in wait of the sums and scores that the draws
// land on (16 us of instructions).
template <typename T>
__global__ void __launch_bounds__(256) k_draw(const T *__restrict__ x, int64_t ld, int64_t V,
                                              int32_t chunks, spdp_rules rules, double scale,
                                              const Part *__restrict__ part,
                                              const double *__restrict__ sums, int32_t share,
                                              int32_t each, int32_t draws,
                                              const double *__restrict__ u, uint64_t seed,
                                              uint32_t step, int64_t draw0,
                                              int32_t *__restrict__ word,
                                              float *__restrict__ logp)
{
    __shared__ Powers powers;
    __shared__ Times times;
    make_powers(powers);
    const int64_t row = blockIdx.x / (uint32_t)share;
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) times.make(r);
    __syncthreads();
    const int64_t t0 = ((int64_t)(blockIdx.x % (uint32_t)share) * 4 + (threadIdx.x >> 6)) * each;
    if (t0 >= draws) return;
    draw_words(x + row * ld, V, r, scale, chunks, part + row * chunks,
               sums + row * chunks * kSums, powers, row * draws + t0,
               (int32_t)(draws - t0 < each ? draws - t0 : each), u, seed, step, draw0, word, logp,
               [&](int32_t base) { return times.of(r, base); });
}

// launch(value of the scores' type, grid), and its error
template <typename F>
hipError_t by_type(int32_t type, int64_t blocks, F launch)
{
    const dim3 grid((unsigned)blocks);
    if (type == SPDP_F32) launch(float{}, grid);
    else if (type == SPDP_F16) launch(_Float16{}, grid);
    else launch(__bf16{}, grid);
    return hipGetLastError();
}

// launch(first row, rows, their scores) for as many rows at a time as their workgroups fit a
// launch, per_row at most for one (2^19 at most: 2^31 words in chunks of 4 096).
template <typename F>
hipError_t by_rows(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t per_row, F launch)
{
    const int64_t step = kLaunchBlocks / per_row, size = type == SPDP_F32 ? 4 : 2;
    for (int64_t row = 0; row < rows; row += step) {
        const int64_t m = rows - row < step ? rows - row : step;
        const hipError_t e = launch(row, m, static_cast<const char *>(x) + row * ld * size);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t chunks_of(int64_t V, int64_t words) { return (V + words - 1) / words; }

// Parts of a row for the best words, of even length: as many as chunks while the rows alone
// leave compute units idle, else several chunks one after another in a workgroup (few
// scores of the later ones pass the bound), all parts of all rows at once on the chip
// (four workgroups a compute unit; 400 rows of 50 000 without rules: two parts 33 us, one 35,
// four 41).  Two chunks are taken by one workgroup, which is sooner done than the parts are
// joined (1 row of 8 192 words 7.6 us, in two parts 10.1; 12 288 words 13.0, in three 10.7).
constexpr int64_t kTopBlocks = 1024;

struct TopShape {
    int64_t parts, words;
};

TopShape top_shape(int64_t rows, int64_t V)
{
    const int64_t chunks = chunks_of(V, kTopThreads * 16);
    int64_t parts = rows > 0 && rows < kTopBlocks ? kTopBlocks / rows : 1;
    parts = chunks <= 2 ? 1 : parts > chunks ? chunks : parts;
    const int64_t per = (chunks + parts - 1) / parts;  // chunks of a part
    parts = (chunks + per - 1) / per;
    const int64_t words = ((V + parts - 1) / parts + 31) / 32 * 32;  // (masks' words)
    return TopShape{(V + words - 1) / words, words};
}

int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

// Rows of one chunk: a row's own workgroup (eight wavefronts, 64 draws each at a time) makes up
// to kDrawAlone draws, and more where there are kRowsAlone rows to fill the chip; else many
// wavefronts do, in a second launch.  (5 000 words, us alone and by many: 1 row, 256 draws 14
// and 11, 1 000 draws 35 and 11; 32 rows, 256 draws 14 and 17, 1 000 draws 36 and 17; 256
// rows, 1 000 draws 37 and 37; 512 rows, 1 000 draws 51 and 60.)
constexpr int64_t kDrawAlone = 384, kRowsAlone = 256;

// (250 draws of 500 rows without rules: 79 us in all with 16 384 wavefronts, 74 with 8 192,
// 76 with 4 096)
constexpr int64_t kDrawWaves = 8192;

int64_t draw_parts_bytes(int64_t rows, int64_t chunks)
{
    return round256(rows * chunks * (int64_t)sizeof(Part));
}

}  // namespace

// Scores above kStreamBytes are streamed (1 000 x 100 000 with all rules: in bf16, 200 MB each
// way, 81 us streamed, 85 not, in fp32 138 and 144; 300 x 100 000 in bf16, 60 MB, 27.6 streamed,
// 25.0 not).
hipError_t launch_adjust(const void *x, int64_t ldx, void *y, int64_t ldy, int32_t type,
                         int64_t rows, int64_t V, const spdp_rules &rules, hipStream_t st)
{
    if (rows == 0 || V == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V, kAdjustThreads * 16);
    return by_rows(x, ldx, type, rows, chunks, [&](int64_t row, int64_t m, const void *from) {
        return by_type(type, m * chunks, [&](auto t, dim3 grid) {
            using T = decltype(t);
            const auto kernel = rows * V * (int64_t)sizeof(T) > kStreamBytes ? k_adjust<T, true>
                                                                             : k_adjust<T, false>;
            hipLaunchKernelGGL(kernel, grid, dim3(kAdjustThreads), 0, st, (const T *)from, ldx,
                               (T *)y + row * ldy, ldy, V, (int32_t)chunks, rules_from(rules, row));
        });
    });
}

int64_t top_work(int64_t rows, int64_t V, int32_t take)
{
    if (rows == 0) return 0;
    // (at least what top_shape's parts need, and no less for more rows)
    const int64_t most = rows * chunks_of(V, kTopThreads * 16);
    const int64_t parts = most < rows + kTopBlocks ? most : rows + kTopBlocks;
    return round256(parts * take * (int64_t)sizeof(u64));
}

int64_t draw_work(int64_t rows, int64_t V)
{
    if (rows == 0) return 0;
    const int64_t chunks = chunks_of(V, kDrawChunk);
    const int64_t apart = chunks > 1 || rows < kRowsAlone ? rows : kRowsAlone;
    return round256(draw_parts_bytes(apart, chunks) + apart * chunks * kSums * 8);
}

hipError_t launch_top(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t V,
                      const spdp_rules &rules, int32_t k, int32_t *word, float *value, void *work,
                      hipStream_t st)
{
    if (rows == 0 || k == 0) return hipSuccess;
    u64 *best = static_cast<u64 *>(work);
    const int64_t chunks = chunks_of(V, kTopThreads * 16);
    return by_rows(x, ld, type, rows, chunks, [&](int64_t row, int64_t m, const void *from) {
        const TopShape s = top_shape(m, V);
        const hipError_t e = by_type(type, m * s.parts, [&](auto t, dim3 grid) {
            using T = decltype(t);
            hipLaunchKernelGGL(k_top_part<T>, grid, dim3(kTopThreads), 0, st, (const T *)from, ld,
                               V, (int32_t)s.parts, s.words, rules_from(rules, row), k, best,
                               word + row * k, value + row * k);
        });
        if (e != hipSuccess || s.parts == 1) return e;
        hipLaunchKernelGGL(k_top_join, dim3((unsigned)m), dim3(kTopThreads), 0, st, best,
                           (int32_t)s.parts, k, word + row * k, value + row * k);
        return hipGetLastError();
    });
}

hipError_t launch_draw(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t V,
                       const spdp_rules &rules, double temperature, int32_t draws,
                       const double *u, uint64_t seed, uint32_t step, int64_t draw0,
                       int32_t *word, float *logp, void *work, hipStream_t st)
{
    if (rows == 0 || draws == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V, kDrawChunk);
    const double scale = kPowers * 1.44269504088896340736 / temperature;
    return by_rows(x, ld, type, rows, chunks, [&](int64_t row, int64_t m, const void *from) {
        Part *part = static_cast<Part *>(work);
        double *sums = reinterpret_cast<double *>(static_cast<char *>(work) +
                                                  draw_parts_bytes(m, chunks));
        const spdp_rules r = rules_from(rules, row);
        const int64_t at = row * draws;
        const double *given = u ? u + at : nullptr;
        const bool alone = chunks == 1 && (draws <= kDrawAlone || m >= kRowsAlone);
        const hipError_t e = by_type(type, m * chunks, [&](auto t, dim3 grid) {
            using T = decltype(t);
            const auto kernel = alone ? k_draw_parts<T, true> : k_draw_parts<T, false>;
            hipLaunchKernelGGL(kernel, grid, dim3(kDrawThreads), 0, st, (const T *)from, ld, V,
                               (int32_t)chunks, r, scale, part, sums, draws, given, seed, step,
                               draw0 + at, word + at, logp + at);
        });
        if (e != hipSuccess || alone) return e;
        // a wavefront per draw while that does not fill the chip, then several each
        int64_t waves = (kDrawWaves + m - 1) / m;
        waves = waves > draws ? draws : waves;
        const int64_t each = (draws + waves - 1) / waves;
        const int64_t share = (draws + 4 * each - 1) / (4 * each);
        return by_type(type, m * share, [&](auto t, dim3 grid) {
            using T = decltype(t);
            hipLaunchKernelGGL(k_draw<T>, grid, dim3(256), 0, st, (const T *)from, ld, V,
                               (int32_t)chunks, r, scale, part, sums, (int32_t)share, (int32_t)each,
                               draws, given, seed, step, draw0 + at, word + at, logp + at);
        });
    });
}

}  // namespace spdp
