// words.hip -- scores under rules, the best words of a row, and words drawn from a
// row's law (gfx950).
#include "words.hpp"

namespace spdp {
namespace {

typedef unsigned long long u64;

template <typename T>
__device__ __forceinline__ float word_score(const T *x, const RowRules &r, int64_t w0, int at,
                                            int64_t V, const int32_t *count)
{
    return ruled(r, (float)x[w0 + at], w0 + at, r.n_words > 0 ? count[at] : 0);
}

// One workgroup per (row, chunk).
template <typename T>
__global__ void __launch_bounds__(kThreads) k_adjust(const T *x, int64_t ldx, T *y, int64_t ldy,
                                                     int64_t V, int64_t chunks, spdp_rules rules)
{
    __shared__ int32_t count[kChunk];
    const int64_t row = blockIdx.x / chunks, w0 = (blockIdx.x % chunks) * kChunk;
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) chunk_counts(r, w0, count);
    for (int at = threadIdx.x; at < kChunk && w0 + at < V; at += kThreads)
        y[row * ldy + w0 + at] = (T)word_score(x + row * ldx, r, w0, at, V, count);
}

// ---------------------------------------------------------------------------
// The best words.  A word of a row is a 64-bit key, its score's order above the
// complement of the word, so that keys are distinct and the k largest keys are
// the k best words with ties to the lowest word.  Key 0: no word.
// ---------------------------------------------------------------------------
__device__ __forceinline__ u64 key_of(float x, int64_t w)
{
    x = x + 0.f;  // -0 and 0 are a tie
    if (!(x > -__builtin_inff())) return 0;  // -inf, NaN
    const uint32_t b = __float_as_uint(x);
    const uint32_t order = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (u64)order << 32 | (uint32_t)~(uint32_t)w;
}

// Largest key below `below` among the workgroup's.
__device__ __forceinline__ u64 block_max(u64 v, u64 *red)
{
    for (int d = 32; d; d >>= 1) {
        const u64 o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int i = 0; i < kThreads / 64; ++i) v = red[i] > v ? red[i] : v;
    return v;
}

// One workgroup per (row, chunk): the chunk's k best, best first.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_top_chunk(const T *__restrict__ x, int64_t ld,
                                                        int64_t V, int64_t chunks,
                                                        spdp_rules rules, int32_t k,
                                                        u64 *__restrict__ best)
{
    constexpr int kPer = kChunk / kThreads;
    __shared__ int32_t count[kChunk];
    __shared__ u64 red[kThreads / 64];
    const int64_t row = blockIdx.x / chunks, w0 = (blockIdx.x % chunks) * kChunk;
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) chunk_counts(r, w0, count);
    u64 key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int at = threadIdx.x + i * kThreads;
        key[i] = w0 + at < V ? key_of(word_score(x + row * ld, r, w0, at, V, count), w0 + at) : 0;
    }
    u64 below = ~0ull;
    for (int32_t t = 0; t < k; ++t) {
        u64 m = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) m = key[i] < below && key[i] > m ? key[i] : m;
        m = block_max(m, red);
        if (threadIdx.x == 0) best[(int64_t)blockIdx.x * k + t] = m;
        below = m;
    }
}

// One workgroup per row: the k best of n keys.
__global__ void __launch_bounds__(kThreads) k_top_join(const u64 *__restrict__ best, int64_t n,
                                                       int32_t k, int32_t *__restrict__ word,
                                                       float *__restrict__ value)
{
    __shared__ u64 red[kThreads / 64];
    const int64_t row = blockIdx.x;
    u64 below = ~0ull;
    for (int32_t t = 0; t < k; ++t) {
        u64 m = 0;
        for (int64_t i = threadIdx.x; i < n; i += kThreads) {
            const u64 v = best[row * n + i];
            m = v < below && v > m ? v : m;
        }
        m = block_max(m, red);
        below = m;
        if (threadIdx.x == 0) {
            const uint32_t order = (uint32_t)(m >> 32);
            word[row * k + t] = m ? (int32_t)~(uint32_t)m : -1;
            value[row * k + t] = m ? __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu
                                                                         : ~order)
                                   : -__builtin_inff();
        }
    }
}

// ---------------------------------------------------------------------------
// Draws.  Word w of a row has the weight exp((x[w] - max x) / T); a draw with
// uniform u is the first word whose prefix of the weights exceeds u times their
// sum.  Two words' border is a sum of up to V weights, and a draw is decided by
// where u falls between borders that lie 1/V apart, so everything is in fp64.
//
// First pass: of every chunk the largest score and the sum of exp((x - largest) /
// T).  Second pass: a chunk holds the draws whose target falls between the sums
// up to it and past it; it finds them in the prefixes of its own weights.
// ---------------------------------------------------------------------------
struct Part {
    double top, sum;  // top: NaN where the row has no law (NaN or inf among its scores)
};

__device__ __forceinline__ double block_max(double v, double *red)
{
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int i = 0; i < kThreads / 64; ++i) v = fmax(v, red[i]);
    return v;
}

// Sum over the workgroup, in a fixed order.
__device__ __forceinline__ double block_sum(double v, double *red)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < kThreads / 64; ++i) s += red[i];
    return s;
}

constexpr int kSegment = kChunk / kThreads;  // consecutive words of a thread

template <typename T>
__global__ void __launch_bounds__(kThreads) k_draw_parts(const T *__restrict__ x, int64_t ld,
                                                         int64_t V, int64_t chunks,
                                                         spdp_rules rules, double inv_t,
                                                         Part *__restrict__ part)
{
    __shared__ int32_t count[kChunk];
    __shared__ double red[kThreads / 64];
    const int64_t row = blockIdx.x / chunks, w0 = (blockIdx.x % chunks) * kChunk;
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) chunk_counts(r, w0, count);
    float v[kSegment];
    double top = -__builtin_inf();
    bool law = true;
#pragma unroll
    for (int i = 0; i < kSegment; ++i) {
        const int at = threadIdx.x * kSegment + i;
        v[i] = w0 + at < V ? word_score(x + row * ld, r, w0, at, V, count) : -__builtin_inff();
        law = law && v[i] < __builtin_inff();
        top = fmax(top, (double)v[i]);
    }
    top = block_max(top, red);
    double s = 0.0;
    if (top > -__builtin_inf() && top < __builtin_inf())
#pragma unroll
        for (int i = 0; i < kSegment; ++i) s += exp(((double)v[i] - top) * inv_t);
    s = block_sum(s, red);
    const bool all = __syncthreads_and(law);
    if (threadIdx.x == 0) part[blockIdx.x] = Part{all ? top : __builtin_nan(""), s};
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_draw(const T *__restrict__ x, int64_t ld, int64_t V,
                                                   int64_t chunks, spdp_rules rules,
                                                   double inv_t,
                                                   const Part *__restrict__ part, int32_t draws,
                                                   const double *__restrict__ u, uint64_t seed,
                                                   uint32_t step, int64_t draw0,
                                                   int32_t *__restrict__ word,
                                                   float *__restrict__ logp)
{
    __shared__ int32_t count[kChunk];
    __shared__ double upto[kThreads];  // sum of the weights up to and with each thread's segment
    const int64_t row = blockIdx.x / chunks, chunk = blockIdx.x % chunks, w0 = chunk * kChunk;
    const Part *p = part + row * chunks;
    double top = -__builtin_inf();
    bool law = true;
    for (int64_t c = 0; c < chunks; ++c) {
        law = law && !(p[c].top != p[c].top);
        top = fmax(top, p[c].top);
    }
    law = law && top > -__builtin_inf();
    if (!law) {
        if (chunk == 0)
            for (int32_t t = threadIdx.x; t < draws; t += kThreads) {
                word[row * draws + t] = -1;
                logp[row * draws + t] = __builtin_nanf("");
            }
        return;
    }
    // sums before the chunk and with it, and which chunk holds the last weight
    double before = 0.0, with = 0.0, total = 0.0;
    int64_t last = 0;
    for (int64_t c = 0; c < chunks; ++c) {
        const double s = p[c].sum > 0.0 ? p[c].sum * exp((p[c].top - top) * inv_t) : 0.0;
        if (c == chunk) before = total;
        total += s;
        if (c == chunk) with = total;
        if (s > 0.0) last = c;
    }
    if (!(with > before) && chunk != last) return;
    // The chunk's own weights are taken relative to its own largest score, which has
    // weight 1, so that they do not all vanish beside the row's.
    const double own = p[chunk].top, scale = exp((own - top) * inv_t);
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) chunk_counts(r, w0, count);
    auto score = [&](int at) { return word_score(x + row * ld, r, w0, at, V, count); };
    auto weight = [&](int at) {
        return w0 + at < V ? exp(((double)score(at) - own) * inv_t) : 0.0;
    };
    double s = 0.0;
    for (int i = 0; i < kSegment; ++i) s += weight(threadIdx.x * kSegment + i);
    upto[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double a = 0.0;
        for (int i = 0; i < kThreads; ++i) {
            a += upto[i];
            upto[i] = a;
        }
    }
    __syncthreads();
    const double log_total = log(total);
    for (int32_t t = threadIdx.x; t < draws; t += kThreads) {
        const int64_t d = row * draws + t;
        const double uniform =
            u ? u[d] : (double)philox_x0(seed, (uint64_t)(draw0 + d), step, kPurposeWord) * 0x1p-32;
        const double target = fmax(uniform * total, 0.0);
        const bool past = !(uniform * total < total);  // also NaN: the last word with weight
        if (past ? chunk != last : !(target >= before && target < with)) continue;
        const double goal = past ? __builtin_inf() : (target - before) / scale;
        // first segment past the goal, else (rounding) the last one with weight
        int seg = -1, best = 0;
        for (int i = 0; i < kThreads && seg < 0; ++i) {
            if (upto[i] > (i ? upto[i - 1] : 0.0)) best = i;
            if (upto[i] > goal) seg = i;
        }
        if (seg < 0) seg = best;
        double a = seg ? upto[seg - 1] : 0.0;
        int got = 0;
        for (int i = 0; i < kSegment; ++i) {
            const double y = weight(seg * kSegment + i);
            a += y;
            if (y > 0.0) {
                got = seg * kSegment + i;
                if (a > goal) break;
            }
        }
        word[d] = (int32_t)(w0 + got);
        logp[d] = (float)(((double)score(got) - top) * inv_t - log_total);
    }
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

int64_t chunks_of(int64_t V) { return (V + kChunk - 1) / kChunk; }

}  // namespace

hipError_t launch_adjust(const void *x, int64_t ldx, void *y, int64_t ldy, int32_t type,
                         int64_t rows, int64_t V, const spdp_rules &rules, hipStream_t st)
{
    if (rows == 0 || V == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V);
    return by_type(type, rows * chunks, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_adjust<T>, grid, dim3(kThreads), 0, st, (const T *)x, ldx, (T *)y, ldy,
                           V, chunks, rules);
    });
}

int64_t words_work(int64_t rows, int64_t V, int32_t take)
{
    const int64_t chunks = chunks_of(V);
    const int64_t top = take * (int64_t)sizeof(u64), part = sizeof(Part);
    return rows * chunks * (top > part ? top : part);
}

int64_t words_blocks(int64_t rows, int64_t V) { return rows * chunks_of(V); }

hipError_t launch_top(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t V,
                      const spdp_rules &rules, int32_t k, int32_t *word, float *value, void *work,
                      hipStream_t st)
{
    if (rows == 0 || k == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V);
    u64 *best = static_cast<u64 *>(work);
    hipError_t e = by_type(type, rows * chunks, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_top_chunk<T>, grid, dim3(kThreads), 0, st, (const T *)x, ld, V,
                           chunks, rules, k, best);
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_top_join, dim3((unsigned)rows), dim3(kThreads), 0, st, best, chunks * k,
                       k, word, value);
    return hipGetLastError();
}

hipError_t launch_draw(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t V,
                       const spdp_rules &rules, double temperature, int32_t draws,
                       const double *u, uint64_t seed, uint32_t step, int64_t draw0,
                       int32_t *word, float *logp, void *work, hipStream_t st)
{
    if (rows == 0 || draws == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V);
    Part *part = static_cast<Part *>(work);
    hipError_t e = by_type(type, rows * chunks, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_draw_parts<T>, grid, dim3(kThreads), 0, st, (const T *)x, ld, V,
                           chunks, rules, 1.0 / temperature, part);
    });
    if (e != hipSuccess) return e;
    return by_type(type, rows * chunks, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_draw<T>, grid, dim3(kThreads), 0, st, (const T *)x, ld, V, chunks,
                           rules, 1.0 / temperature, part, draws, u, seed, step, draw0, word,
                           logp);
    });
}

}  // namespace spdp
