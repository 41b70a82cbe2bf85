// words.hip -- scores under rules, the best words of a row, and words drawn from a
// row's law (gfx950).
#include "words.hpp"

namespace spdp {
namespace {

typedef unsigned long long u64;

// One workgroup per (row, chunk).
constexpr int kAdjustThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kAdjustThreads) k_adjust(const T *x, int64_t ldx, T *y,
                                                           int64_t ldy, int64_t V, int32_t chunks,
                                                           spdp_rules rules)
{
    using C = Chunk<T, kAdjustThreads, 16>;
    __shared__ typename C::Listed listed;
    const int64_t row = blockIdx.x / (uint32_t)chunks;
    const int64_t w0 = (int64_t)(blockIdx.x % (uint32_t)chunks) * C::kWords;
    C c;
    c.request(x + row * ldx, w0, V);
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) C::count(r, w0, listed);
    T *out = y + row * ldy + w0;
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
        float v[C::N];
        c.scores(r, w0, V, listed, u, v);
        Vec<T> k;
#pragma unroll
        for (int i = 0; i < C::N; ++i) k.v[i] = (T)v[i];
        const int a = C::at(u);
        if (w0 + a + C::N <= V) {
            store_vec(out + a, k);
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

__device__ __forceinline__ u64 key_of(uint32_t order, int64_t w)
{
    return order ? (u64)order << 32 | (uint32_t)~(uint32_t)w : 0;
}

// The k best of the keys in buf [0, n), best first, to its front; n <= kKeys.  A bitonic
// sort of the next power of two of them.  All threads call it, with barriers before
// (the keys are written) and after (they can be read).
constexpr int kTopThreads = 256;
constexpr int kKeys = 2048;

__device__ __forceinline__ void sort_keys(u64 *buf, int n)
{
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kTopThreads) buf[i] = 0;
    for (int k = 2; k <= size; k *= 2)
        for (int d = k / 2; d; d /= 2) {
            __syncthreads();
            for (int p = threadIdx.x; p < size / 2; p += kTopThreads) {
                const int i = 2 * p - (p & (d - 1)), j = i + d;  // bit d of i is 0
                const u64 x = buf[i], y = buf[j];
                if ((x < y) == ((i & k) == 0)) {
                    buf[i] = y;
                    buf[j] = x;
                }
            }
        }
    __syncthreads();
}

__device__ __forceinline__ void put_top(u64 key, int32_t *word, float *value)
{
    const uint32_t order = (uint32_t)(key >> 32);
    *word = key ? (int32_t)~(uint32_t)key : -1;
    *value = key ? __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order)
                 : -__builtin_inff();
}

// One workgroup per part of a row: `per` chunks, one after another.  What could be among
// the k best is collected in LDS: keys at or above a bound that at least k of the scores
// seen so far reach, namely the least of the largest scores that groups of threads have
// seen, with at least k groups.  The bound rises as the groups see more, so that after
// the first chunk few scores pass.  Where the collection would overflow (many ties), it
// is cut down to its k best, which raise the bound to the last of them.
template <typename T>
__global__ void __launch_bounds__(kTopThreads) k_top_part(const T *__restrict__ x, int64_t ld,
                                                          int64_t V, int32_t parts, int32_t per,
                                                          spdp_rules rules, int32_t k,
                                                          u64 *__restrict__ best,
                                                          int32_t *__restrict__ word,
                                                          float *__restrict__ value)
{
    using C = Chunk<T, kTopThreads, 16>;
    __shared__ typename C::Listed listed;
    __shared__ u64 buf[kKeys];
    __shared__ uint32_t wave_least[kTopThreads / 64];
    __shared__ int kept, passing;
    const int64_t row = blockIdx.x / (uint32_t)parts;
    const int32_t part = blockIdx.x % (uint32_t)parts;
    const RowRules r = row_rules(rules, row);
    const int64_t chunks = (V + C::kWords - 1) / C::kWords, first = (int64_t)part * per;
    const int64_t last = first + per < chunks ? first + per : chunks;
    int group = 1;  // threads of a group: the most that leaves k groups
    while (kTopThreads / (2 * group) >= k) group *= 2;
    if (threadIdx.x == 0) kept = 0;
    uint32_t mine = 0;    // largest order that this thread has seen
    u64 bound = 1;        // keys below are not among the k best (1: every word's key passes)
    C c;
    if (first < last) c.request(x + row * ld, first * C::kWords, V);
    for (int64_t ch = first; ch < last; ++ch) {
        const int64_t w0 = ch * C::kWords;
        if (r.n_words > 0) C::count(r, w0, listed);
        float v[C::U][C::N];
#pragma unroll
        for (int u = 0; u < C::U; ++u) c.scores(r, w0, V, listed, u, v[u]);
        if (ch + 1 < last) c.request(x + row * ld, w0 + C::kWords, V);
        uint32_t order[C::U][C::N];
#pragma unroll
        for (int u = 0; u < C::U; ++u)
#pragma unroll
            for (int i = 0; i < C::N; ++i) {
                order[u][i] = order_of(v[u][i]);
                mine = order[u][i] > mine ? order[u][i] : mine;
            }
        // least of the groups' largest
        uint32_t g = mine;
        for (int d = 1; d < group && d < 64; d *= 2) {
            const uint32_t o = __shfl_xor(g, d);
            g = o > g ? o : g;
        }
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_xor(g, d);
            g = o < g ? o : g;
        }
        if ((threadIdx.x & 63) == 0) wave_least[threadIdx.x >> 6] = g;
        if (threadIdx.x == 0) passing = 0;
        __syncthreads();
        {
            uint32_t w[kTopThreads / 64];
#pragma unroll
            for (int i = 0; i < kTopThreads / 64; ++i) w[i] = wave_least[i];
            uint32_t least;
            if (group <= 64) {
                least = min(min(w[0], w[1]), min(w[2], w[3]));
            } else if (group == 128) {
                least = min(max(w[0], w[1]), max(w[2], w[3]));
            } else {
                least = max(max(w[0], w[1]), max(w[2], w[3]));
            }
            const u64 b = (u64)least << 32;
            bound = b > bound ? b : bound;
        }
        int n = 0;
#pragma unroll
        for (int u = 0; u < C::U; ++u)
#pragma unroll
            for (int i = 0; i < C::N; ++i)
                n += key_of(order[u][i], w0 + C::at(u) + i) >= bound;
        if (n) atomicAdd(&passing, n);
        __syncthreads();
        const int have = kept;
        if (have + passing <= kKeys) {
            __syncthreads();
            if (n) {
                int to = atomicAdd(&kept, n);
#pragma unroll
                for (int u = 0; u < C::U; ++u)
#pragma unroll
                    for (int i = 0; i < C::N; ++i) {
                        const u64 key = key_of(order[u][i], w0 + C::at(u) + i);
                        if (key >= bound) buf[to++] = key;
                    }
            }
            __syncthreads();
            continue;
        }
        // (kKeys / 2 scores at a time, so that there is room after every cut)
#pragma unroll
        for (int u = 0; u < C::U; ++u)
#pragma unroll
            for (int i = 0; i < C::N; i += 4) {
                __syncthreads();
                const int m = kept;
                __syncthreads();  // (everybody has read it)
                if (m > kKeys / 2) {
                    sort_keys(buf, m);
                    if (m >= k) bound = buf[k - 1] > bound ? buf[k - 1] : bound;
                    __syncthreads();
                    if (threadIdx.x == 0) kept = m < k ? m : k;
                    __syncthreads();
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u64 key = key_of(order[u][i + e], w0 + C::at(u) + i + e);
                    if (key >= bound) buf[atomicAdd(&kept, 1)] = key;
                }
            }
        __syncthreads();
    }
    __syncthreads();
    const int n = kept;
    sort_keys(buf, n);
    for (int t = threadIdx.x; t < k; t += kTopThreads) {
        const u64 key = t < n ? buf[t] : 0;
        if (parts == 1) put_top(key, word + row * k + t, value + row * k + t);
        else best[(int64_t)blockIdx.x * k + t] = key;
    }
}

// One workgroup per row: the k best of its parts' keys, n in all.
__global__ void __launch_bounds__(kTopThreads) k_top_join(const u64 *__restrict__ best, int64_t n,
                                                          int32_t k, int32_t *__restrict__ word,
                                                          float *__restrict__ value)
{
    __shared__ u64 buf[kKeys];
    const int64_t row = blockIdx.x;
    int have = 0;
    for (int64_t from = 0; from < n;) {
        const int take = (int)(n - from < kKeys - have ? n - from : kKeys - have);
        for (int i = threadIdx.x; i < take; i += kTopThreads) buf[have + i] = best[row * n + from + i];
        from += take;
        __syncthreads();
        sort_keys(buf, have + take);
        have = have + take < k ? have + take : k;
    }
    for (int t = threadIdx.x; t < k; t += kTopThreads)
        put_top(t < have ? buf[t] : 0, word + row * k + t, value + row * k + t);
}

// ---------------------------------------------------------------------------
// Draws.  Word w of a row has the weight exp((x[w] - max x) / T); a draw with
// uniform u is the first word whose prefix of the weights exceeds u times their
// sum.  Two words' border is a sum of up to V weights, and a draw is decided by
// where u falls between borders that lie 1/V apart, so everything is in fp64.
//
// One pass over the scores leaves of every chunk its largest score, the sum of its
// weights relative to that (the largest is then 1 in every chunk, and they do not
// vanish beside the row's largest), and the sums of its blocks of 128 words.  A draw
// is then one wavefront's work: the chunk among the chunks' sums, the block among its
// chunk's 64, the word among its block's 128 scores, each by a prefix sum over the
// lanes.
// ---------------------------------------------------------------------------
constexpr int kDrawThreads = 512;
constexpr int kDrawChunk = kDrawThreads * 16;
constexpr int kBlocks = 64, kBlockWords = kDrawChunk / kBlocks;

struct Part {
    double top, sum;  // top: NaN where the chunk holds NaN or +inf
};

// exp(x) for x <= 0, to about 1 ulp: x = n log 2 + r, the series of exp(r) up to r^13
// (|r| <= 0.347, so the rest is below 2^-57 of it), times 2^n.
__device__ __forceinline__ double exp_of(double x)
{
    x = fmax(x, -746.0);  // (whose exponential rounds to 0)
    const double n = rint(x * 1.4426950408889634);
    double r = fma(n, -0x1.62e42fefa39efp-1, x);  // log 2 in two parts
    r = fma(n, -0x1.abc9e3b39803fp-56, r);
    double p = 1.0 / 6227020800.0;
    p = fma(p, r, 1.0 / 479001600.0);
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)n);
}

__device__ __forceinline__ double weight_of(float x, double top, double inv_t)
{
    return exp_of(((double)x - top) * inv_t);
}

// Sum over the lanes up to and with each.
__device__ __forceinline__ double prefix(double v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// A choice among 64 shares: the first lane whose prefix exceeds goal, else (rounding, or
// goal infinite) the last with a share; goal becomes what is left of it, at least 0.
// some share has to be positive.
__device__ __forceinline__ int choose(double share, double &goal)
{
    const double upto = prefix(share);
    const u64 positive = __ballot(share > 0.0);
    const u64 past = __ballot(upto > goal) & positive;
    const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(positive);
    const double before = at ? __shfl(upto, at - 1) : 0.0;
    goal = fmax(goal - before, 0.0);
    return at;
}

// The draws t0, t0 + step.. of a row by one wavefront each.
template <typename T>
__device__ __forceinline__ void draw_words(const T *__restrict__ x, int64_t V, const RowRules &r,
                                           double inv_t, int32_t chunks, const Part *part,
                                           const double *blocks, int32_t t0, int32_t step,
                                           int32_t draws, int64_t d0, const double *__restrict__ u,
                                           uint64_t seed, uint32_t philox_step, int64_t draw0,
                                           int32_t *__restrict__ word, float *__restrict__ logp)
{
    const int lane = threadIdx.x & 63;
    // the row's largest score and the sum of its weights
    double top = -__builtin_inf();
    bool law = true;
    for (int32_t c0 = 0; c0 < chunks; c0 += 64) {
        const double t = c0 + lane < chunks ? part[c0 + lane].top : -__builtin_inf();
        law = law && t == t;
        top = fmax(top, t);
    }
    for (int d = 32; d; d >>= 1) top = fmax(top, __shfl_xor(top, d));
    law = !__any(!law) && top > -__builtin_inf();
    auto share_of = [&](int32_t c) {
        if (c >= chunks) return 0.0;
        const Part p = part[c];
        return p.sum > 0.0 ? p.sum * exp_of((p.top - top) * inv_t) : 0.0;
    };
    double total = 0.0, share = 0.0;
    int32_t last = 0;  // the last 64 chunks that hold some weight
    if (law) {
        for (int32_t c0 = 0; c0 < chunks; c0 += 64) {
            share = share_of(c0 + lane);
            total += __shfl(prefix(share), 63);
            if (__any(share > 0.0)) last = c0;
        }
    }
    const double log_total = log(total);
    for (int32_t t = t0; t < draws; t += step) {
        const int64_t d = d0 + t;
        if (!law) {
            if (lane == 0) {
                word[d] = -1;
                logp[d] = __builtin_nanf("");
            }
            continue;
        }
        const double uniform =
            u ? u[d]
              : (double)philox_x0(seed, (uint64_t)(draw0 + d), philox_step, kPurposeWord) * 0x1p-32;
        // (NaN, and 1 or more: the last word with weight)
        double goal = uniform * total < total ? fmax(uniform * total, 0.0) : __builtin_inf();
        // 64 chunks at a time, the ones whose shares exceed what is left of the goal
        int32_t c0 = 0;
        if (chunks > 64) {
            for (; c0 < last; c0 += 64) {
                share = share_of(c0 + lane);
                const double sum = __shfl(prefix(share), 63);
                if (sum > goal) break;
                goal -= sum;
            }
            share = share_of(c0 + lane);
        }
        const int32_t c = c0 + choose(share, goal);
        const double own = part[c].top;
        goal = goal / exp_of((own - top) * inv_t);
        const int b = choose(blocks[(int64_t)c * kBlocks + lane], goal);
        // the block's words, two a lane
        const int64_t w = (int64_t)c * kDrawChunk + b * kBlockWords + 2 * lane;
        float s[2];
        int32_t n[2] = {0, 0};
        for (int64_t i = 0; i < r.n_words; i += 64) {
            const int64_t at =
                i + lane < r.n_words ? (int64_t)r.words[i + lane] - (w - 2 * lane) : -1;
            u64 hits = __ballot(at >= 0 && at < kBlockWords);
            while (hits) {
                const int from = __builtin_ctzll(hits);
                hits &= hits - 1;
                const int a = __shfl((int)at, from);
                n[0] += a == 2 * lane;
                n[1] += a == 2 * lane + 1;
            }
        }
        double y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = w + i < V ? ruled(r, (float)x[w + i], w + i, n[i]) : -__builtin_inff();
            y[i] = weight_of(s[i], own, inv_t);
        }
        const int l = choose(y[0] + y[1], goal);
        const bool second = !(y[0] > goal) && y[1] > 0.0;
        if (lane == l) {
            word[d] = (int32_t)(w + second);
            logp[d] = (float)(((double)(second ? s[1] : s[0]) - top) * inv_t - log_total);
        }
    }
}

// One workgroup per (row, chunk): its largest score and its sums.  Rows of one chunk are
// drawn from at once.
template <typename T>
__global__ void __launch_bounds__(kDrawThreads) k_draw_parts(
    const T *__restrict__ x, int64_t ld, int64_t V, int32_t chunks, spdp_rules rules, double inv_t,
    Part *__restrict__ part, double *__restrict__ blocks, int32_t draws,
    const double *__restrict__ u, uint64_t seed, uint32_t step, int64_t draw0,
    int32_t *__restrict__ word, float *__restrict__ logp)
{
    using C = Chunk<T, kDrawThreads, 16>;
    constexpr int kLanes = kBlockWords / C::N;  // lanes whose vectors make a block
    __shared__ typename C::Listed listed;
    __shared__ float wave_top[kDrawThreads / 64];
    __shared__ double sum_of[kBlocks];
    __shared__ Part own;
    const int64_t row = blockIdx.x / (uint32_t)chunks;
    const int32_t chunk = blockIdx.x % (uint32_t)chunks;
    const int64_t w0 = (int64_t)chunk * C::kWords;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    C c;
    c.request(x + row * ld, w0, V);
    const RowRules r = row_rules(rules, row);
    if (r.n_words > 0) C::count(r, w0, listed);
    float v[C::U][C::N];
    float top = -__builtin_inff();
    bool law = true;
#pragma unroll
    for (int k = 0; k < C::U; ++k) {
        c.scores(r, w0, V, listed, k, v[k]);
#pragma unroll
        for (int i = 0; i < C::N; ++i) {
            law = law && v[k][i] < __builtin_inff();
            top = fmaxf(top, v[k][i]);
        }
    }
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) wave_top[wave] = top;
    law = !__syncthreads_or(!law);
    for (int i = 0; i < kDrawThreads / 64; ++i) top = fmaxf(top, wave_top[i]);
    const bool some = top > -__builtin_inff() && top < __builtin_inff();
#pragma unroll
    for (int k = 0; k < C::U; ++k) {
        double s = 0.0;
        if (some) {
#pragma unroll
            for (int i = 0; i < C::N; ++i) s += weight_of(v[k][i], top, inv_t);
        }
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) s += __shfl_xor(s, d);
        const int b = C::at(k) / kBlockWords;
        if (lane % kLanes == 0) sum_of[b] = s;
    }
    __syncthreads();
    if (wave == 0) {
        const double s = sum_of[lane], sum = __shfl(prefix(s), 63);
        if (lane == 0) own = Part{law ? (double)top : __builtin_nan(""), sum};
        if (chunks > 1) {
            blocks[(int64_t)blockIdx.x * kBlocks + lane] = s;
            if (lane == 0) part[blockIdx.x] = Part{law ? (double)top : __builtin_nan(""), sum};
        }
    }
    if (chunks > 1) return;
    __syncthreads();
    draw_words(x + row * ld, V, r, inv_t, 1, &own, sum_of, wave, kDrawThreads / 64, draws,
               row * draws, u, seed, step, draw0, word, logp);
}

// `share` workgroups of four wavefronts per row.
template <typename T>
__global__ void __launch_bounds__(256) k_draw(const T *__restrict__ x, int64_t ld, int64_t V,
                                              int32_t chunks, spdp_rules rules, double inv_t,
                                              const Part *__restrict__ part,
                                              const double *__restrict__ blocks, int32_t share,
                                              int32_t draws, const double *__restrict__ u,
                                              uint64_t seed, uint32_t step, int64_t draw0,
                                              int32_t *__restrict__ word,
                                              float *__restrict__ logp)
{
    const int64_t row = blockIdx.x / (uint32_t)share;
    const int32_t t0 = (int32_t)(blockIdx.x % (uint32_t)share) * 4 + (threadIdx.x >> 6);
    if (t0 >= draws) return;
    const RowRules r = row_rules(rules, row);
    draw_words(x + row * ld, V, r, inv_t, chunks, part + row * chunks,
               blocks + row * chunks * kBlocks, t0, 4 * share, draws, row * draws, u, seed, step,
               draw0, word, logp);
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

int64_t chunks_of(int64_t V, int64_t words) { return (V + words - 1) / words; }

// Parts of a row for the best words: as many as chunks while the rows alone leave compute
// units idle, else chunks one after another in a workgroup (few scores of the later ones
// pass the bound), with about six workgroups for a compute unit.
constexpr int64_t kTopBlocks = 1536;

struct TopShape {
    int64_t parts, per;
};

TopShape top_shape(int64_t rows, int64_t V)
{
    const int64_t chunks = chunks_of(V, kTopThreads * 16);
    int64_t parts = rows > 0 ? (kTopBlocks + rows - 1) / rows : 1;
    parts = parts > chunks ? chunks : parts;
    const int64_t per = (chunks + parts - 1) / parts;
    return TopShape{(chunks + per - 1) / per, per};
}

int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

int64_t draw_parts_bytes(int64_t rows, int64_t chunks)
{
    return round256(rows * chunks * (int64_t)sizeof(Part));
}

}  // namespace

hipError_t launch_adjust(const void *x, int64_t ldx, void *y, int64_t ldy, int32_t type,
                         int64_t rows, int64_t V, const spdp_rules &rules, hipStream_t st)
{
    if (rows == 0 || V == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V, kAdjustThreads * 16);
    return by_type(type, rows * chunks, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_adjust<T>, grid, dim3(kAdjustThreads), 0, st, (const T *)x, ldx,
                           (T *)y, ldy, V, (int32_t)chunks, rules);
    });
}

int64_t words_work(int64_t rows, int64_t V, int32_t take)
{
    if (rows == 0) return 0;
    // (at least what top_shape's parts need, and no less for more rows)
    const int64_t most = rows * chunks_of(V, kTopThreads * 16);
    const int64_t parts = most < rows + kTopBlocks ? most : rows + kTopBlocks;
    const int64_t chunks = chunks_of(V, kDrawChunk);
    const int64_t top = parts * take * (int64_t)sizeof(u64);
    const int64_t draw = chunks > 1 ? draw_parts_bytes(rows, chunks) + rows * chunks * kBlocks * 8 : 0;
    return round256(top > draw ? top : draw > 0 ? draw : 1);
}

int64_t words_blocks(int64_t rows, int64_t V) { return rows * chunks_of(V, kTopThreads * 16); }

hipError_t launch_top(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t V,
                      const spdp_rules &rules, int32_t k, int32_t *word, float *value, void *work,
                      hipStream_t st)
{
    if (rows == 0 || k == 0) return hipSuccess;
    const TopShape s = top_shape(rows, V);
    u64 *best = static_cast<u64 *>(work);
    hipError_t e = by_type(type, rows * s.parts, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_top_part<T>, grid, dim3(kTopThreads), 0, st, (const T *)x, ld, V,
                           (int32_t)s.parts, (int32_t)s.per, rules, k, best, word, value);
    });
    if (e != hipSuccess || s.parts == 1) return e;
    hipLaunchKernelGGL(k_top_join, dim3((unsigned)rows), dim3(kTopThreads), 0, st, best,
                       s.parts * k, k, word, value);
    return hipGetLastError();
}

hipError_t launch_draw(const void *x, int64_t ld, int32_t type, int64_t rows, int64_t V,
                       const spdp_rules &rules, double temperature, int32_t draws,
                       const double *u, uint64_t seed, uint32_t step, int64_t draw0,
                       int32_t *word, float *logp, void *work, hipStream_t st)
{
    if (rows == 0 || draws == 0) return hipSuccess;
    const int64_t chunks = chunks_of(V, kDrawChunk);
    const double inv_t = 1.0 / temperature;
    Part *part = static_cast<Part *>(work);
    double *blocks = reinterpret_cast<double *>(static_cast<char *>(work) +
                                                draw_parts_bytes(rows, chunks));
    hipError_t e = by_type(type, rows * chunks, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_draw_parts<T>, grid, dim3(kDrawThreads), 0, st, (const T *)x, ld, V,
                           (int32_t)chunks, rules, inv_t, part, blocks, draws, u, seed, step, draw0,
                           word, logp);
    });
    if (e != hipSuccess || chunks == 1) return e;
    // a wavefront per draw while that leaves the chip's wavefronts enough, then several each
    int64_t share = (draws + 3) / 4;
    const int64_t most = (4096 + rows - 1) / rows;
    share = share > most ? most : share;
    return by_type(type, rows * share, [&](auto t, dim3 grid) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_draw<T>, grid, dim3(256), 0, st, (const T *)x, ld, V, (int32_t)chunks,
                           rules, inv_t, part, blocks, (int32_t)share, draws, u, seed, step, draw0,
                           word, logp);
    });
}

}  // namespace spdp
