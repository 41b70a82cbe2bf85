// words.hpp -- scores of words under rules: what the kernels that adjust scores,
// take the best words and draw words share.
//
// A row holds a document's scores x[w], one per word of the vocabulary.  The rules
// of the row make of them, every step rounded to fp32,
//   c   = times w is among the document's listed words
//   x1  = c > 0 ? (x > 0 ? x / repeat : x * repeat) : x
//   x2  = c > 0 ? x1 - (presence + frequency * c) : x1
//   x3  = x2 + bias[w]
//   out = allowed(w) ? x3 : -inf
// The steps are rounded one by one (no fused multiply-add), so that the kernels
// that store the result and those that choose from it see the same scores.
//
// A row is taken in chunks by workgroups, 16 bytes of scores a load.  Counts of a chunk's
// words are added up in LDS by walking the document's words (integer atomics, so their
// order does not matter); few words of a chunk are listed, and a bitmap says which.
#pragma once

#include "spdp_internal.hpp"

namespace spdp {

// 16 bytes of scores from any element's address (gfx950 reads and writes wide words
// at addresses that are aligned to their parts only).
template <typename T>
struct Vec {
    static constexpr int N = 16 / sizeof(T);
    T v[N];
};

// STREAM: past the caches' usual order, for scores that are more than the caches hold.
template <bool STREAM, typename T>
__device__ __forceinline__ Vec<T> load_vec(const T *p)
{
    typedef int unit __attribute__((ext_vector_type(4), aligned(2)));
    const unit *q = reinterpret_cast<const unit *>(p);
    unit u;
    if constexpr (STREAM) u = __builtin_nontemporal_load(q);
    else u = *q;
    Vec<T> k;
    __builtin_memcpy(&k, &u, sizeof k);
    return k;
}

template <bool STREAM, typename T>
__device__ __forceinline__ void store_vec(T *p, const Vec<T> &k)
{
    typedef int unit __attribute__((ext_vector_type(4), aligned(2)));
    unit u;
    __builtin_memcpy(&u, &k, sizeof k);
    if constexpr (STREAM) __builtin_nontemporal_store(u, reinterpret_cast<unit *>(p));
    else *reinterpret_cast<unit *>(p) = u;
}

// The rules of one row.
struct RowRules {
    const int32_t *words = nullptr;  // the document's words
    int64_t n_words = 0;             // how many (0: the penalties change nothing)
    float repeat = 1.f, presence = 0.f, frequency = 0.f;
    const float *bias = nullptr;     // [V] or null
    const uint32_t *mask = nullptr;  // [(V + 31) / 32] or null
    bool bad = false;                // an index past its table: the row comes out as NaN
};

__device__ __forceinline__ RowRules row_rules(const spdp_rules &r, int64_t row)
{
    // everything that is read of the row is requested before any of it is looked at
    int64_t a = 0, b = 0;
    float repeat = 1.f, presence = 0.f, frequency = 0.f;
    int32_t bias = 0, mask = 0;
    if (r.doc_off) {
        a = r.doc_off[row];
        b = r.doc_off[row + 1];
        repeat = r.penalties[3 * row];
        presence = r.penalties[3 * row + 1];
        frequency = r.penalties[3 * row + 2];
    }
    if (r.bias_of) bias = r.bias_of[row];
    if (r.mask_of) mask = r.mask_of[row];
    RowRules o;
    a = a < 0 ? 0 : a;
    b = b > r.n_listed ? r.n_listed : b;
    if (a < b) {
        o.words = r.words + a;
        o.n_words = b - a;
        o.repeat = repeat;
        o.presence = presence;
        o.frequency = frequency;
    }
    if (r.bias) {
        if (bias >= r.n_bias) o.bad = true;
        else if (bias >= 0) o.bias = r.bias + (int64_t)bias * r.n_words;
    }
    if (r.mask) {
        if (mask >= r.n_masks) o.bad = true;
        else if (mask >= 0) o.mask = r.mask + (int64_t)mask * (((int64_t)r.n_words + 31) / 32);
    }
    return o;
}

// Score x of a word that is listed c > 0 times.
__device__ __forceinline__ float penalised(const RowRules &r, float x, int32_t c)
{
#pragma clang fp contract(off)
    const float y = x > 0.f ? x / r.repeat : x * r.repeat;
    const float fc = r.frequency * (float)c;
    const float amount = r.presence + fc;
    return y - amount;
}

// Score x of word w with count c under the rules.
__device__ __forceinline__ float ruled(const RowRules &r, float x, int64_t w, int32_t c)
{
    if (r.bad) return __builtin_nanf("");
    if (c > 0) x = penalised(r, x, c);
    if (r.bias) x = x + r.bias[w];
    if (r.mask && !((r.mask[w >> 5] >> (w & 31)) & 1u)) x = -__builtin_inff();
    return x;
}

// The chunk of a row that a workgroup of THREADS threads holds, PER scores a thread in
// vectors of 16 bytes: vector u of a thread is at (u THREADS + thread) N of the chunk.
template <typename T, int THREADS, int PER, bool STREAM = false>
struct Chunk {
    static constexpr int kWords = THREADS * PER, N = Vec<T>::N, U = PER / N;
    struct alignas(16) Listed {  // LDS
        uint32_t seen[kWords / 32];
        int32_t count[kWords];
    };
    Vec<T> raw[U];

    static __device__ __forceinline__ int at(int u) { return (u * THREADS + (int)threadIdx.x) * N; }

    // Request the scores of words w0 ..; past the row's end none is read.
    __device__ __forceinline__ void request(const T *row, int64_t w0, int64_t V)
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t w = w0 + at(u);
            if (w + N <= V) {
                raw[u] = load_vec<STREAM>(row + w);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) raw[u].v[i] = w + i < V ? row[w + i] : (T)0;
            }
        }
    }

    // Counts of the chunk's words among the row's listed words.  All threads of the
    // workgroup call it (with the same row); the counts can be read when it returns, and
    // a barrier has to come before it is called again.
    static __device__ __forceinline__ void count(const RowRules &r, int64_t w0, Listed &l)
    {
        // (a thread's first word is on its way while the counts are cleared)
        int32_t word = (int64_t)threadIdx.x < r.n_words ? r.words[threadIdx.x] : -1;
        typedef int quad __attribute__((ext_vector_type(4)));
        quad *clear = reinterpret_cast<quad *>(&l);
        constexpr int kQuads = (int)(sizeof(Listed) / sizeof(quad));
#pragma unroll
        for (int i = 0; i < (kQuads + THREADS - 1) / THREADS; ++i)
            if (i * THREADS + (int)threadIdx.x < kQuads) clear[i * THREADS + threadIdx.x] = quad{0, 0, 0, 0};
        __syncthreads();
        for (int64_t i = threadIdx.x;;) {
            const int64_t a = (int64_t)word - w0;
            if (word >= 0 && a >= 0 && a < kWords) {
                atomicAdd(&l.count[a], 1);
                atomicOr(&l.seen[a >> 5], 1u << (a & 31));
            }
            i += THREADS;
            if (i >= r.n_words) break;
            word = r.words[i];
        }
        __syncthreads();
    }

    // What the row's bias and mask hold for a vector of scores.
    struct Held {
        float bias[N];
        uint32_t allowed;
    };

    // Request them for vector u, to be under way while the listed words are counted.
    static __device__ __forceinline__ void hold(const RowRules &r, int64_t w0, int64_t V, int u,
                                                Held &h)
    {
        const int64_t w = w0 + at(u);
        if (w + N > V) return;  // (the scores at a row's end look up their own)
        if (r.bias) {
            typedef float quad __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const quad b = *reinterpret_cast<const quad *>(r.bias + w + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) h.bias[i + k] = b[k];
            }
        }
        // (w is a multiple of N, so its bits lie in one byte)
        if (r.mask) h.allowed = reinterpret_cast<const uint8_t *>(r.mask)[w >> 3];
    }

    // The scores of vector u under the rules; -inf past the row's end.  Without `held` (for
    // kernels that have no registers to hold them) bias and mask are read here.
    __device__ __forceinline__ void scores(const RowRules &r, int64_t w0, int64_t V,
                                           const Listed &l, int u, float (&x)[N],
                                           const Held *held = nullptr) const
    {
        const int a = at(u);
        const int64_t w = w0 + a;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)raw[u].v[i];
        if (w + N > V) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool seen = r.n_words > 0 && (l.seen[a >> 5] >> ((a & 31) + i) & 1u);
                x[i] = w + i < V ? ruled(r, x[i], w + i, seen ? l.count[a + i] : 0)
                                 : -__builtin_inff();
            }
            return;
        }
        if (r.n_words > 0) {
            const uint32_t seen = l.seen[a >> 5] >> (a & 31);
            if (seen & ((1u << N) - 1)) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (seen >> i & 1u) x[i] = penalised(r, x[i], l.count[a + i]);
            }
        }
        Held own;
        if (!held) hold(r, w0, V, u, own);
        const Held &h = held ? *held : own;
        if (r.bias) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = x[i] + h.bias[i];
        }
        if (r.mask) {
            const uint32_t ok = h.allowed >> (w & 7);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = ok >> i & 1u ? x[i] : -__builtin_inff();
        }
        if (r.bad) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = __builtin_nanf("");
        }
    }
};

}  // namespace spdp
