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
// A row is taken in chunks of kChunk words by workgroups of kThreads threads.
// The counts c of a chunk's words are made in LDS: the workgroup walks the
// document's words and counts those that fall into the chunk (integer atomics,
// so the order does not matter).
#pragma once

#include "spdp_internal.hpp"

namespace spdp {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;

template <typename T, int N>
struct alignas(sizeof(T)) Pack {
    T v[N];
};

// N consecutive values from any element's address (gfx950 reads and writes wide
// words at addresses that are aligned to their parts only).
template <typename T, int N>
__device__ __forceinline__ void load_n(const T *p, float (&out)[N])
{
    Pack<T, N> k;
    __builtin_memcpy(&k, p, sizeof k);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = (float)k.v[i];
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
    RowRules o;
    if (r.doc_off && r.penalties) {
        int64_t a = r.doc_off[row], b = r.doc_off[row + 1];
        a = a < 0 ? 0 : a;
        b = b > r.n_listed ? r.n_listed : b;
        if (a < b) {
            o.words = r.words + a;
            o.n_words = b - a;
            o.repeat = r.penalties[3 * row];
            o.presence = r.penalties[3 * row + 1];
            o.frequency = r.penalties[3 * row + 2];
        }
    }
    if (r.bias) {
        const int32_t k = r.bias_of ? r.bias_of[row] : 0;
        if (k >= r.n_bias) o.bad = true;
        else if (k >= 0) o.bias = r.bias + (int64_t)k * r.n_words;
    }
    if (r.mask) {
        const int32_t k = r.mask_of ? r.mask_of[row] : 0;
        if (k >= r.n_masks) o.bad = true;
        else if (k >= 0) o.mask = r.mask + (int64_t)k * (((int64_t)r.n_words + 31) / 32);
    }
    return o;
}

// Counts of the words [w0, w0 + kChunk) among the row's listed words.  All threads
// of the workgroup call it; the counts can be read when it returns.
__device__ __forceinline__ void chunk_counts(const RowRules &r, int64_t w0, int32_t *count)
{
    for (int i = threadIdx.x; i < kChunk; i += kThreads) count[i] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < r.n_words; i += kThreads) {
        const int64_t at = (int64_t)r.words[i] - w0;
        if (at >= 0 && at < kChunk) atomicAdd(&count[at], 1);
    }
    __syncthreads();
}

// Score x of word w with count c under the rules.
__device__ __forceinline__ float ruled(const RowRules &r, float x, int64_t w, int32_t c)
{
#pragma clang fp contract(off)
    if (r.bad) return __builtin_nanf("");
    if (c > 0) {
        const float y = x > 0.f ? x / r.repeat : x * r.repeat;
        const float fc = r.frequency * (float)c;
        const float amount = r.presence + fc;
        x = y - amount;
    }
    if (r.bias) x = x + r.bias[w];
    if (r.mask && !((r.mask[w >> 5] >> (w & 31)) & 1u)) x = -__builtin_inff();
    return x;
}

}  // namespace spdp
