// rows8.hip -- rows in 8-bit floating point with a scale for each block of 128
// columns, and products of such rows on the matrix cores (gfx950).
//
// A document's word probabilities are p(w | d) = sum_k theta[d][k] phi[w][k]:
// over all words of the vocabulary a product of the estimates' rows.  Both are
// stored topics contiguous, so both operands run along the sum, as the matrix
// cores read them.  In 8 bits (e4m3: 4 bits of exponent, 3 of fraction, largest
// 448, no infinities) phi of the largest workload takes 51 MB a group instead of
// the estimates' 400 MB.  A block of 128 columns of a row has a scale of its own,
// a power of two, so that multiplying by it rounds nothing.
//
// The products run on the bf16 matrix instructions, on values that are converted, and
// scaled in the same instruction, without rounding.  The instructions on 8-bit operands
// (with or without scales) would take the rows as they are at up to twice the rate,
// but they cut products that are small beside the largest one: sums over 512 columns
// with the values' whole range of exponents were off by up to 1e-4 of the sum, all to
// the same side, where the bf16 instructions stay within 5e-7.
#include "spdp_internal.hpp"

namespace spdp {
namespace {

constexpr int kBlock = kBlock8;  // columns that share a scale

typedef unsigned long long u64;

// Exponent that |x| alone would ask of its block's scale, before it is cut to [-127, 127]:
// the least e with |x| <= 448 2^e.  |x| = f 2^p with f in [1/2, 1), and 448 = 7/8 2^9, so
// e = p - 9, and one more where f > 7/8: where adding all but the last of the
// fraction's upper quarter carries into the exponent.  What is not finite asks for none.
__device__ __forceinline__ int scale_exponent(double x)
{
    const u64 bits = __builtin_bit_cast(u64, x) & ~(1ull << 63);
    const int e = (int)((bits + 0x3FFFFFFFFFFFFull) >> 52) - 1031;
    return bits < 0x7FF0000000000000ull ? e : -2000;
}

// x 2^-e as fp32 for the 8-bit conversion, which rounds fp32 to nearest even: cut to fp32
// with the last bit set where anything was cut off (rounding to odd), so that the two
// steps round as one.  What the conversion takes to 0 may be 0 here; what is not finite or
// beyond 448 becomes NaN.
__device__ __forceinline__ float scaled_odd(double x, int e)
{
    const u64 bits = __builtin_bit_cast(u64, x);
    const uint32_t high = (uint32_t)(bits >> 32), low = (uint32_t)bits;
    // of the scaled value, 1023 for 1; at most what fp32 has for infinities and NaN, where those
    // of fp64 come out too
    const int exponent = min((int)(high >> 20 & 0x7FF) - e, 1151);
    uint32_t f = (uint32_t)((bits & 0xFFFFFFFFFFFFFull) >> 29) | ((low & 0x1FFFFFFF) ? 1u : 0u);
    f |= (uint32_t)(exponent - 896) << 23;
    f = exponent < 1000 ? 0u : f;  // (below 2^-23)
    f = f <= 0x43E00000u ? f : 0x7FC00000u;
    return __uint_as_float(f | (high & 0x80000000u));
}

// The largest of 32 lanes' values, in each of them.
__device__ __forceinline__ int max32(int v)
{
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false));   // lane ^ 1
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false));   // lane ^ 2
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, false));  // other 4 of 8
    v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x140, 0xF, 0xF, false));  // other 8 of 16
    return max(v, __shfl_xor(v, 16));
}

// Half a wavefront per (row, block), four columns a lane, UNITS blocks whose columns are all
// requested first; whole numbers throughout, as the scale is an exponent and the rounding
// bits.  Bound by the read: 100 000 rows of 500 doubles (400 MB, 52 written) take 78 us (5.8
// TB/s), of floats 55 us in twos (4.6 TB/s).
template <typename T, int UNITS>
__global__ void __launch_bounds__(256) k_pack8(const T *__restrict__ x, uint32_t units,
                                               int32_t cols, int64_t ld, int32_t nb,
                                               uint8_t *__restrict__ q, uint8_t *__restrict__ e)
{
    typedef T quad __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t first = (blockIdx.x * 8 + (threadIdx.x >> 5)) * UNITS;
    const int lane = threadIdx.x & 31;
    double v[UNITS][4];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const uint32_t unit = first + i < units ? first + i : units - 1;
        const uint32_t row = unit / (uint32_t)nb;
        const int32_t c = (int32_t)(unit - row * (uint32_t)nb) * kBlock + 4 * lane;
        const T *src = x + row * ld + c;
        if (c + 4 <= cols) {
            const quad a = *reinterpret_cast<const quad *>(src);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = a[k];
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = c + k < cols ? (double)src[k] : 0.0;
        }
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        int ex = -127;
#pragma unroll
        for (int k = 0; k < 4; ++k) ex = max(ex, scale_exponent(v[i][k]));
        ex = min(max32(ex), 127);
        int word = 0;
        word = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_odd(v[i][0], ex), scaled_odd(v[i][1], ex),
                                               word, false);
        word = __builtin_amdgcn_cvt_pk_fp8_f32(scaled_odd(v[i][2], ex), scaled_odd(v[i][3], ex),
                                               word, true);
        if (first + i < units) {
            *reinterpret_cast<int *>(q + (int64_t)(first + i) * kBlock + 4 * lane) = word;
            if (lane == 0) e[first + i] = (uint8_t)(ex + 127);
        }
    }
}

typedef __bf16 b2v __attribute__((ext_vector_type(2)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef int i4v __attribute__((ext_vector_type(4)));

// 8 packed values times their block's scale as bf16.  This rounds nothing for scales of
// 2^-124 to 2^119: a value has 4 significant bits, and bf16 has the exponents of fp32.
__device__ __forceinline__ b8v unpack8(uint32_t lo, uint32_t hi, float scale)
{
    const b2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const b2v b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const b2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const b2v d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return b8v{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 2^(e - 127)
__device__ __forceinline__ float scale_of(uint32_t e)
{
    return __uint_as_float(e ? e << 23 : 1u << 22);
}

template <typename T>
__device__ __forceinline__ T out_as(float v);
template <>
__device__ __forceinline__ float out_as<float>(float v) { return v; }
template <>
__device__ __forceinline__ _Float16 out_as<_Float16>(float v)
{
    // (the value is rounded to fp32 first: a multiplication and the conversion in one instruction
    // would round once, here and there, and the kernels' results would differ)
    asm("" : "+v"(v));
    return (_Float16)v;
}
template <>
__device__ __forceinline__ __bf16 out_as<__bf16>(float v) { return (__bf16)v; }

// Natural logarithms of N sums: the hardware's base-2 logarithm (1 ulp, normal
// arguments only) times log 2.  Sums below the normal range, zeros and negative ones
// among them, are rare enough to be looked for in all of a wavefront's sums at once.
template <int N>
__device__ __forceinline__ void log_of(float (&v)[N])
{
    constexpr float kLog2 = 0.693147180559945f;
    float least = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) least = fminf(least, v[i]);
    if (__any(least < 0x1p-126f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool tiny = v[i] < 0x1p-126f;
            const float l = __builtin_amdgcn_logf(tiny ? v[i] * 0x1p+32f : v[i]);
            v[i] = (tiny ? l - 32.f : l) * kLog2;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_logf(v[i]) * kLog2;
    }
}

// N values at c, whose address is aligned to one value.
template <typename T, int N>
__device__ __forceinline__ void store_n(T *c, const T (&v)[N])
{
    __builtin_memcpy(c, v, sizeof v);
}

// 16 bytes at p, whose address is aligned to 2; STREAM: past the caches' usual order.
template <bool STREAM, typename T>
__device__ __forceinline__ void store_unit(T *p, i4v v)
{
    typedef int unit __attribute__((ext_vector_type(4), aligned(2)));
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<unit *>(p));
    else *reinterpret_cast<unit *>(p) = v;
}

// c[i][j] = sum_k a[i][k] b[j][k], or its logarithm, for documents a and words b.
//
// A workgroup keeps 16 FD documents in LDS, converted to bf16 once and laid out as
// the matrix instructions read them (every read is 64 lanes x 16 bytes in a row).
// Its eight wavefronts then go over the words on their own, without a barrier, 64
// words at a time: words come from memory in 8 bits straight into the registers of
// the one wavefront that uses them, a block of 128 columns ahead of the products,
// and are converted there.  So one wavefront's stores and logarithms run under
// another's products, LDS is read once per FW products, and a word is converted once
// per 16 FD documents.
//
// Instruction j (of 4) of a block sums the columns 32 p + 8 j .. + 7, p = 0 .. 3
// (p = lane / 16): a lane's 32 bytes of a row lie together.  The order of a sum does not
// depend on FW and FD, nor an output on how many rows are multiplied at a time.
//
// Words are the matrix instruction's rows, so that a lane ends with words that lie
// next to each other in c; the words of a wavefront are dealt to its fragments so that
// they make stores of kPer values, 16 bytes where FW allows.
//
// Columns past kLdsBlocks / FD blocks do not fit the LDS at once: then documents are
// staged again, part by part, for every round of words.
//
// 2 000 x 100 000 x 500 (512 padded) to logarithms in bf16: 180 us, 1 140 TFLOP/s of the
// padded products; 137 us without stores and logarithms, where a large product of the library
// takes 140 at its best rate (1 430 TFLOP/s at 8 192 cubed, and 404 us for these sizes).  The
// stores, 400 MB, and the logarithms run under other wavefronts' products only in part.
constexpr int kWordFragments = 4;
constexpr int kLdsBlocks = 32;  // (blocks of columns) x (document fragments) in 128 KB

template <typename T, bool LOG, int FD, bool STREAM>
__global__ void __launch_bounds__(512, 2) k_product8(
    const uint8_t *__restrict__ aq, const uint8_t *__restrict__ ae, int32_t m,
    const uint8_t *__restrict__ bq, const uint8_t *__restrict__ be, int32_t n, int32_t nb,
    T *__restrict__ c, int64_t ld, int32_t tiles_d, int32_t ranges, int32_t rounds)
{
    constexpr int FW = kWordFragments;
    constexpr int kPer = 16 / sizeof(T);      // values of a store
    constexpr int kJoin = kPer / 4;           // fragments of a store
    constexpr int kMost = kLdsBlocks / FD;    // blocks in LDS at a time
    extern __shared__ uint4 docs[];           // [block][j][document fragment][lane]
    // Workgroups go to the 8 XCDs in turn; each XCD takes consecutive ones of the order
    // (range, documents), so that its workgroups read the same words at a time.
    const int32_t total = tiles_d * ranges, per = (total + 7) / 8;
    const int32_t order = (int32_t)(blockIdx.x & 7) * per + (int32_t)(blockIdx.x >> 3);
    if ((int32_t)(blockIdx.x >> 3) >= per || order >= total) return;
    const int32_t d0 = order % tiles_d * (16 * FD), range = order / tiles_d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, part = lane >> 4;
    const int64_t pitch = (int64_t)nb * kBlock;

    auto stage = [&](int32_t b0, int32_t blocks) {
        for (int u = wave; u < blocks * FD; u += 8) {
            const int b = u / FD, y = u % FD;
            // (documents past the end repeat the last one; nothing of them is stored)
            const int32_t d = d0 + y * 16 + r < m ? d0 + y * 16 + r : m - 1;
            const uint4 *q = reinterpret_cast<const uint4 *>(aq + d * pitch +
                                                             (int64_t)(b0 + b) * kBlock + part * 32);
            const uint4 lo = q[0], hi = q[1];
            const float f = scale_of(ae[(int64_t)d * nb + b0 + b]);
            b8v *to = reinterpret_cast<b8v *>(docs) + (b * 4 * FD + y) * 64 + lane;
            to[0] = unpack8(lo.x, lo.y, f);
            to[FD * 64] = unpack8(lo.z, lo.w, f);
            to[2 * FD * 64] = unpack8(hi.x, hi.y, f);
            to[3 * FD * 64] = unpack8(hi.z, hi.w, f);
        }
    };
    const bool fits = nb <= kMost;

    // This wavefront's words of a round: fragment x, row r.  The last tile is moved back
    // to be a whole one (its first words are then made twice, the same).
    uint32_t off[FW], eoff[FW];
#pragma unroll
    for (int x = 0; x < FW; ++x) {
        const uint32_t row = x / kJoin * (16 * kJoin) + (r >> 2) * kPer + x % kJoin * 4 + (r & 3);
        off[x] = row * (uint32_t)pitch + part * 32;
        eoff[x] = row * (uint32_t)nb;
    }
    auto first_word = [&](int32_t tile) {
        const int32_t w0 = tile * (16 * FW);
        return w0 > n - 16 * FW ? n - 16 * FW : w0;
    };
    uint4 q[FW][2];
    uint32_t scale[FW];
    // (half a block of the next block's columns is requested as soon as the present
    // block's half is converted)
    auto request = [&](int32_t w0, int32_t b, int half) {
        const uint8_t *wq = bq + w0 * pitch + (int64_t)b * kBlock + 16 * half;
        const uint8_t *we = be + w0 * (int64_t)nb + b;
#pragma unroll
        for (int x = 0; x < FW; ++x) {
            q[x][half] = *reinterpret_cast<const uint4 *>(wq + off[x]);
            if (half) scale[x] = we[eoff[x]];
        }
    };
    b8v fw[FW], fd[2];
    float f[FW];
    auto convert = [&](int j) {
#pragma unroll
        for (int x = 0; x < FW; ++x) {
            const uint4 v = q[x][j >> 1];
            fw[x] = j & 1 ? unpack8(v.z, v.w, f[x]) : unpack8(v.x, v.y, f[x]);
        }
    };
    const b8v *held = reinterpret_cast<const b8v *>(docs) + lane;
    const int32_t tiles_w = (n + 16 * FW - 1) / (16 * FW), stride = ranges * 8;
    int32_t tile = range * 8 + wave;
    int32_t w0 = first_word(tile < tiles_w ? tile : 0);
    if (fits) {
        stage(0, nb);
        __syncthreads();
    }
    request(w0, 0, 0);
    request(w0, 0, 1);
    fd[0] = held[0];
    fd[1] = held[64];
    for (int32_t round = 0; round < rounds; ++round, tile += stride) {
        if (fits && tile >= tiles_w) return;
        const bool here = tile < tiles_w;
        // (past the last tile, the present one is requested again)
        const int32_t then_w0 = first_word(tile + stride < tiles_w ? tile + stride : here ? tile : 0);
        f4v acc[FW][FD];
#pragma unroll
        for (int x = 0; x < FW; ++x)
#pragma unroll
            for (int y = 0; y < FD; ++y) acc[x][y] = f4v{0.f, 0.f, 0.f, 0.f};
        for (int32_t b0 = 0; b0 < nb; b0 += kMost) {
            const int32_t b1 = b0 + kMost < nb ? b0 + kMost : nb;
            if (!fits) {
                __syncthreads();
                stage(b0, b1 - b0);
                __syncthreads();
                if (!here) continue;
                fd[0] = held[0];
                fd[1] = held[64];
            }
            for (int32_t b = b0; b < b1; ++b) {
                const b8v *now = held + (b - b0) * 4 * FD * 64;
                const b8v *then = b + 1 < b1 ? now + 4 * FD * 64 : held;
                const int32_t next_b = b + 1 < nb ? b + 1 : 0, next_w0 = b + 1 < nb ? w0 : then_w0;
#pragma unroll
                for (int x = 0; x < FW; ++x) f[x] = scale_of(scale[x]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    convert(j);
                    if (j & 1) request(next_w0, next_b, j >> 1);
#pragma unroll
                    for (int y = 0; y < FD; ++y) {
                        const int i = j * FD + y;
                        const b8v d = fd[i & 1];
                        fd[i & 1] = i + 2 < 4 * FD ? now[(i + 2) * 64] : then[(i + 2 - 4 * FD) * 64];
#pragma unroll
                        for (int x = 0; x < FW; ++x)
                            acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[x], d, acc[x][y],
                                                                                0, 0, 0);
                        if constexpr (FD >= 4) {  // one LDS read ahead of every FW products
                            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                            __builtin_amdgcn_sched_group_barrier(0x008, FW, 0);
                        }
                    }
                }
            }
        }
        if (!here) continue;
        // Value v of a lane: word row 4 part + v of the fragment, document column r.  A unit
        // of kPer words of a document is a 16-byte store; four lanes have a document's
        // unit u side by side.  Lanes r and r ^ 8 trade units u and u + 1, so that a store
        // instruction writes 128 bytes of 8 documents and not 64 of 16.
#pragma unroll
        for (int y = 0; y < FD; ++y) {
            float v[4 * FW];
#pragma unroll
            for (int i = 0; i < 4 * FW; ++i) v[i] = acc[i / 4][y][i % 4];
            if constexpr (LOG) log_of(v);
            const bool hi = r & 8;
            const int32_t d = d0 + y * 16 + (r & 7);
            T *to = c + d * ld + w0 + (hi ? 16 * kJoin : 0) + part * kPer;
#pragma unroll
            for (int u = 0; u < FW / kJoin; u += 2) {
                i4v one[2];  // units u and u + 1 of document r
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    T out[kPer];
#pragma unroll
                    for (int i = 0; i < kPer; ++i) out[i] = out_as<T>(v[(u + e) * kPer + i]);
                    __builtin_memcpy(&one[e], out, sizeof out);
                }
                i4v low, high;  // unit u (hi: u + 1) of documents r & 7 and (r & 7) + 8
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int got = __builtin_amdgcn_mov_dpp(hi ? one[0][i] : one[1][i],
                                                             0x128, 0xF, 0xF, true);  // ror 8
                    low[i] = hi ? got : one[0][i];
                    high[i] = hi ? one[1][i] : got;
                }
                if (d < m) store_unit<STREAM>(to + u * 16 * kJoin, low);
                if (d + 8 < m) store_unit<STREAM>(to + 8 * ld + u * 16 * kJoin, high);
            }
        }
        w0 = then_w0;
    }
}

// The same for few documents, or few words: a wavefront makes 16 x 16 outputs.  Here the
// words' bytes are all there is to wait for, so four blocks of them are requested at
// once, by as many wavefronts as the chip holds, before the documents' blocks are
// converted into LDS for the workgroup's four wavefronts.  (Documents read from the
// caches by every wavefront instead: 17.3 us for 16 x 100 000 x 500, 13.2 so, 4.4 TB/s of the
// 58 MB read and written.)
template <typename T, bool LOG>
__global__ void __launch_bounds__(256) k_product8_few(
    const uint8_t *__restrict__ aq, const uint8_t *__restrict__ ae, int32_t m,
    const uint8_t *__restrict__ bq, const uint8_t *__restrict__ be, int32_t n, int32_t nb,
    T *__restrict__ c, int64_t ld, int32_t tiles_d)
{
    constexpr int kAhead = 4;
    __shared__ b8v docs[kAhead][4][64];  // [block][j][lane]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, part = lane >> 4;
    const int64_t d0 = (int64_t)(blockIdx.x % tiles_d) * 16;
    const int64_t w0 = ((int64_t)(blockIdx.x / tiles_d) * 4 + wave) * 16;
    const int64_t pitch = (int64_t)nb * kBlock;
    // (rows past the end repeat the last one; nothing of them is stored)
    const int64_t d = d0 + r < m ? d0 + r : m - 1, w = w0 + r < n ? w0 + r : n - 1;
    const uint4 *qd = reinterpret_cast<const uint4 *>(aq + d * pitch + part * 32);
    const uint4 *qw = reinterpret_cast<const uint4 *>(bq + w * pitch + part * 32);
    const uint8_t *ed = ae + d * nb, *ew = be + w * nb;
    f4v acc = {0.f, 0.f, 0.f, 0.f};
    for (int32_t b = 0; b < nb; b += kAhead) {
        uint4 x[kAhead][2];
        uint32_t scale[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int32_t at = b + i < nb ? b + i : nb - 1;
            x[i][0] = qw[at * 8];
            x[i][1] = qw[at * 8 + 1];
            scale[i] = ew[at];
        }
        if (b) __syncthreads();
        if (b + wave < nb) {
            const uint4 lo = qd[(b + wave) * 8], hi = qd[(b + wave) * 8 + 1];
            const float f = scale_of(ed[b + wave]);
            docs[wave][0][lane] = unpack8(lo.x, lo.y, f);
            docs[wave][1][lane] = unpack8(lo.z, lo.w, f);
            docs[wave][2][lane] = unpack8(hi.x, hi.y, f);
            docs[wave][3][lane] = unpack8(hi.z, hi.w, f);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (b + i >= nb) break;
            const float f = scale_of(scale[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 v = x[i][j >> 1];
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    j & 1 ? unpack8(v.z, v.w, f) : unpack8(v.x, v.y, f), docs[i][j][lane], acc, 0,
                    0, 0);
            }
        }
    }
    float v[4] = {acc[0], acc[1], acc[2], acc[3]};
    if constexpr (LOG) log_of(v);
    if (d0 + r >= m || w0 >= n) return;
    T out[4], *to = c + (d0 + r) * ld + w0 + part * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = out_as<T>(v[i]);
    if (w0 + 16 <= n) {
        store_n(to, out);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (w0 + part * 4 + i < n) to[i] = out[i];
    }
}

// How a product is shared out: document tiles, workgroups that share a document
// tile's words, the rounds of words that each of their wavefronts takes, and what that
// costs.  A compute unit takes `turns` workgroups one after another; a round takes as long
// as its products or 3 more document fragments' (its words' conversion and stores), a
// workgroup's start as long as 2 of them.  (What it costs to stage documents part by part, past
// kLdsBlocks / fd blocks of columns, is not counted.)
struct Shares {
    int64_t tiles_d, ranges, rounds, cost;
};

Shares shares_of(int64_t m, int64_t n, int32_t fd, int64_t turns)
{
    const int64_t tw = (n + 16 * kWordFragments - 1) / (16 * kWordFragments), most = (tw + 7) / 8;
    Shares s;
    s.tiles_d = (m + 16 * fd - 1) / (16 * fd);
    s.ranges = 256 * turns / s.tiles_d;
    if (s.ranges > most) s.ranges = most;
    if (s.ranges < 1) s.ranges = 1;
    s.rounds = (tw + 8 * s.ranges - 1) / (8 * s.ranges);
    s.cost = (s.tiles_d * s.ranges + 255) / 256 * (s.rounds * (fd + 3) + 2);
    return s;
}

// Scores above kStreamBytes are written past the caches' usual order: they would push out
// the words, which every tile of documents reads again (2 000 x 100 000 of 500 topics: in bf16,
// 400 MB, 180 us streamed, 230 not; in fp32 218 and 270; 1 000 x 100 000 of 64 topics in fp16,
// 200 MB, 57 streamed, 70 not).  Less than that stays in the last level cache for whoever reads
// it next, and takes less time too (777 x 14 724 of 64 topics in fp16, 23 MB: 12.9 us streamed,
// 11.0 not).  Rows have to start at multiples of 64 bytes: lines that are written in parts are
// not put together past the caches (2 000 x 99 999 of 500 topics in bf16: 388 us streamed, 274
// not; 2 000 x 100 016, rows at multiples of 32 bytes: 257 streamed, 233 not; of 700 topics,
// where more work hides the stores, 301 streamed, 340 not).
template <typename T, bool LOG, int FD, bool STREAM>
hipError_t product(const spdp_rows8 &a, const spdp_rows8 &b, void *c, int64_t ld, const Shares &s,
                   hipStream_t st)
{
    const int32_t nb = blocks8(a.cols), held = nb < kLdsBlocks / FD ? nb : kLdsBlocks / FD;
    const int64_t per = (s.tiles_d * s.ranges + 7) / 8;
    hipLaunchKernelGGL((k_product8<T, LOG, FD, STREAM>), dim3((unsigned)(per * 8)), dim3(512),
                       held * FD * 4096, st, a.q, a.e, (int32_t)a.rows, b.q, b.e, (int32_t)b.rows,
                       nb, (T *)c, ld, (int32_t)s.tiles_d, (int32_t)s.ranges, (int32_t)s.rounds);
    return hipGetLastError();
}

template <typename T, bool LOG, int FD>
hipError_t product(const spdp_rows8 &a, const spdp_rows8 &b, void *c, int64_t ld, const Shares &s,
                   hipStream_t st)
{
    const bool lines = ((uintptr_t)c | (uintptr_t)(ld * (int64_t)sizeof(T))) % 64 == 0;
    return lines && a.rows * b.rows * (int64_t)sizeof(T) > kStreamBytes
               ? product<T, LOG, FD, true>(a, b, c, ld, s, st)
               : product<T, LOG, FD, false>(a, b, c, ld, s, st);
}

// Document fragments of a workgroup and turns: those that cost least.
template <typename T, bool LOG>
hipError_t product(const spdp_rows8 &a, const spdp_rows8 &b, void *c, int64_t ld, hipStream_t st)
{
    if (a.rows <= 16 || b.rows < 16 * kWordFragments) {
        const int64_t td = (a.rows + 15) / 16, blocks = td * ((b.rows + 63) / 64);
        hipLaunchKernelGGL((k_product8_few<T, LOG>), dim3((unsigned)blocks), dim3(256), 0, st, a.q,
                           a.e, (int32_t)a.rows, b.q, b.e, (int32_t)b.rows, blocks8(a.cols), (T *)c,
                           ld, (int32_t)td);
        return hipGetLastError();
    }
    int32_t best = 0;
    Shares s{};
    for (int32_t fd : {2, 4, 6, 8})
        for (int64_t turns = 1; turns <= 8; ++turns) {
            const Shares o = shares_of(a.rows, b.rows, fd, turns);
            if (!best || o.cost < s.cost) {
                s = o;
                best = fd;
            }
        }
    switch (best) {
        case 2: return product<T, LOG, 2>(a, b, c, ld, s, st);
        case 4: return product<T, LOG, 4>(a, b, c, ld, s, st);
        case 6: return product<T, LOG, 6>(a, b, c, ld, s, st);
        default: return product<T, LOG, 8>(a, b, c, ld, s, st);
    }
}

template <typename T>
hipError_t product(const spdp_rows8 &a, const spdp_rows8 &b, bool log, void *c, int64_t ld,
                   hipStream_t st)
{
    return log ? product<T, true>(a, b, c, ld, st) : product<T, false>(a, b, c, ld, st);
}

}  // namespace

hipError_t launch_pack8(const void *x, int32_t type, int64_t rows, int32_t cols, int64_t ld,
                        uint8_t *q, uint8_t *e, hipStream_t st)
{
    const int32_t nb = blocks8(cols);
    if (rows == 0 || nb == 0) return hipSuccess;
    // rows of a launch: nb is at most 2^17, and units stay below 8 kLaunchBlocks < 2^26
    const int64_t step = kLaunchBlocks / nb * 8;
    for (int64_t row = 0; row < rows; row += step) {
        const uint32_t units = (uint32_t)((rows - row < step ? rows - row : step) * nb);
        const auto blocks = [&](uint32_t per) {
            return dim3((units + 8 * per - 1) / (8 * per));
        };
        uint8_t *to = q + row * nb * kBlock, *scales = e + row * nb;
        if (type == SPDP_F64)
            hipLaunchKernelGGL((k_pack8<double, 1>), blocks(1), dim3(256), 0, st,
                               (const double *)x + row * ld, units, cols, ld, nb, to, scales);
        else
            hipLaunchKernelGGL((k_pack8<float, 2>), blocks(2), dim3(256), 0, st,
                               (const float *)x + row * ld, units, cols, ld, nb, to, scales);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

hipError_t launch_product8(const spdp_rows8 &a, const spdp_rows8 &b, bool log, void *c,
                           int32_t type, int64_t ld, hipStream_t st)
{
    // (launches hold 2^24 documents and 2^28 words: 2^20 tiles of 16 documents, or 2^22 of 64
    // words for up to 16 documents)
    constexpr int64_t kDocs = 1 << 24, kWords = 1 << 28;
    const int64_t nb = blocks8(a.cols), size = type == SPDP_F32 ? 4 : 2;
    for (int64_t d = 0; d < a.rows; d += kDocs)
        for (int64_t w = 0; w < b.rows; w += kWords) {
            const spdp_rows8 docs{a.rows - d < kDocs ? a.rows - d : kDocs, a.cols,
                                  a.q + d * nb * kBlock, a.e + d * nb};
            const spdp_rows8 words{b.rows - w < kWords ? b.rows - w : kWords, b.cols,
                                   b.q + w * nb * kBlock, b.e + w * nb};
            void *to = static_cast<char *>(c) + (d * ld + w) * size;
            const hipError_t e = type == SPDP_F32   ? product<float>(docs, words, log, to, ld, st)
                                 : type == SPDP_F16 ? product<_Float16>(docs, words, log, to, ld, st)
                                                    : product<__bf16>(docs, words, log, to, ld, st);
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace spdp
