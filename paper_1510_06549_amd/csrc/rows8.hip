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
constexpr float kMax8 = 448.0f;  // largest e4m3 value

// Exponent of a block's scale: the least e in [-127, 127] with amax <= 448 2^e.
// amax = f 2^p with f in [1/2, 1), and 448 = 7/8 2^9.
__device__ __forceinline__ int scale_exponent(double amax)
{
    if (!(amax > 0.0)) return -127;
    int p;
    const double f = frexp(amax, &p);
    const int e = p - 9 + (f > 0.875 ? 1 : 0);
    return e < -127 ? -127 : e > 127 ? 127 : e;
}

// v (already scaled) for the 8-bit conversion, which rounds fp32 to nearest even:
// the value is cut to fp32 with the last bit set where anything was cut off
// (rounding to odd), so that the two steps round as one.
__device__ __forceinline__ float odd_f32(double v)
{
    if (!(fabs(v) <= (double)kMax8)) return __builtin_nanf("");
    const float f = __double2float_rz(v);
    return (double)f == v ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// One wavefront per (row, block): two columns a lane, the largest finite magnitude
// over the wavefront, then both values in one 16-bit store.
template <typename T>
__global__ void __launch_bounds__(256) k_pack8(const T *__restrict__ x, int64_t rows, int32_t cols,
                                               int64_t ld, int32_t nb, uint8_t *__restrict__ q,
                                               uint8_t *__restrict__ e)
{
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= rows * nb) return;
    const int lane = threadIdx.x & 63;
    const int64_t row = unit / nb;
    const int32_t c = (int32_t)(unit - row * nb) * kBlock + 2 * lane;
    const T *src = x + row * ld + c;
    const double a = c < cols ? (double)src[0] : 0.0;
    const double b = c + 1 < cols ? (double)src[1] : 0.0;
    double m = fmax(isfinite(a) ? fabs(a) : 0.0, isfinite(b) ? fabs(b) : 0.0);
    for (int d = 32; d; d >>= 1) m = fmax(m, __shfl_xor(m, d));
    const int ex = scale_exponent(m);
    const float fa = odd_f32(ldexp(a, -ex)), fb = odd_f32(ldexp(b, -ex));
    const int pair = __builtin_amdgcn_cvt_pk_fp8_f32(fa, fb, 0, false);
    *reinterpret_cast<uint16_t *>(q + unit * kBlock + 2 * lane) = (uint16_t)pair;
    if (lane == 0) e[unit] = (uint8_t)(ex + 127);
}

typedef __bf16 b2v __attribute__((ext_vector_type(2)));
typedef __bf16 b8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));

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
__device__ __forceinline__ _Float16 out_as<_Float16>(float v) { return (_Float16)v; }
template <>
__device__ __forceinline__ __bf16 out_as<__bf16>(float v) { return (__bf16)v; }

// c[i][j] = sum_k a[i][k] b[j][k], or its logarithm: one wavefront per 16 x 16
// outputs.  A lane gives 8 columns of row (lane & 15) of either operand to an
// instruction; which columns does not matter to the sum as long as both operands
// agree.
template <typename T, bool LOG>
__global__ void __launch_bounds__(256) k_product8(const uint8_t *__restrict__ aq,
                                                  const uint8_t *__restrict__ ae, int64_t m,
                                                  const uint8_t *__restrict__ bq,
                                                  const uint8_t *__restrict__ be, int64_t n,
                                                  int32_t nb, T *__restrict__ c, int64_t ld,
                                                  int64_t tiles_j, int64_t tiles)
{
    const int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const int lane = threadIdx.x & 63, r = lane & 15, part = lane >> 4;
    const int64_t i0 = tile / tiles_j * 16, j0 = tile % tiles_j * 16;
    // rows past the end repeat the last one; their outputs are not stored
    const int64_t ia = i0 + r < m ? i0 + r : m - 1, jb = j0 + r < n ? j0 + r : n - 1;
    const uint8_t *pa = aq + ia * nb * kBlock + part * 32, *pb = bq + jb * nb * kBlock + part * 32;
    f4v acc = {0.f, 0.f, 0.f, 0.f};
    for (int32_t b = 0; b < nb; ++b) {
        const float sa = scale_of(ae[ia * nb + b]), sb = scale_of(be[jb * nb + b]);
        for (int h = 0; h < 2; ++h) {
            const uint4 x = *reinterpret_cast<const uint4 *>(pa + b * kBlock + 16 * h);
            const uint4 y = *reinterpret_cast<const uint4 *>(pb + b * kBlock + 16 * h);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(unpack8(x.x, x.y, sa),
                                                          unpack8(y.x, y.y, sb), acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(unpack8(x.z, x.w, sa),
                                                          unpack8(y.z, y.w, sb), acc, 0, 0, 0);
        }
    }
    // result: value v of a lane is row 4 (lane >> 4) + v, column lane & 15
    if (j0 + r >= n) return;
    for (int v = 0; v < 4; ++v) {
        const int64_t i = i0 + 4 * part + v;
        if (i < m) c[i * ld + j0 + r] = out_as<T>(LOG ? logf(acc[v]) : acc[v]);
    }
}

template <typename T>
hipError_t product(const spdp_rows8 &a, const spdp_rows8 &b, bool log, void *c, int64_t ld,
                   hipStream_t st)
{
    const int64_t tj = (b.rows + 15) / 16, tiles = (a.rows + 15) / 16 * tj;
    const dim3 grid((unsigned)((tiles + 3) / 4));
    const int32_t nb = blocks8(a.cols);
    if (log)
        hipLaunchKernelGGL((k_product8<T, true>), grid, dim3(256), 0, st, a.q, a.e, a.rows, b.q,
                           b.e, b.rows, nb, (T *)c, ld, tj, tiles);
    else
        hipLaunchKernelGGL((k_product8<T, false>), grid, dim3(256), 0, st, a.q, a.e, a.rows, b.q,
                           b.e, b.rows, nb, (T *)c, ld, tj, tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_pack8(const void *x, int32_t type, int64_t rows, int32_t cols, int64_t ld,
                        uint8_t *q, uint8_t *e, hipStream_t st)
{
    const int32_t nb = blocks8(cols);
    if (rows == 0 || nb == 0) return hipSuccess;
    const dim3 grid((unsigned)((rows * nb + 3) / 4));
    if (type == SPDP_F64)
        hipLaunchKernelGGL(k_pack8<double>, grid, dim3(256), 0, st, (const double *)x, rows, cols,
                           ld, nb, q, e);
    else
        hipLaunchKernelGGL(k_pack8<float>, grid, dim3(256), 0, st, (const float *)x, rows, cols,
                           ld, nb, q, e);
    return hipGetLastError();
}

hipError_t launch_product8(const spdp_rows8 &a, const spdp_rows8 &b, bool log, void *c,
                           int32_t type, int64_t ld, hipStream_t st)
{
    if (a.rows == 0 || b.rows == 0) return hipSuccess;
    if (type == SPDP_F32) return product<float>(a, b, log, c, ld, st);
    if (type == SPDP_F16) return product<_Float16>(a, b, log, c, ld, st);
    return product<__bf16>(a, b, log, c, ld, st);
}

}  // namespace spdp
