// Products in 8-bit integers with a scale for each token and each output feature: what the sources of them share.
#pragma once

#include "gemm.hpp"

namespace sf {

__device__ __forceinline__ uint32_t pack4_i8(int a, int b, int c, int d)
{
    return (uint32_t)(a & 255) | ((uint32_t)(b & 255) << 8) | ((uint32_t)(c & 255) << 16) | ((uint32_t)d << 24);
}

// One row's quantiser.  code = rne(127 x / a) with a the row's largest magnitude, scale = a / 127; a = 0: codes and scale 0; an infinity or
// NaN in the row: codes 0 and scale NaN, so that every product with the row is NaN.
struct RowCode {
    float amax, r, pre, scale;          // pre: rows of magnitudes below 2^-60 are brought up first, by a power of two (exact)
    __device__ explicit RowCode(uint32_t amax_bits)
    {
        const float a = __uint_as_float(amax_bits);
        const bool fine = amax_bits < 0x7f800000u && amax_bits != 0;
        pre = a < 0x1p-60f ? 0x1p80f : 1.0f;
        amax = a * pre;
        r = fine ? 127.0f / amax : 0.f;
        if (!fine) pre = 0.f;
        scale = amax_bits < 0x7f800000u ? a / 127.0f : __uint_as_float(0x7fc00000u);
    }
    // Eight codes: a rounded quotient that stays away from the borders is the code, and where one of the eight does not, operator() decides all
    __device__ __forceinline__ uint2 eight(const float *x) const
    {
        float c[8], off = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = x[e] * pre * r;
            c[e] = __builtin_rintf(t);
            off = fmaxf(off, fabsf(t - c[e]));
        }
        int k[8];
        if (off < 0.5f - 2e-5f && r != 0.f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) k[e] = (int)c[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) k[e] = (*this)(x[e]);
        }
        return make_uint2(pack4_i8(k[0], k[1], k[2], k[3]), pack4_i8(k[4], k[5], k[6], k[7]));
    }
    // x r differs from 127 x / a by less than 1.6e-5 (two roundings of values up to 127): only there a border between two codes is decided in
    // 64 bits, where 254 x and (2 k + 1) a are exact
    __device__ int operator()(float x) const
    {
        if (r == 0.f) return 0;                              // 0 x infinity
        const float t = x * pre * r, m = fabsf(t), k = floorf(m), f = m - k;
        float c = __builtin_rintf(t);
        if (fabsf(f - 0.5f) < 2e-5f) {
            const double lhs = 254.0 * (double)fabsf(x * pre), rhs = (2.0 * (double)k + 1.0) * (double)amax;
            const float up = lhs > rhs || (lhs == rhs && ((int)k & 1)) ? k + 1.f : k;
            c = __builtin_copysignf(up, t);
        }
        return (int)c;
    }
};

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// As pair_sum, for the larger one
template <int O>
__device__ __forceinline__ uint32_t pair_max(uint32_t x)
{
    uint32_t y, z = x;
    if constexpr (O == 32 || O == 16) {
        const auto r = O == 32 ? __builtin_amdgcn_permlane32_swap(x, x, false, false) : __builtin_amdgcn_permlane16_swap(x, x, false, false);
        y = r[0]; z = r[1];
    } else {
        constexpr int ctrl = O == 8 ? 0x128 : O == 4 ? 0x124 : O == 2 ? 0x4e : 0xb1;
        y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, false);
    }
    return y > z ? y : z;
}
// Largest and sum of each LANES lanes of a wave (16, 32, 64), in each of them
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x)
{
    if constexpr (LANES > 32) x = pair_max<32>(x);
    if constexpr (LANES > 16) x = pair_max<16>(x);
    return pair_max<1>(pair_max<2>(pair_max<4>(pair_max<8>(x))));
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x)
{
    if constexpr (LANES > 32) x = pair_sum<32>(x);
    if constexpr (LANES > 16) x = pair_sum<16>(x);
    return pair_sum<1>(pair_sum<2>(pair_sum<4>(pair_sum<8>(x))));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) { return lanes_max<64>(x); }

// p[n .. n + 3], zeros from N on
__device__ __forceinline__ f32x4 four(const float *p, int n, int N)
{
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (n + 4 <= N && !((uintptr_t)(p + n) & 15)) return *reinterpret_cast<const f32x4 *>(p + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) if (n + e < N) o[e] = p[n + e];
    return o;
}
__device__ __forceinline__ f32x4 four(const h16 *p, int n, int N)
{
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (n + 4 <= N && !((uintptr_t)(p + n) & 7)) {
        const h16x4 t = *reinterpret_cast<const h16x4 *>(p + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (float)t[e];
        return o;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) if (n + e < N) o[e] = (float)p[n + e];
    return o;
}

// T: what the value is rounded to afterwards.  gelu_erf() is good enough for 16 bits and for codes
template <class T>
__device__ __forceinline__ float activate(int act, float z)
{
    if (act == ACT_RELU) return z < 0.f ? 0.f : z;                   // a NaN stays one
    if (act == ACT_GELU) return sizeof(T) == 4 ? 0.5f * z * (1.0f + erff(z * 0.70710678f)) : gelu_erf(z);
    return z;
}

// Rows of X (fp32 when x_f32, else 16 bits), LayerNorm first when ln_g != NULL: codes [rows, K] (K % 16 == 0, stride K) and scales.
struct I8Rows {
    const void *X; int64_t ldx; bool x_f32;
    int64_t rows; int K;
    const void *ln_g, *ln_b; float eps;      // 16-bit
    int8_t *codes; float *scale;
};
bool i8_rows_vector(const I8Rows &a);        // 16-byte accesses; the LayerNorm needs them
void quantize_i8(const I8Rows &a, hipStream_t st);

// C[row, n] = epilogue(sum_k A[row, k] W[p, n, k]); row = b L + i, p the pattern of sample b.
enum I8Mode { I8_OUT, I8_AMAX, I8_CODES };
struct GemmI8 {
    const int8_t *A; int64_t lda; const float *sa;                       // codes, a scale per row; lda % 16 == 0
    const int8_t *W; int64_t ldw, w_pstride; const float *sw; int64_t sw_pstride;
    const void *bias; int64_t bias_pstride; int bias_f32;                // NULL: none
    const int32_t *pattern_id; int P;                                    // P > 1: a tile's rows are one sample's
    int64_t B, L; int N, K;
    int act;                                                             // ACT_*
    const void *R; int64_t ldr;                                          // I8_OUT: residual, type of C
    void *C; int64_t ldc; int c_f32;                                     // I8_OUT
    float *part;                                                         // I8_AMAX out, I8_CODES in: [n_parts, B L] largest |value| of a
                                                                         // row over each tile of features
    int8_t *codes; float *scale;                                         // I8_CODES: [B L, N] and the row's scale
    float *top;                                                          // I8_CODES: scratch, [B L]
};
int gemm_i8_parts(const GemmI8 &a);                                      // n_parts
int32_t gemm_i8(I8Mode mode, const GemmI8 &a, hipStream_t st);

}  // namespace sf
