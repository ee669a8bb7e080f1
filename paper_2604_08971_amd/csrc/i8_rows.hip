// Quantisers of rows to 8-bit integers, one scale per row: alone and behind a LayerNorm.
//
// A row is read once and stays in registers (a wave per row, up to 4096 elements), so what bounds it is memory: es bytes read and one
// written per element.
#include "i8.hpp"

namespace sf {

namespace {

template <class T, int NCH, bool LN>
__global__ __launch_bounds__(256) void i8_rows_kernel(const T *__restrict__ X, int64_t ldx, int64_t rows, int n, const h16 *__restrict__ g,
                                                      const h16 *__restrict__ b, float eps, int8_t *__restrict__ codes, int64_t ldc,
                                                      float *__restrict__ scale)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const T *x = X + row * ldx;
    float v[NCH][8];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int at = (lane + c * 64) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = 0.f;
        if (at < n) {
            if constexpr (sizeof(T) == 2) {
                const h16x8 t = *reinterpret_cast<const h16x8 *>(x + at);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[c][e] = (float)t[e];
            } else {
                const f32x4 t0 = *reinterpret_cast<const f32x4 *>(x + at), t1 = *reinterpret_cast<const f32x4 *>(x + at + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[c][e] = t0[e]; v[c][4 + e] = t1[e]; }
            }
            if constexpr (LN) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += v[c][e];
            }
        }
    }
    if constexpr (LN) {
        const float mean = wave_sum(sum) / n;
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
            if ((lane + c * 64) * 8 < n) {
#pragma unroll
                for (int e = 0; e < 8; ++e) { v[c][e] -= mean; q = fmaf(v[c][e], v[c][e], q); }
            }
        const float inv = 1.0f / sqrtf(wave_sum(q) / n + eps);
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int at = (lane + c * 64) * 8;
            if (at >= n) continue;
            const h16x8 gm = *reinterpret_cast<const h16x8 *>(g + at), bt = *reinterpret_cast<const h16x8 *>(b + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = fmaf(v[c][e] * inv, (float)gm[e], (float)bt[e]);
        }
    }
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) { const uint32_t u = abs_bits(v[c][e]); m = m > u ? m : u; }
    const RowCode code(wave_max_u32(m));
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int at = (lane + c * 64) * 8;
        if (at >= n) continue;
        uint2 o;
        o.x = pack4_i8(code(v[c][0]), code(v[c][1]), code(v[c][2]), code(v[c][3]));
        o.y = pack4_i8(code(v[c][4]), code(v[c][5]), code(v[c][6]), code(v[c][7]));
        *reinterpret_cast<uint2 *>(codes + row * ldc + at) = o;
    }
    if (lane == 0) scale[row] = code.scale;
}

// Rows of any length, stride and alignment: a workgroup per row, read twice
template <class T>
__global__ __launch_bounds__(256) void i8_rows_any_kernel(const T *__restrict__ X, int64_t ldx, int64_t rows, int n, int8_t *__restrict__ codes,
                                                          int64_t ldc, float *__restrict__ scale)
{
    __shared__ uint32_t most[4];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *x = X + row * ldx;
        uint32_t m = 0;
        for (int i = threadIdx.x; i < n; i += 256) { const uint32_t u = abs_bits(to_f32(x[i])); m = m > u ? m : u; }
        m = wave_max_u32(m);
        __syncthreads();                                     // the last row's values have been read
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) m = m > most[w] ? m : most[w];
        const RowCode code(m);
        for (int i = threadIdx.x; i < n; i += 256) codes[row * ldc + i] = (int8_t)code(to_f32(x[i]));
        if (threadIdx.x == 0) scale[row] = code.scale;
    }
}

template <class T>
void launch_rows(const I8Rows &a, int64_t ldc, bool vec, hipStream_t st)
{
    const T *X = (const T *)a.X;
    if (!vec || a.K > 4096) {
        const unsigned grid = (unsigned)(a.rows < 65536 ? a.rows : 65536);
        hipLaunchKernelGGL(i8_rows_any_kernel<T>, dim3(grid), dim3(256), 0, st, X, a.ldx, a.rows, a.K, a.codes, ldc, a.scale);
        return;
    }
    const dim3 grid((unsigned)((a.rows + 3) / 4));
#define SF_I8_ROWS(NCH, LN)                                                                                                      \
    hipLaunchKernelGGL((i8_rows_kernel<T, NCH, LN>), grid, dim3(256), 0, st, X, a.ldx, a.rows, a.K, (const h16 *)a.ln_g, (const h16 *)a.ln_b, \
                       a.eps, a.codes, ldc, a.scale)
#define SF_I8_ROWS_N(LN)                                                                                                         \
    do {                                                                                                                         \
        if (a.K <= 512) SF_I8_ROWS(1, LN);                                                                                       \
        else if (a.K <= 1024) SF_I8_ROWS(2, LN);                                                                                 \
        else if (a.K <= 2048) SF_I8_ROWS(4, LN);                                                                                 \
        else SF_I8_ROWS(8, LN);                                                                                                  \
    } while (0)
    if constexpr (sizeof(T) == 2) {
        if (a.ln_g) { SF_I8_ROWS_N(true); return; }
    }
    SF_I8_ROWS_N(false);
#undef SF_I8_ROWS_N
#undef SF_I8_ROWS
}

bool rows_aligned(const void *X, int64_t ldx, int es, int n, const void *codes, int64_t ldc)
{
    return !((uintptr_t)X & 15) && (ldx * es) % 16 == 0 && n % 8 == 0 && !((uintptr_t)codes & 7) && ldc % 8 == 0;
}

}  // namespace

bool i8_rows_vector(const I8Rows &a) { return a.K <= 4096 && rows_aligned(a.X, a.ldx, a.x_f32 ? 4 : 2, a.K, a.codes, a.K); }

void quantize_i8(const I8Rows &a, hipStream_t st)
{
    if (a.x_f32) launch_rows<float>(a, a.K, i8_rows_vector(a), st);
    else launch_rows<h16>(a, a.K, i8_rows_vector(a), st);
}

}  // namespace sf

using namespace sf;

extern "C" int32_t sf_quantize_i8_rows(const void *x, int32_t dtype, int64_t rows, int32_t n, int64_t ldx, int8_t *codes, int64_t ldc,
                                       float *scale, void *stream)
{
    if (dtype == SF_DTYPE_16_OTHER)
        return fail(SF_ERR_UNSUPPORTED, "quantize_i8_rows: rows of this 16-bit type take the other build of the library");
    if (dtype != SF_F32 && dtype != SF_DTYPE_16) return fail(SF_ERR_UNSUPPORTED, "quantize_i8_rows: unknown dtype");
    if (rows < 0 || n < 1 || ldx < n || ldc < n) return fail(SF_ERR_INVALID_ARG, "quantize_i8_rows: needs rows >= 0, n >= 1 and strides of at least n");
    if (rows == 0) return SF_OK;
    if (!x || !codes || !scale) return fail(SF_ERR_INVALID_ARG, "quantize_i8_rows: NULL argument");
    if (rows > (int64_t)1 << 30) return fail(SF_ERR_SHAPE, "quantize_i8_rows: more than 2^30 rows");
    const int es = dtype == SF_F32 ? 4 : 2;
    if (((uintptr_t)x % es) || ((uintptr_t)scale & 3)) return fail(SF_ERR_INVALID_ARG, "quantize_i8_rows: x and scale aligned to their elements required");
    I8Rows a{};
    a.X = x; a.ldx = ldx; a.x_f32 = dtype == SF_F32; a.rows = rows; a.K = n; a.codes = codes; a.scale = scale;
    const bool vec = rows_aligned(x, ldx, es, n, codes, ldc);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.x_f32) launch_rows<float>(a, ldc, vec, st);
    else launch_rows<h16>(a, ldc, vec, st);
    return check_launch("quantize_i8_rows");
}
