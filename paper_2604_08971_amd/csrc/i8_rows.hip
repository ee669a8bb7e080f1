// Quantisers of rows to 8-bit integers, one scale per row: alone and behind a LayerNorm.
//
// A row is read once and stays in registers (up to 4096 elements), so what bounds it is memory: es bytes read and one written per element.  A
// wave per row has too little on its way where rows are short: 65 536 rows of 64, 512 and 768 bf16 elements took 27, 29 and 35 us that way, and take 7,
// 21 and 28 with the rows of a wave's lanes next to each other and four (two) of them at once; behind a LayerNorm 49 and now 45 us for 768.
#include "i8.hpp"

namespace sf {

namespace {

template <class T> struct Raw;
template <> struct Raw<h16> { typedef h16x8 type; };
template <> struct Raw<float> { typedef __attribute__((ext_vector_type(8), aligned(16))) float type; };

// LANES lanes a row, NCH times eight elements each, NR rows of a lane with their loads in flight together
template <class T, int NCH, int LANES, int NR, bool LN>
__global__ __launch_bounds__(256) void i8_rows_kernel(const T *__restrict__ X, int64_t ldx, int64_t rows, int n, const h16 *__restrict__ g,
                                                      const h16 *__restrict__ b, float eps, int8_t *__restrict__ codes, int64_t ldc,
                                                      float *__restrict__ scale)
{
    constexpr int SIDE = 64 / LANES;                         // rows next to each other in a wave
    const int lane = threadIdx.x & (LANES - 1);
    const int64_t row0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (NR * SIDE) + (threadIdx.x & 63) / LANES;
    typedef typename Raw<T>::type Eight;
    Eight raw[NR][NCH];
    h16x8 gm[LN ? NCH : 1], bt[LN ? NCH : 1];
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int at = (lane + c * LANES) * 8;
            raw[i][c] = Eight{};
            if (at < n && row0 + i * SIDE < rows) raw[i][c] = *reinterpret_cast<const Eight *>(X + (row0 + i * SIDE) * ldx + at);
        }
    if constexpr (LN) {
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int at = (lane + c * LANES) * 8;
            gm[c] = bt[c] = h16x8{};
            if (at < n) { gm[c] = *reinterpret_cast<const h16x8 *>(g + at); bt[c] = *reinterpret_cast<const h16x8 *>(b + at); }
        }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int64_t row = row0 + i * SIDE;
        if (row >= rows) break;
        float v[NCH][8];
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = (float)raw[i][c][e];
        if constexpr (LN) {
            float sum = 0.f, q = 0.f;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += v[c][e];
            const float mean = lanes_sum<LANES>(sum) / n;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                if ((lane + c * LANES) * 8 < n) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) { v[c][e] -= mean; q = fmaf(v[c][e], v[c][e], q); }
                }
            const float inv = 1.0f / sqrtf(lanes_sum<LANES>(q) / n + eps);
#pragma unroll
            for (int c = 0; c < NCH; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[c][e] = fmaf(v[c][e] * inv, (float)gm[c][e], (float)bt[c][e]);       // zeros behind the row
        }
        uint32_t m = 0;
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) { const uint32_t u = abs_bits(v[c][e]); m = m > u ? m : u; }
        const RowCode code(lanes_max<LANES>(m));
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int at = (lane + c * LANES) * 8;
            if (at < n) *reinterpret_cast<uint2 *>(codes + row * ldc + at) = code.eight(v[c]);
        }
        if (lane == 0) scale[row] = code.scale;
    }
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
#define SF_I8_ROWS(NCH, LANES, NR, LN)                                                                                           \
    hipLaunchKernelGGL((i8_rows_kernel<T, NCH, LANES, NR, LN>), dim3((unsigned)((a.rows + 256 / LANES * NR - 1) / (256 / LANES * NR))),   \
                       dim3(256), 0, st, X, a.ldx, a.rows, a.K, (const h16 *)a.ln_g, (const h16 *)a.ln_b, a.eps, a.codes, ldc, a.scale)
    // a wave for every row until the chip holds no more of them (8192); well above that, more rows on their way in each
    const bool many = a.rows >= (a.K <= 512 ? 16384 : 32768);
#define SF_I8_ROWS_N(LN)                                                                                                         \
    do {                                                                                                                         \
        if (many && a.K <= 128) SF_I8_ROWS(1, 16, 4, LN);                                                                        \
        else if (many && a.K <= 256) SF_I8_ROWS(1, 32, 4, LN);                                                                   \
        else if (many && a.K <= 512) SF_I8_ROWS(1, 64, 4, LN);                                                                   \
        else if (many && a.K <= 1024) SF_I8_ROWS(2, 64, 2, LN);                                                                  \
        else if (a.K <= 512) SF_I8_ROWS(1, 64, 1, LN);                                                                           \
        else if (a.K <= 1024) SF_I8_ROWS(2, 64, 1, LN);                                                                          \
        else if (a.K <= 2048) SF_I8_ROWS(4, 64, 1, LN);                                                                          \
        else SF_I8_ROWS(8, 64, 1, LN);                                                                                           \
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
