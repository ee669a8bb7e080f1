// Projections and the pruned FFN in 8-bit integers: the path of few rows, and the entry points.
#include "i8.hpp"

namespace sf {

namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr int FEW_ROWS = 8, FEW_K = 4096, FEW_FEATURES = 16;

// sum of a row of 16 lanes, in each of them
__device__ __forceinline__ int row16_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);      // row_ror 8, 4, 2, 1
    x += __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false);
    return x;
}

// Quantiser and product of up to R rows in one launch (blockIdx.y: sample).  What bounds it is the weights, read once, and one memory round
// trip each for them, the rows and the reduction.  Every workgroup quantises the rows for itself, into LDS, while its first weights are on
// their way; 16 lanes then share a feature, 16 bytes of K each at a time (v_dot4), and join their sums at the end.  Up to eight rows of up to 4096:
// one row, 512 x 512 3.1 us (quantiser and product in launches of their own 5.7), eight rows 4.8 (6.3), eight of 4096 x 768 15.7 (17.0).
struct FewI8 {
    const void *X; int64_t ldx; int64_t x_bstride; int rows, K;          // rows of a sample
    const void *ln_g, *ln_b; float eps;
    const int8_t *W; int64_t ldw, w_pstride; const float *sw; int64_t sw_pstride;
    const void *bias; int64_t bias_pstride; int bias_f32; const int32_t *pattern_id; int P;
    int N, act;
    const void *R; int64_t ldr; void *C; int64_t ldc, c_bstride; int c_f32;
};

template <class T, bool LN, int R, int NCH>
__global__ __launch_bounds__(256) void i8_few_kernel(FewI8 a)
{
    __shared__ __attribute__((aligned(16))) int8_t xq[R][NCH * 512];
    __shared__ float xs[R];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15;
    const int b = blockIdx.y, p = a.P > 1 && a.pattern_id ? a.pattern_id[b] : 0;
    const int n = blockIdx.x * FEW_FEATURES + wave * 4 + (lane >> 4), chunks = a.K >> 4;
    const int8_t *W = a.W + p * a.w_pstride + (int64_t)(n < a.N ? n : a.N - 1) * a.ldw;
    constexpr int AHEAD = 4;
    i32x4 w[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int c = c16 + j * 16;
        w[j] = i32x4{0, 0, 0, 0};
        if (c < chunks) w[j] = *reinterpret_cast<const i32x4 *>(W + c * 16);
    }
    for (int r = wave; r < R; r += 4) {
        float v[NCH][8];
        const T *x = (const T *)a.X + b * a.x_bstride + (int64_t)(r < a.rows ? r : 0) * a.ldx;
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int at = (lane + c * 64) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = 0.f;
            if (at < a.K) {
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
            const float mean = wave_sum(sum) / a.K;
            float q = 0.f;
#pragma unroll
            for (int c = 0; c < NCH; ++c)
                if ((lane + c * 64) * 8 < a.K) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) { v[c][e] -= mean; q = fmaf(v[c][e], v[c][e], q); }
                }
            const float inv = 1.0f / sqrtf(wave_sum(q) / a.K + a.eps);
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                const int at = (lane + c * 64) * 8;
                if (at >= a.K) continue;
                const h16x8 gm = *reinterpret_cast<const h16x8 *>((const h16 *)a.ln_g + at), bt = *reinterpret_cast<const h16x8 *>((const h16 *)a.ln_b + at);
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
        for (int c = 0; c < NCH; ++c) *reinterpret_cast<uint2 *>(&xq[r][(lane + c * 64) * 8]) = code.eight(v[c]);
        if (lane == 0) xs[r] = code.scale;
    }
    __syncthreads();
    int acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0;
    for (int c0 = c16; c0 < chunks; c0 += 16 * AHEAD) {
        i32x4 next[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int c = c0 + (j + AHEAD) * 16;
            next[j] = i32x4{0, 0, 0, 0};
            if (c < chunks) next[j] = *reinterpret_cast<const i32x4 *>(W + c * 16);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (c0 + j * 16 >= chunks) break;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const i32x4 x = *reinterpret_cast<const i32x4 *>(&xq[r][(c0 + j * 16) * 16]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[r] = __builtin_amdgcn_sdot4(w[j][e], x[e], acc[r], false);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) w[j] = next[j];
    }
    int mine = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) { const int s = row16_sum(acc[r]); if (c16 == r) mine = s; }
    if (c16 < R && c16 < a.rows && n < a.N) {
        float z = (float)mine * xs[c16] * a.sw[p * a.sw_pstride + n];
        if (a.bias) z += a.bias_f32 ? ((const float *)a.bias)[p * a.bias_pstride + n] : (float)((const h16 *)a.bias)[p * a.bias_pstride + n];
        const int64_t row = (int64_t)b * a.rows + c16;
        if (a.c_f32) {
            z = activate<float>(a.act, z);
            if (a.R) z += ((const float *)a.R)[row * a.ldr + n];
            ((float *)a.C)[row * a.ldc + n] = z;
        } else {
            z = activate<h16>(a.act, z);
            if (a.R) z += (float)((const h16 *)a.R)[row * a.ldr + n];
            ((h16 *)a.C)[row * a.ldc + n] = from_f32<h16>(z);
        }
    }
}

void few(const FewI8 &a, bool x_f32, int samples, hipStream_t st)
{
    const dim3 grid((unsigned)ceil_div(a.N, FEW_FEATURES), (unsigned)samples);
#define SF_FEW(T, LN, R, NCH) hipLaunchKernelGGL((i8_few_kernel<T, LN, R, NCH>), grid, dim3(256), 0, st, a)
#define SF_FEW_R(T, LN, NCH)                                                                                          \
    do {                                                                                                              \
        if (a.rows == 1) SF_FEW(T, LN, 1, NCH);                                                                       \
        else if (a.rows <= 4) SF_FEW(T, LN, 4, NCH);                                                                  \
        else SF_FEW(T, LN, 8, NCH);                                                                                   \
    } while (0)
#define SF_FEW_K(T, LN)                                                                                               \
    do {                                                                                                              \
        if (a.K <= 1024) SF_FEW_R(T, LN, 2);                                                                          \
        else SF_FEW_R(T, LN, 8);                                                                                      \
    } while (0)
    if (x_f32) SF_FEW_K(float, false);
    else if (a.ln_g) SF_FEW_K(h16, true);
    else SF_FEW_K(h16, false);
#undef SF_FEW_K
#undef SF_FEW_R
#undef SF_FEW
}

int act_of(int act) { return act == SF_GELU_ERF ? ACT_GELU : act == SF_RELU ? ACT_RELU : ACT_NONE; }

struct LinearWs { int8_t *q; float *s; size_t bytes; };
LinearWs linear_ws(int64_t rows, int K, void *ws)
{
    Carver c(ws);
    LinearWs w{};
    w.q = c.take<int8_t>((size_t)rows * K);
    w.s = c.take<float>((size_t)rows);
    w.bytes = c.off;
    return w;
}

// Few rows: hid holds them in fp32 between the two launches
struct FfnI8Ws { int8_t *xq, *hq; float *sx, *sh, *part, *top, *hid; size_t bytes; };
bool ffn_few(const Dims &D, int Fp) { return D.d <= FEW_K && Fp <= FEW_K && (D.P > 1 ? D.L <= FEW_ROWS && D.B <= 8 : (int64_t)D.B * D.L <= FEW_ROWS); }
FfnI8Ws ffn_ws(const Dims &D, int Fp, void *ws)
{
    Carver c(ws);
    FfnI8Ws w{};
    const size_t rows = (size_t)D.B * D.L;
    w.xq = c.take<int8_t>(rows * D.d);
    w.sx = c.take<float>(rows);
    w.hq = c.take<int8_t>(rows * Fp);
    w.sh = c.take<float>(rows);
    w.part = c.take<float>(rows * ceil_div(Fp, 32));      // the most parts that any kernel makes
    w.top = c.take<float>(rows);
    w.hid = ffn_few(D, Fp) ? c.take<float>(rows * Fp) : nullptr;
    w.bytes = c.off;
    return w;
}

int32_t check_ffn_i8(const char *who, const Dims &D, int32_t k_ffn)
{
    if (D.dtype != SF_BF16) return fail(SF_ERR_UNSUPPORTED, "%s: the integer path takes 16-bit activations, not fp32", who);
    if (k_ffn < 1 || k_ffn > D.F) return fail(SF_ERR_INVALID_ARG, "%s: k_ffn out of range", who);
    if (D.d % 16 || D.d > 4096) return fail(SF_ERR_SHAPE, "%s: d_model must be a multiple of 16, at most 4096", who);
    if (D.F > 65472) return fail(SF_ERR_SHAPE, "%s: d_ff <= 65472 required", who);
    return SF_OK;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" size_t sf_linear_i8_workspace_bytes(int64_t rows, int32_t K)
{
    if (rows < 1 || rows > (int64_t)1 << 30 || K < 1 || K > 65536) return 0;
    return linear_ws(rows, K, nullptr).bytes;
}

extern "C" int32_t sf_linear_i8_forward(const sf_linear_i8 *lin, int32_t dtype, int64_t rows, const void *X, int64_t ldx, int32_t act,
                                        const void *R, int64_t ldr, void *Y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    if (dtype == SF_DTYPE_16_OTHER) return fail(SF_ERR_UNSUPPORTED, "linear_i8: rows of this 16-bit type take the other build of the library");
    if (dtype != SF_F32 && dtype != SF_DTYPE_16) return fail(SF_ERR_UNSUPPORTED, "linear_i8: unknown dtype");
    if (act != SF_ACT_NONE && act != SF_RELU && act != SF_GELU_ERF) return fail(SF_ERR_UNSUPPORTED, "linear_i8: unknown activation");
    if (!lin) return fail(SF_ERR_INVALID_ARG, "linear_i8: NULL argument");
    const int N = lin->N, K = lin->K;
    if (N < 1 || K < 1 || rows < 0) return fail(SF_ERR_INVALID_ARG, "linear_i8: needs N >= 1, K >= 1 and rows >= 0");
    if (K % 16 || K > 65536) return fail(SF_ERR_SHAPE, "linear_i8: K must be a multiple of 16, at most 65536");
    if (rows > (int64_t)1 << 30) return fail(SF_ERR_SHAPE, "linear_i8: more than 2^30 rows");
    if (lin->ldw < K || lin->ldw % 16 || lin->ldw > 1 << 22)
        return fail(SF_ERR_INVALID_ARG, "linear_i8: ldw must be a multiple of 16, at least K and at most 2^22");
    if (ldx < K || ldy < N || (R && ldr < N)) return fail(SF_ERR_INVALID_ARG, "linear_i8: row strides shorter than the rows");
    if (rows == 0) return SF_OK;
    if (!lin->W || !lin->s || !X || !Y) return fail(SF_ERR_INVALID_ARG, "linear_i8: NULL argument");
    if (X == Y) return fail(SF_ERR_INVALID_ARG, "linear_i8: Y may not alias X");
    if (R == Y && ldr != ldy) return fail(SF_ERR_INVALID_ARG, "linear_i8: R is Y with rows of another stride");
    const int es = dtype == SF_F32 ? 4 : 2;
    if (((uintptr_t)lin->W & 15) || ((uintptr_t)lin->s & 3) || (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)R | (uintptr_t)lin->bias) % es))
        return fail(SF_ERR_INVALID_ARG, "linear_i8: W aligned to 16 bytes, the others to their elements required");
    const LinearWs w = linear_ws(rows, K, workspace);
    if (!workspace || workspace_bytes < w.bytes || ((uintptr_t)workspace & 255))
        return fail(SF_ERR_WORKSPACE, "linear_i8: workspace of %zu bytes (256-byte aligned) required, got %zu", w.bytes, workspace_bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    I8Rows q{};
    q.X = X; q.ldx = ldx; q.x_f32 = es == 4; q.rows = rows; q.K = K; q.codes = w.q; q.scale = w.s;
    if (rows <= FEW_ROWS && K <= FEW_K && i8_rows_vector(q)) {
        FewI8 f{};
        f.X = X; f.ldx = ldx; f.rows = (int)rows; f.K = K; f.W = (const int8_t *)lin->W; f.ldw = lin->ldw; f.sw = lin->s;
        f.bias = lin->bias; f.bias_f32 = es == 4; f.P = 1; f.N = N; f.act = act_of(act); f.R = R; f.ldr = ldr; f.C = Y; f.ldc = ldy; f.c_f32 = es == 4;
        few(f, es == 4, 1, st);
        return check_launch("linear_i8_forward");
    }
    quantize_i8(q, st);
    GemmI8 g{};
    g.A = w.q; g.lda = K; g.sa = w.s; g.W = (const int8_t *)lin->W; g.ldw = lin->ldw; g.sw = lin->s; g.bias = lin->bias; g.bias_f32 = es == 4;
    g.P = 1; g.B = 1; g.L = rows; g.N = N; g.K = K; g.act = act_of(act); g.R = R; g.ldr = ldr; g.C = Y; g.ldc = ldy; g.c_f32 = es == 4;
    if (int32_t rc = gemm_i8(I8_OUT, g, st)) return rc;
    return check_launch("linear_i8_forward");
}

extern "C" size_t sf_pruned_ffn_i8_workspace_bytes(const sf_desc *desc, int32_t k_ffn)
{
    Dims D;
    if (read_desc(desc, D) || check_ffn_i8("pruned_ffn_i8", D, k_ffn)) return 0;
    return ffn_ws(D, (int)align_up((size_t)k_ffn, D.ffn_pad), nullptr).bytes;
}

extern "C" int32_t sf_pruned_ffn_i8_forward(const sf_desc *desc, const sf_ffn_i8 *f, const void *X, const int32_t *pattern_id, int32_t pre_ln,
                                            int32_t add_residual, void *Y, void *workspace, size_t workspace_bytes, void *stream)
{
    Dims D;
    if (int32_t rc = read_desc(desc, D)) return rc;
    if (!f) return fail(SF_ERR_INVALID_ARG, "pruned_ffn_i8: NULL argument");
    if (int32_t rc = check_ffn_i8("pruned_ffn_i8", D, f->k_ffn)) return rc;
    if (!X || !Y || !f->W1q || !f->s1 || !f->W2Tq || !f->s2 || (pre_ln && (!f->ln2_g || !f->ln2_b)))
        return fail(SF_ERR_INVALID_ARG, "pruned_ffn_i8: NULL argument");
    if (X == Y) return fail(SF_ERR_INVALID_ARG, "pruned_ffn_i8: Y may not alias X");
    if (D.P > 1 && !pattern_id) return fail(SF_ERR_INVALID_ARG, "pruned_ffn_i8: pattern_id required when P > 1");
    if (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)f->W1q | (uintptr_t)f->W2Tq | (pre_ln ? (uintptr_t)f->ln2_g | (uintptr_t)f->ln2_b : 0)) & 15)
        return fail(SF_ERR_INVALID_ARG, "pruned_ffn_i8: 16-byte aligned X, Y, weights and LayerNorm vectors required");
    if ((((uintptr_t)f->s1 | (uintptr_t)f->s2) & 3) || (((uintptr_t)f->b1 | (uintptr_t)f->b2) & 1))
        return fail(SF_ERR_INVALID_ARG, "pruned_ffn_i8: scales and biases aligned to their elements required");
    const int Fp = (int)align_up((size_t)f->k_ffn, D.ffn_pad);
    const FfnI8Ws w = ffn_ws(D, Fp, workspace);
    if (!workspace || workspace_bytes < w.bytes || ((uintptr_t)workspace & 255))
        return fail(SF_ERR_WORKSPACE, "pruned_ffn_i8: workspace of %zu bytes (256-byte aligned) required, got %zu", w.bytes, workspace_bytes);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t rows = (int64_t)D.B * D.L;
    if (ffn_few(D, Fp)) {
        const int samples = D.P > 1 ? D.B : 1, per = (int)(rows / samples);
        FewI8 u{};
        u.X = X; u.ldx = D.d; u.x_bstride = (int64_t)per * D.d; u.rows = per; u.K = D.d;
        u.ln_g = pre_ln ? f->ln2_g : nullptr; u.ln_b = f->ln2_b; u.eps = D.eps;
        u.W = f->W1q; u.ldw = D.d; u.w_pstride = (int64_t)Fp * D.d; u.sw = f->s1; u.sw_pstride = Fp; u.bias = f->b1; u.bias_pstride = Fp;
        u.pattern_id = pattern_id; u.P = D.P; u.N = Fp; u.act = act_of(D.act); u.C = w.hid; u.ldc = Fp; u.c_f32 = 1;
        few(u, false, samples, st);
        FewI8 v{};
        v.X = w.hid; v.ldx = Fp; v.x_bstride = (int64_t)per * Fp; v.rows = per; v.K = Fp;
        v.W = f->W2Tq; v.ldw = Fp; v.w_pstride = (int64_t)D.d * Fp; v.sw = f->s2; v.bias = f->b2;
        v.pattern_id = pattern_id; v.P = D.P; v.N = D.d; v.act = ACT_NONE; v.R = add_residual ? X : nullptr; v.ldr = D.d; v.C = Y; v.ldc = D.d;
        few(v, true, samples, st);
        return check_launch("pruned_ffn_i8_forward");
    }
    I8Rows q{};
    q.X = X; q.ldx = D.d; q.rows = rows; q.K = D.d; q.ln_g = pre_ln ? f->ln2_g : nullptr; q.ln_b = f->ln2_b; q.eps = D.eps; q.codes = w.xq; q.scale = w.sx;
    quantize_i8(q, st);
    // A hidden row's codes need its largest value first.  The product is done twice: once for that value alone, once for the codes.
    GemmI8 u{};
    u.A = w.xq; u.lda = D.d; u.sa = w.sx; u.W = f->W1q; u.ldw = D.d; u.w_pstride = (int64_t)Fp * D.d; u.sw = f->s1; u.sw_pstride = Fp;
    u.bias = f->b1; u.bias_pstride = Fp; u.pattern_id = pattern_id; u.P = D.P; u.B = D.B; u.L = D.L; u.N = Fp; u.K = D.d; u.act = act_of(D.act);
    u.part = w.part; u.top = w.top; u.codes = w.hq; u.scale = w.sh;
    if (int32_t rc = gemm_i8(I8_AMAX, u, st)) return rc;
    if (int32_t rc = gemm_i8(I8_CODES, u, st)) return rc;
    GemmI8 v{};
    v.A = w.hq; v.lda = Fp; v.sa = w.sh; v.W = f->W2Tq; v.ldw = Fp; v.w_pstride = (int64_t)D.d * Fp; v.sw = f->s2; v.bias = f->b2;
    v.pattern_id = pattern_id; v.P = D.P; v.B = D.B; v.L = D.L; v.N = D.d; v.K = Fp; v.act = ACT_NONE;
    v.R = add_residual ? X : nullptr; v.ldr = D.d; v.C = Y; v.ldc = D.d;
    if (int32_t rc = gemm_i8(I8_OUT, v, st)) return rc;
    return check_launch("pruned_ffn_i8_forward");
}
