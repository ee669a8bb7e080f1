// C = epilogue(A W^T) on the integer matrix cores: codes of rows and of output features, exact sums in 32 bits (a product of two codes is at
// most 2^14, so K up to 65 536 cannot overflow).
//
// A workgroup owns BM rows x BN features.  Both operands go straight from memory into LDS, 128 bytes of K a stage, two stages; a wave of it
// computes 32 x 32 blocks with mfma_i32_32x32x32_i8.  W is the instruction's first operand, so that a lane ends up with one row and runs of four
// features.  What lies past the last row, feature or K reads as zeros: the buffer loads are out of range there.
#include "i8.hpp"

namespace sf {

namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((address_space(3))) void lds_void;

template <int BM, int BN, int WM, int WN, int MODE, int ACT, class TC>
__global__ __launch_bounds__(WM *WN * 64) void gemm_i8_kernel(GemmI8 a, int tiles_n, int tiles_l, int n_parts)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int BK = 128;                                                        // bytes of K per stage
    constexpr int NT = WM * WN * 64, LX = BM * 8 / NT, LW = BN * 8 / NT;           // 16-byte pieces a thread moves per stage
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32, STAGE = (BM + BN) * BK;
    __shared__ __attribute__((aligned(128))) char lds[2 * STAGE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / WN, wn = wave % WN;
    // an XCD walks a contiguous run of tiles, the features of a row tile one after the other: its L2 reads the rows once
    const int total = gridDim.x, q8 = total / 8, r8 = total % 8, xcd = blockIdx.x % 8;
    const int t = xcd * q8 + (xcd < r8 ? xcd : r8) + blockIdx.x / 8;
    const int tn = t % tiles_n, tm = t / tiles_n;
    const int64_t b = tm / tiles_l, i0 = (int64_t)(tm % tiles_l) * BM, row0 = b * a.L + i0;
    const int64_t left = a.L - i0;                                                 // rows of this sample from row0 on
    const int rows = left < BM ? (int)left : BM, n0 = tn * BN;
    const int p = a.P > 1 && a.pattern_id ? a.pattern_id[b] : 0;
    const int8_t *A = a.A + row0 * a.lda, *W = a.W + p * a.w_pstride + (int64_t)n0 * a.ldw;
    const int feats = a.N - n0 < BN ? a.N - n0 : BN;
    const auto ar = __builtin_amdgcn_make_buffer_rsrc((void *)A, 0, (int)((rows - 1) * a.lda + a.K), 0x00020000);
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, (int)((feats - 1) * a.ldw + a.K), 0x00020000);
    // piece q of a stage: row q / 8, chunk (q % 8) ^ (row % 8) of its eight, so that 16 lanes of a fragment read meet no bank twice
    const int chunk = (threadIdx.x & 7) ^ ((threadIdx.x >> 3) & 7);
    int xoff[LX], woff[LW];
#pragma unroll
    for (int j = 0; j < LX; ++j) xoff[j] = (j * (NT / 8) + (threadIdx.x >> 3)) * (int)a.lda + chunk * 16;
#pragma unroll
    for (int j = 0; j < LW; ++j) woff[j] = (j * (NT / 8) + (threadIdx.x >> 3)) * (int)a.ldw + chunk * 16;
    auto fetch = [&](int kt, int s) {
        char *base = lds + s * STAGE + wave * 1024;
        const bool in = kt * BK + chunk * 16 < a.K;
#pragma unroll
        for (int j = 0; j < LX; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (lds_void *)(base + j * (NT * 16)), 16, in ? xoff[j] + kt * BK : 0x7ffffff0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < LW; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void *)(base + BM * BK + j * (NT * 16)), 16, in ? woff[j] + kt * BK : 0x7ffffff0, 0, 0, 0);
    };
    i32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const int kts = (a.K + BK - 1) / BK, r = lane & 31, hi = lane >> 5;
    fetch(0, 0);
    for (int kt = 0; kt < kts; ++kt) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                                     // stage kt is there, and nobody reads the other one any more
        if (kt + 1 < kts) fetch(kt + 1, (kt + 1) & 1);
        const char *xs = lds + (kt & 1) * STAGE + (wm * TM * 32 + r) * BK, *ws = lds + (kt & 1) * STAGE + (BM + wn * TN * 32 + r) * BK;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = ((k * 2 + hi) ^ (r & 7)) * 16;
            i32x4 xf[TM], wf[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) xf[i] = *reinterpret_cast<const i32x4 *>(xs + i * 32 * BK + at);
#pragma unroll
            for (int j = 0; j < TN; ++j) wf[j] = *reinterpret_cast<const i32x4 *>(ws + j * 32 * BK + at);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[j], xf[i], acc[i][j], 0, 0, 0);
        }
    }
    const float *sw = a.sw + p * a.sw_pstride;
    [[maybe_unused]] uint32_t most[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) most[i] = 0;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int li = (wm * TM + i) * 32 + r;                // row inside the tile
        const bool there = li < rows;
        const int64_t row = row0 + li;
        const float sa = there ? a.sa[row] : 0.f;
        [[maybe_unused]] float cr = 0.f;
        if constexpr (MODE == I8_CODES) {
            uint32_t m = 0;
            if (there)
                for (int t2 = 0; t2 < n_parts; ++t2) { const uint32_t u = __float_as_uint(a.part[(int64_t)t2 * (a.B * a.L) + row]); m = m > u ? m : u; }
            // below 2^-100 a row counts as zeros: 127 / amax would overflow
            const float top = __uint_as_float(m);
            cr = m < 0x7f800000u && top >= 0x1p-100f ? 127.0f / top : 0.f;
            if (tn == 0 && wn == 0 && hi == 0 && there) a.scale[row] = m < 0x7f800000u ? top / 127.0f : __uint_as_float(0x7fc00000u);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + (wn * TN + j) * 32 + q * 8 + hi * 4;
                const f32x4 s = four(sw, n, a.N);
                f32x4 z;
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = (float)acc[i][j][q * 4 + e] * sa * s[e];
                if (a.bias) {
                    const f32x4 bv = a.bias_f32 ? four((const float *)a.bias + p * a.bias_pstride, n, a.N) : four((const h16 *)a.bias + p * a.bias_pstride, n, a.N);
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] += bv[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = activate<TC>(ACT, z[e]);
                if constexpr (MODE == I8_AMAX) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) { const uint32_t u = abs_bits(z[e]); most[i] = most[i] > u ? most[i] : u; }
                } else if constexpr (MODE == I8_CODES) {
                    // a value at the border of two codes carries the rounding of its own fp32 sum: no exact decision here
                    int c[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[e] = cr == 0.f ? 0 : (int)__builtin_rintf(z[e] * cr);
                    if (there && n < a.N) *reinterpret_cast<uint32_t *>(a.codes + row * a.N + n) = pack4_i8(c[0], c[1], c[2], c[3]);
                } else if (there) {
                    TC *C = (TC *)a.C + row * a.ldc + n;
                    if (a.R) {
                        const f32x4 rv = four((const TC *)a.R + row * a.ldr, n, a.N);
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[e] += rv[e];
                    }
                    if (n + 4 <= a.N && !((uintptr_t)C & (sizeof(TC) * 4 - 1))) {
                        if constexpr (sizeof(TC) == 2) *reinterpret_cast<uint2 *>(C) = make_uint2(pack2_h16(z[0], z[1]), pack2_h16(z[2], z[3]));
                        else *reinterpret_cast<f32x4 *>(C) = z;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) if (n + e < a.N) C[e] = from_f32<TC>(z[e]);
                    }
                }
            }
        }
    }
    if constexpr (MODE == I8_AMAX) {
        uint32_t *red = reinterpret_cast<uint32_t *>(lds);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const uint32_t o = (uint32_t)__shfl_xor((int)most[i], 32);
            if (hi == 0) red[wn * BM + (wm * TM + i) * 32 + r] = most[i] > o ? most[i] : o;
        }
        __syncthreads();
        for (int l = threadIdx.x; l < rows; l += NT) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < WN; ++w) { const uint32_t u = red[w * BM + l]; m = m > u ? m : u; }
            a.part[(int64_t)tn * (a.B * a.L) + row0 + l] = __uint_as_float(m);
        }
    }
#endif
}

template <int BM, int BN, int WM, int WN, int MODE, class TC>
int32_t launch_act(const GemmI8 &a, hipStream_t st)
{
    const int64_t tiles_l = (a.L + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN, grid = a.B * tiles_l * tiles_n;
    if (grid > 0x7fffffff) return fail(SF_ERR_SHAPE, "gemm_i8: too many tiles");
    const int parts = gemm_i8_parts(a);
#define SF_I8_GEMM(ACT)                                                                                                           \
    hipLaunchKernelGGL((gemm_i8_kernel<BM, BN, WM, WN, MODE, ACT, TC>), dim3((unsigned)grid), dim3(WM * WN * 64), 0, st, a, (int)tiles_n, \
                       (int)tiles_l, parts)
    if (a.act == ACT_GELU) SF_I8_GEMM(ACT_GELU);
    else if (a.act == ACT_RELU) SF_I8_GEMM(ACT_RELU);
    else if constexpr (MODE == I8_OUT) SF_I8_GEMM(ACT_NONE);
#undef SF_I8_GEMM
    return check_launch("gemm_i8");
}

}  // namespace

int gemm_i8_parts(const GemmI8 &a) { return ceil_div(a.N, 128); }

int32_t gemm_i8(I8Mode mode, const GemmI8 &a0, hipStream_t st)
{
    GemmI8 a = a0;
    if (a.P <= 1) { a.L *= a.B; a.B = 1; }                   // one weight set: tiles may hold rows of several samples
    if (mode == I8_AMAX) return launch_act<128, 128, 2, 2, I8_AMAX, h16>(a, st);
    if (mode == I8_CODES) return launch_act<128, 128, 2, 2, I8_CODES, h16>(a, st);
    if (a.c_f32) return launch_act<128, 128, 2, 2, I8_OUT, float>(a, st);
    return launch_act<128, 128, 2, 2, I8_OUT, h16>(a, st);
}

}  // namespace sf
