// C = epilogue(A W^T) on the integer matrix cores: codes of rows and of output features, exact sums in 32 bits (a product of two codes is at
// most 2^14, so K up to 65 536 cannot overflow).
//
// A workgroup owns BM rows x BN features.  Both operands go straight from memory into LDS, 128 bytes of K a stage; a wave of it
// computes 32 x 32 blocks with mfma_i32_32x32x32_i8.  W is the instruction's first operand, so that a lane ends up with one row and runs of four
// features.  What lies past the last row, feature or K reads as zeros: the buffer loads are out of range there.
#include <atomic>

#include "i8.hpp"

namespace sf {

namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;
typedef __attribute__((address_space(3))) void lds_void;

// BM x BN values a workgroup, WM x WN waves, NS stages of 128 bytes of K in LDS
template <int BM, int BN, int WM, int WN, int NS, int MODE, int ACT, class TC>
__global__ __launch_bounds__(WM *WN * 64) void gemm_i8_kernel(GemmI8 a, int tiles_n, int tiles_l, int n_parts)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int BK = 128, NT = WM * WN * 64, LX = BM * 8 / NT, LW = BN * 8 / NT;           // 16-byte pieces a thread moves per stage
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32, STAGE = (BM + BN) * BK;
    static_assert(LX > 0 && LW > 0 && NT % 64 == 0, "every thread moves the same number of pieces");
    extern __shared__ __attribute__((aligned(128))) char lds[];                    // NS stages
    __shared__ __attribute__((aligned(16))) float sws[BN], bs[BN];
    __shared__ uint32_t red[MODE == I8_OUT ? 1 : WN * BM];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, hi = lane >> 5;
    const int wm = wave / WN, wn = wave % WN;
    // an XCD walks a contiguous run of tiles, the features of a row tile one after the other: its L2 reads the rows once
    const int total = gridDim.x, q8 = total / 8, r8 = total % 8, xcd = blockIdx.x % 8;
    const int t = xcd * q8 + (xcd < r8 ? xcd : r8) + blockIdx.x / 8;
    const int tn = t % tiles_n, tm = t / tiles_n;
    const int64_t b = tm / tiles_l, i0 = (int64_t)(tm % tiles_l) * BM, row0 = b * a.L + i0, all_rows = a.B * a.L;
    const int64_t left = a.L - i0;                                                 // rows of this sample from row0 on
    const int rows = left < BM ? (int)left : BM, n0 = tn * BN;
    const int p = a.P > 1 && a.pattern_id ? a.pattern_id[b] : 0;
    const int8_t *A = a.A + row0 * a.lda, *W = a.W + p * a.w_pstride + (int64_t)n0 * a.ldw;
    const int feats = a.N - n0 < BN ? a.N - n0 : BN;
    const auto ar = __builtin_amdgcn_make_buffer_rsrc((void *)A, 0, (int)((rows - 1) * a.lda + a.K), 0x00020000);
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, (int)((feats - 1) * a.ldw + a.K), 0x00020000);
    // piece q of a stage: row q / 8, chunk (q % 8) ^ (row % 8) of its eight, so that 16 lanes of a fragment read meet no bank twice
    const int chunk = (threadIdx.x & 7) ^ ((threadIdx.x >> 3) & 7);
    const int xoff = (threadIdx.x >> 3) * (int)a.lda + chunk * 16, woff = (threadIdx.x >> 3) * (int)a.ldw + chunk * 16;
    const int xstep = NT / 8 * (int)a.lda, wstep = NT / 8 * (int)a.ldw;
    auto fetch = [&](int kt, int s) {
        char *base = lds + s * STAGE + wave * 1024;
        const bool in = kt * BK + chunk * 16 < a.K;
        const int xo = in ? xoff + kt * BK : 0x7ffffff0 - LX * xstep, wo = in ? woff + kt * BK : 0x7ffffff0 - LW * wstep;
#pragma unroll
        for (int j = 0; j < LX; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (lds_void *)(base + j * (NT * 16)), 16, xo + j * xstep, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < LW; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void *)(base + BM * BK + j * (NT * 16)), 16, wo + j * wstep, 0, 0, 0);
    };
    const int kts = (a.K + BK - 1) / BK;
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) fetch(s, s);            // past the last one: zeros
    // what the end needs, while the first stages come in
    const float *sw = a.sw + p * a.sw_pstride;
    for (int n = threadIdx.x; n < BN; n += NT) {
        const bool in = n0 + n < a.N;
        sws[n] = in ? sw[n0 + n] : 0.f;
        bs[n] = !in || !a.bias ? 0.f : a.bias_f32 ? ((const float *)a.bias)[p * a.bias_pstride + n0 + n] : (float)((const h16 *)a.bias)[p * a.bias_pstride + n0 + n];
    }
    float sa[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) { const int l = (wm * TM + i) * 32 + r; sa[i] = l < rows ? a.sa[row0 + l] : 0.f; }
    if constexpr (MODE == I8_CODES) {
        for (int l = threadIdx.x; l < rows; l += NT) {
            uint32_t m = 0;
            for (int q = 0; q < n_parts; ++q) { const uint32_t u = __float_as_uint(a.part[q * all_rows + row0 + l]); m = m > u ? m : u; }
            red[l] = m;
            if (tn == 0) a.scale[row0 + l] = m < 0x7f800000u ? __uint_as_float(m) / 127.0f : __uint_as_float(0x7fc00000u);
        }
    }
    i32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    int slot = 0, ahead = NS - 1;
    for (int kt = 0; kt < kts; ++kt) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * (LX + LW)) : "memory");
        lds_barrier();                                       // stage kt is there, and nobody reads the one before it any more
        fetch(kt + NS - 1, ahead);
        const char *xs = lds + slot * STAGE + (wm * TM * 32 + r) * BK, *ws = lds + slot * STAGE + (BM + wn * TN * 32 + r) * BK;
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
        slot = slot + 1 == NS ? 0 : slot + 1;
        ahead = ahead + 1 == NS ? 0 : ahead + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // the zeros past the end are in LDS: the launch's memory is its own again
    if constexpr (MODE == I8_CODES) __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int li = (wm * TM + i) * 32 + r;                // row inside the tile
        const bool there = li < rows;
        const int64_t row = row0 + li;
        [[maybe_unused]] float cr = 0.f;
        [[maybe_unused]] uint32_t most = 0;
        if constexpr (MODE == I8_CODES) {
            // below 2^-100 a row counts as zeros: 127 / amax would overflow
            const uint32_t m = there ? red[li] : 0;
            cr = m < 0x7f800000u && __uint_as_float(m) >= 0x1p-100f ? 127.0f / __uint_as_float(m) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            [[maybe_unused]] uint32_t w[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int nl = (wn * TN + j) * 32 + q * 8 + hi * 4, n = n0 + nl;
                const f32x4 s = *reinterpret_cast<const f32x4 *>(sws + nl), bv = *reinterpret_cast<const f32x4 *>(bs + nl);
                f32x4 z;
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = activate<TC>(ACT, (float)acc[i][j][q * 4 + e] * sa[i] * s[e] + bv[e]);
                if constexpr (MODE == I8_AMAX) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) { const uint32_t u = abs_bits(z[e]); most = most > u ? most : u; }
                } else if constexpr (MODE == I8_CODES) {
                    // a value at the border of two codes carries the rounding of its own fp32 sum: no exact decision here
                    int c[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[e] = cr == 0.f ? 0 : (int)__builtin_rintf(z[e] * cr);
                    w[q] = pack4_i8(c[0], c[1], c[2], c[3]);
                } else {
                    if (a.R && there) {
                        const f32x4 rv = four((const TC *)a.R + row * a.ldr, n, a.N);
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[e] += rv[e];
                    }
                    if constexpr (sizeof(TC) == 2) { w[2 * q] = pack2_h16(z[0], z[1]); w[2 * q + 1] = pack2_h16(z[2], z[3]); }
                    else if (there) {
                        float *C = (float *)a.C + row * a.ldc + n;
                        if (n + 4 <= a.N && !((uintptr_t)C & 15)) *reinterpret_cast<f32x4 *>(C) = z;
                        else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) if (n + e < a.N) C[e] = z[e];
                        }
                    }
                }
            }
            // a lane has four features of every eight, its other half the others: swapped, each has sixteen bytes in a row
            if constexpr (MODE == I8_CODES) {
                const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                const int n = n0 + (wn * TN + j) * 32 + hi * 16;
                if (there && n < a.N) *reinterpret_cast<uint4 *>(a.codes + row * a.N + n) = make_uint4(x[0], x[1], y[0], y[1]);      // N % 64 == 0
            } else if constexpr (MODE == I8_OUT && sizeof(TC) == 2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const auto x = __builtin_amdgcn_permlane32_swap(w[4 * h], w[4 * h + 2], false, false), y = __builtin_amdgcn_permlane32_swap(w[4 * h + 1], w[4 * h + 3], false, false);
                    const int n = n0 + (wn * TN + j) * 32 + h * 16 + hi * 8;
                    h16 *C = (h16 *)a.C + row * a.ldc + n;
                    const uint4 o = make_uint4(x[0], y[0], x[1], y[1]);
                    if (!there) continue;
                    if (n + 8 <= a.N && !((uintptr_t)C & 15)) *reinterpret_cast<uint4 *>(C) = o;
                    else {
                        const h16x8 v = __builtin_bit_cast(h16x8, o);
#pragma unroll
                        for (int e = 0; e < 8; ++e) if (n + e < a.N) C[e] = v[e];
                    }
                }
            }
        }
        if constexpr (MODE == I8_AMAX) {
            const auto o = __builtin_amdgcn_permlane32_swap(most, most, false, false);
            if (hi == 0) red[wn * BM + li] = o[0] > o[1] ? o[0] : o[1];
        }
    }
    if constexpr (MODE == I8_AMAX) {
        __syncthreads();
        for (int l = threadIdx.x; l < rows; l += NT) {
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < WN; ++w) { const uint32_t u = red[w * BM + l]; m = m > u ? m : u; }
            a.part[tn * all_rows + row0 + l] = __uint_as_float(m);
        }
    }
#endif
}

template <int BM, int BN, int WM, int WN, int NS, int MODE, int ACT, class TC>
int32_t launch(const GemmI8 &a, hipStream_t st)
{
    const int64_t tiles_l = (a.L + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN, grid = a.B * tiles_l * tiles_n;
    if (grid > 0x7fffffff) return fail(SF_ERR_SHAPE, "gemm_i8: too many tiles");
    auto kern = gemm_i8_kernel<BM, BN, WM, WN, NS, MODE, ACT, TC>;
    constexpr int LDS = NS * (BM + BN) * 128;
    static std::atomic<bool> attr_set{false};     // setting the attribute twice is harmless
    if (!attr_set) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess)
            return fail(SF_ERR_HIP, "gemm_i8: cannot reserve LDS");
        attr_set = true;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(WM * WN * 64), LDS, st, a, (int)tiles_n, (int)tiles_l, gemm_i8_parts(a));
    return check_launch("gemm_i8");
}
template <int BM, int BN, int WM, int WN, int NS, int MODE, class TC>
int32_t launch_act(const GemmI8 &a, hipStream_t st)
{
    if (a.act == ACT_GELU) return launch<BM, BN, WM, WN, NS, MODE, ACT_GELU, TC>(a, st);
    if (a.act == ACT_RELU) return launch<BM, BN, WM, WN, NS, MODE, ACT_RELU, TC>(a, st);
    if constexpr (MODE == I8_OUT) return launch<BM, BN, WM, WN, NS, MODE, ACT_NONE, TC>(a, st);
    return fail(SF_ERR_UNSUPPORTED, "gemm_i8: this mode takes an activation");
}

// Tiles: 128 x 128 where they give every compute unit one, 64 x 64 or 32 x 64 with more stages ahead where they do not
enum Tile { BIG, MIDDLE, SMALL };
Tile tile_of(const GemmI8 &a)
{
    const int64_t samples = a.P > 1 ? a.B : 1, L = a.P > 1 ? a.L : a.B * a.L;
    auto tiles = [&](int m, int n) { return samples * ((L + m - 1) / m) * ((a.N + n - 1) / n); };
    return tiles(128, 128) >= 256 ? BIG : tiles(64, 64) >= 256 ? MIDDLE : SMALL;
}
template <int MODE, class TC>
int32_t launch_tile(const GemmI8 &a, hipStream_t st)
{
    switch (tile_of(a)) {
    case BIG: return launch_act<128, 128, 2, 2, 2, MODE, TC>(a, st);
    case MIDDLE: return launch_act<64, 64, 2, 2, 4, MODE, TC>(a, st);
    default: return launch_act<32, 64, 1, 2, 5, MODE, TC>(a, st);
    }
}

}  // namespace

int gemm_i8_parts(const GemmI8 &a) { return ceil_div(a.N, tile_of(a) == BIG ? 128 : 64); }

int32_t gemm_i8(I8Mode mode, const GemmI8 &a0, hipStream_t st)
{
    GemmI8 a = a0;
    if (a.P <= 1) { a.L *= a.B; a.B = 1; }                   // one weight set: tiles may hold rows of several samples
    if (mode == I8_AMAX) return launch_tile<I8_AMAX, h16>(a, st);
    if (mode == I8_CODES) return launch_tile<I8_CODES, h16>(a, st);
    if (a.c_f32) return launch_tile<I8_OUT, float>(a, st);
    return launch_tile<I8_OUT, h16>(a, st);
}

}  // namespace sf
