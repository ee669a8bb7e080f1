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

__device__ __forceinline__ float plain_nan(float x) { return x == x ? x : __uint_as_float(0x7fc00000u); }

// A value that is the same in all lanes, where the compiler does not see it
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// Between stages: this wave's LDS reads have returned.  Not __syncthreads() nor a fence of LDS alone: both wait for the fetches into LDS of later stages.
__device__ __forceinline__ void barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The largest |activation| of a lane's values, as bits (a NaN is larger than everything).  GELU is evaluated at three of them: |gelu| rises up to its
// bump at z = -0.7518, falls to 0 and rises again, so its largest value is at the largest z or next to the bump, from either side.
// ReLU: as integers, negative values are below zero (a NaN comes without a sign: scales and biases are brought to that).
template <int ACT> struct Largest {
    int m = 0;
    __device__ __forceinline__ void take(float z) { const int u = __float_as_int(z); m = m > u ? m : u; }
    __device__ __forceinline__ uint32_t bits() const { return (uint32_t)m; }
};
template <> struct Largest<ACT_GELU> {
    float top = -INFINITY, below = -INFINITY, above = INFINITY, bad = 0.f;
    __device__ __forceinline__ void take(float z)
    {
        top = fmaxf(top, z);
        below = fmaxf(below, z <= -0.7518f ? z : -INFINITY);
        above = fminf(above, z >= -0.7518f ? z : INFINITY);
        bad = fmaf(z, 0.f, bad);                             // NaN from a NaN or an infinity: both make codes of NaN
    }
    __device__ __forceinline__ uint32_t bits() const
    {
        if (!(bad == 0.f)) return 0x7fc00000u;
        float m = top > 0.f ? gelu_erf(top) : 0.f;
        if (below > -INFINITY) m = fmaxf(m, fabsf(gelu_erf(below)));
        if (above < INFINITY) m = fmaxf(m, fabsf(gelu_erf(above)));
        return __float_as_uint(m);
    }
};

// Four features from n on of a row of fp32
__device__ __forceinline__ void store4(float *row, int n, int N, f32x4 z)
{
    float *C = row + n;
    if (n + 4 <= N && !((uintptr_t)C & 15)) *reinterpret_cast<f32x4 *>(C) = z;
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (n + e < N) C[e] = z[e];
    }
}
// A lane has four features of every eight of a block of 32, its other half the others: swapped, each has sixteen bytes in a row.
// Codes, four to a word (N % 64 == 0)
__device__ __forceinline__ void store_codes(const GemmI8 &a, const uint32_t *w, int64_t row, int n32, int hi, bool there)
{
    const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const int n = n32 + hi * 16;
    if (there && n < a.N) *reinterpret_cast<uint4 *>(a.codes + row * a.N + n) = make_uint4(x[0], x[1], y[0], y[1]);
}
// 16-bit values, two to a word
__device__ __forceinline__ void store_halves(const GemmI8 &a, const uint32_t *w, int64_t row, int n32, int hi, bool there)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const auto x = __builtin_amdgcn_permlane32_swap(w[4 * h], w[4 * h + 2], false, false), y = __builtin_amdgcn_permlane32_swap(w[4 * h + 1], w[4 * h + 3], false, false);
        const int n = n32 + h * 16 + hi * 8;
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
        sws[n] = in ? plain_nan(sw[n0 + n]) : 0.f;
        bs[n] = !in || !a.bias ? 0.f : plain_nan(a.bias_f32 ? ((const float *)a.bias)[p * a.bias_pstride + n0 + n] : (float)((const h16 *)a.bias)[p * a.bias_pstride + n0 + n]);
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
        barrier();                                       // stage kt is there, and nobody reads the one before it any more
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
        [[maybe_unused]] Largest<ACT> most;
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
                for (int e = 0; e < 4; ++e) z[e] = fmaf((float)acc[i][j][q * 4 + e] * sa[i], s[e], bv[e]);
                if constexpr (MODE != I8_AMAX) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] = activate<TC>(ACT, z[e]);
                }
                if constexpr (MODE == I8_AMAX) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) most.take(z[e]);
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
                    else if (there) store4((float *)a.C + row * a.ldc, n, a.N, z);
                }
            }
            if constexpr (MODE == I8_CODES) store_codes(a, w, row, n0 + (wn * TN + j) * 32, hi, there);
            else if constexpr (MODE == I8_OUT && sizeof(TC) == 2) store_halves(a, w, row, n0 + (wn * TN + j) * 32, hi, there);
        }
        if constexpr (MODE == I8_AMAX) {
            const uint32_t m = most.bits();
            const auto o = __builtin_amdgcn_permlane32_swap(m, m, false, false);
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

// Many rows and features: 256 x 256 values a workgroup, 128 x 128 a wave, one wave per SIMD.  A wave then reads eight fragments for sixteen products
// and the LDS keeps ahead of the matrix cores (1536 of 2048 clocks per stage, with its writes; tiles of 128 x 128 need 1536 of 1024 and took 181 us for
// 65 536 x 768 with K 2176, these 146).  Stages of 128 bytes of K - whole lines: with stages of 64 or 32 bytes the fetches were what took the time, 173 and 228 us.
// Fragments are read one step of 32 bytes ahead, across the stages: the wait for the next one stands before a stage's last step.
template <int ACT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
void gemm_i8_wide_kernel(GemmI8 a, int tiles_n, int tiles_l, int in_line)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int BM = 256, BN = 256, BK = 128, STAGE = (BM + BN) * BK;
    extern __shared__ __attribute__((aligned(128))) char lds[];                    // [NS][rows, features][128]
    __shared__ __attribute__((aligned(16))) float sws[BN], bs[BN];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, hi = lane >> 5;
    const int wm = wave >> 1, wn = wave & 1, kts = (a.K + BK - 1) / BK;
    // an XCD walks a contiguous run of tiles, the features of a row tile one after the other: its L2 reads the rows once
    const int total = gridDim.x, q8 = total / 8, r8 = total % 8, xcd = blockIdx.x % 8;
    const int t = xcd * q8 + (xcd < r8 ? xcd : r8) + blockIdx.x / 8;
    const int tn = t % tiles_n, tm = t / tiles_n;
    const int64_t b = tm / tiles_l, i0 = (int64_t)(tm % tiles_l) * BM, row0 = uniform(b * a.L + i0), left = a.L - i0;
    const int rows = __builtin_amdgcn_readfirstlane(left < BM ? (int)left : BM), n0 = tn * BN, feats = a.N - n0 < BN ? a.N - n0 : BN;
    const int p = a.P > 1 && a.pattern_id ? __builtin_amdgcn_readfirstlane(a.pattern_id[b]) : 0;
    const auto ar = __builtin_amdgcn_make_buffer_rsrc((void *)(a.A + uniform(row0 * a.lda)), 0, __builtin_amdgcn_readfirstlane((rows - 1) * (int)a.lda + a.K), 0x00020000);
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void *)(a.W + uniform(p * a.w_pstride + (int64_t)n0 * a.ldw)), 0,
                                                      __builtin_amdgcn_readfirstlane((feats - 1) * (int)a.ldw + a.K), 0x00020000);
    // piece q of a stage: row q / 8, chunk (q % 8) ^ (row % 8) of its eight, so that 16 lanes of a fragment read meet no bank twice
    const int chunk = (threadIdx.x & 7) ^ ((threadIdx.x >> 3) & 7);
    const int xoff = (threadIdx.x >> 3) * (int)a.lda + chunk * 16, woff = (threadIdx.x >> 3) * (int)a.ldw + chunk * 16;
    const int xstep = 32 * (int)a.lda, wstep = 32 * (int)a.ldw;
    // the wave's j-th KB of a stage, rows (0 .. 7) and features (8 .. 15); past the last stage zeros
    auto fetch = [&](int kt, int s, int j) {
        char *base = lds + s * STAGE + wave * 1024 + j * 4096;
        const bool in = kt * BK + chunk * 16 < a.K;
        if (j < 8) __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (lds_void *)base, 16, in ? xoff + kt * BK + j * xstep : 0x7ffffff0, 0, 0, 0);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void *)base, 16, in ? woff + kt * BK + (j - 8) * wstep : 0x7ffffff0, 0, 0, 0);
    };
#pragma unroll
    for (int j = 0; j < 16; ++j) fetch(0, 0, j);
    {
        const int n = n0 + threadIdx.x;
        const bool in = n < a.N;
        sws[threadIdx.x] = in ? a.sw[p * a.sw_pstride + n] : 0.f;
        bs[threadIdx.x] = !in || !a.bias ? 0.f : a.bias_f32 ? ((const float *)a.bias)[p * a.bias_pstride + n] : (float)((const h16 *)a.bias)[p * a.bias_pstride + n];
    }
    float sa[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const int l = (wm * 4 + i) * 32 + r; sa[i] = l < rows ? a.sa[row0 + l] : 0.f; }
    __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0): from here on the compiler has nothing of its own to wait for
    i32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const int xrow = (wm * 128 + r) * BK, wrow = BM * BK + (wn * 128 + r) * BK;
    int at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = ((k * 2 + hi) ^ (r & 7)) * 16;
    i32x4 xf[2][4], wf[2][4];
    auto read = [&](int slot, int k) {
        const char *base = lds + slot * STAGE + at[k];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            xf[k & 1][i] = *reinterpret_cast<const i32x4 *>(base + xrow + i * 32 * BK);
            wf[k & 1][i] = *reinterpret_cast<const i32x4 *>(base + wrow + i * 32 * BK);
        }
        __builtin_amdgcn_sched_barrier(0);                   // in this order: the reads return while the products run
    };
    // A fetch holds up its wave's issue for some 100 clocks where others stand before it (all sixteen in a row: 157 us for K 2176): one or two, then four
    // products
    auto multiply = [&](int k, int kt, int slot, int from, int to) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[k & 1][j], xf[k & 1][i], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int f = from + i * (to - from) / 4; f < from + (i + 1) * (to - from) / 4; ++f) fetch(kt, slot, f);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    barrier();
#pragma unroll
    for (int j = 0; j < 6; ++j) fetch(1, 1, j);
    read(0, 0);
    for (int kt = 0; kt < kts; ++kt) {
        const int slot = kt & 1;
        read(slot, 1);
        multiply(0, kt + 1, slot ^ 1, 6, 12);
        read(slot, 2);
        multiply(1, kt + 1, slot ^ 1, 12, 16);
        read(slot, 3);
        multiply(2, 0, 0, 0, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        barrier();                                           // stage kt + 1 is there, and nobody reads kt any more
        read(slot ^ 1, 0);                                   // behind the last stage: zeros, multiplied by nobody
        multiply(3, kt + 2, slot, 0, 6);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                      // the zeros past the end are in LDS: the launch's memory is its own again
    // Whole features, rows that start on 16 bytes: stores and residual through buffers that end behind the last row.  The residual comes sixteen
    // bytes in a row, as the values leave, and is exchanged between the halves as they are.
    if (in_line && n0 + BN <= a.N) {
        const auto cr = __builtin_amdgcn_make_buffer_rsrc((void *)((h16 *)a.C + uniform(row0 * a.ldc + n0)), 0,
                                                          __builtin_amdgcn_readfirstlane(((rows - 1) * (int)a.ldc + BN) * 2), 0x00020000);
        const auto rr = __builtin_amdgcn_make_buffer_rsrc((void *)((const h16 *)a.R + uniform(row0 * a.ldr + n0)), 0,
                                                          a.R ? __builtin_amdgcn_readfirstlane(((rows - 1) * (int)a.ldr + BN) * 2) : 0, 0x00020000);
        int co[4], ro[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int l = (wm * 4 + i) * 32 + r, col = (wn * 128 + hi * 8) * 2;
            co[i] = l < rows ? l * (int)a.ldc * 2 + col : 0x7fff0000;
            ro[i] = l < rows ? l * (int)a.ldr * 2 + col : 0x7fff0000;
        }
        i32x4 res[2][4][2];
        auto residual = [&](int j) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) res[j & 1][i][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rr, ro[i] + j * 64 + h * 32, 0, 0));
        };
        if (a.R) residual(0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (a.R && j < 3) residual(j + 1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 s[2], bv[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int nl = (wn * 4 + j) * 32 + (2 * h + q) * 8 + hi * 4;
                    s[q] = *reinterpret_cast<const f32x4 *>(sws + nl);
                    bv[q] = *reinterpret_cast<const f32x4 *>(bs + nl);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 z[2];
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[q][e] = activate<h16>(ACT, fmaf((float)acc[i][j][(2 * h + q) * 4 + e] * sa[i], s[q][e], bv[q][e]));
                    if (a.R) {
                        const i32x4 v = res[j & 1][i][h];
                        const auto x = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false), y = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const h16x4 rv = __builtin_bit_cast(h16x4, make_uint2(x[q], y[q]));
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[q][e] += (float)rv[e];
                        }
                    }
                    const auto x = __builtin_amdgcn_permlane32_swap(pack2_h16(z[0][0], z[0][1]), pack2_h16(z[1][0], z[1][1]), false, false);
                    const auto y = __builtin_amdgcn_permlane32_swap(pack2_h16(z[0][2], z[0][3]), pack2_h16(z[1][2], z[1][3]), false, false);
                    __builtin_amdgcn_raw_buffer_store_b128(i32x4{(int)x[0], (int)y[0], (int)x[1], (int)y[1]}, cr, co[i] + j * 64 + h * 32, 0, 0);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int li = (wm * 4 + i) * 32 + r;            // row inside the tile
            const bool there = li < rows;
            const int64_t row = row0 + li;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[8];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int nl = (wn * 4 + j) * 32 + q * 8 + hi * 4;
                    const f32x4 s = *reinterpret_cast<const f32x4 *>(sws + nl), bv = *reinterpret_cast<const f32x4 *>(bs + nl);
                    f32x4 z;
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[e] = activate<h16>(ACT, fmaf((float)acc[i][j][q * 4 + e] * sa[i], s[e], bv[e]));
                    if (a.R && there) {
                        const f32x4 rv = four((const h16 *)a.R + row * a.ldr, n0 + nl, a.N);
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[e] += rv[e];
                    }
                    w[2 * q] = pack2_h16(z[0], z[1]);
                    w[2 * q + 1] = pack2_h16(z[2], z[3]);
                }
                store_halves(a, w, row, n0 + (wn * 4 + j) * 32, hi, there);
            }
        }
    }
#endif
}

// Many rows, short K, codes out: the weights stay in registers.  One wave per SIMD holds TF x 32 features whole (KS steps of 32 bytes of K: 24 of
// three blocks are 288 of its 512 registers), and every 32 rows pass by it once, through LDS.  A tile kernel reads a row and a feature fragment
// from LDS for every two or four products; here a row fragment serves TF of them and the features none.  The values of one step are finished (scales,
// activation, codes) between the products of the next, into whose accumulators they do not go.  A workgroup owns a group of features and a run of
// rows; where the run comes to a sample of another pattern the weights are fetched again.  65 536 rows, K 768, 2176 features: largest values 114 us, codes
// 124 (tiles of 128 x 128: 145 and 230).
// Waiting: a wave's memory operations complete in order as far as vmcnt tells, and it issues the same number each step: F fetches into LDS and E
// stores (out of range where there is nothing to store).  The last fetch of step s may be the last operation of the turn that issues it; NS - 2 turns
// follow before it is waited for.
template <int KS, int TF, int MODE, int ACT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
void gemm_i8_held_kernel(GemmI8 a, int groups, int per, int steps_l, int total_steps)
{
#if defined(__HIP_DEVICE_COMPILE__)
    static_assert(MODE != I8_OUT, "codes, or their rows' largest values");
    constexpr int RB = KS * 32, TILE = 32 * RB, SLOT = TILE + 512, NS = KS <= 16 ? 6 : 4, CH = KS * 2, NF = 4 * TF * 32;
    constexpr int F = KS / 4 + (MODE == I8_CODES ? 2 : 1), E = MODE == I8_CODES ? TF : 1;
    extern __shared__ __attribute__((aligned(128))) char lds[];                    // [NS][32 rows of codes, 64 scales, 64 largest values]
    __shared__ __attribute__((aligned(16))) float sws[NF], bs[NF];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, hi = lane >> 5;
    const int group = blockIdx.x % groups, at = blockIdx.x / groups, blocks = gridDim.x / groups;
    const int first = __builtin_amdgcn_readfirstlane((int)((int64_t)total_steps * at / blocks));
    const int last = __builtin_amdgcn_readfirstlane((int)((int64_t)total_steps * (at + 1) / blocks));
    if (first >= last) return;
    const int64_t all_rows = a.B * a.L;
    const int f0 = group * per * TF * 32, n0 = f0 + wave * TF * 32;
    const bool works = wave < per && n0 < a.N;
    struct Step { int64_t row0; int b, rows; };
    auto step_of = [&](int s) {
        const int b = s / steps_l, i0 = (s - b * steps_l) * 32;
        const int64_t left = a.L - i0;
        return Step{uniform(b * a.L + i0), b, __builtin_amdgcn_readfirstlane(left < 32 ? (int)left : 32)};
    };
    // a wave fetches KS / 4 KB of the 32 rows; chunk c of row r lies at c ^ (r % 8), so that 16 lanes of a fragment read meet no bank twice
    int off[KS / 4];
#pragma unroll
    for (int j = 0; j < KS / 4; ++j) {
        const int q = (j * 4 + wave) * 64 + lane, row = q / CH, chunk = (q - row * CH) ^ (row & 7);
        off[j] = chunk * 16 < a.K ? row * (int)a.lda + chunk * 16 : 0x7ffffff0;
    }
    // the wave's j-th fetch of a step: KS / 4 KB of codes, the scales, the largest values; past the last step zeros
    struct Aim { int64_t a, row0; int an, rows; char *base; };
    auto aim = [&](int s, int slot) {
        const Step st = step_of(s < last ? s : last - 1);
        const int rows = s < last ? st.rows : 0;
        return Aim{uniform(st.row0 * a.lda), st.row0, __builtin_amdgcn_readfirstlane(rows ? (rows - 1) * (int)a.lda + a.K : 0), rows, lds + slot * SLOT};
    };
    auto fetch = [&](const Aim &m, int j) {
        if (j < KS / 4) {
            const auto ar = __builtin_amdgcn_make_buffer_rsrc((void *)(a.A + m.a), 0, m.an, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (lds_void *)(m.base + (j * 4 + wave) * 1024), 16, off[j], 0, 0, 0);
        } else {
            // every wave brings the same 32 values (and 32 zeros): the count of its operations is what matters
            const auto sr = __builtin_amdgcn_make_buffer_rsrc((void *)((j == KS / 4 ? a.sa : a.top) + m.row0), 0, __builtin_amdgcn_readfirstlane(m.rows * 4), 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, (lds_void *)(m.base + TILE + (j - KS / 4) * 256), 4, lane * 4, 0, 0, 0);
        }
    };
    i32x4 w[TF][KS];
    auto weights = [&](int p) {
        const int8_t *W = a.W + p * a.w_pstride;
        const int feats = a.N - n0 < TF * 32 ? a.N - n0 : TF * 32;
        const auto wr = __builtin_amdgcn_make_buffer_rsrc((void *)(W + uniform((int64_t)n0 * a.ldw)), 0,
                                                          __builtin_amdgcn_readfirstlane(works ? (feats - 1) * (int)a.ldw + a.K : 0), 0x00020000);
#pragma unroll
        for (int j = 0; j < TF; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int c = (k * 2 + hi) * 16;
                w[j][k] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, c < a.K ? (j * 32 + r) * (int)a.ldw + c : 0x7ffffff0, 0, 0));
            }
        for (int i = threadIdx.x; i < NF; i += 256) {
            const int n = f0 + i;
            sws[i] = n < a.N ? plain_nan(a.sw[p * a.sw_pstride + n]) : 0.f;
            bs[i] = n >= a.N || !a.bias ? 0.f : plain_nan(a.bias_f32 ? ((const float *)a.bias)[p * a.bias_pstride + n] : (float)((const h16 *)a.bias)[p * a.bias_pstride + n]);
        }
    };
    // the last step's rows and what belongs to them
    Step prev{0, 0, 0};
    float sa = 0.f, cr = 0.f;
    [[maybe_unused]] Largest<ACT> most;
    [[maybe_unused]] uint32_t o[4];
    f32x4 sv[2], bv[2];
    auto scales = [&](int g) {                               // of the g-th four features of a wave
        const int nl = wave * TF * 32 + g * 8 + hi * 4;
        sv[g & 1] = *reinterpret_cast<const f32x4 *>(sws + nl);
        bv[g & 1] = *reinterpret_cast<const f32x4 *>(bs + nl);
    };
    [[maybe_unused]] uint32_t c4[4];
    i32x16 done[TF];                                         // the sums of the step before
#pragma unroll
    for (int j = 0; j < TF; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) done[j][e] = 0;
    auto value = [&](int v) {                                // the v-th of a lane's values of the last step
        const int j = v / 16, g = v / 4, q = g % 4, e = v % 4;
        if (e == 0 && g + 1 < 4 * TF) scales(g + 1);
        const float z = fmaf((float)done[j][v % 16] * sa, sv[g & 1][e], bv[g & 1][e]);
        if constexpr (MODE == I8_AMAX) most.take(z);
        else {
            // rounded by the addition of 1.5 2^23: the code is the low byte of the sum, 0 where it is NaN
            c4[e] = __float_as_uint(fmaf(ACT == ACT_RELU ? fmaxf(z, 0.f) : activate<h16>(ACT, z), cr, 12582912.f));
            if (e == 3) o[q] = __builtin_amdgcn_perm(c4[1], c4[0], 0x0c0c0400u) | __builtin_amdgcn_perm(c4[3], c4[2], 0x04000c0cu);
            if (e == 3 && q == 3) {
                const auto x = __builtin_amdgcn_permlane32_swap(o[0], o[2], false, false), y = __builtin_amdgcn_permlane32_swap(o[1], o[3], false, false);
                const int n = n0 + j * 32 + hi * 16;
                const auto cr_ = __builtin_amdgcn_make_buffer_rsrc((void *)(a.codes + uniform(prev.row0 * a.N)), 0, __builtin_amdgcn_readfirstlane(prev.rows * a.N), 0x00020000);
                __builtin_amdgcn_raw_buffer_store_b128(i32x4{(int)x[0], (int)x[1], (int)y[0], (int)y[1]}, cr_, works && n < a.N ? r * a.N + n : 0x7ffffff0, 0, 0);
            }
        }
    };
    auto finish = [&]() {                                    // the last step's rows: their largest values
        if constexpr (MODE == I8_AMAX) {
            const uint32_t m = most.bits();
            const auto x = __builtin_amdgcn_permlane32_swap(m, m, false, false);
            const auto pr = __builtin_amdgcn_make_buffer_rsrc((void *)(a.part + uniform((group * per + wave) * all_rows + prev.row0)), 0,
                                                              __builtin_amdgcn_readfirstlane(prev.rows * 4), 0x00020000);
            __builtin_amdgcn_raw_buffer_store_b32((int)(x[0] > x[1] ? x[0] : x[1]), pr, works && hi == 0 ? r * 4 : 0x7ffffff0, 0, 0);
            most = Largest<ACT>();
        }
    };
    auto flush = [&]() {
        scales(0);
#pragma unroll
        for (int v = 0; v < 16 * TF; ++v) value(v);
        finish();
    };
    int slot = 0, ahead = NS - 1;
    // step s, while the one before is finished
    auto turn = [&](int s) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 2) * (F + E) < 63 ? (NS - 2) * (F + E) : 63) : "memory");
        barrier();                                           // step s is there, and nobody reads the one before it any more
        const Aim m = aim(s + NS - 1, ahead);
        const char *xs = lds + slot * SLOT + r * RB;
        const float *xsc = reinterpret_cast<const float *>(lds + slot * SLOT + TILE);
        const float sa_now = xsc[r];
        [[maybe_unused]] const float top_now = MODE == I8_CODES ? xsc[64 + r] : 0.f;
        i32x16 acc[TF];
#pragma unroll
        for (int j = 0; j < TF; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[j][e] = 0;
        i32x4 xf[2];
        xf[0] = *reinterpret_cast<const i32x4 *>(xs + (hi ^ (r & 7)) * 16);
        scales(0);
        __builtin_amdgcn_sched_barrier(0);
        // A wave issues in order: vector instructions behind the last product of a step of K overlap with that one alone (a step took 4250 clocks for
        // 2304 of products so).  They are spread: between two products stands a value's share, and nothing moves across.
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (k + 1 < KS) xf[(k + 1) & 1] = *reinterpret_cast<const i32x4 *>(xs + (((k + 1) * 2 + hi) ^ (r & 7)) * 16);
#pragma unroll
            for (int j = 0; j < TF; ++j) {
                acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[j][k], xf[k & 1], acc[j], 0, 0, 0);
                constexpr int SLOTS = KS * TF;
#pragma unroll
                for (int v = 16 * TF * (k * TF + j) / SLOTS; v < 16 * TF * (k * TF + j + 1) / SLOTS; ++v) value(v);
#pragma unroll
                for (int f = F * (k * TF + j) / SLOTS; f < F * (k * TF + j + 1) / SLOTS; ++f) fetch(m, f);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        finish();
#pragma unroll
        for (int j = 0; j < TF; ++j) done[j] = acc[j];
        prev = step_of(s);
        sa = sa_now;
        if constexpr (MODE == I8_CODES)                      // below 2^-100 a row counts as zeros: 127 / amax would overflow
            cr = __float_as_uint(top_now) < 0x7f800000u && top_now >= 0x1p-100f ? 127.0f / top_now : 0.f;
        slot = slot + 1 == NS ? 0 : slot + 1;
        ahead = ahead + 1 == NS ? 0 : ahead + 1;
    };
    for (int s = 0; s < NS - 1; ++s) {
        const Aim m = aim(first + s, s);
#pragma unroll
        for (int j = 0; j < F; ++j) fetch(m, j);
    }
    for (int s = first; s < last;) {
        // a run of steps of one pattern
        const int b0 = step_of(s).b, p = a.P > 1 && a.pattern_id ? __builtin_amdgcn_readfirstlane(a.pattern_id[b0]) : 0;
        int end = last;
        if (a.P > 1 && a.pattern_id)
            for (int b = b0 + 1; (int64_t)b * steps_l < last; ++b)
                if (__builtin_amdgcn_readfirstlane(a.pattern_id[b]) != p) { end = b * steps_l; break; }
        if (s > first) barrier();                            // the last pattern's scales have been read
        weights(p);
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0), as the compiler understands it: it would wait for the weights at their use
        barrier();
        for (; s < end; ++s) turn(s);
        flush();
        prev.rows = 0;                                       // finished: the next turn stores nothing
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                      // the zeros past the end are in LDS: the launch's memory is its own again
#endif
}

// The largest of a row's parts, and the row's scale
__global__ __launch_bounds__(256) void i8_top_kernel(const float *__restrict__ part, int n_parts, int64_t rows, float *__restrict__ top, float *__restrict__ scale)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= rows) return;
    uint32_t m = 0;
#pragma unroll 8
    for (int q = 0; q < n_parts; ++q) { const uint32_t u = __float_as_uint(part[q * rows + row]); m = m > u ? m : u; }
    top[row] = __uint_as_float(m);
    scale[row] = m < 0x7f800000u ? __uint_as_float(m) / 127.0f : __uint_as_float(0x7fc00000u);
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

// Tiles: 256 x 256 (for 16-bit values alone) where K is long and whole rounds of one per compute unit are at least 7/8 full: a workgroup's start and end
// have nothing beside them.  65 536 x 512, 256 x 256 against 128 x 128: K 512 34 and 31 us, K 1024 46 and 45 (2048 features: 181 and 184), K 2048 76
// and 100; a round 3/4 full, K 2048: 82 and 74.  128 x 128 where they give every compute unit one, 64 x 64 or 32 x 64 with more stages ahead where they do not.
enum Tile { WIDE, BIG, MIDDLE, SMALL };
Tile tile_of(const GemmI8 &a, bool values)
{
    const int64_t samples = a.P > 1 ? a.B : 1, L = a.P > 1 ? a.L : a.B * a.L;
    auto tiles = [&](int m, int n) { return samples * ((L + m - 1) / m) * ((a.N + n - 1) / n); };
    const int64_t rounds = (tiles(256, 256) + 255) / 256;
    if (values && a.K >= 1024 && 8 * samples * L * a.N >= 7 * rounds * 256 * 65536) return WIDE;
    return tiles(128, 128) >= 256 ? BIG : tiles(64, 64) >= 256 ? MIDDLE : SMALL;
}

// The kernel with held weights, by K: three or four blocks of features a wave up to 768, two up to 1024; rows enough for some steps of 32 per workgroup
struct Held { int ks, tf, groups, per, steps_l; int64_t steps; };
bool held(const GemmI8 &a, Held &h)
{
    const int64_t samples = a.P > 1 ? a.B : 1, L = a.P > 1 ? a.L : a.B * a.L;
    if (a.K > 1024 || a.lda > 1 << 20 || (L + 31) / 32 > 1 << 24) return false;
    h.ks = a.K <= 256 ? 8 : a.K <= 512 ? 16 : a.K <= 768 ? 24 : 32;
    h.tf = h.ks <= 16 ? 4 : h.ks == 24 ? 3 : 2;
    const int units = ceil_div(a.N, h.tf * 32);
    h.groups = ceil_div(units, 4);
    h.per = ceil_div(units, h.groups);
    h.steps_l = (int)((L + 31) / 32);
    h.steps = samples * h.steps_l;
    return h.steps <= 1 << 30 && h.groups <= 64 && h.steps * h.groups >= 256 * 4;
}
template <int KS, int TF, int MODE, int ACT>
int32_t launch_held(const GemmI8 &a, const Held &h, hipStream_t st)
{
    auto kern = gemm_i8_held_kernel<KS, TF, MODE, ACT>;
    constexpr int LDS = (KS <= 16 ? 6 : 4) * (KS * 1024 + 512);
    static std::atomic<bool> attr_set{false};     // setting the attribute twice is harmless
    if (!attr_set) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess)
            return fail(SF_ERR_HIP, "gemm_i8: cannot reserve LDS");
        attr_set = true;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(256 / h.groups * h.groups)), dim3(256), LDS, st, a, h.groups, h.per, h.steps_l, (int)h.steps);
    return check_launch("gemm_i8");
}
template <int MODE, int ACT>
int32_t launch_held_k(const GemmI8 &a, const Held &h, hipStream_t st)
{
    switch (h.ks) {
    case 8: return launch_held<8, 4, MODE, ACT>(a, h, st);
    case 16: return launch_held<16, 4, MODE, ACT>(a, h, st);
    case 24: return launch_held<24, 3, MODE, ACT>(a, h, st);
    default: return launch_held<32, 2, MODE, ACT>(a, h, st);
    }
}

template <int ACT>
int32_t launch_wide(const GemmI8 &a, hipStream_t st)
{
    auto kern = gemm_i8_wide_kernel<ACT>;
    constexpr int LDS = 2 * 512 * 128;
    static std::atomic<bool> attr_set{false};     // setting the attribute twice is harmless
    if (!attr_set) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess)
            return fail(SF_ERR_HIP, "gemm_i8: cannot reserve LDS");
        attr_set = true;
    }
    const int64_t tiles_l = (a.L + 255) / 256, tiles_n = (a.N + 255) / 256, grid = a.B * tiles_l * tiles_n;
    if (grid > 0x7fffffff) return fail(SF_ERR_SHAPE, "gemm_i8: too many tiles");
    const bool in_line = a.ldc % 8 == 0 && !((uintptr_t)a.C & 15) && (!a.R || (a.ldr % 8 == 0 && !((uintptr_t)a.R & 15))) && a.ldc < 1 << 21 && a.ldr < 1 << 21;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), LDS, st, a, (int)tiles_n, (int)tiles_l, (int)in_line);
    return check_launch("gemm_i8");
}
template <int MODE, class TC>
int32_t launch_tile(const GemmI8 &a, hipStream_t st)
{
    if constexpr (MODE != I8_OUT) {
        Held h;
        if (held(a, h)) {
            if (MODE == I8_CODES)
                hipLaunchKernelGGL(i8_top_kernel, dim3((unsigned)((a.B * a.L + 255) / 256)), dim3(256), 0, st, a.part, gemm_i8_parts(a), a.B * a.L, a.top, a.scale);
            return a.act == ACT_GELU ? launch_held_k<MODE, ACT_GELU>(a, h, st) : launch_held_k<MODE, ACT_RELU>(a, h, st);
        }
    }
    switch (tile_of(a, MODE == I8_OUT && sizeof(TC) == 2)) {
    case WIDE:
        if constexpr (MODE == I8_OUT && sizeof(TC) == 2)
            return a.act == ACT_GELU ? launch_wide<ACT_GELU>(a, st) : a.act == ACT_RELU ? launch_wide<ACT_RELU>(a, st) : launch_wide<ACT_NONE>(a, st);
    case BIG: return launch_act<128, 128, 2, 2, 2, MODE, TC>(a, st);
    case MIDDLE: return launch_act<64, 64, 2, 2, 4, MODE, TC>(a, st);
    default: return launch_act<32, 64, 1, 2, 5, MODE, TC>(a, st);
    }
}

}  // namespace

int gemm_i8_parts(const GemmI8 &a)
{
    Held h;
    return held(a, h) ? ceil_div(a.N, h.tf * 32) : ceil_div(a.N, tile_of(a, false) == BIG ? 128 : 64);
}

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
