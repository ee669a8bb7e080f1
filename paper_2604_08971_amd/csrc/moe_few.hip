// The Sparse-MoE FFN block of a few tokens (Sec. 4.5) in two launches.  What bounds it is the chosen experts' weights, read once, and latency.
//
//   up:    every workgroup normalises the tokens and routes them for itself (LayerNorm, logits, Top-k), then takes channels of one of the
//          chosen (pattern, expert) pairs: hidden rows in fp32, one per (token, slot)
//   down:  four features of every token: the pairs' products, the slots' sum with their weights in the order of the slots, the residual
//
// The products run on the matrix cores, weights as the first operand, tokens as the second.  An activation goes in as a sum of
// 16-bit terms, so that nothing is rounded on the way: two terms (16 bits in bfloat16, 22 in binary16) for the experts' products, three for
// the logits, whose order decides.  fp32 models take the fp32 instruction.
#include <algorithm>
#include <atomic>

#include "gemm.hpp"

namespace sf {

namespace {

constexpr int FEW = SF_MOE_FEW_TOKENS, TILE_T = 16, MAX_D = 1024, WAVES = 8, NT = WAVES * 64, STEPS = MAX_D / 32 / WAVES;      // K steps of 32 of a wave
constexpr int DOWN_WAVES = 16;
constexpr int XT_BYTES = 100 * 1024;                        // LDS that normalised tokens may take: all of them up to here, else sixteen at a time
#ifdef SF_HALF_F16
#define SF_MFMA_16X16 __builtin_amdgcn_mfma_f32_16x16x32_f16
#define SF_MFMA_4X4(w, x, acc) __builtin_amdgcn_mfma_f32_4x4x4f16(w, x, acc, 0, 0, 0)
#else
#define SF_MFMA_16X16 __builtin_amdgcn_mfma_f32_16x16x32_bf16
typedef __attribute__((ext_vector_type(4))) short s16x4;
#define SF_MFMA_4X4(w, x, acc) __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4, w), __builtin_bit_cast(s16x4, x), acc, 0, 0, 0)
#endif

struct FewMoe {
    const void *X, *Wr, *br, *ln_g, *ln_b, *W1, *b1, *W2T, *b2x;
    const int32_t *pattern_id, *forced, *k_ffn;
    int T, L, d, E, P, top_k, ffn_pad, Fp, act; float eps; int add_residual;
    int segs, by_slot, slices, parts;                        // pairs looked at (by_slot: those of each (token, slot), else all there are);
                                                             // workgroups of a pair (up), ranges of its channels (down)
    int per, feats;                                          // channels of a range; features of a workgroup (down)
    int tile_rows;                                           // normalised tokens in LDS at a time
    uint64_t *route; float *weight;                          // workspace, eight slots a token: experts in bytes (255: none, or listed again in a
                                                             // later slot), weights
    void *hid;                                               // [T k, Fp] fp32, or the two terms [2, T k, Fp] in 16 bits
    void *Y; int32_t *route_out; float *weight_out, *logit_out;
};

// Eight K elements of an operand: 16-bit models as terms whose sum they are, fp32 models as they stand
template <class T> struct Operand;
template <> struct Operand<h16> {
    h16x8 t[3];
    template <int TERMS> __device__ __forceinline__ static Operand split(const float *v)
    {
        Operand o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float r = v[e];
#pragma unroll
            for (int k = 0; k < TERMS; ++k) { const h16 h = (h16)r; o.t[k][e] = h; r -= (float)h; }
        }
        return o;
    }
    template <int TERMS> __device__ __forceinline__ f32x4 times(h16x8 w, f32x4 acc) const
    {
#pragma unroll
        for (int k = TERMS - 1; k >= 0; --k) acc = SF_MFMA_16X16(w, t[k], acc, 0, 0, 0);
        return acc;
    }
};
struct f32x8 { f32x4 a, b; };
template <> struct Operand<float> {
    f32x4 a, b;
    template <int> __device__ __forceinline__ static Operand split(const float *v) { return {{v[0], v[1], v[2], v[3]}, {v[4], v[5], v[6], v[7]}}; }
    template <int> __device__ __forceinline__ f32x4 times(f32x8 w, f32x4 acc) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w.a[e], a[e], acc, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w.b[e], b[e], acc, 0, 0, 0);
        return acc;
    }
};
template <class T> struct Weights;
template <> struct Weights<h16> { typedef h16x8 type; };
template <> struct Weights<float> { typedef f32x8 type; };
// Loads without branches, so that they stay in flight together: what is not `in` (and all of a NULL tensor) is out of range and reads as zero
typedef __amdgpu_buffer_rsrc_t Span;
__device__ __forceinline__ Span span_of(const void *p, int64_t bytes) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, __builtin_amdgcn_readfirstlane(p ? (int)bytes : 0), 0x00020000); }
constexpr int NOWHERE = 0x7ff00000;
template <class V> __device__ __forceinline__ V load16(Span s, int byte, int further)
{
    return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(s, byte, further, 0));
}
// eight elements `ahead` (a constant) and `further` (the same for all lanes) behind the lane's own
template <class T> __device__ __forceinline__ typename Weights<T>::type load8(Span s, int at, bool in, int ahead = 0, int further = 0)
{
    const int S = sizeof(T), byte = (in ? at * S : NOWHERE) + ahead * S;
    if constexpr (S == 2) return load16<h16x8>(s, byte, further * S);
    else return {load16<f32x4>(s, byte, further * S), load16<f32x4>(s, byte + 16, further * S)};
}
template <class T> __device__ __forceinline__ float load1(Span s, int at, bool in)
{
    if constexpr (sizeof(T) == 2) return (float)__builtin_bit_cast(h16, __builtin_amdgcn_raw_buffer_load_b16(s, in ? at * 2 : NOWHERE, 0, 0));
    else return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(s, in ? at * 4 : NOWHERE, 0, 0));
}

template <class T>
__device__ __forceinline__ float activated(int act, float z)
{
    if (act == ACT_RELU) return z < 0.f ? 0.f : z;
    return sizeof(T) == 4 ? 0.5f * z * (1.0f + erff(z * 0.70710678f)) : gelu_erf(z);
}

// Pattern of a lane's token
__device__ __forceinline__ int pattern_of(const FewMoe &a, int t)
{
    const int p = __builtin_amdgcn_raw_buffer_load_b32(span_of(a.pattern_id, a.T / a.L * 4), t < a.T ? t / a.L * 4 : NOWHERE, 0, 0);
    return min(max(p, 0), a.P - 1);
}

// The `nth` pair looked at: its number (pattern E + expert), and the (token, slot) in which the lane's token chose it or -1.  by_slot: the pair of
// (token, slot) nth.  picks: the experts of the lane's token, a byte each.  Registers of one wave only.
struct Pair { int seg, at, expert; };
__device__ __forceinline__ Pair find_pair(const FewMoe &a, uint64_t picks, int pattern, int nth)
{
    const int lane = threadIdx.x & 63;
    Pair p{nth, -1, 0};
    if (a.by_slot) {
        const int t = nth / a.top_k, s = nth - t * a.top_k;
        const uint64_t of = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(picks >> 32), t) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)picks, t);
        const int e = (int)(of >> (8 * s)) & 255;
        if (e == 255) return p;
        p.seg = __builtin_amdgcn_readlane(pattern, t) * a.E + e;
    }
    const uint32_t e = (uint32_t)(p.seg - pattern * a.E);    // the pair's expert, where the lane's token has its pattern
    const uint64_t x = picks ^ (uint64_t)e * 0x0101010101010101ull;                  // a zero byte where the expert is; E <= 64: none carries into the next
    const uint64_t zero = ~((((x & 0x7f7f7f7f7f7f7f7full) + 0x7f7f7f7f7f7f7f7full) | x) | 0x7f7f7f7f7f7f7f7full);
    if (e < (uint32_t)a.E && zero) p.at = lane * a.top_k + (__ffsll((unsigned long long)zero) - 1) / 8;
    const uint64_t chose = __ballot(p.at >= 0);
    if (chose) p.expert = __builtin_amdgcn_readlane((int)e, __ffsll((unsigned long long)chose) - 1);
    return p;
}
// The tokens that chose the pair: a list per wave, which that wave alone writes and reads.  0: not looked at here (none, or an earlier
// (token, slot) is of the same pair)
__device__ __forceinline__ int list_tokens(const FewMoe &a, const Pair &p, int nth, short *slots)
{
    const uint64_t chose = __ballot(p.at >= 0);
    if (a.by_slot && __ballot(p.at >= 0 && p.at < nth)) return 0;
    if (p.at >= 0) slots[__popcll(chose & ((1ull << (threadIdx.x & 63)) - 1))] = (short)p.at;
    return __popcll(chose);
}

// Channels of an expert, padded as its weights are
__device__ __forceinline__ int width_of(const FewMoe &a, int kept)
{
    const int w = (kept + a.ffn_pad - 1) / a.ffn_pad * a.ffn_pad;
    return w < a.Fp ? w : a.Fp;
}

// One wave's 16 x 16 sums over its part of K are added up in LDS: [8 waves][64][17].
//
// A launch runs this code once, so its length counts: 35 KB of it, with every loop unrolled, took 24 500 clocks for one token of eight experts, of which
// the choice of two experts alone was 5700; what is not a load ahead of its use is a loop here.
// G: runs of sixteen channels per round of a workgroup, so that its weights are on their way together.
template <class T, int G>
__global__ __launch_bounds__(NT) void moe_few_up_kernel(FewMoe a)
{
    // [tile_rows][dp + 4] normalised tokens (rows 16 bytes apart over the banks), then partial sums, then logits [T][E + 1]
    extern __shared__ __attribute__((aligned(16))) float xt[];
    __shared__ float mean[FEW], rstd[FEW];
    __shared__ uint64_t picks[FEW];
    __shared__ short slots[WAVES][FEW];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kq = (lane >> 4) * 8;
    const int d = a.d, dp = (d + 31) / 32 * 32, ld = dp + 4, steps = dp / 32, lgs = a.E + 1;
    float *red = xt + a.tile_rows * ld, *lg = red + WAVES * 64 * (TILE_T + 1);
    auto part = [&](int w, int e, int r) -> float & { return red[(w * 64 + e) * (TILE_T + 1) + r]; };
    const T *X = (const T *)a.X;
    constexpr int NCH = MAX_D / 512;
    typedef typename Weights<T>::type Eight;
    auto to_floats = [](const Eight &q, float *v) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)q[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = q.a[e]; v[4 + e] = q.b[e]; }
        }
    };
    // what does not depend on the tokens is on its way first
    const int pattern = pattern_of(a, lane), kept = __builtin_amdgcn_raw_buffer_load_b32(span_of(a.k_ffn, a.E * 4), lane * 4, 0, 0);
    const int S = sizeof(T);
    const Span xs = span_of(X, (int64_t)a.T * d * S), rs = span_of(a.Wr, (int64_t)a.E * d * S), gs = span_of(a.ln_g, d * S), bs = span_of(a.ln_b, d * S);
    Eight gq[NCH], bq[NCH], wr[STEPS];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int at = (lane + j * 64) * 8;
        gq[j] = load8<T>(gs, at, at < d);
        bq[j] = load8<T>(bs, at, at < d);
    }
#pragma unroll
    for (int j = 0; j < STEPS; ++j) wr[j] = load8<T>(rs, c * d + (wave + j * WAVES) * 32 + kq, c < a.E && (wave + j * WAVES) * 32 + kq < d);

    // Channels of a pair, a round: G runs of sixteen, G 16 x 16 values over the waves' K; a thread stores up to two of them for one (token, slot).
    // Where every pair there is has its workgroups, the first round's weights are on their way while the logits are made.
    const int nth = blockIdx.x / a.slices, g0 = blockIdx.x % a.slices * G, r = threadIdx.x & 15, ch0 = threadIdx.x >> 4;
    constexpr int EACH = G == 1 ? 1 : G / 2;
    int seg = nth, groups = 0;
    Eight w[G][STEPS];
    float bias[EACH];
    auto fetch = [&](int g) {
        const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane(seg) * a.Fp;
        const Span ws = span_of((const T *)a.W1 + first * d, (int64_t)a.Fp * d * S), b1 = span_of(a.b1 ? (const T *)a.b1 + first : nullptr, a.Fp * S);
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const int k = (wave + j * WAVES) * 32 + kq;
                w[i][j] = load8<T>(ws, ((g + i) * 16 + c) * d + k, g + i < groups && k < d);
            }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int ch = g * 16 + ch0 + i * 32;
            bias[i] = load1<T>(b1, ch, ch < groups * 16);
        }
    };

    // ---- route
    const bool resident = a.T <= a.tile_rows;
    for (int base = 0; base < a.T; base += a.tile_rows) {
        const int rows = a.T - base < a.tile_rows ? a.T - base : a.tile_rows;
        // two tokens of a wave at a time, the next two on their way
        Eight next[2][NCH];
        auto load_tokens = [&](int i) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int at = (lane + j * 64) * 8;
                    next[u][j] = load8<T>(xs, (base + i + u * WAVES) * d + at, at < d && i + u * WAVES < rows);
                }
        };
        load_tokens(wave);
        for (int i = wave; i < rows; i += 2 * WAVES) {
            Eight xq[2][NCH];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < NCH; ++j) xq[u][j] = next[u][j];
            load_tokens(i + 2 * WAVES);
            float v[2][NCH][8], m[2], inv[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                m[u] = 0.f;
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    to_floats(xq[u][j], v[u][j]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) m[u] += v[u][j][e];
                }
            }
            if (a.ln_g) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    m[u] = wave_sum(m[u]) / d;
                    inv[u] = 0.f;
#pragma unroll
                    for (int j = 0; j < NCH; ++j)
                        if ((lane + j * 64) * 8 < d) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) inv[u] = fmaf(v[u][j][e] - m[u], v[u][j][e] - m[u], inv[u]);
                        }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) inv[u] = 1.0f / sqrtf(wave_sum(inv[u]) / d + a.eps);
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    float gm[8], bt[8];
                    to_floats(gq[j], gm);
                    to_floats(bq[j], bt);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[u][j][e] = fmaf((v[u][j][e] - m[u]) * inv[u], gm[e], bt[e]);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = i + u * WAVES;
                if (r >= rows) break;
                if (lane == 0 && a.ln_g) { mean[base + r] = m[u]; rstd[base + r] = inv[u]; }
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    const int at = (lane + j * 64) * 8;
                    if (at >= dp) continue;                  // zeros from d to the next multiple of 32
                    float *o = xt + r * ld + at;
                    const bool in = at < d;
                    *reinterpret_cast<f32x4 *>(o) = in ? f32x4{v[u][j][0], v[u][j][1], v[u][j][2], v[u][j][3]} : f32x4{0.f, 0.f, 0.f, 0.f};
                    *reinterpret_cast<f32x4 *>(o + 4) = in ? f32x4{v[u][j][4], v[u][j][5], v[u][j][6], v[u][j][7]} : f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
        }
        if (!a.by_slot && base + a.tile_rows >= a.T) {
            groups = width_of(a, __builtin_amdgcn_readlane(kept, seg % a.E)) / 16;
            fetch(g0);
        }
        __syncthreads();
        // logits in blocks of 16 experts x 16 tokens, four blocks between two barriers
        const int tiles_e = (a.E + 15) / 16, blocks = tiles_e * ((rows + TILE_T - 1) / TILE_T);
        for (int b0 = 0; b0 < blocks; b0 += 4) {
            const int nb = blocks - b0 < 4 ? blocks - b0 : 4;
            for (int i = 0; i < nb; ++i) {
                const int e0 = (b0 + i) % tiles_e * 16, r = (b0 + i) / tiles_e * TILE_T + c;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const int s = wave + j * WAVES;
                    if (s >= steps) break;
                    Eight w = wr[j];
                    if (e0) w = load8<T>(rs, (e0 + c) * d + s * 32 + kq, e0 + c < a.E && s * 32 + kq < d);
                    float v[8];
                    const float *p = xt + (r < rows ? r : 0) * ld + s * 32 + kq;      // columns from `rows` on: another's sums, not stored
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = p[e];
                    acc = Operand<T>::template split<3>(v).template times<3>(w, acc);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) part(wave, i * 16 + (lane >> 4) * 4 + e, c) = acc[e];
            }
            __syncthreads();
            for (int i = threadIdx.x; i < nb * 256; i += NT) {
                const int e = (b0 + i / 256) % tiles_e * 16 + (i >> 4) % 16, r = (b0 + i / 256) / tiles_e * TILE_T + (i & 15);
                if (e >= a.E || r >= rows) continue;
                float q = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) q += part(w, i >> 4, i & 15);
                lg[(base + r) * lgs + e] = q + (a.br ? to_f32(((const T *)a.br)[e]) : 0.f);
            }
            __syncthreads();
        }
    }
    // An expert's rank is the number of those before it: higher logits, and equal ones of lower numbers; a NaN ranks below every number.  An
    // expert that the caller lists twice counts in its last slot.
    uint8_t *pk = reinterpret_cast<uint8_t *>(picks);
    for (int i = threadIdx.x; i < a.T * 8; i += NT) if (i % 8 >= a.top_k) pk[i] = 255;
    if (a.forced) {
        for (int i = threadIdx.x; i < a.T * a.top_k; i += NT) {
            const int t = i / a.top_k, s = i - t * a.top_k, e = min(max(a.forced[i], 0), a.E - 1);
            bool again = false;
            for (int q = s + 1; q < a.top_k; ++q) again = again || min(max(a.forced[t * a.top_k + q], 0), a.E - 1) == e;
            pk[t * 8 + s] = again ? 255 : (uint8_t)e;
        }
    } else {
        for (int i = threadIdx.x; i < a.T * a.E; i += NT) {
            const int t = i / a.E, e = i - t * a.E;
            const float *l = lg + t * lgs;
            const float mine = l[e] == l[e] ? l[e] : -INFINITY;
            int rank = 0;
#pragma unroll 8
            for (int q = 0; q < a.E; ++q) {
                const float u = l[q] == l[q] ? l[q] : -INFINITY;
                rank += u > mine || (u == mine && q < e);
            }
            if (rank < a.top_k) pk[t * 8 + rank] = (uint8_t)e;
        }
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        if (a.logit_out) for (int i = threadIdx.x; i < a.T * a.E; i += NT) a.logit_out[i] = lg[i / a.E * lgs + i % a.E];
        if (threadIdx.x < a.T) {
            const int t = threadIdx.x;
            float most = -INFINITY, den = 0.f;
            auto logit = [&](int s) { const int e = pk[t * 8 + s]; return e == 255 || !(lg[t * lgs + e] == lg[t * lgs + e]) ? -INFINITY : lg[t * lgs + e]; };
            for (int s = 0; s < a.top_k; ++s) most = fmaxf(most, logit(s));
            for (int s = 0; s < a.top_k; ++s) den += pk[t * 8 + s] == 255 ? 0.f : expf(logit(s) - most);
            for (int s = 0; s < a.top_k; ++s) {
                const float w = pk[t * 8 + s] == 255 ? 0.f : expf(logit(s) - most) / den;
                a.weight[t * 8 + s] = w;
                if (a.weight_out) a.weight_out[t * a.top_k + s] = w;
                if (a.route_out) a.route_out[t * a.top_k + s] = a.forced ? min(max(a.forced[t * a.top_k + s], 0), a.E - 1) : pk[t * 8 + s];
            }
            a.route[t] = picks[t];
        }
    }
    const uint64_t mine_picks = lane < a.T ? picks[lane] : ~0ull;

    // ---- the pair's channels
    const Pair pair = find_pair(a, mine_picks, pattern, nth);
    const int n_all = list_tokens(a, pair, nth, slots[wave]);
    if (!n_all) return;
    if (a.by_slot) {
        seg = pair.seg;
        groups = width_of(a, __builtin_amdgcn_readlane(kept, pair.expert)) / 16;
    }
    for (int t0 = 0; t0 < n_all; t0 += TILE_T) {
        if (a.by_slot || t0) fetch(g0);
        const int n = n_all - t0 < TILE_T ? n_all - t0 : TILE_T;
        const int token = slots[wave][t0 + (c < n ? c : 0)] / a.top_k;        // columns from n on: another's sums, not stored
        Operand<T> x[STEPS];
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            const int k = (wave + j * WAVES) * 32 + kq;
            if (wave + j * WAVES >= steps) break;
            float v[8];
            if (resident) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = xt[token * ld + k + e];
            } else {                                         // normalised again, from memory
                to_floats(load8<T>(xs, token * d + k, k < d), v);
                if (a.ln_g) {
                    float gm[8], bt[8];
                    to_floats(load8<T>(gs, k, k < d), gm);
                    to_floats(load8<T>(bs, k, k < d), bt);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mean[token]) * rstd[token], gm[e], bt[e]);
                }
            }
            x[j] = Operand<T>::template split<2>(v);
        }
        const int mine = r < n ? slots[wave][t0 + r] : -1;
        for (int g = g0; g < groups; g += a.slices * G) {
            f32x4 acc[G];
            float bv[EACH];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) if (wave + j * WAVES < steps) acc[i] = x[j].template times<2>(w[i][j], acc[i]);
            }
#pragma unroll
            for (int i = 0; i < EACH; ++i) bv[i] = bias[i];
            fetch(g + a.slices * G);
            __syncthreads();                                 // the last round's sums have been read
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) part(wave, i * 16 + (lane >> 4) * 4 + e, c) = acc[i][e];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int at_ch = ch0 + i * 32, ch = g * 16 + at_ch;
                if (mine < 0 || at_ch >= G * 16 || ch >= groups * 16) continue;
                float z = bv[i];
#pragma unroll
                for (int v = 0; v < WAVES; ++v) z += part(v, at_ch, r);
                z = activated<T>(a.act, z);
                const int64_t at = (int64_t)mine * a.Fp + ch;
                if constexpr (sizeof(T) == 2) {
                    const h16 hi = (h16)z;
                    ((h16 *)a.hid)[at] = hi;
                    ((h16 *)a.hid)[(int64_t)a.T * a.top_k * a.Fp + at] = (h16)(z - (float)hi);
                } else ((float *)a.hid)[at] = z;
            }
        }
    }
}

// Two or four features of all tokens.  A wave takes ranges of the pairs' channels as they come and multiplies in sixteen 4 x 4 blocks at once, four
// features by four tokens, each over channels of its own: 16 bytes of a lane are eight channels of one feature.  Every (range, slot) has its own
// place in LDS, and the end adds them up in order.  What bounds it is how much one compute unit keeps on its way, so the features are as few as still
// leave it one workgroup: two where d <= 512 (34 tokens, sixteen experts of d 512: 24.5 us, with four 27.5), else four.
template <class T>
__global__ __launch_bounds__(DOWN_WAVES * 64) void moe_few_down_kernel(FewMoe a)
{
    extern __shared__ __attribute__((aligned(16))) float zs[];         // [parts][T k][4]
    __shared__ short slots[DOWN_WAVES][2][FEW];             // of this pair and of the next
    __shared__ float weight[FEW][8];
    __shared__ uint64_t route[FEW];
    __shared__ int taken;
    if (threadIdx.x == 0) taken = 0;
    for (int i = threadIdx.x; i < a.parts * a.T * a.top_k * 4; i += DOWN_WAVES * 64) zs[i] = 0.f;      // ranges past an expert's width stay so
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q4 = lane & 3, k8 = (lane >> 2) * 8;
    const int n0 = blockIdx.x * a.feats, d = a.d, all = a.T * a.top_k;
    const uint64_t picks = lane < a.T ? a.route[lane] : ~0ull;
    const int pattern = pattern_of(a, lane), kept = __builtin_amdgcn_raw_buffer_load_b32(span_of(a.k_ffn, a.E * 4), lane * 4, 0, 0);
    // what the end needs: a thread's feature and token, at most 64 tokens x 4, and one of the weights
    const int f = threadIdx.x & 3, t = threadIdx.x >> 2;
    const bool ends = t < a.T && f < a.feats && n0 + f < d;
    const float y = load1<T>(span_of(a.X, (int64_t)a.T * d * (int)sizeof(T)), t * d + n0 + f, ends && a.add_residual);
    const float one = load1<float>(span_of(a.weight, a.T * 32), threadIdx.x, true);
    // Chunks of a wave: the channels of an item, up to sixteen tokens at a time, four to a product.  The weights of the next chunk, or of the next
    // pair's first one, take the place of this one's as they are used.
    constexpr int TT = 4, AHEAD = sizeof(T) == 2 ? 8 : 4, CHUNK = 128 * AHEAD, TERMS = sizeof(T) == 2 ? 2 : 1;
    struct At { int item, buf, seg, prt, n_all, t0, from, to, k; };
    auto advance = [&](At s) {
        if (s.k + CHUNK < s.to) { s.k += CHUNK; return s; }
        s.k = s.from;
        s.t0 += 16;
        if (s.t0 < s.n_all) return s;
        for (;;) {                                           // the next item that no wave has: which wave sums it does not matter to the sum
            if (s.item < 0) s.item = wave;
            else {
                int i = 0;
                if (lane == 0) i = atomicAdd(&taken, 1);
                s.item = DOWN_WAVES + __builtin_amdgcn_readfirstlane(i);
            }
            if (s.item >= a.segs * a.parts) break;
            int nth = s.item, prt = 0;
            for (; nth >= a.segs; nth -= a.segs) ++prt;
            const Pair pair = find_pair(a, picks, pattern, nth);
            const int n_all = list_tokens(a, pair, nth, slots[wave][s.buf ^ 1]);
            if (!n_all) continue;
            const int width = width_of(a, __builtin_amdgcn_readlane(kept, pair.expert)), from = prt * a.per;
            if (from >= width && prt) continue;
            return At{s.item, s.buf ^ 1, pair.seg, prt, n_all, 0, from, from + a.per < width ? from + a.per : width, from};
        }
        return At{s.item, s.buf, 0, 0, 0, 0, 0, 0, 0};
    };
    const Span hs = span_of(a.hid, (int64_t)all * a.Fp * 4);
    typename Weights<T>::type w[AHEAD];
    auto fetch = [&](const At &s, int j) {
        const Span ws = span_of((const T *)a.W2T + ((int64_t)__builtin_amdgcn_readfirstlane(s.seg) * d + n0) * a.Fp, (int64_t)(d - n0) * a.Fp * (int)sizeof(T));
        w[j] = load8<T>(ws, q4 * a.Fp + s.k + k8, s.k + k8 < (q4 < a.feats && n0 + q4 < d ? s.to - j * 128 : 0), j * 128);
    };
    At cur = advance(At{-1, 0, 0, 0, 0, 0, 0, 0, 0});
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) fetch(cur, j);
    int at[TT];
    f32x4 acc[TT], bias;
    while (cur.n_all) {
        if (cur.k == cur.from) {
#pragma unroll
            for (int u = 0; u < TT; ++u) {
                at[u] = cur.t0 + u * 4 + q4 < cur.n_all ? slots[wave][cur.buf][cur.t0 + u * 4 + q4] : -1;
                acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            const Span b2 = span_of(a.b2x ? (const T *)a.b2x + (int64_t)__builtin_amdgcn_readfirstlane(cur.seg) * d + n0 : nullptr, (d - n0) * (int)sizeof(T));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                bias[e] = load1<T>(b2, e, cur.prt == 0);
        }
        const At next = advance(cur);
        const int left = cur.n_all - cur.t0;
#pragma unroll
        for (int u = 0; u < TT; ++u) {
            if (u * 4 >= left) break;
            const bool last = u + 1 == TT || (u + 1) * 4 >= left;
#pragma unroll
            for (int j0 = 0; j0 < AHEAD; j0 += 4) {
                typename Weights<T>::type x[4][TERMS];       // hidden channels of four products on their way together
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int v = 0; v < TERMS; ++v) {
                        const int k = cur.k + k8;
                        x[j][v] = load8<T>(hs, at[u] * a.Fp + k, k < (at[u] < 0 ? 0 : cur.to - (j0 + j) * 128), (j0 + j) * 128, v * all * a.Fp);
                    }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (sizeof(T) == 2) {
#define SF_QUARTER(x, i) __builtin_shufflevector(x, x, (i) * 4, (i) * 4 + 1, (i) * 4 + 2, (i) * 4 + 3)
#pragma unroll
                        for (int v = TERMS - 1; v >= 0; --v) {
                            acc[u] = SF_MFMA_4X4(SF_QUARTER(w[j0 + j], 0), SF_QUARTER(x[j][v], 0), acc[u]);
                            acc[u] = SF_MFMA_4X4(SF_QUARTER(w[j0 + j], 1), SF_QUARTER(x[j][v], 1), acc[u]);
                        }
#undef SF_QUARTER
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[u] = __builtin_amdgcn_mfma_f32_4x4x1f32(w[j0 + j].a[e], x[j][0].a[e], acc[u], 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[u] = __builtin_amdgcn_mfma_f32_4x4x1f32(w[j0 + j].b[e], x[j][0].b[e], acc[u], 0, 0, 0);
                    }
                }
            }
            if (last) {
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) fetch(next, j);
            }
        }
        if (next.item != cur.item || next.t0 != cur.t0) {
#pragma unroll
            for (int u = 0; u < TT; ++u) {
                if (u * 4 >= left) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[u][e] = pair_sum<4>(pair_sum<8>(pair_sum<16>(pair_sum<32>(acc[u][e])))) + bias[e];
                if (lane < 4 && at[u] >= 0) *reinterpret_cast<f32x4 *>(zs + (cur.prt * all + at[u]) * 4) = acc[u];
            }
        }
        cur = next;
    }
    if (threadIdx.x < FEW * 8) weight[threadIdx.x / 8][threadIdx.x % 8] = one;
    if (threadIdx.x < FEW) route[threadIdx.x] = picks;
    __syncthreads();
    if (!ends) return;
    const uint64_t slot_of = route[t];
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        if (s >= a.top_k) break;
        if (((slot_of >> (8 * s)) & 255) == 255) continue;
        float z = 0.f;
        for (int q = 0; q < a.parts; ++q) z += zs[(q * all + t * a.top_k + s) * 4 + f];
        sum = fmaf(weight[t][s], z, sum);
    }
    ((T *)a.Y)[(int64_t)t * d + n0 + f] = from_f32<T>(y + sum);
}

struct FewWs { uint64_t *route; float *weight; void *hid; int Fp, segs, by_slot, slices, groups, parts, per; size_t bytes; };
FewWs few_ws(const Dims &D, const sf_moe_compact &m, void *ws)
{
    Carver c(ws);
    FewWs w{};
    const int T = D.B * D.L, pairs = T * m.top_k;
    w.Fp = (int)align_up((size_t)m.k_ffn_max, (size_t)D.ffn_pad);
    w.by_slot = pairs < D.P * m.n_experts;
    w.segs = w.by_slot ? pairs : D.P * m.n_experts;
    // a workgroup per compute unit: each routes for itself, so more of them would do that more often
    w.slices = std::max(1, 256 / w.segs);
    const int together = D.dtype == SF_BF16 ? 4 : 2;          // fp32 weights take twice the registers
    w.groups = w.Fp / 16 >= together * w.slices ? together : 1;
    w.slices = std::min(ceil_div(w.Fp / 16, w.groups), w.slices);
    // ranges of 1024 channels, where few pairs share a workgroup's waves as many as there are waves; their sums take at most 48 KB
    w.parts = std::max(1, std::min(std::max(ceil_div(w.Fp, 1024), DOWN_WAVES / w.segs), 48 * 1024 / (pairs * 16)));
    w.per = align_up((size_t)ceil_div(w.Fp, w.parts), 64);
    w.route = c.take<uint64_t>((size_t)T);
    w.weight = c.take<float>((size_t)T * 8);
    w.hid = c.take<float>((size_t)pairs * w.Fp);
    w.bytes = c.off;
    return w;
}

int32_t check_few(const Dims &D, const sf_moe_compact *m)
{
    if (!m) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: NULL argument");
    if (m->n_experts < 1 || m->n_experts > 64 || m->top_k < 1 || m->top_k > m->n_experts || m->top_k > 8)
        return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: needs 1 <= top_k <= min(8, n_experts), n_experts <= 64");
    if (m->k_ffn_max < 1 || m->k_ffn_max > D.F) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: k_ffn_max out of range");
    if (m->k_ffn_max > 1 << 18) return fail(SF_ERR_SHAPE, "moe_ffn_few: at most 2^18 channels an expert");
    if (!m->k_ffn) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: k_ffn (device keep counts) missing");
    if ((int64_t)D.B * D.L > FEW) return fail(SF_ERR_SHAPE, "moe_ffn_few: at most %d tokens (sf_moe_ffn_forward takes any number)", FEW);
    if ((int64_t)D.P * m->n_experts > 4096) return fail(SF_ERR_SHAPE, "moe_ffn_few: more than 4096 (pattern, expert) pairs");
    if (D.d % 8 || D.d > MAX_D) return fail(SF_ERR_SHAPE, "moe_ffn_few: d_model must be a multiple of 8, at most %d", MAX_D);
    return SF_OK;
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" size_t sf_moe_ffn_few_workspace_bytes(const sf_desc *desc, const sf_moe_compact *m)
{
    Dims D;
    if (read_desc(desc, D) || check_few(D, m)) return 0;
    return few_ws(D, *m, nullptr).bytes;
}

extern "C" int32_t sf_moe_ffn_few_forward(const sf_desc *desc, const sf_moe_compact *m, const void *X, const int32_t *pattern_id, int32_t pre_ln,
                                          int32_t add_residual, const int32_t *forced_route, void *Y, int32_t *route_out, float *weight_out,
                                          float *logit_out, void *workspace, size_t workspace_bytes, void *stream)
{
    Dims D;
    if (int32_t rc = read_desc(desc, D)) return rc;
    if (int32_t rc = check_few(D, m)) return rc;
    if (!X || !Y) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: NULL argument");
    if (X == Y) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: Y may not alias X");
    if (!m->Wr || !m->W1 || !m->W2T || (pre_ln && (!m->ln_g || !m->ln_b))) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: NULL parameter pointer");
    if (D.P > 1 && !pattern_id) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: pattern_id required when P > 1");
    if (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)m->Wr | (uintptr_t)m->W1 | (uintptr_t)m->W2T | (pre_ln ? (uintptr_t)m->ln_g | (uintptr_t)m->ln_b : 0)) & 15)
        return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: X, Y, Wr, W1, W2T, ln_g and ln_b must be 16-byte aligned");
    const FewWs w = few_ws(D, *m, workspace);
    if (!workspace || workspace_bytes < w.bytes || ((uintptr_t)workspace & 255))
        return fail(SF_ERR_WORKSPACE, "moe_ffn_few: workspace of %zu bytes (256-byte aligned) required, got %zu", w.bytes, workspace_bytes);
    FewMoe a{};
    a.X = X; a.Wr = m->Wr; a.br = m->br; a.ln_g = pre_ln ? m->ln_g : nullptr; a.ln_b = m->ln_b; a.W1 = m->W1; a.b1 = m->b1; a.W2T = m->W2T; a.b2x = m->b2x;
    a.pattern_id = D.P > 1 ? pattern_id : nullptr; a.forced = forced_route; a.k_ffn = m->k_ffn;
    a.T = D.B * D.L; a.L = D.L; a.d = D.d; a.E = m->n_experts; a.P = D.P; a.top_k = m->top_k; a.ffn_pad = D.ffn_pad; a.Fp = w.Fp;
    a.act = D.act == SF_GELU_ERF ? ACT_GELU : ACT_RELU; a.eps = D.eps; a.add_residual = add_residual;
    a.segs = w.segs; a.by_slot = w.by_slot; a.slices = w.slices; a.parts = w.parts; a.per = w.per;
    a.route = w.route; a.weight = w.weight; a.hid = w.hid;
    a.Y = Y; a.route_out = route_out; a.weight_out = weight_out; a.logit_out = logit_out;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const size_t row = (align_up((size_t)D.d, 32) + 4) * sizeof(float);
    a.tile_rows = a.T * row <= XT_BYTES ? a.T : std::min(a.T, TILE_T);
    const size_t lds = a.tile_rows * row + ((size_t)WAVES * 64 * (TILE_T + 1) + (size_t)a.T * (a.E + 1)) * sizeof(float);
    const bool bf = D.dtype == SF_BF16;
    auto kern = w.groups > 1 ? (bf ? moe_few_up_kernel<h16, 4> : moe_few_up_kernel<float, 2>) : (bf ? moe_few_up_kernel<h16, 1> : moe_few_up_kernel<float, 1>);
    static std::atomic<bool> attr_set[4];         // setting the attribute twice is harmless
    const int which = bf + 2 * (w.groups > 1);
    if (!attr_set[which]) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 156 * 1024) != hipSuccess)
            return fail(SF_ERR_HIP, "moe_ffn_few: cannot reserve LDS");
        attr_set[which] = true;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(w.segs * w.slices)), dim3(NT), lds, st, a);
    a.feats = D.d <= 2 * 256 ? 2 : 4;                        // 256 compute units
    const dim3 down((unsigned)ceil_div(D.d, a.feats));
    const size_t zs = (size_t)w.parts * a.T * a.top_k * 4 * sizeof(float);
    if (bf) hipLaunchKernelGGL(moe_few_down_kernel<h16>, down, dim3(DOWN_WAVES * 64), zs, st, a);
    else hipLaunchKernelGGL(moe_few_down_kernel<float>, down, dim3(DOWN_WAVES * 64), zs, st, a);
    return check_launch("moe_ffn_few_forward");
}
