// The Sparse-MoE FFN block of a few tokens (Sec. 4.5) in two launches.  What bounds it is the chosen experts' weights, read once, and latency.
//
//   up:    every workgroup normalises the tokens and routes them for itself (LayerNorm, logits, Top-k), then takes channels of one of the
//          chosen (pattern, expert) pairs: hidden rows in fp32, one per (token, slot)
//   down:  features of one pair over a range of its channels; the workgroup that finishes a run of features last adds up the slots,
//          in their order, with their weights, and the residual
//
// The products run on the matrix cores, weights as the first operand, sixteen tokens as the second.  An activation goes in as a sum of
// 16-bit terms, so that nothing is rounded on the way: two terms (16 bits in bfloat16, 22 in binary16) for the experts' products, three for
// the logits, whose order decides.  fp32 models take the fp32 instruction.
#include <algorithm>
#include <atomic>

#include "gemm.hpp"

namespace sf {

namespace {

constexpr int FEW = SF_MOE_FEW_TOKENS, TILE_T = 16, MAX_D = 1024, MAX_SEGS = 4096, STEPS = MAX_D / 32 / 4;      // K steps of 32 that a wave of four owns
#ifdef SF_HALF_F16
#define SF_MFMA_16X16 __builtin_amdgcn_mfma_f32_16x16x32_f16
#else
#define SF_MFMA_16X16 __builtin_amdgcn_mfma_f32_16x16x32_bf16
#endif

struct FewMoe {
    const void *X, *Wr, *br, *ln_g, *ln_b, *W1, *b1, *W2T, *b2x;
    const int32_t *pattern_id, *forced, *k_ffn;
    int T, L, d, E, P, top_k, ffn_pad, Fp, act; float eps; int add_residual;
    int segs, slices, parts;                                 // most pairs in use; workgroups of a pair (up), ranges of its channels (down)
    int32_t *route; float *weight; int32_t *done; float *hid, *z;      // workspace: [T k] (-1: listed again in a later slot), [T k],
                                                             // [features / 16], [T k, Fp], [parts, T k, d]
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
__device__ __forceinline__ h16x8 load8(const h16 *p, bool in) { return in ? *reinterpret_cast<const h16x8 *>(p) : h16x8{}; }
__device__ __forceinline__ f32x8 load8(const float *p, bool in)
{
    f32x8 o{};
    if (in) { o.a = *reinterpret_cast<const f32x4 *>(p); o.b = *reinterpret_cast<const f32x4 *>(p + 4); }
    return o;
}

template <class T>
__device__ __forceinline__ float activated(int act, float z)
{
    if (act == ACT_RELU) return z < 0.f ? 0.f : z;
    return sizeof(T) == 4 ? 0.5f * z * (1.0f + erff(z * 0.70710678f)) : gelu_erf(z);
}

// The pairs in use: seg of every (token, slot), whether it is the first of its seg, and the tokens of the n-th seg in use
struct Pairs {
    short slot[FEW];                                         // of the seg looked for: its (token, slot) numbers
    int n, seg;
};
__device__ __forceinline__ int pattern_of(const FewMoe &a, int t)
{
    return a.pattern_id ? min(max(a.pattern_id[t / a.L], 0), a.P - 1) : 0;
}
// route(i): the expert of (token, slot) i, negative where it does not count; first: LDS for P E numbers, the lowest (token, slot) of a pair.
// All 256 threads.  false: fewer than `nth` + 1 pairs are in use
template <class Route>
__device__ bool find_pairs(const FewMoe &a, Pairs &p, int *first, int nth, Route route)
{
    const int n = a.T * a.top_k, lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < a.P * a.E; i += 256) first[i] = 0x7fffffff;
    if (threadIdx.x == 0) p.seg = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += 256) {
        const int e = route(i);
        if (e >= 0) atomicMin(&first[pattern_of(a, i / a.top_k) * a.E + e], i);
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        int before = 0;
        for (int i0 = 0; i0 < n && before <= nth; i0 += 64) {
            const int i = i0 + lane, e = i < n ? route(i) : -1;
            const int s = e >= 0 ? pattern_of(a, i / a.top_k) * a.E + e : -1;
            const uint64_t is_first = __ballot(s >= 0 && first[s < 0 ? 0 : s] == i);
            const int rank = before + __popcll(is_first & ((1ull << lane) - 1));
            if ((is_first >> lane & 1) && rank == nth) p.seg = s;
            before += __popcll(is_first);
        }
    }
    __syncthreads();
    if (p.seg < 0) return false;
    if (threadIdx.x < 64) {
        int at = -1;
        if (lane < a.T && pattern_of(a, lane) == p.seg / a.E)
            for (int s = 0; s < a.top_k; ++s) if (route(lane * a.top_k + s) == p.seg % a.E) at = lane * a.top_k + s;
        const uint64_t m = __ballot(at >= 0);
        if (at >= 0) p.slot[__popcll(m & ((1ull << lane) - 1))] = (short)at;
        if (lane == 0) p.n = __popcll(m);
    }
    __syncthreads();
    return true;
}

// Channels of seg's expert, padded as its weights are
__device__ __forceinline__ int width_of(const FewMoe &a, int seg)
{
    const int w = (a.k_ffn[seg % a.E] + a.ffn_pad - 1) / a.ffn_pad * a.ffn_pad;
    return w < a.Fp ? w : a.Fp;
}

template <class T>
__global__ __launch_bounds__(256) void moe_few_up_kernel(FewMoe a)
{
    extern __shared__ __attribute__((aligned(16))) float xt[];         // [16][dp + 4] normalised tokens: rows 16 bytes apart over the banks
    __shared__ Pairs pairs;
    __shared__ float mean[FEW], rstd[FEW], red[4][64][TILE_T + 1];
    static_assert(sizeof(red) >= MAX_SEGS * sizeof(int), "find_pairs");
    __shared__ signed char pick[FEW * 8];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kq = (lane >> 4) * 8;
    const int d = a.d, dp = (d + 31) / 32 * 32, ld = dp + 4, steps = dp / 32, lgs = a.E + 1;
    float *lg = xt + TILE_T * ld;                            // [T][E + 1]
    const T *X = (const T *)a.X;
    // token t normalised into row r of xt; statistics the first time
    auto normalise = [&](int t, int r, bool first) {
        const T *x = X + (int64_t)t * d;
        float v[MAX_D / 64], sum = 0.f;
#pragma unroll
        for (int j = 0; j < MAX_D / 64; ++j) {
            const int at = lane + j * 64;
            v[j] = at < d ? to_f32(x[at]) : 0.f;
            sum += v[j];
        }
        if (a.ln_g) {
            float m, inv;
            if (first) {
                m = wave_sum(sum) / d;
                float q = 0.f;
#pragma unroll
                for (int j = 0; j < MAX_D / 64; ++j) if (lane + j * 64 < d) q = fmaf(v[j] - m, v[j] - m, q);
                inv = 1.0f / sqrtf(wave_sum(q) / d + a.eps);
                if (lane == 0) { mean[t] = m; rstd[t] = inv; }
            } else { m = mean[t]; inv = rstd[t]; }
#pragma unroll
            for (int j = 0; j < MAX_D / 64; ++j) {
                const int at = lane + j * 64;
                if (at < d) v[j] = fmaf((v[j] - m) * inv, to_f32(((const T *)a.ln_g)[at]), to_f32(((const T *)a.ln_b)[at]));
            }
        }
#pragma unroll
        for (int j = 0; j < MAX_D / 64; ++j) if (lane + j * 64 < dp) xt[r * ld + lane + j * 64] = v[j];
    };
    auto clear = [&](int r) { for (int at = lane; at < dp; at += 64) xt[r * ld + at] = 0.f; };

    // ---- route
    for (int t0 = 0; t0 < a.T; t0 += TILE_T) {
        __syncthreads();
        for (int r = wave; r < TILE_T; r += 4) {
            if (t0 + r < a.T) normalise(t0 + r, r, true);
            else clear(r);
        }
        __syncthreads();
        f32x4 acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int s = wave; s < steps; s += 4) {
            const auto x = Operand<T>::template split<3>(xt + c * ld + s * 32 + kq);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i * 16 >= a.E) break;
                const int e = i * 16 + c;
                acc[i] = x.template times<3>(load8((const T *)a.Wr + (int64_t)e * d + s * 32 + kq, e < a.E && s * 32 + kq < d), acc[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][i * 16 + (lane >> 4) * 4 + e][c] = acc[i][e];
        __syncthreads();
        for (int i = threadIdx.x; i < a.E * TILE_T; i += 256) {
            const int e = i / TILE_T, r = i % TILE_T;
            const float *p = &red[0][e][r];
            constexpr int W = 64 * (TILE_T + 1);
            if (t0 + r < a.T) lg[(t0 + r) * lgs + e] = (p[0] + p[W]) + (p[2 * W] + p[3 * W]) + (a.br ? to_f32(((const T *)a.br)[e]) : 0.f);
        }
    }
    __syncthreads();
    const bool one = blockIdx.x == 0;
    if ((int)threadIdx.x < a.T) {
        // ties go to the lower expert, a NaN ranks below every number; an expert that the caller lists twice counts in its last slot
        const int t = threadIdx.x;
        unsigned long long taken = 0;
        float most = -INFINITY, den = 0.f, v[8];
        int who[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            who[s] = -1;
            v[s] = -INFINITY;
            if (s >= a.top_k) continue;
            int be = -1;
            float bv = -INFINITY;
            if (a.forced) {
                be = min(max(a.forced[t * a.top_k + s], 0), a.E - 1);
                bv = lg[t * lgs + be];
                bv = bv == bv ? bv : -INFINITY;
            } else {
                for (int e = 0; e < a.E; ++e) {
                    float u = lg[t * lgs + e];
                    u = u == u ? u : -INFINITY;
                    if (!(taken >> e & 1) && (be < 0 || u > bv)) { be = e; bv = u; }
                }
                taken |= 1ull << be;
            }
            who[s] = be;
            v[s] = bv;
        }
        bool again[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            again[s] = false;
#pragma unroll
            for (int q = s + 1; q < 8; ++q) again[s] = again[s] || (q < a.top_k && who[q] == who[s]);
            if (!again[s]) most = fmaxf(most, v[s]);
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            v[s] = s < a.top_k && !again[s] ? expf(v[s] - most) : 0.f;
            den += v[s];
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if (s >= a.top_k) continue;
            const int i = t * a.top_k + s;
            pick[i] = (signed char)(again[s] ? -1 : who[s]);
            if (one) {
                a.route[i] = pick[i];
                a.weight[i] = v[s] / den;
                if (a.route_out) a.route_out[i] = who[s];
                if (a.weight_out) a.weight_out[i] = v[s] / den;
            }
        }
    }
    if (one) {
        if (a.logit_out) for (int i = threadIdx.x; i < a.T * a.E; i += 256) a.logit_out[i] = lg[i / a.E * lgs + i % a.E];
        for (int i = threadIdx.x; i < (d + 15) / 16; i += 256) a.done[i] = 0;
    }
    __syncthreads();
    if (!find_pairs(a, pairs, reinterpret_cast<int *>(red), blockIdx.x / a.slices, [&](int i) { return (int)pick[i]; })) return;

    // ---- channels of the pair
    const int seg = pairs.seg, groups = width_of(a, seg) / 16;
    const T *W1 = (const T *)a.W1 + (int64_t)seg * a.Fp * d, *b1 = a.b1 ? (const T *)a.b1 + (int64_t)seg * a.Fp : nullptr;
    const int g0 = blockIdx.x % a.slices;
    for (int t0 = 0; t0 < (a.T <= TILE_T ? 1 : pairs.n); t0 += TILE_T) {
        // up to sixteen tokens in all: they lie in xt already, and the columns of those that chose otherwise are not stored
        const bool all = a.T <= TILE_T;
        if (!all) {
            __syncthreads();
            for (int r = wave; r < TILE_T; r += 4) {
                if (t0 + r < pairs.n) normalise(pairs.slot[t0 + r] / a.top_k, r, false);
                else clear(r);
            }
            __syncthreads();
        }
        Operand<T> x[STEPS];
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            const int s = wave + j * 4;
            if (s < steps) x[j] = Operand<T>::template split<2>(xt + c * ld + s * 32 + kq);
        }
        // (token, slot) that this thread stores, channel threadIdx.x % 16 of the group
        const int r = threadIdx.x >> 4;
        int mine = -1;
        if (!all) { if (t0 + r < pairs.n) mine = pairs.slot[t0 + r]; }
        else
            for (int i = 0; i < pairs.n; ++i) if (pairs.slot[i] / a.top_k == r) mine = pairs.slot[i];
        typename Weights<T>::type w[STEPS];
        auto fetch = [&](int g) {
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const int k = (wave + j * 4) * 32 + kq;
                w[j] = load8(W1 + (int64_t)(g * 16 + c) * d + k, g < groups && k < d);
            }
        };
        fetch(g0);
        for (int g = g0, b = 0; g < groups; g += a.slices, b ^= 1) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < STEPS; ++j) if (wave + j * 4 < steps) acc = x[j].template times<2>(w[j], acc);
            fetch(g + a.slices);
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][b * 16 + (lane >> 4) * 4 + e][c] = acc[e];
            __syncthreads();                                 // two buffers: the next round's values go into the other one
            if (mine >= 0) {
                const int ch = threadIdx.x & 15, at = b * 16 + ch;
                const float z = (red[0][at][r] + red[1][at][r]) + (red[2][at][r] + red[3][at][r]);
                a.hid[(int64_t)mine * a.Fp + g * 16 + ch] = activated<T>(a.act, z + (b1 ? to_f32(b1[g * 16 + ch]) : 0.f));
            }
        }
        __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(256) void moe_few_down_kernel(FewMoe a)
{
    __shared__ Pairs pairs;
    __shared__ int first[MAX_SEGS];
    __shared__ float red[4][16][TILE_T + 1];
    __shared__ int last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, kq = (lane >> 4) * 8;
    const int n0 = blockIdx.x * 16, d = a.d, pair_no = blockIdx.y / a.parts, part = blockIdx.y % a.parts, all = a.T * a.top_k;
    if (find_pairs(a, pairs, first, pair_no, [&](int i) { return a.route[i]; })) {
        const int seg = pairs.seg, steps = width_of(a, seg) / 32, from = steps * part / a.parts, to = steps * (part + 1) / a.parts;
        const int n = n0 + c < d ? n0 + c : d - 1;
        const T *W = (const T *)a.W2T + ((int64_t)seg * d + n) * a.Fp + kq;
        for (int t0 = 0; t0 < pairs.n; t0 += TILE_T) {
            const float *h = a.hid + (int64_t)pairs.slot[t0 + c < pairs.n ? t0 + c : t0] * a.Fp + kq;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            constexpr int AHEAD = 4;
            for (int s = from + wave; s < to; s += 4 * AHEAD) {
                typename Weights<T>::type w[AHEAD];
                float v[AHEAD][8];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const bool in = s + j * 4 < to;
                    w[j] = load8(W + (s + j * 4) * 32, in);
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        f32x4 q = {0.f, 0.f, 0.f, 0.f};
                        if (in) q = *reinterpret_cast<const f32x4 *>(h + (s + j * 4) * 32 + e);
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[j][e + k] = q[k];
                    }
                }
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) acc = Operand<T>::template split<2>(v[j]).template times<2>(w[j], acc);
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e) red[wave][(lane >> 4) * 4 + e][c] = acc[e];
            __syncthreads();
            const int r = threadIdx.x >> 4, f = threadIdx.x & 15;
            if (t0 + r < pairs.n && n0 + f < d)
                a.z[((int64_t)part * all + pairs.slot[t0 + r]) * d + n0 + f] = (red[0][f][r] + red[1][f][r]) + (red[2][f][r] + red[3][f][r]);
        }
    }
    // the last workgroup of these features adds the slots up
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(&a.done[blockIdx.x], 1) == (int)gridDim.y - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int f = threadIdx.x & 15;
    if (n0 + f >= d) return;
    for (int t = threadIdx.x >> 4; t < a.T; t += 16) {
        float y = a.add_residual ? to_f32(((const T *)a.X)[(int64_t)t * d + n0 + f]) : 0.f;
        const int p = pattern_of(a, t);
        float sum = 0.f;
        for (int s = 0; s < a.top_k; ++s) {
            const int i = t * a.top_k + s, e = a.route[i];
            if (e < 0) continue;
            float z = a.b2x ? to_f32(((const T *)a.b2x)[((int64_t)p * a.E + e) * d + n0 + f]) : 0.f;
            for (int q = 0; q < a.parts; ++q) z += a.z[((int64_t)q * all + i) * d + n0 + f];
            sum = fmaf(a.weight[i], z, sum);
        }
        ((T *)a.Y)[(int64_t)t * d + n0 + f] = from_f32<T>(y + sum);
    }
}

struct FewWs { int32_t *route; float *weight; int32_t *done; float *hid, *z; int Fp, segs, slices, parts; size_t bytes; };
FewWs few_ws(const Dims &D, const sf_moe_compact &m, void *ws)
{
    Carver c(ws);
    FewWs w{};
    const int T = D.B * D.L, pairs = T * m.top_k, tiles = ceil_div(D.d, 16);
    w.Fp = (int)align_up((size_t)m.k_ffn_max, (size_t)D.ffn_pad);
    w.segs = pairs < D.P * m.n_experts ? pairs : D.P * m.n_experts;
    // two workgroups per compute unit: each routes for itself, so more of them would do that more often
    w.slices = std::min(w.Fp / 16, std::max(1, 512 / w.segs));
    w.parts = std::min(8, std::max(1, 512 / (w.segs * tiles)));
    w.route = c.take<int32_t>((size_t)pairs);
    w.weight = c.take<float>((size_t)pairs);
    w.done = c.take<int32_t>((size_t)tiles);
    w.hid = c.take<float>((size_t)pairs * w.Fp);
    w.z = c.take<float>((size_t)w.parts * pairs * D.d);
    w.bytes = c.off;
    return w;
}

int32_t check_few(const Dims &D, const sf_moe_compact *m)
{
    if (!m) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: NULL argument");
    if (m->n_experts < 1 || m->n_experts > 64 || m->top_k < 1 || m->top_k > m->n_experts || m->top_k > 8)
        return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: needs 1 <= top_k <= min(8, n_experts), n_experts <= 64");
    if (m->k_ffn_max < 1 || m->k_ffn_max > D.F) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: k_ffn_max out of range");
    if (!m->k_ffn) return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: k_ffn (device keep counts) missing");
    if ((int64_t)D.B * D.L > FEW) return fail(SF_ERR_SHAPE, "moe_ffn_few: at most %d tokens (sf_moe_ffn_forward takes any number)", FEW);
    if ((int64_t)D.P * m->n_experts > MAX_SEGS) return fail(SF_ERR_SHAPE, "moe_ffn_few: more than %d (pattern, expert) pairs", MAX_SEGS);
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
    if (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)m->Wr | (uintptr_t)m->W1 | (uintptr_t)m->W2T) & 15)
        return fail(SF_ERR_INVALID_ARG, "moe_ffn_few: X, Y, Wr, W1 and W2T must be 16-byte aligned");
    const FewWs w = few_ws(D, *m, workspace);
    if (!workspace || workspace_bytes < w.bytes || ((uintptr_t)workspace & 255))
        return fail(SF_ERR_WORKSPACE, "moe_ffn_few: workspace of %zu bytes (256-byte aligned) required, got %zu", w.bytes, workspace_bytes);
    FewMoe a{};
    a.X = X; a.Wr = m->Wr; a.br = m->br; a.ln_g = pre_ln ? m->ln_g : nullptr; a.ln_b = m->ln_b; a.W1 = m->W1; a.b1 = m->b1; a.W2T = m->W2T; a.b2x = m->b2x;
    a.pattern_id = D.P > 1 ? pattern_id : nullptr; a.forced = forced_route; a.k_ffn = m->k_ffn;
    a.T = D.B * D.L; a.L = D.L; a.d = D.d; a.E = m->n_experts; a.P = D.P; a.top_k = m->top_k; a.ffn_pad = D.ffn_pad; a.Fp = w.Fp;
    a.act = D.act == SF_GELU_ERF ? ACT_GELU : ACT_RELU; a.eps = D.eps; a.add_residual = add_residual;
    a.segs = w.segs; a.slices = w.slices; a.parts = w.parts;
    a.route = w.route; a.weight = w.weight; a.done = w.done; a.hid = w.hid; a.z = w.z;
    a.Y = Y; a.route_out = route_out; a.weight_out = weight_out; a.logit_out = logit_out;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 up((unsigned)(w.segs * w.slices)), down((unsigned)ceil_div(D.d, 16), (unsigned)(w.segs * w.parts));
    const size_t lds = ((size_t)TILE_T * (align_up((size_t)D.d, 32) + 4) + (size_t)a.T * (a.E + 1)) * sizeof(float);
    const bool bf = D.dtype == SF_BF16;
    auto kern = bf ? moe_few_up_kernel<h16> : moe_few_up_kernel<float>;
    static std::atomic<bool> attr_set[2] = {{false}, {false}};      // setting the attribute twice is harmless
    if (!attr_set[bf]) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (TILE_T * (MAX_D + 4) + FEW * 65) * 4) != hipSuccess)
            return fail(SF_ERR_HIP, "moe_ffn_few: cannot reserve LDS");
        attr_set[bf] = true;
    }
    hipLaunchKernelGGL(kern, up, dim3(256), lds, st, a);
    if (bf) hipLaunchKernelGGL(moe_few_down_kernel<h16>, down, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(moe_few_down_kernel<float>, down, dim3(256), 0, st, a);
    return check_launch("moe_ffn_few_forward");
}
