// Cross attention: query tokens over states of another length, K/V groups shared by heads.
//
// The rows of a group are its heads' queries, one head after the other, so K and V are read once for all of them.  A workgroup owns a run
// of rows of one (sample, group) and walks the keys in tiles of 64; scores, softmax and the weighted sum stay in registers:
//   S^T = K Q^T    a lane owns one row and 16 of 32 keys, so the running maximum, sum and rescaling are its own
//   O^T += V^T P^T the probabilities go from accumulators straight into the second operand: the rows of K are dealt to the first product
//                  in the order in which its accumulators are those operands
// exp2 takes the scale along; the running maximum moves only where a tile exceeds it by 2^8, so that most tiles rescale nothing.  The sum is
// that of the probabilities as rounded to 16 bits, which the second product adds up as well.
// Few rows: the four waves of a workgroup take tiles in turn and join at the end; too few workgroups: key ranges in workgroups of their own,
// joined by a second launch.  Keys that are not allowed: a tile without any is not read, a row of one is fetched as zeros (out of range for
// the buffer load), whatever it holds.
#include <atomic>

#include "common.hpp"

namespace sf {

namespace {

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int SEG_KEYS = 8192;              // keys whose masks are held in LDS at a time
constexpr float LOG2E = 1.44269504f;

struct CrossArgs {
    const void *Q, *K, *V; sf_strides sq, sk, sv;
    const int32_t *head_group, *pattern_id; const uint8_t *key_valid;
    void *O; int64_t ldo;
    float *part, *ml;                       // splits > 1: sums [splits, B nH Lq, dh], maximum and sum of weights [splits, B nH Lq, 2]
    int B, Lq, Lk, nH, nG, dh, splits, tiles_per_split;
    float scale;
};

// Which rows a workgroup owns: run t of the runs of `rows` rows of all groups, one group after the other
struct Rows { uint64_t heads; int g, first, n; };
__device__ __forceinline__ Rows find_rows(const CrossArgs &a, int b, int t, int rows)
{
    const int lane = threadIdx.x & 63;
    const int32_t *hg = a.head_group + (a.pattern_id ? (int64_t)a.pattern_id[b] * a.nH : 0);
    const int mine = lane < a.nH ? hg[lane] : -1;
    Rows r{0, 0, 0, 0};
    for (int g = 0; g < a.nG; ++g) {
        const uint64_t heads = __ballot(mine == g);
        const int n = __popcll(heads) * a.Lq, runs = (n + rows - 1) / rows;
        if (t < runs) { r.heads = heads; r.g = g; r.first = t * rows; r.n = n; return r; }
        t -= runs;
    }
    return r;
}
// head and query of row i
__device__ __forceinline__ void row_of(const CrossArgs &a, uint64_t heads, int i, int &h, int &q)
{
    const int j = i / a.Lq;
    q = i - j * a.Lq;
    for (int k = 0; k < j; ++k) heads &= heads - 1;
    h = __ffsll((unsigned long long)heads) - 1;
}

__device__ __forceinline__ float both_halves_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The tiles of KT keys of [k0, k1) that hold an allowed key, in LDS: their numbers and the bits of their keys.  All threads of the workgroup.
template <int KT, bool MASK>
struct KeyTiles {
    static constexpr int MOST = SEG_KEYS / KT;
    uint64_t bits[MASK ? MOST : 1];
    uint16_t list[MASK ? MOST : 1];
    int n;
};
template <int KT, bool MASK>
__device__ __forceinline__ int tiles_of(KeyTiles<KT, MASK> &t, const uint8_t *valid, int k0, int k1)
{
    if constexpr (!MASK) return (k1 - k0 + KT - 1) / KT;
    else {
        const int tiles = (k1 - k0 + KT - 1) / KT, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        __syncthreads();                                     // the last segment's masks have been read
        for (int i = wave; i < (k1 - k0 + 63) / 64; i += waves) {
            const int k = k0 + i * 64 + lane;
            const uint64_t m = __ballot(k < k1 && valid[k] != 0);
            if (lane == 0) {
                if constexpr (KT == 64) t.bits[i] = m;
                else { t.bits[2 * i] = m & 0xffffffffu; if (2 * i + 1 < tiles) t.bits[2 * i + 1] = m >> 32; }
            }
        }
        __syncthreads();
        if (wave == 0) {
            int n = 0;
            for (int i = 0; i < tiles; i += 64) {
                const bool some = i + lane < tiles && t.bits[i + lane] != 0;
                const uint64_t m = __ballot(some);
                if (some) t.list[n + __popcll(m & ((1ull << lane) - 1))] = (uint16_t)(i + lane);
                n += __popcll(m);
            }
            if (lane == 0) t.n = n;
        }
        __syncthreads();
        return t.n;
    }
}

// ------------------------------------------------------------------------------------------------- 16-bit models
// WQ waves along the rows (QB blocks of 32 each), WK along the keys.  Two blocks a wave read a fragment of K and V once for both: 16 samples of 2048
// queries and keys, twelve heads of 64 gained 1 % (239 to 236 us), 64 samples of 512 lost 13 % (49 to 56) - one block it is.
template <int DH, int WQ, int WK, bool MASK>
__global__ __launch_bounds__(WQ *WK * 64, DH == 128 && WK == 4 ? 1 : 2) void cross_kernel(CrossArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int QB = 1, KT = WK == 4 ? 32 : 64, RB = DH * 2, CH = DH / 8;       // keys of a tile, bytes and 16-byte chunks of a row
    constexpr int TILE = KT * RB, STAGE = WK * 2 * TILE, PIECES = TILE / 1024, ROWS = WQ * QB * 32;
    constexpr int JOIN = WK > 1 ? WK * 32 * (DH + 2) * 4 : 0;
    __shared__ __attribute__((aligned(128))) char lds[2 * STAGE > JOIN ? 2 * STAGE : JOIN];
    __shared__ KeyTiles<KT, MASK> tiles;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wq = wave % WQ, wk = wave / WQ;
    const int r = lane & 31, hi = lane >> 5;
    const int b = blockIdx.y, split = blockIdx.z;
    const Rows own = find_rows(a, b, blockIdx.x, ROWS);
    if (own.n == 0) return;
    const h16 *Kg = (const h16 *)a.K + b * a.sk.b + own.g * a.sk.h, *Vg = (const h16 *)a.V + b * a.sv.b + own.g * a.sv.h;
    const float c = a.scale * LOG2E;
    // binary16: probabilities stand 2^4 higher, so that those down to 2^-18 of the largest keep all their bits
    constexpr float LIFT = SF_DTYPE_16 == SF_F16 ? 4.f : 0.f, SLACK = 8.f;

    h16x8 qf[QB][DH / 16];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int i = own.first + (wq * QB + qb) * 32 + r;
        int h, q;
        row_of(a, own.heads, i < own.n ? i : 0, h, q);
        const h16 *p = (const h16 *)a.Q + b * a.sq.b + h * a.sq.h + q * a.sq.l + hi * 8;
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) qf[qb][ks] = *reinterpret_cast<const h16x8 *>(p + ks * 16);
    }
    f32x16 o[QB][DH / 32];
    float m[QB], l[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        l[qb] = 0.f;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[qb][d][e] = 0.f;
    }
    // a piece of a stage is 1024 bytes: 1024 / RB rows; chunk c of row k lies at c ^ f(k), so that a fragment read meets no bank twice
    constexpr int PR = 1024 / RB;
    const int lk = lane / CH, lc = lane % CH;
    const int fk = DH == 32 ? (lk >> 1) & 3 : lk & 7, fv = DH == 32 ? lk & 2 : 2 * (lk & 3);      // rows of a piece start on a multiple of 4
    auto chunk_k = [&](int piece) { return DH == 128 ? lc ^ ((piece * PR + lk) & 7) : lc ^ fk; };
    const int kl = (int)a.sk.l * 2, vl = (int)a.sv.l * 2;
    auto fetch = [&](int key0, uint64_t bits, int s) {
        char *base = lds + s * STAGE + wk * 2 * TILE;
        const auto kr = __builtin_amdgcn_make_buffer_rsrc((void *)(Kg + (int64_t)key0 * a.sk.l), 0, (KT - 1) * kl + RB, 0x00020000);
        const auto vr = __builtin_amdgcn_make_buffer_rsrc((void *)(Vg + (int64_t)key0 * a.sv.l), 0, (KT - 1) * vl + RB, 0x00020000);
#pragma unroll
        for (int j = 0; j < (PIECES + WQ - 1) / WQ; ++j) {
            const int piece = wq + j * WQ;
            if (PIECES % WQ && piece >= PIECES) break;
            const int key = piece * PR + lk;
            const bool in = (bits >> key) & 1;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void *)(base + piece * 1024), 16, in ? key * kl + chunk_k(piece) * 16 : 0x7ffffff0, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void *)(base + TILE + piece * 1024), 16, in ? key * vl + (lc ^ fv) * 16 : 0x7ffffff0, 0, 0, 0);
        }
    };
    // K: accumulator i of a lane is key 16 (i / 8) + 8 hi + i % 8 when row m = 8 a + 4 b + c of the operand is key 16 (a / 2) + 8 b + 4 (a % 2) + c
    const int krow = 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
    const int kswz = DH == 32 ? (krow >> 1) & 3 : krow & 7;
    // V: four lanes of 16 address four dims of one key each, and get four keys of one dim
    const int vkey = hi * 8 + ((lane & 15) >> 2), vchunk = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const int vswz = DH == 32 ? ((lane & 15) >> 2) & 2 : 2 * ((lane & 15) >> 2);

    const int range0 = split * a.tiles_per_split * KT;
    const int range1 = a.Lk < range0 + a.tiles_per_split * KT ? a.Lk : range0 + a.tiles_per_split * KT;
    for (int seg = range0; seg < range1; seg += SEG_KEYS) {
        const int seg1 = range1 < seg + SEG_KEYS ? range1 : seg + SEG_KEYS;
        const int n = tiles_of<KT, MASK>(tiles, a.key_valid + (int64_t)b * a.Lk, seg, seg1);
        auto tile_at = [&](int i, int &key0) -> uint64_t {
            if (i >= n) return 0;
            const uint64_t all = KT == 64 ? ~0ull : 0xffffffffull;
            if constexpr (MASK) {
                const int t = __builtin_amdgcn_readfirstlane(tiles.list[i]);
                key0 = seg + t * KT;
                const uint64_t w = tiles.bits[t];
                return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(w >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)w);
            } else {
                key0 = seg + i * KT;
                const int left = seg1 - key0;
                return left >= KT ? all : (1ull << left) - 1;
            }
        };
        int key_next = 0;
        uint64_t next = tile_at(wk, key_next);
        if (next) fetch(key_next, next, 0);
        for (int i = 0, s = 0; i < n; i += WK, s ^= 1) {
            const uint64_t bits = next;
            // this stage is there, and nobody reads the other one any more
            if constexpr (WQ > 1) {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
            } else {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            }
            next = tile_at(i + WK + wk, key_next);
            if (next) fetch(key_next, next, s ^ 1);
            if (!bits) continue;
            const char *ks_ = lds + s * STAGE + wk * 2 * TILE, *vs_ = ks_ + TILE;
            f32x16 sc[QB][KT / 32];
#pragma unroll
            for (int sub = 0; sub < KT / 32; ++sub) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sc[qb][sub][e] = 0.f;
#pragma unroll
                for (int ks = 0; ks < DH / 16; ++ks) {
                    const h16x8 kf = *reinterpret_cast<const h16x8 *>(ks_ + (sub * 32 + krow) * RB + ((ks * 2 + hi) ^ kswz) * 16);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) sc[qb][sub] = SF_MFMA16(kf, qf[qb][ks], sc[qb][sub], 0, 0, 0);
                }
            }
            const bool whole = bits == (KT == 64 ? ~0ull : 0xffffffffull);
            uint32_t pk[QB][KT / 32][8];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float top = -INFINITY;
#pragma unroll
                for (int sub = 0; sub < KT / 32; ++sub) {
                    if (!whole) {
                        const uint32_t w = (uint32_t)(bits >> (sub * 32)) >> (8 * hi);
#pragma unroll
                        for (int e = 0; e < 16; ++e) if (!((w >> (16 * (e / 8) + e % 8)) & 1)) sc[qb][sub][e] = -INFINITY;
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, sc[qb][sub][e]);
                }
                top = both_halves_max(top);
                if (__ballot(top * c > m[qb] + SLACK)) {
                    const float mn = fmaxf(m[qb], top * c), f = m[qb] == mn ? 1.f : __builtin_amdgcn_exp2f(m[qb] - mn);
                    m[qb] = mn;
                    l[qb] *= f;
#pragma unroll
                    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[qb][d][e] *= f;
                }
                const float off = LIFT - (m[qb] == -INFINITY ? 0.f : m[qb]);    // all scores so far are -inf: weights of 0
#pragma unroll
                for (int sub = 0; sub < KT / 32; ++sub)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t w = pack2_h16(__builtin_amdgcn_exp2f(fmaf(sc[qb][sub][2 * e], c, off)),
                                                     __builtin_amdgcn_exp2f(fmaf(sc[qb][sub][2 * e + 1], c, off)));
                        pk[qb][sub][e] = w;
                        l[qb] = SF_FDOT2(__builtin_bit_cast(h16x2, w), (h16x2){(h16)1.f, (h16)1.f}, l[qb], false);
                    }
            }
#pragma unroll
            for (int kb = 0; kb < KT / 16; ++kb)
#pragma unroll
                for (int d = 0; d < DH / 32; ++d) {
                    const char *p = vs_ + (kb * 16 + vkey) * RB + ((d * 4 + vchunk) ^ vswz) * 16 + (lane & 1) * 8;
                    struct { s16x4 a, b; } v = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p),
                                                __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * RB))};
                    const h16x8 vf = __builtin_bit_cast(h16x8, v);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) {
                        const uint32_t *w = &pk[qb][kb / 2][(kb & 1) * 4];
                        const h16x8 pf = __builtin_bit_cast(h16x8, make_uint4(w[0], w[1], w[2], w[3]));
                        o[qb][d] = SF_MFMA16(vf, pf, o[qb][d], 0, 0, 0);
                    }
                }
        }
        if constexpr (WQ > 1) __syncthreads();               // the next segment's first stage
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[qb]), __float_as_uint(l[qb]), false, false);
        l[qb] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    const int64_t all_rows = (int64_t)a.B * a.nH * a.Lq;
    if constexpr (WK == 1) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const int i = own.first + (wq * QB + qb) * 32 + r;
            int h, q;
            row_of(a, own.heads, i < own.n ? i : 0, h, q);
            if (a.splits > 1) {
                if (i < own.n) {
                    const int64_t row = ((int64_t)b * a.nH + h) * a.Lq + q + split * all_rows;
#pragma unroll
                    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            *reinterpret_cast<f32x4 *>(a.part + row * DH + d * 32 + e * 8 + hi * 4) =
                                f32x4{o[qb][d][4 * e], o[qb][d][4 * e + 1], o[qb][d][4 * e + 2], o[qb][d][4 * e + 3]};
                    if (hi == 0) *reinterpret_cast<float2 *>(a.ml + row * 2) = make_float2(m[qb], l[qb]);
                }
            } else {
                const float inv = l[qb] == 0.f ? 0.f : 1.0f / l[qb];
                h16 *out = (h16 *)a.O + ((int64_t)b * a.Lq + q) * a.ldo + h * DH;
#pragma unroll
                for (int d = 0; d < DH / 32; ++d)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        // dims 8 e + 4 hi .. of both halves: swapped, a lane has eight dims in a row
                        const auto x = __builtin_amdgcn_permlane32_swap(pack2_h16(o[qb][d][4 * e] * inv, o[qb][d][4 * e + 1] * inv),
                                                                        pack2_h16(o[qb][d][4 * e + 4] * inv, o[qb][d][4 * e + 5] * inv), false, false);
                        const auto y = __builtin_amdgcn_permlane32_swap(pack2_h16(o[qb][d][4 * e + 2] * inv, o[qb][d][4 * e + 3] * inv),
                                                                        pack2_h16(o[qb][d][4 * e + 6] * inv, o[qb][d][4 * e + 7] * inv), false, false);
                        if (i < own.n) *reinterpret_cast<uint4 *>(out + d * 32 + e * 8 + hi * 8) = make_uint4(x[0], y[0], x[1], y[1]);
                    }
            }
        }
    } else {
        // join the waves that walked the keys in turn: [wk][row][dh], then maxima and sums
        float *po = reinterpret_cast<float *>(lds), *pm = po + WK * WQ * 32 * DH;
        static_assert(WQ == 1 && QB == 1, "one block of rows");
        __syncthreads();
        if (hi == 0) pm[wk * 32 + r] = m[0];
        __syncthreads();
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < WK; ++w) M = fmaxf(M, pm[w * 32 + r]);
        const float f = m[0] == M ? 1.f : __builtin_amdgcn_exp2f(m[0] - M);
        if (hi == 0) pm[(WK + wk) * 32 + r] = l[0] * f;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<f32x4 *>(po + (wk * 32 + r) * DH + d * 32 + e * 8 + hi * 4) =
                    f32x4{o[0][d][4 * e] * f, o[0][d][4 * e + 1] * f, o[0][d][4 * e + 2] * f, o[0][d][4 * e + 3] * f};
        __syncthreads();
        constexpr int PER = 32 * DH / (WK * 64);              // dims of a thread: 4, 8 or 16
        const int row = threadIdx.x / (DH / PER), d0 = threadIdx.x % (DH / PER) * PER, i = own.first + row;
        if (i >= own.n) return;
        int h, q;
        row_of(a, own.heads, i, h, q);
        float L = 0.f, v[PER];
#pragma unroll
        for (int w = 0; w < WK; ++w) L += pm[(WK + w) * 32 + row];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            v[e] = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) v[e] += po[(w * 32 + row) * DH + d0 + e];
        }
        if (a.splits > 1) {
            const int64_t at = ((int64_t)b * a.nH + h) * a.Lq + q + split * all_rows;
#pragma unroll
            for (int e = 0; e < PER; e += 4) *reinterpret_cast<f32x4 *>(a.part + at * DH + d0 + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
            float Mr = -INFINITY;
#pragma unroll
            for (int w = 0; w < WK; ++w) Mr = fmaxf(Mr, pm[w * 32 + row]);
            if (d0 == 0) *reinterpret_cast<float2 *>(a.ml + at * 2) = make_float2(Mr, L);
        } else {
            const float inv = L == 0.f ? 0.f : 1.0f / L;
            h16 *out = (h16 *)a.O + ((int64_t)b * a.Lq + q) * a.ldo + h * DH + d0;
#pragma unroll
            for (int e = 0; e < PER; e += 4)
                *reinterpret_cast<uint2 *>(out + e) = make_uint2(pack2_h16(v[e] * inv, v[e + 1] * inv), pack2_h16(v[e + 2] * inv, v[e + 3] * inv));
        }
    }
#endif
}

// ------------------------------------------------------------------------------------------------- fp32 models
// The same with mfma_f32_32x32x2: a lane's accumulators are the second operand of the second product as they stand.  Rows of dh + 1 floats.
template <int WQ, int WK, bool MASK>
__global__ __launch_bounds__(256) void cross_f32_kernel(CrossArgs a)
{
    constexpr int KT = 32, KEYS = WK * KT, ROWS = WQ * 32;
    extern __shared__ __attribute__((aligned(16))) float smem[];
    __shared__ KeyTiles<KT, MASK> tiles;
    const int dh = a.dh, ld = dh + 1;
    float *ksm = smem, *vsm = smem + KEYS * ld;              // 32 floats behind the last row of V: dims past dh are read and not used
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wq = wave % WQ, wk = wave / WQ;
    const int r = lane & 31, hi = lane >> 5;
    const int b = blockIdx.y, split = blockIdx.z;
    const Rows own = find_rows(a, b, blockIdx.x, ROWS);
    if (own.n == 0) return;
    const float *Kg = (const float *)a.K + b * a.sk.b + own.g * a.sk.h, *Vg = (const float *)a.V + b * a.sv.b + own.g * a.sv.h;
    const float c = a.scale * LOG2E;
    const int i = own.first + wq * 32 + r;
    int h, q;
    row_of(a, own.heads, i < own.n ? i : 0, h, q);
    const float *Qr = (const float *)a.Q + b * a.sq.b + h * a.sq.h + q * a.sq.l;
    f32x16 o[4];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    const int range0 = split * a.tiles_per_split * KT;
    const int range1 = a.Lk < range0 + a.tiles_per_split * KT ? a.Lk : range0 + a.tiles_per_split * KT;
    for (int seg = range0; seg < range1; seg += SEG_KEYS) {
        const int seg1 = range1 < seg + SEG_KEYS ? range1 : seg + SEG_KEYS;
        const int n = tiles_of<KT, MASK>(tiles, a.key_valid + (int64_t)b * a.Lk, seg, seg1);
        for (int i0 = 0; i0 < n; i0 += WK) {
            __syncthreads();                                 // the last tiles have been read
            for (int t = 0; t < WK && i0 + t < n; ++t) {
                const int at = MASK ? tiles.list[i0 + t] : i0 + t, key0 = seg + at * KT;
                const uint64_t bits = MASK ? tiles.bits[at] : ~0ull;
                for (int x = threadIdx.x; x < KT * dh; x += 256) {
                    const int k = x / dh, e = x - k * dh;
                    const bool in = key0 + k < seg1 && ((bits >> k) & 1);
                    ksm[(t * KT + k) * ld + e] = in ? Kg[(key0 + k) * a.sk.l + e] : 0.f;
                    vsm[(t * KT + k) * ld + e] = in ? Vg[(key0 + k) * a.sv.l + e] : 0.f;
                }
            }
            __syncthreads();
            if (i0 + wk >= n) continue;
            const int at = MASK ? tiles.list[i0 + wk] : i0 + wk, left = seg1 - (seg + at * KT);
            const uint32_t bits = MASK ? (uint32_t)tiles.bits[at] : left >= KT ? ~0u : (1u << left) - 1;
            const float *kt = ksm + (wk * KT + r) * ld + hi, *vt = vsm + wk * KT * ld + r;
            f32x16 sc;
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = 0.f;
            for (int k = 0; k < dh; k += 2) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(kt[k], Qr[k + hi], sc, 0, 0, 0);
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (!((bits >> (8 * (e / 4) + 4 * hi + e % 4)) & 1)) sc[e] = -INFINITY;
                top = fmaxf(top, sc[e]);
            }
            const float mn = fmaxf(m, both_halves_max(top)), f = m == mn ? 1.f : __builtin_amdgcn_exp2f((m - mn) * c);
            m = mn;
            l *= f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sc[e] = __builtin_amdgcn_exp2f((sc[e] - (m == -INFINITY ? 0.f : m)) * c);       // all scores so far are -inf: weights of 0
                l += sc[e];
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                if (d * 32 >= dh) break;
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= f;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vt[(8 * (e / 4) + 4 * hi + e % 4) * ld + d * 32], sc[e], o[d], 0, 0, 0);
            }
        }
    }
    {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
        l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    m *= c;                                                  // maxima of both kernels are held in powers of two
    const int64_t all_rows = (int64_t)a.B * a.nH * a.Lq;
    float M = m, L = l;
    if constexpr (WK > 1) {
        static_assert(WQ == 1, "one block of rows");
        float *po = smem, *pm = smem + WK * 32 * ld;
        __syncthreads();
        if (hi == 0) pm[wk * 32 + r] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WK; ++w) M = fmaxf(M, pm[w * 32 + r]);
        const float f = m == M ? 1.f : __builtin_amdgcn_exp2f(m - M);
        if (hi == 0) pm[(WK + wk) * 32 + r] = l * f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int dim = d * 32 + 8 * (e / 4) + 4 * hi + e % 4;
                if (dim < dh) po[(wk * 32 + r) * ld + dim] = o[d][e] * f;
            }
        __syncthreads();
        if (wk) return;
        L = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) L += pm[(WK + w) * 32 + r];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int dim = d * 32 + 8 * (e / 4) + 4 * hi + e % 4;
                if (dim >= dh) continue;
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < WK; ++w) v += po[(w * 32 + r) * ld + dim];
                o[d][e] = v;
            }
    }
    if (i >= own.n) return;
    const int64_t row = ((int64_t)b * a.nH + h) * a.Lq + q + split * all_rows;
    const float inv = a.splits > 1 ? 1.f : L == 0.f ? 0.f : 1.0f / L;
    float *out = a.splits > 1 ? a.part + row * dh : (float *)a.O + ((int64_t)b * a.Lq + q) * a.ldo + h * dh;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int dim = d * 32 + 8 * (e / 4) + 4 * hi + e % 4;
            if (dim < dh) out[dim] = o[d][e] * inv;
        }
    if (a.splits > 1 && hi == 0) *reinterpret_cast<float2 *>(a.ml + row * 2) = make_float2(M, L);
}

// O of a row from its key ranges: sums of exp2(m_s - M) parts over that of the weights.  A thread takes four dims and up to JOIN_RANGES ranges, whose
// loads are all in flight at once; `groups` threads along the ranges join in LDS.
constexpr int JOIN_RANGES = 8;
template <class T>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossArgs a, int groups)
{
    __shared__ f32x4 sums[256];
    __shared__ float2 mls[256];
    const int64_t all_rows = (int64_t)a.B * a.nH * a.Lq;
    const int per = a.dh / 4, team = per * groups, rows = 256 / team, t = threadIdx.x % team, d = t % per * 4, y = t / per;
    const int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / team;
    const bool in = (int)threadIdx.x < rows * team && row < all_rows;
    const int h = (int)(row / a.Lq % a.nH), q = (int)(row % a.Lq);
    const int64_t b = row / ((int64_t)a.nH * a.Lq);
    int g = -1;
    if (in) g = a.head_group[(a.pattern_id ? (int64_t)a.pattern_id[b] * a.nH : 0) + h];
    const bool computed = g >= 0 && g < a.nG;                // otherwise its parts were not written
    float2 ml[JOIN_RANGES];
    f32x4 p[JOIN_RANGES], v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < JOIN_RANGES; ++i) {
        const int s = y + i * groups;
        ml[i] = make_float2(-INFINITY, 0.f);
        p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (computed && s < a.splits) {
            ml[i] = *reinterpret_cast<const float2 *>(a.ml + (s * all_rows + row) * 2);
            p[i] = *reinterpret_cast<const f32x4 *>(a.part + (s * all_rows + row) * a.dh + d);
        }
    }
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN_RANGES; ++i) M = fmaxf(M, ml[i].x);
#pragma unroll
    for (int i = 0; i < JOIN_RANGES; ++i) {
        const float f = ml[i].x == M ? 1.f : __builtin_amdgcn_exp2f(ml[i].x - M);
        L = fmaf(f, ml[i].y, L);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(f, p[i][e], v[e]);
    }
    if (groups > 1) {
        mls[threadIdx.x] = make_float2(M, L);
        sums[threadIdx.x] = v;
        __syncthreads();
        if (y) return;
        const float own = M;
        for (int k = 1; k < groups; ++k) M = fmaxf(M, mls[threadIdx.x + k * per].x);
        const float f0 = own == M ? 1.f : __builtin_amdgcn_exp2f(own - M);
        L *= f0;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= f0;
        for (int k = 1; k < groups; ++k) {
            const float2 o = mls[threadIdx.x + k * per];
            const f32x4 w = sums[threadIdx.x + k * per];
            const float f = o.x == M ? 1.f : __builtin_amdgcn_exp2f(o.x - M);
            L = fmaf(f, o.y, L);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(f, w[e], v[e]);
        }
    }
    if (!computed) return;
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    T *out = (T *)a.O + (b * a.Lq + q) * a.ldo + (int64_t)h * a.dh + d;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(out) = make_uint2(pack2_h16(v[0] * inv, v[1] * inv), pack2_h16(v[2] * inv, v[3] * inv));
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = v[e] * inv;
    }
}

// How a call runs: waves along rows and keys, key ranges.
// Waves along the keys where a group has at most one block of rows, so that none idles (64 samples of ten queries, 1024 keys: 17.7 us, along the rows
// 18.8; 256 of four, 480 keys: 26.4 and 26.8; eight of eight, 2048 keys: 13.0 and 11.4).  Key ranges of workgroups of their own where these are fewer
// than the compute units, towards two for each (one query, 4096 keys: 8.7 us, without 22.6; four samples of 128, 4096 keys: 18 and 56).
struct CrossPlan { int wq, wk, kt, runs, splits, tiles_per_split; size_t part, bytes; };
CrossPlan cross_plan(const Dims &D, int64_t Lk, int nH, int nG)
{
    CrossPlan p{};
    const bool half = D.dtype == SF_BF16;
    const int64_t rows = (int64_t)nH * D.L;                   // of all groups of a sample
    const int64_t mean = (rows + nG - 1) / nG;
    p.wq = 4; p.wk = 1;
    if (mean <= 32) { p.wq = 1; p.wk = 4; }
    p.kt = half && p.wk == 1 ? 64 : 32;
    const int own = p.wq * 32;
    p.runs = (int)(rows / own) + nG;                          // at least the runs of all groups, whatever the heads' map
    const int64_t blocks = (int64_t)D.B * ((rows + own - 1) / own > nG ? (rows + own - 1) / own : nG);
    const int64_t tiles = (Lk + p.kt - 1) / p.kt;
    int64_t s = blocks >= 256 ? 1 : (512 + blocks - 1) / blocks;
    const int64_t most = (tiles + p.wk - 1) / p.wk;           // a tile for every wave at least
    s = s < most ? s : most;
    s = s < 64 ? s : 64;
    p.tiles_per_split = (int)((tiles + s - 1) / s);
    p.splits = (int)((tiles + p.tiles_per_split - 1) / p.tiles_per_split);
    Carver c(nullptr);
    if (p.splits > 1) {
        c.take<float>((size_t)p.splits * D.B * rows * D.dh);
        p.part = c.off;
        c.take<float>((size_t)p.splits * D.B * rows * 2);
    }
    p.bytes = c.off;
    return p;
}

int32_t check_cross(const Dims &D, int32_t Lk, int32_t nH, int32_t nG)
{
    if (nH < 1 || nG < 1 || Lk < 1) return fail(SF_ERR_INVALID_ARG, "cross_gqa: nH, nG and Lk must be positive");
    if (nH > 64 || nG > 64) return fail(SF_ERR_SHAPE, "cross_gqa: at most 64 heads and 64 groups");
    if (D.dtype == SF_BF16 ? D.dh != 32 && D.dh != 64 && D.dh != 128 : D.dh % 8 || D.dh > 128)
        return fail(SF_ERR_SHAPE, "cross_gqa: head dim must be 32, 64 or 128 (16 bits) or a multiple of 8 up to 128 (fp32)");
    if (D.B > 65535 || (int64_t)D.L * nH > 1 << 30 || Lk > 1 << 30) return fail(SF_ERR_SHAPE, "cross_gqa: too many samples, rows or keys");
    return SF_OK;
}

template <int DH, int WQ, int WK>
void launch16(const CrossArgs &a, const CrossPlan &p, hipStream_t st)
{
    const dim3 grid((unsigned)p.runs, (unsigned)a.B, (unsigned)p.splits), block(WQ * WK * 64);
    if (a.key_valid) hipLaunchKernelGGL((cross_kernel<DH, WQ, WK, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((cross_kernel<DH, WQ, WK, false>), grid, block, 0, st, a);
}
template <int DH>
void launch_dh(const CrossArgs &a, const CrossPlan &p, hipStream_t st)
{
    if (p.wk == 4) launch16<DH, 1, 4>(a, p, st);
    else launch16<DH, 4, 1>(a, p, st);
}
template <int WQ, int WK, bool MASK>
int32_t launch32(const CrossArgs &a, const CrossPlan &p, hipStream_t st)
{
    auto kern = cross_f32_kernel<WQ, WK, MASK>;
    const size_t lds = ((size_t)2 * WK * 32 * (a.dh + 1) + 32 + (WK > 1 ? 2 * WK * 32 : 0)) * sizeof(float);
    static std::atomic<bool> attr_set{false};     // setting the attribute twice is harmless
    if (!attr_set) {
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 140 * 1024) != hipSuccess)
            return fail(SF_ERR_HIP, "cross_gqa: cannot reserve LDS");
        attr_set = true;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)p.runs, (unsigned)a.B, (unsigned)p.splits), dim3(256), lds, st, a);
    return SF_OK;
}
template <int WQ, int WK>
int32_t launch32(const CrossArgs &a, const CrossPlan &p, hipStream_t st)
{
    return a.key_valid ? launch32<WQ, WK, true>(a, p, st) : launch32<WQ, WK, false>(a, p, st);
}

}  // namespace

}  // namespace sf

using namespace sf;

extern "C" size_t sf_cross_gqa_workspace_bytes(const sf_desc *desc, int32_t Lk, int32_t nH, int32_t nG)
{
    Dims D;
    if (read_desc(desc, D) || check_cross(D, Lk, nH, nG)) return 0;
    return cross_plan(D, Lk, nH, nG).bytes;
}

extern "C" int32_t sf_cross_gqa_forward(const sf_desc *desc, int32_t nH, int32_t nG, int32_t Lk, const void *Q, sf_strides sq, const void *K,
                                        sf_strides sk, const void *V, sf_strides sv, const int32_t *head_group, const int32_t *pattern_id,
                                        const uint8_t *key_valid, void *O, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    Dims D;
    if (int32_t rc = read_desc(desc, D)) return rc;
    if (int32_t rc = check_cross(D, Lk, nH, nG)) return rc;
    if (!Q || !K || !V || !head_group || !O) return fail(SF_ERR_INVALID_ARG, "cross_gqa: NULL argument");
    if (ldo < (int64_t)nH * D.dh) return fail(SF_ERR_INVALID_ARG, "cross_gqa: ldo shorter than nH * dh");
    for (const sf_strides &s : {sq, sk, sv})
        if (s.b < 0 || s.h < 0 || s.l < 0 || s.l > 1 << 22) return fail(SF_ERR_SHAPE, "cross_gqa: strides must not be negative, that of a token at most 2^22 elements");
    if (D.dtype == SF_BF16) {
        for (const sf_strides &s : {sq, sk, sv})
            if ((s.b | s.h | s.l) % 8) return fail(SF_ERR_SHAPE, "cross_gqa: strides of 16-bit tensors must be multiples of 8 elements");
        if ((((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O) & 15) || ldo % 8)
            return fail(SF_ERR_INVALID_ARG, "cross_gqa: 16-byte aligned tensors and rows of O required");
    } else if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O) & 3)
        return fail(SF_ERR_INVALID_ARG, "cross_gqa: tensors aligned to their elements required");
    if (O == Q || O == K || O == V) return fail(SF_ERR_INVALID_ARG, "cross_gqa: O may not alias an input");
    const CrossPlan p = cross_plan(D, Lk, nH, nG);
    if (p.bytes && (!workspace || workspace_bytes < p.bytes || ((uintptr_t)workspace & 255)))
        return fail(SF_ERR_WORKSPACE, "cross_gqa: workspace of %zu bytes (256-byte aligned) required, got %zu", p.bytes, workspace_bytes);
    CrossArgs a{};
    a.Q = Q; a.K = K; a.V = V; a.sq = sq; a.sk = sk; a.sv = sv;
    a.head_group = head_group; a.pattern_id = pattern_id; a.key_valid = key_valid; a.O = O; a.ldo = ldo;
    if (p.splits > 1) { a.part = (float *)workspace; a.ml = (float *)((char *)workspace + p.part); }
    a.B = D.B; a.Lq = D.L; a.Lk = Lk; a.nH = nH; a.nG = nG; a.dh = D.dh; a.splits = p.splits; a.tiles_per_split = p.tiles_per_split;
    a.scale = 1.0f / sqrtf((float)D.dh);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (D.dtype != SF_BF16) {
        if (int32_t rc = p.wk == 4 ? launch32<1, 4>(a, p, st) : launch32<4, 1>(a, p, st)) return rc;
    } else if (D.dh == 32) launch_dh<32>(a, p, st);
    else if (D.dh == 64) launch_dh<64>(a, p, st);
    else launch_dh<128>(a, p, st);
    if (p.splits > 1) {
        const int groups = (p.splits + JOIN_RANGES - 1) / JOIN_RANGES, rows = 256 / (D.dh / 4 * groups);       // at most 64 ranges, 32 threads each
        const dim3 grid((unsigned)(((int64_t)D.B * nH * D.L + rows - 1) / rows));
        if (D.dtype == SF_BF16) hipLaunchKernelGGL(cross_join_kernel<h16>, grid, dim3(256), 0, st, a, groups);
        else hipLaunchKernelGGL(cross_join_kernel<float>, grid, dim3(256), 0, st, a, groups);
    }
    return check_launch("cross_gqa_forward");
}
