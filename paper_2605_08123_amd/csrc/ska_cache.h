// Softmax attention on caches for gfx950 (sinkhorn_attn_cache.h): keys and values in 8 bits, bf16 or fp32, and a prefix that the items
// of a batch share.
//
// A wavefront holds up to NQ blocks of 16 query rows and walks over tiles of keys:
//   S^T = K Q^T  (16x16x32 products, keys as rows),  P = exp(S - m),  O^T += V^T P^T.
// Nothing passes through LDS on the way: the operand layouts are met by the loads.
//   K: lane (x, g) = (lane & 15, lane >> 4) has 16 adjacent bytes of token x: the features that a product sums over may come in any order, so
//      these are whole operands, and 4 lanes read 64 adjacent bytes of a row.
//   V: the second product sums over tokens.  Lane (x, g) reads features x F ... x F + F - 1 (F = d / 16) of the tokens 4 g ... 4 g + 3 of each tile:
//      the tokens whose P this lane has in the accumulators' layout, and F products' operands of 8 tokens after a transposition of bytes
//      inside the lane.  Product j gives features x F + j, so that a lane ends up with d / 4 adjacent features of a row.
// Codes in 8 bits are exact in bf16.  A key's scale is a factor of its score, a value's scale one of its P.
#pragma once
#include "ska_softmax.h"

namespace {

struct E4M3 { unsigned char c; };
struct INT8 { signed char c; };
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Keys and values of one side: the items' own, or the prefix.
struct CaSide {
    SmTensor k, v;                    // (b of the prefix: 0)
    const float *ks, *vs;             // scales, null where there are none
    long ks_b, ks_h, vs_b, vs_h;
    const unsigned char *mask;        // [B][L], prefix: [L]
    const int *len;                   // [B], prefix: [1]
    int L;
    int rows;                         // query rows of a problem: Lq G, prefix: B Lq G
    int problems;                     // B Hk, prefix: Hk
    int ks_waves;                     // wavefronts of a workgroup that share rows and split the keys (1, 2, 4)
    int blocks, parts, wgs;           // blocks of rows, parts of a walk, workgroups: blocks * parts * problems
    SmDiv by_problems, by_blocks, by_span;   // problems, blocks, parts * ks_waves
};
struct CaArgs {
    SmTensor q, o;
    float *lse;
    CaSide side[2];                   // the items' own, the prefix
    const int *start, *len_q;
    const unsigned char *mask_q;
    float *part, *part_lse;           // [parts][B Hk][Lq G][D], [parts][B Hk][Lq G]: the own ones first
    int B, Hk, G, Lq, W, causal;
    int parts;                        // of both sides
    SmDiv by_g, by_hk, by_r;          // G, Hk, Lq G
    float c2;                         // log2(e) / (eps sqrt d)
};

template <typename S> struct CaStore {
    static constexpr int BYTES = (int)sizeof(S);
    static constexpr bool SCALED = BYTES == 1;
    static constexpr int NT = BYTES == 4 ? 1 : 2;   // tiles of 16 keys at a time
    static constexpr int KT = 16 * NT;
};

// Loads through a buffer descriptor: what lies beyond its bytes is not read and comes as 0.
typedef __amdgpu_buffer_rsrc_t CaBuf;
__device__ __forceinline__ CaBuf ca_buffer(const unsigned char *base, unsigned bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(sm_uniform(base)), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
template <int BYTES> __device__ __forceinline__ void ca_load(unsigned *to, CaBuf b, unsigned at)
{
    if constexpr (BYTES == 2) to[0] = __builtin_amdgcn_raw_buffer_load_b16(b, at, 0, 0);
    else if constexpr (BYTES == 4) to[0] = __builtin_amdgcn_raw_buffer_load_b32(b, at, 0, 0);
    else if constexpr (BYTES == 8) {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(b, at, 0, 0);
        to[0] = x[0]; to[1] = x[1];
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(b, at + 16 * i, 0, 0);
#pragma unroll
            for (int w = 0; w < 4; ++w) to[4 * i + w] = x[w];
        }
    }
}

// KT keys and values as they come from memory
template <typename S, int D> struct CaTile {
    using ST = CaStore<S>;
    static constexpr int NT = ST::NT, KB = D * ST::BYTES / 4, KP = KB < 16 ? KB : 16, VB = D / 16 * ST::BYTES;   // bytes per lane of a key, of a load, of a value
    unsigned k[NT][KB / 4], v[NT][4][VB < 4 ? 1 : VB / 4];
    float ks[NT][4], vs[NT][4];
    unsigned char act;
    // rows 0 ... rows - 1 (>= 1) of the tile at token j0 exist
    __device__ __forceinline__ void load(const CaSide &s, const unsigned char *kb, const unsigned char *vb, const float *ksb, const float *vsb,
                                         const unsigned char *mask, int j0, int rows, int x, int g)
    {
        const unsigned kst = (unsigned)(s.k.l * ST::BYTES), vst = (unsigned)(s.v.l * ST::BYTES);
        const unsigned last = (unsigned)(min(rows, ST::KT) - 1);
        const CaBuf bk = ca_buffer(kb + (long)j0 * kst, last * kst + D * ST::BYTES), bv = ca_buffer(vb + (long)j0 * vst, last * vst + D * ST::BYTES);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int p = 0; p < KB / KP; ++p) ca_load<KP>(&k[n][p * KP / 4], bk, (unsigned)(16 * n + x) * kst + (unsigned)(p * 4 * KP + g * KP));
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) ca_load<VB>(v[n][e], bv, (unsigned)(16 * n + 4 * g + e) * vst + (unsigned)(x * VB));
        if constexpr (ST::SCALED) {
            const CaBuf b0 = ca_buffer(reinterpret_cast<const unsigned char *>(ksb + j0), 4 * last + 4), b1 = ca_buffer(reinterpret_cast<const unsigned char *>(vsb + j0), 4 * last + 4);
            if (rows >= ST::KT) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    ca_load<16>(reinterpret_cast<unsigned *>(ks[n]), b0, (unsigned)(16 * n + 4 * g) * 4);
                    ca_load<16>(reinterpret_cast<unsigned *>(vs[n]), b1, (unsigned)(16 * n + 4 * g) * 4);
                }
            } else {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ca_load<4>(reinterpret_cast<unsigned *>(&ks[n][e]), b0, (unsigned)(16 * n + 4 * g + e) * 4);
                        ca_load<4>(reinterpret_cast<unsigned *>(&vs[n][e]), b1, (unsigned)(16 * n + 4 * g + e) * 4);
                    }
            }
        }
        if (mask) act = mask[j0 + min(x + 16 * (g & 1), (int)last)];
    }
};

// 8 codes as bf16
__device__ __forceinline__ bf16x2 ca_pair(float a, float b) { return bf16x2{(__bf16)a, (__bf16)b}; }
template <typename S> __device__ __forceinline__ bf16x8 ca_codes(unsigned a, unsigned b)
{
    bf16x8 r;
    const unsigned w[2] = {a, b};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        bf16x2 lo, hi;
        if constexpr (std::is_same<S, E4M3>::value) {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, true);
        } else {
            lo = ca_pair((float)(signed char)w[i], (float)(signed char)(w[i] >> 8));
            hi = ca_pair((float)(signed char)(w[i] >> 16), (float)(signed char)(w[i] >> 24));
        }
        r[4 * i] = lo[0]; r[4 * i + 1] = lo[1]; r[4 * i + 2] = hi[0]; r[4 * i + 3] = hi[1];
    }
    return r;
}
// feature j (of the lane's F) of two tokens whose words that hold it are a and b
template <typename S> __device__ __forceinline__ bf16x2 ca_feature(unsigned a, unsigned b, int j)
{
    if constexpr (std::is_same<S, E4M3>::value) {
        // bytes a0 b0 a1 b1, or a2 b2 a3 b3
        const unsigned w = (j & 3) < 2 ? __builtin_amdgcn_perm(b, a, 0x05010400u) : __builtin_amdgcn_perm(b, a, 0x07030602u);
        return j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
    } else if constexpr (std::is_same<S, INT8>::value) {
        const int at = 8 * (j & 3);
        return ca_pair((float)(signed char)(a >> at), (float)(signed char)(b >> at));
    } else {
        return __builtin_bit_cast(bf16x2, j & 1 ? __builtin_amdgcn_perm(b, a, 0x07060302u) : __builtin_amdgcn_perm(b, a, 0x05040100u));
    }
}

// Query rows as operands: lane (x, g) has of row x the features that its pieces of a key hold.  fp32 queries of 8-bit caches are the
// sum of three bf16 numbers, cut off and not rounded: all 24 bits, and none overflows.
template <typename S, typename T, int D> struct CaQuery {
    static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    bf16x8 v[PARTS][D / 32];
    __device__ __forceinline__ void load(const T *row, int g)
    {
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            // 8 bits: 16 features adjacent (d = 32: 8), two operands; bf16: 8
            const int at = CaStore<S>::BYTES == 1 && D > 32 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            if constexpr (PARTS == 1) v[0][s] = *reinterpret_cast<const bf16x8 *>(row + at);
            else {
                float f[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) load4<float>(reinterpret_cast<const float *>(row) + at + 4 * i, reinterpret_cast<float(&)[4]>(f[4 * i]));
#pragma unroll
                for (int p = 0; p < 3; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float cut = __uint_as_float(__float_as_uint(f[i]) & 0xffff0000u);
                        v[p][s][i] = __builtin_bit_cast(__bf16, (unsigned short)(__float_as_uint(f[i]) >> 16));
                        f[i] = isinf(f[i]) ? 0.f : f[i] - cut;
                    }
            }
        }
    }
};
template <int D> struct CaQuery<float, float, D> {
    float v[D / 4];   // 16 c + 4 g + j at 4 c + j
    __device__ __forceinline__ void load(const float *row, int g)
    {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) load4<float>(row + 16 * c + 4 * g, reinterpret_cast<float(&)[4]>(v[4 * c]));
    }
};

__device__ __forceinline__ float ca_max_groups(float x)   // over the four lanes that share a row
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return sm_max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// A row of a problem: item, query, head
struct CaRow { int b, i, hq, at; };   // at: row of (b, hk)'s Lq G
__device__ __forceinline__ CaRow ca_row(const CaArgs &a, bool prefix, int b, int hk, int r)
{
    CaRow w;
    w.b = prefix ? a.by_r(r) : b;
    w.at = prefix ? r - w.b * (a.Lq * a.G) : r;
    w.i = a.by_g(w.at);
    w.hq = hk * a.G + (w.at - w.i * a.G);
    return w;
}

// Results of a row from its running maximum (powers of two), sum and whether it has met a key: factor of the accumulators, LSE
__device__ __forceinline__ float ca_finish(float m, float sum, bool live, bool parts, float &lse)
{
    // (a row without a key is zeros, one that a NaN or an infinite score has poisoned is NaN; scores of -inf alone are 0 / 0, in a part they weigh nothing)
    const bool nothing = sum == 0.f;
    lse = !live ? -INFINITY : !nothing ? (m + fast_log2(sum)) * LN2 : parts ? SM_NOTHING : NAN;
    return nothing && parts ? 0.f : 1.f / sum;
}

template <typename S, typename T, int D, int NQ>
__global__ __launch_bounds__(256, 1) void ca_attn_kernel(const CaArgs a)
{
    using ST = CaStore<S>;
    using TL = CaTile<S, D>;
    constexpr int NT = ST::NT, KT = ST::KT, F = D / 16, PITCH = D + 4;
    constexpr int PP = sizeof(T) == 4 ? 3 : 2;   // bf16 parts of P
    __shared__ __align__(16) float red[4][16][PITCH];
    __shared__ float red_m[4][16], red_l[4][16];
    __shared__ int red_live[4][16];

    const bool prefix = (int)blockIdx.x >= a.side[0].wgs;
    const CaSide &s = a.side[prefix ? 1 : 0];
    int at = (int)blockIdx.x - (prefix ? a.side[0].wgs : 0);
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), x = lane & 15, g = lane >> 4;
    // problems fastest, then blocks, then parts
    int rest = s.by_problems(at);
    const int prob = at - rest * s.problems, part = s.by_blocks(rest), blk = rest - part * s.blocks;
    const int b0 = prefix ? 0 : a.by_hk(prob), hk = prefix ? prob : prob - b0 * a.Hk;
    const int kw = s.ks_waves, rw = wv / kw, kq = wv - rw * kw;
    const int r0 = (blk * (4 / kw) + rw) * 16 * NQ;
    const int P = prefix ? sm_len(s.len, 0, s.L) : 0, up = a.causal ? 0 : a.W;
    const int nb_live = min(NQ, (s.rows - r0 + 15) >> 4);   // blocks of rows that exist (may be <= 0)

    // this lane's rows
    CaQuery<S, T, D> q[NQ];
    int my_lo[NQ], my_hi[NQ];
    unsigned live = 0, keys = 0;   // a bit per block: the row takes part; it has met a key
    int lo = 0x7fffffff, hi = -1, all_lo = 0, all_hi = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int r = r0 + 16 * n + x;
        const CaRow w = ca_row(a, prefix, b0, hk, min(r, s.rows - 1));
        bool on = r < s.rows && w.i < sm_len(a.len_q, w.b, a.Lq);
        if (on && a.mask_q) on = a.mask_q[(long)w.b * a.Lq + w.i] != 0;
        const int p = (a.start ? min(max(a.start[w.b], 0), 1 << 24) : 0) + w.i;   // behind the prefix
        my_lo[n] = max(0, prefix ? P + p - a.W : p - a.W);
        my_hi[n] = prefix ? P - 1 : min(p + up, sm_len(s.len, w.b, s.L) - 1);
        if (n < nb_live) q[n].load(reinterpret_cast<const T *>(a.q.p) + w.b * a.q.b + w.hq * a.q.h + w.i * a.q.l, g);
        if (on) {
            live |= 1u << n;
            lo = min(lo, my_lo[n]); hi = max(hi, my_hi[n]);
            all_lo = max(all_lo, my_lo[n]); all_hi = min(all_hi, my_hi[n]);
        } else {
            my_lo[n] = 0x3fffffff; my_hi[n] = -1;
        }
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        lo = min(lo, __shfl_xor(lo, d)); hi = max(hi, __shfl_xor(hi, d));
        all_lo = max(all_lo, __shfl_xor(all_lo, d)); all_hi = min(all_hi, __shfl_xor(all_hi, d));
    }
    lo = __builtin_amdgcn_readfirstlane(lo); hi = __builtin_amdgcn_readfirstlane(hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo); all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    // this wavefront's tiles: every kw-th of the part's
    const int tiles = hi < lo ? 0 : (hi - lo + KT) / KT;
    const int per = s.by_span(tiles + s.parts * kw - 1) * kw;
    const int t1 = min(tiles, (part + 1) * per);
    int t = part * per + kq;

    f32x4 acc[NQ][F];
    float m[NQ], sum[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int j = 0; j < F; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const unsigned char *kb = reinterpret_cast<const unsigned char *>(s.k.p) + (b0 * s.k.b + hk * s.k.h) * ST::BYTES;
    const unsigned char *vb = reinterpret_cast<const unsigned char *>(s.v.p) + (b0 * s.v.b + hk * s.v.h) * ST::BYTES;
    const float *ksb = ST::SCALED ? s.ks + b0 * s.ks_b + hk * s.ks_h : nullptr, *vsb = ST::SCALED ? s.vs + b0 * s.vs_b + hk * s.vs_h : nullptr;
    const unsigned char *mk = s.mask ? s.mask + (long)b0 * s.L : nullptr;
    const float c2 = sm_vector(a.c2), none = sm_vector(-INFINITY);

    auto fetch = [&](TL &tl, int t) __attribute__((always_inline)) {
        const int j0 = lo + t * KT;
        tl.load(s, kb, vb, ksb, vsb, mk, j0, hi + 1 - j0, x, g);
    };
    auto step = [&](TL &tl, int t) __attribute__((always_inline)) {
        const int j0 = lo + t * KT;
        unsigned on = sm_bits(0, hi - j0);
        if (mk) on &= (unsigned)__ballot(tl.act != 0);   // (lanes 0 ... 31: keys 0 ... 31)
        if constexpr (KT == 16) on &= 0xffffu;
        constexpr unsigned FULL = KT == 32 ? 0xffffffffu : 0xffffu;
        const bool whole = on == FULL && j0 >= all_lo && j0 + KT - 1 <= all_hi;
        if (on != FULL) {   // what does not count must not meet a product: P is 0 there, and may be 0 times anything
            const unsigned mine = on >> (4 * g);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool ok = mine >> (16 * n + e) & 1;
#pragma unroll
                    for (int w = 0; w < (TL::VB < 4 ? 1 : TL::VB / 4); ++w) tl.v[n][e][w] = ok ? tl.v[n][e][w] : 0u;
                    if constexpr (ST::SCALED) tl.vs[n][e] = ok ? tl.vs[n][e] : 0.f;
                }
        }
        if (whole) keys = ~0u;
        bf16x8 kf[NT][D / 32], vf[F];
        float kc[NT][4];
        if constexpr (ST::BYTES == 1) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < D / 32; ++c) kf[n][c] = ca_codes<S>(tl.k[n][2 * c], tl.k[n][2 * c + 1]);
        } else if constexpr (ST::BYTES == 2) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
                    kf[n][c] = __builtin_bit_cast(bf16x8, u32x4{tl.k[n][4 * c], tl.k[n][4 * c + 1], tl.k[n][4 * c + 2], tl.k[n][4 * c + 3]});
        }
        if constexpr (ST::BYTES < 4) {
#pragma unroll
            for (int j = 0; j < F; ++j) {
                constexpr int PER = 4 / ST::BYTES;   // features of a word
#pragma unroll
                for (int i = 0; i < 4; ++i) {        // tokens 2 i, 2 i + 1 of the operand's 8: four of each tile
                    const bf16x2 y = ca_feature<S>(tl.v[i >> 1][2 * (i & 1)][j / PER], tl.v[i >> 1][2 * (i & 1) + 1][j / PER], j);
                    vf[j][2 * i] = y[0]; vf[j][2 * i + 1] = y[1];
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) kc[n][e] = ST::SCALED ? tl.ks[n][e] * c2 : c2;
#pragma unroll
        for (int nb = 0; nb < NQ; ++nb) {
            if (nb >= nb_live) break;
            f32x4 sc[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                sc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
                if constexpr (ST::BYTES == 4) {
#pragma unroll
                    for (int c = 0; c < D / 4; ++c) sc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tl.k[n][c]), q[nb].v[c], sc[n], 0, 0, 0);
                } else {
#pragma unroll
                    for (int p = CaQuery<S, T, D>::PARTS - 1; p >= 0; --p)   // (the smallest part first)
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n][c], q[nb].v[p][c], sc[n], 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[n][e] *= kc[n][e];
            }
            if (!whole) {
                const unsigned own = sm_bits(my_lo[nb] - j0, my_hi[nb] - j0) & on, keep = own >> (4 * g);
                if (own) keys |= 1u << nb;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[n][e] = sm_keep(sc[n][e], keep, 16 * n + e, none);
            }
            // The running maximum moves when a score of any lane exceeds it by 2^SM_LAZY: lanes are compared with no exchange between them
            float top = sc[0][0];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[n][e]);
            if (__any(top > m[nb] + SM_LAZY)) {
                const float mn = fmaxf(m[nb], ca_max_groups(top)), f = mn > -INFINITY ? fast_exp2(m[nb] - mn) : 1.f;
                sum[nb] *= f;
#pragma unroll
                for (int j = 0; j < F; ++j) acc[nb][j] *= f;
                m[nb] = mn;
            }
            const float mu = m[nb] > -INFINITY ? m[nb] : 0.f;
            float p[4 * NT];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[4 * n + e] = fast_exp2(sc[n][e] - mu);
                    sum[nb] += p[4 * n + e];
                    if constexpr (ST::SCALED) p[4 * n + e] *= tl.vs[n][e];
                }
            if constexpr (ST::BYTES == 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < F; ++j) acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tl.v[0][e][j]), p[e], acc[nb][j], 0, 0, 0);
            } else {
#pragma unroll
                for (int h = 0; h < PP; ++h) {
                    const bf16x8 pf = pack8(p);
#pragma unroll
                    for (int j = 0; j < F; ++j) acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j], pf, acc[nb][j], 0, 0, 0);
                    if (h + 1 < PP) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] -= (float)pf[e];
                    }
                }
            }
        }
    };
    TL ta, tb;
    if (t < t1) fetch(ta, t);
    while (t < t1) {
        if (t + kw < t1) fetch(tb, t + kw);
        SM_READ_FIRST();
        step(ta, t);
        t += kw;
        if (t >= t1) break;
        if (t + kw < t1) fetch(ta, t + kw);
        SM_READ_FIRST();
        step(tb, t);
        t += kw;
    }

    const long rows = (long)a.B * a.Hk * a.Lq * a.G;
    const int slot = part + (prefix ? a.side[0].parts : 0);
    // four adjacent features of a row, from feature f on
    auto put = [&](const CaRow &w, int f, const f32x4 &y) {
        if (a.parts > 1) *reinterpret_cast<f32x4 *>(a.part + ((slot * rows + ((long)w.b * a.Hk + hk) * (a.Lq * a.G) + w.at) * D + f)) = y;
        else store4<T>(reinterpret_cast<T *>(const_cast<void *>(a.o.p)) + w.b * a.o.b + w.hq * a.o.h + w.i * a.o.l + f, y[0], y[1], y[2], y[3]);
    };
    auto put_lse = [&](const CaRow &w, float lse) {
        if (a.parts > 1) a.part_lse[slot * rows + ((long)w.b * a.Hk + hk) * (a.Lq * a.G) + w.at] = lse;
        else a.lse[((long)w.b * a.G * a.Hk + w.hq) * a.Lq + w.i] = lse;
    };
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        float l = sum[n] + __shfl_xor(sum[n], 16);
        l += __shfl_xor(l, 32);
        const bool met = (live >> n & 1) && (keys >> n & 1);
        if (kw == 1) {
            const int r = r0 + 16 * n + x;
            if (r < s.rows) {
                const CaRow w = ca_row(a, prefix, b0, hk, r);
                float lse;
                const float scale = ca_finish(m[n], l, met, a.parts > 1, lse);
#pragma unroll
                for (int f = 0; f < F; ++f) {   // features (4 g + e) F + j, four at a time
                    f32x4 y;
#pragma unroll
                    for (int c = 0; c < 4; ++c) y[c] = met ? acc[n][(4 * f + c) % F][(4 * f + c) / F] * scale : 0.f;
                    put(w, 4 * F * g + 4 * f, y);
                }
                if (g == 0) put_lse(w, lse);
            }
        } else {
            if (n) __syncthreads();
#pragma unroll
            for (int f = 0; f < F; ++f) {
                f32x4 y;
#pragma unroll
                for (int c = 0; c < 4; ++c) y[c] = acc[n][(4 * f + c) % F][(4 * f + c) / F];
                *reinterpret_cast<f32x4 *>(&red[wv][x][4 * F * g + 4 * f]) = y;
            }
            if (g == 0) {
                red_m[wv][x] = m[n];
                red_l[wv][x] = l;
                red_live[wv][x] = met;
            }
            __syncthreads();
            // the kw wavefronts of the same rows: each of their threads takes four features of a row at a time
            for (int u = kq * 64 + lane; u < 16 * (D / 4); u += kw * 64) {
                const int row = u / (D / 4), f = (u % (D / 4)) * 4, r = r0 + 16 * n + row;
                float M = -INFINITY, L = 0.f;
                bool any = false;
                for (int k = 0; k < kw; ++k) {
                    M = fmaxf(M, red_m[rw * kw + k][row]);
                    any |= red_live[rw * kw + k][row] != 0;
                }
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
                for (int k = 0; k < kw; ++k) {
                    const float mk2 = red_m[rw * kw + k][row], c = mk2 > -INFINITY ? fast_exp2(mk2 - M) : 0.f;
                    L = fmaf(red_l[rw * kw + k][row], c, L);
                    y += *reinterpret_cast<const f32x4 *>(&red[rw * kw + k][row][f]) * c;
                }
                if (r < s.rows) {
                    const CaRow w = ca_row(a, prefix, b0, hk, r);
                    float lse;
                    const float scale = ca_finish(M, L, any, a.parts > 1, lse);
                    put(w, f, any ? y * scale : f32x4{0.f, 0.f, 0.f, 0.f});
                    if (f == 0) put_lse(w, lse);
                }
            }
        }
    }
}

// Joins the parts of a row: weighted by exp(their LSE - the largest).  A thread takes four features over every slices-th part; parts
// without a key are not read.
template <typename T, int D> __global__ __launch_bounds__(NTHREADS) void ca_join_kernel(const CaArgs a, int slices)
{
    constexpr int FT = D / 4;
    __shared__ f32x4 sx[NTHREADS];
    __shared__ float sm[NTHREADS], sl[NTHREADS];
    const int R = a.Lq * a.G, f = (threadIdx.x % FT) * 4, rest = threadIdx.x / FT, slice = rest % slices;
    const long rows = (long)a.B * a.Hk * R, row = (long)blockIdx.x * (NTHREADS / FT / slices) + rest / slices;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (row < rows) {
#pragma unroll 4
        for (int s = slice; s < a.parts; s += slices) {
            const float lse = a.part_lse[s * rows + row];
            if (lse == -INFINITY) continue;
            const f32x4 y = *reinterpret_cast<const f32x4 *>(a.part + (s * rows + row) * D + f);
            // (fmaxf passes over a NaN, so that m never is one; c is, and l and x from there on)
            const float mn = fmaxf(m, lse), old = m > -INFINITY ? fast_exp2((m - mn) * LOG2E) : 0.f, c = fast_exp2((lse - mn) * LOG2E);
            l = fmaf(l, old, c);
            x = x * old + y * c;
            m = mn;
        }
    }
    if (slices > 1) {
        sx[threadIdx.x] = x;
        sm[threadIdx.x] = m;
        sl[threadIdx.x] = l;
        __syncthreads();
        if (slice) return;
        for (int s = 1; s < slices; ++s) {
            const int o = threadIdx.x + s * FT;
            const float mo = sm[o], lo = sl[o];
            const float mn = fmaxf(m, mo), old = m > -INFINITY ? fast_exp2((m - mn) * LOG2E) : 1.f, c = mo > -INFINITY ? fast_exp2((mo - mn) * LOG2E) : 1.f;
            l = l * old + lo * c;   // (a slice that has met nothing but NaN has m = -inf and l = NaN)
            x = x * old + sx[o] * c;
            m = mn;
        }
    }
    if (row >= rows) return;
    const int prob = (int)(row / R), r = (int)(row - (long)prob * R), b = a.by_hk(prob), hk = prob - b * a.Hk;
    const CaRow w = ca_row(a, false, b, hk, r);
    if (m == SM_NOTHING) l = NAN;   // (keys, whose scores are all -inf)
    const float c = l == 0.f ? 0.f : 1.f / l;
    store4<T>(reinterpret_cast<T *>(const_cast<void *>(a.o.p)) + w.b * a.o.b + w.hq * a.o.h + w.i * a.o.l + f, x[0] * c, x[1] * c, x[2] * c, x[3] * c);
    if (f == 0) a.lse[((long)b * a.Hk * a.G + w.hq) * a.Lq + w.i] = l == 0.f ? -INFINITY : m + fast_log2(l) * LN2;
}

}  // namespace
