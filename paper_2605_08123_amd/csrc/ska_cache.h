// Softmax attention on caches for gfx950 (sinkhorn_attn_cache.h): keys and values in 8 bits, bf16 or fp32, and a prefix that the items
// of a batch share.
//
// A wavefront holds NQ blocks of 16 query rows and walks over tiles of keys:
//   S^T = K Q^T  (16x16x32 products, keys as rows),  P = exp(S - m),  O^T += V^T P^T.
// Eight wavefronts of a workgroup have the same rows and take every eighth tile each; their sums are joined in LDS at the end, parts of a
// walk in other workgroups by ca_join_kernel.  The queries' operands lie in LDS, read again for each tile; keys and values go straight from memory
// into registers (keys in bf16 by way of LDS, mostly), where the operand layouts are met by the loads:
//   K: lane (x, g) = (lane & 15, lane >> 4) has 16 adjacent bytes of token x: the features that a product sums over may come in any order, so
//      these are whole operands, and 4 lanes read 64 adjacent bytes of a row.
//   V: the second product sums over tokens.  Lane (x, g) reads features x F ... x F + F - 1 (F = d / 16) of the tokens 4 g ... 4 g + 3 of each tile:
//      the tokens whose P this lane has in the accumulators' layout, and F products' operands of 8 tokens after a transposition of bytes
//      inside the lane.  Product j gives features x F + j, so that a lane ends up with d / 4 adjacent features of a row.
// Codes in 8 bits are exact in bf16 and in fp16.  A key's scale is a factor of its score, a value's scale one of its P.
//
// What bounds it, in us of the kernel alone: few rows, memory (a token of 8 items, 16 heads on 4 of d = 128, int8 caches of 32768: 46, 4.5 TB/s; four
// items, 8 heads on 2 of d = 64, e4m3, 65536: 14.6, 3.7 TB/s, of which about 5 are the first loads' and the last sums' latency).  Many rows,
// vector instructions and products, which do not cover each other (2048 tokens of 8 heads on 2, d = 64, 16384 keys in e4m3: 71; a wavefront issues 187 of
// the former beside the 32 products of a tile of 32 keys and 64 rows: 115 for P, 40 that turn codes into operands, 16 for the values' scales; they take 65 %
// of the time that a CU is busy, products 28 %, with two wavefronts to a SIMD).  fp32 queries: six products for two (the same 142: 58 % and 41 %).  One look at
// a tile decides for all blocks whether a maximum moves (a maximum per tile and block: 81).  bf16 caches, d = 128, 32 rows: the only instance
// that does not fit its registers (24 spilled; two tokens of 64 items, 2 heads on 1, 216039 shared keys: 78).
#pragma once
#include "ska_cache_plan.h"
#include "ska_softmax.h"

namespace {

struct E4M3 { unsigned char c; };
struct INT8 { signed char c; };
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

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
    int blocks, parts;                // blocks of a workgroup's rows in a problem, parts of a walk
    int units, wgs;                   // blocks * parts * problems; the same as a multiple of 8
    int order;                        // CaOrder
    SmDiv by_problems, by_blocks, by_parts, by_span;   // problems, blocks, parts, parts * wavefronts of a workgroup
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

// KT keys and values as they come from memory.  Keys as they are used, 16 rows of 16 bytes a quarter of a load, unless STAGED: bf16 rows of 128
// and 256 bytes are loaded as they lie, 1024 adjacent bytes at a time (C lanes a row), and handed over in LDS, where chunk c of 16 bytes of row
// r lies at c ^ turn(r), so that 8 rows' chunks are in 8 groups of banks.  The cache's lines are asked for once instead of four times: five
// queries of 16 items on 262144 keys, d = 128, 252 -> 178 us; one of 64 items, 4 key heads, 2048 behind 16384, d = 64, 38 -> 33.  Others lose by LDS,
// which has the queries too, or wait for products (four blocks of rows, d = 64: 40 -> 42 us for 94 items on 97725; fp32, d = 128: 145 -> 154 for 128
// rows on 100039; e4m3, d = 64: 70 -> 77 for 2048 tokens on 16384; int8, d = 128: 76 -> 85).
template <typename S, int D, int NQ> struct CaTile {
    using ST = CaStore<S>;
    static constexpr int NT = ST::NT, RB = D * ST::BYTES, C = RB / 16, KB = RB / 4, KP = KB < 16 ? KB : 16, VB = RB / 16;   // bytes of a row, of a lane of a key, of its load, of a value
    static constexpr bool STAGED = ST::BYTES == 2 && RB >= (NQ <= 2 ? 128 : 256);
    static constexpr int PER = 64 / C, LOADS = ST::KT / PER;   // rows of a load, loads
    unsigned k[NT][KB / 4], v[NT][4][VB < 4 ? 1 : VB / 4];
    float ks, vs;   // of key lane & 31
    unsigned char act;
    static __device__ __forceinline__ int turn(int r) { return r & 7; }
    // Rows 0 ... rows - 1 (>= 1) of the tile at token j0 exist.  Keys, with all scales and activity:
    __device__ __forceinline__ void load_keys(unsigned st, const unsigned char *kb, const float *ksb, const float *vsb, const unsigned char *mask, int j0, int rows,
                                              int x, int g)
    {
        const unsigned last = (unsigned)(min(rows, ST::KT) - 1), mine = (unsigned)min(x + 16 * (g & 1), (int)last);
        const CaBuf b = ca_buffer(kb + (long)j0 * st, last * st + RB);
        if constexpr (STAGED) {
            const int lane = 16 * g + x, r = lane / C;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) ca_load<16>(&k[0][4 * i], b, (unsigned)(i * PER + r) * st + 16u * (lane % C ^ turn(i * PER + r)));
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int p = 0; p < KB / KP; ++p) ca_load<KP>(&k[n][p * KP / 4], b, (unsigned)(16 * n + x) * st + (unsigned)(p * 4 * KP + g * KP));
        }
        if constexpr (ST::SCALED) {
            ks = ksb[j0 + mine];
            vs = vsb[j0 + mine];
        }
        if (mask) act = mask[j0 + mine];
    }
    __device__ __forceinline__ void put_keys(u32x4 *to, int lane) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) to[i * 64 + lane] = u32x4{(&k[0][0])[4 * i], (&k[0][0])[4 * i + 1], (&k[0][0])[4 * i + 2], (&k[0][0])[4 * i + 3]};
    }
    // the lane's 16 bytes p of key 16 n + x
    __device__ __forceinline__ u32x4 key(const u32x4 *staged, int n, int p, int x, int g) const
    {
        if constexpr (STAGED) return staged[(16 * n + x) * C + (4 * p + g ^ turn(x))];
        else return u32x4{k[n][4 * p], k[n][4 * p + 1], k[n][4 * p + 2], k[n][4 * p + 3]};
    }
    __device__ __forceinline__ void load_values(unsigned st, const unsigned char *vb, int j0, int rows, int x, int g)
    {
        const unsigned last = (unsigned)(min(rows, ST::KT) - 1);
        const CaBuf b = ca_buffer(vb + (long)j0 * st, last * st + D * ST::BYTES);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) ca_load<VB>(v[n][e], b, (unsigned)(16 * n + 4 * g + e) * st + (unsigned)(x * VB));
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

// the same in fp16, of codes in 8 bits
template <typename S> __device__ __forceinline__ f16x2 ca_feature_half(unsigned a, unsigned b, int j)
{
    if constexpr (std::is_same<S, E4M3>::value) {
        const unsigned w = (j & 3) < 2 ? __builtin_amdgcn_perm(b, a, 0x05010400u) : __builtin_amdgcn_perm(b, a, 0x07030602u);
        return j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
    } else {
        // 1024 + (128 + c) as fp16 numbers, whose last bits are a byte (three instructions for two codes; conversions are nine for four)
        const unsigned w = __builtin_amdgcn_perm(b, a, 0x0c040c00u + 0x00010001u * (j & 3)) ^ 0x64806480u;
        return __builtin_bit_cast(f16x2, w) - f16x2{(_Float16)1152.f, (_Float16)1152.f};
    }
}

// Query rows as operands in LDS, a piece of 16 bytes for each lane: lane (x, g) has of row x the features that its pieces of a key hold.
// fp32 queries of 8-bit caches are the sum of three bf16 numbers, cut off and not rounded: all 24 bits, and none overflows.
template <typename S, typename T, int D> struct CaQuery {
    static constexpr bool PLAIN = CaStore<S>::BYTES == 4;                  // products in fp32
    static constexpr int PARTS = !PLAIN && sizeof(T) == 4 ? 3 : 1, STEPS = PLAIN ? D / 16 : D / 32, PIECES = PARTS * STEPS;   // of a block of 16 rows
    static constexpr int WORDS = PARTS == 1 ? 4 : 8;
    unsigned w[WORDS];   // of step s of a block whose row x is at `row`
    __device__ __forceinline__ void load(const T *row, int s, int g)
    {
        // 8 bits: 16 features adjacent (d = 32: 8), two operands; bf16: 8; fp32: 4
        const int at = PLAIN ? 16 * s + 4 * g : CaStore<S>::BYTES == 1 && D > 32 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) {
            const uint4 y = *reinterpret_cast<const uint4 *>(row + at + 4 * i);
            w[4 * i] = y.x; w[4 * i + 1] = y.y; w[4 * i + 2] = y.z; w[4 * i + 3] = y.w;
        }
    }
    // into `to`: the block's pieces, this lane's 16 bytes of each
    __device__ __forceinline__ void put(uint4 *to, int s, bool on) const
    {
        const auto keep = [&](uint4 y) { return on ? y : make_uint4(0, 0, 0, 0); };
        if constexpr (PARTS == 1) to[s * 64] = keep(make_uint4(w[0], w[1], w[2], w[3]));
        else {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                unsigned y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_perm(__float_as_uint(f[2 * i + 1]), __float_as_uint(f[2 * i]), 0x07060302u);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = isinf(f[i]) ? 0.f : f[i] - __uint_as_float(__float_as_uint(f[i]) & 0xffff0000u);
                to[(p * STEPS + s) * 64] = keep(make_uint4(y[0], y[1], y[2], y[3]));
            }
        }
    }
};

__device__ __forceinline__ float ca_max_groups(float x)   // over the four lanes that share a row
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return sm_max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

// A row of a problem: item, query, head
struct CaRow { int b, i, hq, at; };   // at: row of (b, hk)'s Lq G
__device__ __forceinline__ CaRow ca_row(const CaArgs &a, bool shared, int b, int hk, int r)
{
    CaRow w;
    w.b = shared ? a.by_r(r) : b;
    w.at = shared ? r - w.b * (a.Lq * a.G) : r;
    w.i = a.by_g(w.at);
    w.hq = hk * a.G + (w.at - w.i * a.G);
    return w;
}

constexpr float CA_LEAST = -3.402823466e38f;   // a running maximum before the first score

// Results of a row from its running maximum (powers of two), sum and whether it has met a key: factor of the accumulators, LSE
__device__ __forceinline__ float ca_finish(float m, float sum, bool live, bool parts, float &lse)
{
    // (a row without a key is zeros, one that a NaN or an infinite score has poisoned is NaN; scores of -inf alone are 0 / 0, in a part they weigh nothing)
    const bool nothing = sum == 0.f;
    lse = !live ? -INFINITY : !nothing ? (m + fast_log2(sum)) * LN2 : parts ? SM_NOTHING : NAN;
    return nothing && parts ? 0.f : 1.f / sum;
}

// BOTH: an item's workgroups walk over the prefix too, which has none of its own (its `wgs` is 0)
template <typename S, typename T, int D, int NQ, bool BOTH>
__global__ __launch_bounds__(64 * CA_WAVES, NQ == 1 && D < 128 ? 4 : 2) void ca_attn_kernel(const CaArgs a)
{
    using ST = CaStore<S>;
    using TL = CaTile<S, D, NQ>;
    using QL = CaQuery<S, T, D>;
    constexpr int NW = CA_WAVES, NT = ST::NT, KT = ST::KT, F = D / 16, PITCH = D + 4;
    // P in fp16 times 2^4 (HALF: codes in 8 bits for bf16 results), as the sum of two bf16 numbers (bf16 caches) or three (codes for fp32
    // results), in fp32 (fp32 caches).  Its sums are in fp32: of two bf16 numbers by a product with ones, else of P before it is rounded.
    constexpr bool HALF = ST::BYTES == 1 && sizeof(T) == 2, ONES = ST::BYTES == 2;
    constexpr int PP = HALF ? 1 : sizeof(T) == 4 ? 3 : 2;
    constexpr float BIAS = HALF ? 4.f : 0.f;
    // What the sum over a tile (ONES), a lane's part of it (HALF) or a lane's exponent may come to before a row's maximum is moved to its
    // scores: fp16 is infinite from 2^16 on, so that a maximum may grow by 2^9 and more, and P keeps its bits down to 2^-18; the others may
    // grow by 2^16.  So that products of a P that has grown are no larger than their values, P is counted in 2^16 there, by a maximum that
    // stands 16 above the scores (ONES: 2^-20 of P, which is 2^-16 as two numbers) or after the exponential (fp32 caches), and in tiles with
    // values' scales of more than FAR it may not (codes for fp32 results)
    constexpr float MANY = HALF ? 65504.f : ONES ? 1.f : 16.f, ABOVE = ONES ? 16.f : 0.f, SMALL = ST::BYTES == 4 ? 0x1p-16f : 1.f, FAR = 0x1p64f;
    union Lds {
        struct {
            uint4 q[NQ][QL::PIECES][64];
            u32x4 keys[NW][TL::STAGED ? KT * TL::C : 1];
        };
        float red[NW][16 * NQ][PITCH];
    };
    __shared__ __align__(16) Lds lds;
    __shared__ float red_m[NW][16 * NQ], red_l[NW][16 * NQ];
    __shared__ int red_met[NW][16 * NQ];
    __shared__ __align__(16) float scales[NW][ST::SCALED ? 64 : 4];   // of a wavefront's tile: keys' times c2, values'
    __shared__ __align__(16) _Float16 halves[NW][HALF ? 32 : 4];       // HALF: values' next to the unit
    __shared__ int row_at[16 * NQ], row_live[16 * NQ], reach[2];

    // both sides' workgroups in turn, eight of each, while there are any: one waits for memory while the other computes
    int id = (int)blockIdx.x;
    const int both = min(a.side[0].wgs, a.side[1].wgs);
    bool shared = !BOTH && id - both >= a.side[0].wgs;   // rows of all items, on the prefix's keys
    if (!BOTH && id < 2 * both) {
        shared = id >> 3 & 1;
        id = (id >> 4) * 8 + (id & 7);
    } else id -= both;
    const CaSide &s = a.side[shared ? 1 : 0];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), x = lane & 15, g = lane >> 4;
    int prob, part, blk;
    if (s.order == CA_NEIGHBOURS) {
        const int u = (id & 7) * (s.wgs >> 3) + (id >> 3), v = s.by_blocks(u);
        if (u >= s.units) return;
        prob = s.by_parts(v); part = v - prob * s.parts; blk = u - v * s.blocks;
    } else {
        if (id >= s.units) return;
        const int u = s.by_problems(id), v = s.by_parts(u);
        prob = id - u * s.problems; part = u - v * s.parts; blk = s.blocks - 1 - v;
    }
    const int b0 = shared ? 0 : a.by_hk(prob), hk = shared ? prob : prob - b0 * a.Hk;
    const int r0 = blk * (16 * NQ), R1 = a.Lq * a.G;
    bool front = BOTH || shared;                        // the prefix's keys, which come first, or the items' own
    const int P = front ? sm_len(a.side[1].len, 0, a.side[1].L) : 0, up = a.causal ? 0 : a.W;
    const int nb_live = min(NQ, (s.rows - r0 + 15) >> 4);   // blocks of rows that exist

    const unsigned char *kb, *vb, *mk;
    const float *ksb, *vsb;
    unsigned kst, vst;
    auto keys_of = [&](const CaSide &y, int b) __attribute__((always_inline)) {
        kb = reinterpret_cast<const unsigned char *>(y.k.p) + (b * y.k.b + hk * y.k.h) * ST::BYTES;
        vb = reinterpret_cast<const unsigned char *>(y.v.p) + (b * y.v.b + hk * y.v.h) * ST::BYTES;
        ksb = ST::SCALED ? y.ks + b * y.ks_b + hk * y.ks_h : nullptr;
        vsb = ST::SCALED ? y.vs + b * y.vs_b + hk * y.vs_h : nullptr;
        kst = (unsigned)(y.k.l * ST::BYTES);
        vst = (unsigned)(y.v.l * ST::BYTES);
        mk = y.mask ? y.mask + (long)b * y.L : nullptr;
    };

    // Keys that any, and that all, of the rows reach; tiles of the part, of which this wavefront takes every NW-th.  Of several items' rows
    // (prefix) the starts decide: the first tiles are asked for as if one stood at the prefix's end, where that is not so once more.
    int lo, hi, all_lo, all_hi, t = 0, t1 = 0;
    TL ta;
    auto fetch_keys = [&](TL &tl, int t) __attribute__((always_inline)) { tl.load_keys(kst, kb, ksb, vsb, mk, lo + t * KT, hi + 1 - lo - t * KT, x, g); };
    auto fetch_values = [&](TL &tl, int t) __attribute__((always_inline)) { tl.load_values(vst, vb, lo + t * KT, hi + 1 - lo - t * KT, x, g); };
    auto begin = [&]() __attribute__((always_inline)) {
        const int tiles = hi < lo ? 0 : (hi - lo + KT) / KT;
        const int per = s.by_span(tiles + s.parts * NW - 1) * NW;
        t = part * per + wv;
        t1 = min(tiles, (part + 1) * per);
        // (of a place that exists where there is nothing to do: loads under a condition are waited for with all that come after them)
        const int j0 = t < t1 ? lo + t * KT : 0, rows = t < t1 ? hi + 1 - j0 : 1;
        ta.load_keys(kst, kb, ksb, vsb, mk, j0, rows, x, g);
        ta.load_values(vst, vb, j0, rows, x, g);
    };
    const int start0 = a.start && !shared ? min(max(a.start[b0], 0), 1 << 24) : 0, lq0 = sm_len(a.len_q, b0, a.Lq);
    const int first0 = start0 + a.by_g(r0), last0 = start0 + min(a.by_g(min(r0 + 16 * NQ, s.rows) - 1), lq0 - 1);
    auto range = [&]() __attribute__((always_inline)) {
        if (shared) {
            lo = max(0, P - a.W); hi = P - 1;
            all_lo = 0; all_hi = hi;
        } else {
            const int off = front ? P : 0, end = front ? P - 1 : sm_len(s.len, b0, s.L) - 1;   // (all queries stand behind the prefix)
            lo = max(0, off + first0 - a.W); hi = last0 < first0 ? -1 : front ? end : min(last0 + up, end);
            all_lo = off + last0 - a.W; all_hi = front ? end : min(first0 + up, end);
        }
    };
    // The rows' operands are asked for before the first tile and put into LDS while that is under way.  Rows that do not take part are zeros, so
    // that what they hold decides nothing.
    constexpr int QSTEPS = NQ * QL::STEPS, QN = (QSTEPS + NW - 1) / NW;
    QL rows_q[QN];
    bool on_q[QN];
#pragma unroll
    for (int i = 0; i < QN; ++i) {
        const int j = min(wv + i * NW, QSTEPS - 1), n = j / QL::STEPS, r = r0 + 16 * n + x;
        const CaRow w = ca_row(a, shared, b0, hk, min(r, s.rows - 1));
        rows_q[i].load(reinterpret_cast<const T *>(a.q.p) + w.b * a.q.b + w.hq * a.q.h + w.i * a.q.l, j - n * QL::STEPS, g);
        on_q[i] = r < s.rows && w.i < (shared ? sm_len(a.len_q, w.b, a.Lq) : lq0);
        if (a.mask_q) on_q[i] = on_q[i] && a.mask_q[(long)w.b * a.Lq + w.i] != 0;
    }
    keys_of(a.side[front ? 1 : 0], front ? 0 : b0);
    range();
    begin();
    SM_READ_FIRST();
#pragma unroll
    for (int i = 0; i < QN; ++i) {
        const int j = wv + i * NW, n = j / QL::STEPS;
        if (j < QSTEPS) rows_q[i].put(&lds.q[n][0][lane], j - n * QL::STEPS, on_q[i]);
    }
    if (wv == 0) {   // (16 NQ rows at most: one wavefront has them all)
        const int r = r0 + lane;
        const CaRow w = ca_row(a, shared, b0, hk, min(r, s.rows - 1));
        const int lq = shared ? sm_len(a.len_q, w.b, a.Lq) : lq0, start = shared && a.start ? min(max(a.start[w.b], 0), 1 << 24) : start0;
        bool on = lane < 16 * NQ && r < s.rows && w.i < lq;
        const int p = start + w.i;
        if (shared) {
            int first = on ? P + p - a.W : 0x7fffffff, last = on ? P + p - a.W : 0;
#pragma unroll
            for (int d = 1; d < 16 * NQ; d <<= 1) first = min(first, __shfl_xor(first, d)), last = max(last, __shfl_xor(last, d));
            if (lane == 0) reach[0] = first, reach[1] = last;
        }
        if (on && a.mask_q) on = a.mask_q[(long)w.b * a.Lq + w.i] != 0;
        if (lane < 16 * NQ) row_at[lane] = p, row_live[lane] = on;
    }
    __syncthreads();
    if (shared) {
        const int first = max(0, __builtin_amdgcn_readfirstlane(reach[0]));
        all_lo = __builtin_amdgcn_readfirstlane(reach[1]);
        if (first != lo) {
            lo = first;
            begin();
        }
    }
    unsigned keys = 0;   // a bit per block: this lane's row has met a key

    f32x4 acc[NQ][F];
    float unit = 0x1p-126f, inv = 0x1p126f;   // HALF: the power of two that accumulators count in, at least the largest scale of a value so far
    float m[NQ], sum[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = CA_LEAST;
        sum[n] = 0.f;
#pragma unroll
        for (int j = 0; j < F; ++j) acc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const float c2 = sm_vector(a.c2), none = sm_vector(-INFINITY);

    constexpr unsigned FULL = KT == 32 ? 0xffffffffu : 0xffffu;
    // scores of a block of rows with the tile's keys (which: of all of them, one after another, or of one)
    auto scores = [&](auto &sc, const TL &tl, int nb0, int ql) __attribute__((always_inline)) {
        constexpr int NB = (int)(sizeof(sc) / sizeof(sc[0]));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int n = 0; n < NT; ++n) sc[nb][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (ST::BYTES == 4) {
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                const u32x4 kw = tl.key(lds.keys[wv], 0, c, x, g);
                u32x4 qw[NB];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) qw[nb] = *reinterpret_cast<const u32x4 *>(&lds.q[nb0 + nb][c][ql]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        sc[nb][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[i]), __uint_as_float(qw[nb][i]), sc[nb][0], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                bf16x8 kf[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    if constexpr (ST::BYTES == 1) kf[n] = ca_codes<S>(tl.k[n][2 * c], tl.k[n][2 * c + 1]);
                    else kf[n] = __builtin_bit_cast(bf16x8, tl.key(lds.keys[wv], n, c, x, g));
#pragma unroll
                for (int p = QL::PARTS - 1; p >= 0; --p)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        const bf16x8 qf = *reinterpret_cast<const bf16x8 *>(&lds.q[nb0 + nb][p * QL::STEPS + c][ql]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) sc[nb][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[n], qf, sc[nb][n], 0, 0, 0);
                    }
            }
        }
    };
    // what the four keys of a lane's accumulators are multiplied by
    auto key_factors = [&](float (&kc)[NT][4]) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            f32x4 y = {c2, c2, c2, c2};
            if constexpr (ST::SCALED) y = *reinterpret_cast<const f32x4 *>(&scales[wv][16 * n + 4 * g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) kc[n][e] = y[e];
        }
    };
    auto value_factors = [&](float (&vc)[NT][4]) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(&scales[wv][32 + 16 * n + 4 * g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) vc[n][e] = y[e];
        }
    };
    // (apart: in a branch, whose conversions the compiler must not take together with those of the way past it)
    auto value_operand = [&](const TL &tl, int j, bool apart) __attribute__((always_inline)) -> bf16x8 {
        constexpr int PER = ST::BYTES < 4 ? 4 / ST::BYTES : 1;   // features of a word
        bf16x8 vf;
#pragma unroll
        for (int i = 0; i < 4; ++i) {        // tokens 2 i, 2 i + 1 of the operand's 8: four of each tile
            unsigned a0 = tl.v[(i >> 1) % NT][2 * (i & 1)][j / PER], a1 = tl.v[(i >> 1) % NT][2 * (i & 1) + 1][j / PER];
            if (apart) asm("" : "+v"(a0), "+v"(a1));
            const bf16x2 y = ca_feature<S>(a0, a1, j);
            vf[2 * i] = y[0]; vf[2 * i + 1] = y[1];
        }
        return vf;
    };
    auto sum_of = [&](const float (&p)[4 * NT]) __attribute__((always_inline)) {
        float y[4 * NT];
#pragma unroll
        for (int e = 0; e < 4 * NT; ++e) y[e] = p[e];
#pragma unroll
        for (int d = 2 * NT; d; d >>= 1)
#pragma unroll
            for (int e = 0; e < d; ++e) y[e] += y[e + d];
        return y[0];
    };
    // p as the sum of N bf16 numbers
    auto split = [&](auto &pf, float (&p)[4 * NT]) __attribute__((always_inline)) {
        constexpr int N = (int)(sizeof(pf) / sizeof(pf[0]));
#pragma unroll
        for (int h = 0; h < N; ++h) {
            pf[h] = pack8(p);
            if (h + 1 < N) {
                const u32x4 w = __builtin_bit_cast(u32x4, pf[h]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {   // (by bits: as conversions each number would be rounded once more by itself)
                    p[2 * i] -= __uint_as_float(w[i] << 16);
                    p[2 * i + 1] -= __uint_as_float(w[i] & 0xffff0000u);
                }
            }
        }
    };

    auto tile = [&](auto which, TL &tl) __attribute__((always_inline)) {
        constexpr int NB = decltype(which)::value;   // blocks of rows at work
        int ql = lane;
        asm volatile("" : "+v"(ql));   // (queries are read from LDS in every tile, and not kept in registers that the loop has not)
        const int j0 = lo + t * KT;
        unsigned on = sm_bits(0, hi - j0) & FULL;
        if (mk) on &= (unsigned)__ballot(tl.act != 0);   // (lanes 0 ... 31: keys 0 ... 31)
        const bool inside = j0 >= all_lo && j0 + KT - 1 <= all_hi;   // of all rows' reach
        float many = MANY;
        bool even = true;   // HALF: the values' scales are taken as fp16 numbers next to the unit
        if constexpr (ST::SCALED) {   // from a key per lane to the four of its accumulators
            float rel = tl.vs;
            if (__builtin_expect(on != FULL, 0)) rel = on >> (lane & 31) & 1 ? rel : 0.f;
            if constexpr (HALF) {
                if (__builtin_expect(__any(rel > unit), 0)) {   // (at the first tile, and where a value is larger than all before)
                    float v = rel <= 0x1p127f ? rel : 0.f;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
                    const unsigned bits = (__float_as_uint(fmaxf(v, unit)) + 0x7fffffu) & 0x7f800000u;   // the next power of two
                    const float u = __uint_as_float((unsigned)__builtin_amdgcn_readfirstlane((int)bits)), f = unit / u;
                    unit = u;
                    inv = 1.f / u;   // (exact, a subnormal number at the end)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int j = 0; j < F; ++j) acc[nb][j] *= f;
                }
                rel *= inv;
                // (P times a scale is rounded to a multiple of 2^-24, with P in 2^-4: 2^-19 of a value by itself at 2^-9 of the unit)
                even = __all(rel >= 0x1p-9f && rel <= 1.f);
                if (__builtin_expect(!even, 0)) even = __all(!(on >> (lane & 31) & 1) || (rel >= 0x1p-9f && rel <= 1.f));
                halves[wv][lane & 31] = even ? (_Float16)rel : (_Float16)0;
            } else if (__any(rel > FAR)) many = 0.f;
            scales[wv][lane] = lane < 32 ? tl.ks * c2 : rel;
        }
        // The keys of the next tile are asked for as soon as these are used up (or in LDS), its values likewise; the last one asks for
        // itself again, since loads under a condition are waited for with all that come after them
        const int ahead = min(t + NW, t1 - 1);
        f32x4 sc[NB][NT];
        if constexpr (TL::STAGED) tl.put_keys(lds.keys[wv], lane);
        else scores(sc, tl, 0, ql);
        SM_READ_FIRST();
        fetch_keys(tl, ahead);
        SM_READ_FIRST();
        if constexpr (TL::STAGED) scores(sc, tl, 0, ql);
        float kc[NT][4];
        key_factors(kc);
        if (__builtin_expect(!inside, 0)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int at = row_at[16 * nb + x] + (front ? P : 0) - j0;
                const unsigned mine = sm_bits(at - a.W, front ? 31 : at + up) & on, keep = mine >> (4 * g);
                if (mine) keys |= 1u << nb;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[nb][n][e] = sm_keep(sc[nb][n][e] * kc[n][e], keep, 16 * n + e, none);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) kc[n][e] = 1.f;
        } else if (on) keys = ~0u;
        if (__builtin_expect(on != FULL, 0)) {   // what does not count must not meet a product: P is 0 there, and may be 0 times anything
            const unsigned mine = on >> (4 * g);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool y = mine >> (16 * n + e) & 1;
                    kc[n][e] = y ? kc[n][e] : 1.f;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) sc[nb][n][e] = y ? sc[nb][n][e] : none;
#pragma unroll
                    for (int w = 0; w < (TL::VB < 4 ? 1 : TL::VB / 4); ++w) tl.v[n][e][w] = y ? tl.v[n][e][w] : 0u;
                }
        }
        float p[NB][4 * NT], much[NB];
        bf16x8 pf[NB][PP];
        f16x8 ph[NB];
        // P of a block from its scores, and what is compared with MANY; ONES, HALF: also as operands (of two bf16 numbers the second is NaN
        // where P is infinite)
        auto probabilities = [&](int nb) __attribute__((always_inline)) -> float {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[nb][4 * n + e] = fmaf(sc[nb][n][e], kc[n][e], BIAS - m[nb]);
            float top = p[nb][0];
            if constexpr (!ONES && !HALF) {
#pragma unroll
                for (int e = 1; e < 4 * NT; ++e) top = fmaxf(top, p[nb][e]);
            }
#pragma unroll
            for (int e = 0; e < 4 * NT; ++e) p[nb][e] = fast_exp2(p[nb][e]) * SMALL;
            if constexpr (HALF) {
#pragma unroll
                for (int e = 0; e < 8; ++e) ph[nb][e] = (_Float16)p[nb][e];
                return sum_of(p[nb]);
            } else if constexpr (ONES) {
                const bf16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
                f32x4 y = {0.f, 0.f, 0.f, 0.f};
                split(pf[nb], p[nb]);
#pragma unroll
                for (int h = PP - 1; h >= 0; --h) y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[nb][h], y, 0, 0, 0);
                return y[0];
            } else return top;
        };
        __builtin_amdgcn_s_setprio(1);   // (of a SIMD's two wavefronts the one in these instructions goes first, the other's products meanwhile: 80 -> 76 us)
        bool fits = true;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) much[nb] = probabilities(nb);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) fits = fits && (ST::BYTES == 2 ? much[nb] <= many : !(much[nb] > many));
        if (__builtin_expect(!__all(fits), 0)) {   // a row's maximum moves: lanes are compared with no exchange between them before
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float top = -INFINITY;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[nb][n][e] * kc[n][e]);
                const float high = ca_max_groups(top), mn = fmaxf(m[nb], ONES ? high + ABOVE : high), f = fast_exp2(m[nb] - mn);
                m[nb] = mn;
                sum[nb] *= f;
#pragma unroll
                for (int j = 0; j < F; ++j) acc[nb][j] *= f;
                much[nb] = probabilities(nb);
            }
        }
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) sum[nb] += ONES || HALF ? much[nb] : sum_of(p[nb]);
        if constexpr (ST::BYTES == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < F; ++j)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tl.v[0][e][j]), p[nb][e], acc[nb][j], 0, 0, 0);
        } else if constexpr (HALF) {
            if (__builtin_expect(!even, 0)) {   // scales far apart: in fp32, as two bf16 numbers, a block of rows after another; zeros below
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    SM_READ_FIRST();
                    float vc[NT][4], y[8];
                    value_factors(vc);
                    bf16x8 pw[2];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = (float)ph[nb][e] * vc[e >> 2][e & 3];
                    split(pw, y);
#pragma unroll
                    for (int j = 0; j < F; ++j) {
                        const bf16x8 vf = value_operand(tl, j, true);
                        acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pw[1], acc[nb][j], 0, 0, 0);
                        acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pw[0], acc[nb][j], 0, 0, 0);
                        SM_READ_FIRST();
                    }
                    ph[nb] *= (_Float16)0;
                }
            }
            const f16x4 v0 = *reinterpret_cast<const f16x4 *>(&halves[wv][4 * g]), v1 = *reinterpret_cast<const f16x4 *>(&halves[wv][16 + 4 * g]);
            const f16x8 v8 = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) ph[nb] *= v8;
#pragma unroll
            for (int j = 0; j < F; ++j) {
                f16x8 vf;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f16x2 y = ca_feature_half<S>(tl.v[i >> 1][2 * (i & 1)][j / 4], tl.v[i >> 1][2 * (i & 1) + 1][j / 4], j);
                    vf[2 * i] = y[0]; vf[2 * i + 1] = y[1];
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, ph[nb], acc[nb][j], 0, 0, 0);
            }
        } else {
            if constexpr (ST::SCALED) {
                float vc[NT][4];
                value_factors(vc);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[nb][e] *= vc[e >> 2][e & 3];
                    split(pf[nb], p[nb]);
                }
            }
#pragma unroll
            for (int j = 0; j < F; ++j) {
                const bf16x8 vf = value_operand(tl, j, false);
#pragma unroll
                for (int h = 0; h < PP; ++h)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) acc[nb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[nb][h], acc[nb][j], 0, 0, 0);
            }
        }
        SM_READ_FIRST();
        fetch_values(tl, ahead);
        SM_READ_FIRST();
        t += NW;
    };
    auto walk = [&](auto which) __attribute__((always_inline)) {
#pragma unroll 1
        while (t < t1) {
            tile(which, ta);
        }
    };
    if constexpr (BOTH) {
#pragma unroll 1
        for (;;) {
            walk(std::integral_constant<int, NQ>{});
            if (!front) break;
            front = false;
            keys_of(s, b0);
            range();
            begin();
        }
    } else if (nb_live <= 1) walk(std::integral_constant<int, 1>{});
    else walk(std::integral_constant<int, NQ>{});

    const long rows = (long)a.B * a.Hk * a.Lq * a.G;
    const int slot = part + (shared ? a.side[0].parts : 0);
    // four adjacent features of a row, from feature f on
    auto put = [&](const CaRow &w, int f, const f32x4 &y) {
        if (a.parts > 1) *reinterpret_cast<f32x4 *>(a.part + ((slot * rows + ((long)w.b * a.Hk + hk) * (a.Lq * a.G) + w.at) * D + f)) = y;
        else store4<T>(reinterpret_cast<T *>(const_cast<void *>(a.o.p)) + w.b * a.o.b + w.hq * a.o.h + w.i * a.o.l + f, y[0], y[1], y[2], y[3]);
    };
    auto put_lse = [&](const CaRow &w, float lse) {
        if (a.parts > 1) a.part_lse[slot * rows + ((long)w.b * a.Hk + hk) * (a.Lq * a.G) + w.at] = lse;
        else a.lse[((long)w.b * a.G * a.Hk + w.hq) * a.Lq + w.i] = lse;
    };
    bool met[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        if constexpr (!ONES) {
            sum[n] += __shfl_xor(sum[n], 16);
            sum[n] += __shfl_xor(sum[n], 32);
        }
        if constexpr (HALF) {
            sum[n] *= 1.f / 16.f;   // (BIAS)
            float f = unit * (1.f / 16.f);
            if (unit > FAR) {   // a row's weights, of a maximum that may lag, are brought below 1 first
                const int e = __builtin_amdgcn_frexp_expf(sum[n]);
                sum[n] = ldexpf(sum[n], -e);
                f = ldexpf(f, -e);
                m[n] += (float)e;
            }
#pragma unroll
            for (int j = 0; j < F; ++j) acc[n][j] *= f;
        }
        met[n] = row_live[16 * n + x] && (keys >> n & 1);
    }
    // features (4 g + e) F + j of a row, four at a time
    auto piece = [&](int n, int f) __attribute__((always_inline)) {
        f32x4 y;
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = acc[n][(4 * f + c) % F][(4 * f + c) / F];
        return y;
    };
    __syncthreads();   // (the queries' LDS is used for the results)
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        if (n >= nb_live) break;
#pragma unroll
        for (int f = 0; f < F; ++f) *reinterpret_cast<f32x4 *>(&lds.red[wv][16 * n + x][4 * F * g + 4 * f]) = piece(n, f);
        if (g == 0) {
            red_m[wv][16 * n + x] = m[n];
            red_l[wv][16 * n + x] = sum[n];
            red_met[wv][16 * n + x] = met[n];
        }
    }
    __syncthreads();
    // a thread takes four features of a row at a time
    const int here = min(16 * NQ, s.rows - r0) * (D / 4);
    for (int u = threadIdx.x; u < here; u += NW * 64) {
        const int row = u / (D / 4), f = (u % (D / 4)) * 4;
        float M = CA_LEAST, L = 0.f;
        bool any = false;
        for (int k = 0; k < NW; ++k) {
            M = fmaxf(M, red_m[k][row]);
            any |= red_met[k][row] != 0;
        }
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < NW; ++k) {
            const float c = fast_exp2(red_m[k][row] - M);
            L = fmaf(red_l[k][row], c, L);
            y += *reinterpret_cast<const f32x4 *>(&lds.red[k][row][f]) * c;
        }
        const CaRow w = ca_row(a, shared, b0, hk, r0 + row);
        float lse;
        const float scale = ca_finish(M, L * (1.f / SMALL), any, a.parts > 1, lse) * (1.f / SMALL);
        put(w, f, any ? y * scale : f32x4{0.f, 0.f, 0.f, 0.f});
        if (f == 0) put_lse(w, lse);
    }
}

// Joins the parts of a row: weighted by exp(their LSE - the largest).  A thread takes four features over every slices-th part, four parts
// asked for at a time (a part without a key has LSE = -inf and zeros); the slices are joined by LDS in their order.  first: the launch's first row.
template <typename T, int D> __global__ __launch_bounds__(NTHREADS) void ca_join_kernel(const CaArgs a, long first, int slices)
{
    constexpr int FT = D / 4, U = 4;
    __shared__ f32x4 sx[NTHREADS];
    __shared__ float sm[NTHREADS], sl[NTHREADS];
    const int R = a.Lq * a.G, f = (threadIdx.x % FT) * 4, rest = threadIdx.x / FT, slice = rest % slices;
    const long rows = (long)a.B * a.Hk * R, row = first + (long)blockIdx.x * (NTHREADS / FT / slices) + rest / slices, from = min(row, rows - 1);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float m = CA_LEAST, l = 0.f;
    for (int s0 = slice; s0 < a.parts; s0 += U * slices) {
        f32x4 y[U];
        float lse[U], top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u * slices, a.parts - 1);
            lse[u] = a.part_lse[s * rows + from];
            y[u] = *reinterpret_cast<const f32x4 *>(a.part + (s * rows + from) * D + f);
            if (s0 + u * slices >= a.parts) lse[u] = -INFINITY;
        }
        // (fmaxf passes over a NaN, so that m never is one; a weight is, and l and x from there on)
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, lse[u]);
        const float old = fast_exp2((m - top) * LOG2E);
        l *= old;
        x *= old;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float c = lse[u] == -INFINITY ? 0.f : fast_exp2((lse[u] - top) * LOG2E);
            l += c;
            x += y[u] * c;
        }
        m = top;
    }
    if (slices > 1) {
        sx[threadIdx.x] = x;
        sm[threadIdx.x] = m;
        sl[threadIdx.x] = l;
        __syncthreads();
        if (slice) return;
        float top = m;
        for (int s = 1; s < slices; ++s) top = fmaxf(top, sm[threadIdx.x + s * FT]);
        const float c0 = fast_exp2((m - top) * LOG2E);
        l *= c0;
        x *= c0;
        for (int s = 1; s < slices; ++s) {
            const int o = threadIdx.x + s * FT;
            const float c = fast_exp2((sm[o] - top) * LOG2E);
            l = fmaf(sl[o], c, l);
            x += sx[o] * c;
        }
        m = top;
    }
    if (row >= rows) return;
    const int prob = (int)(row / R), r = (int)(row - (long)prob * R), b = a.by_hk(prob), hk = prob - b * a.Hk;
    const CaRow w = ca_row(a, false, b, hk, r);
    // A row with keys whose scores are all -inf has parts of SM_NOTHING and no others: l counts them, and they are 0 / 0
    if (m == SM_NOTHING && l > 0.f) l = NAN;
    const float c = l == 0.f ? 0.f : 1.f / l;
    store4<T>(reinterpret_cast<T *>(const_cast<void *>(a.o.p)) + w.b * a.o.b + w.hq * a.o.h + w.i * a.o.l + f, x[0] * c, x[1] * c, x[2] * c, x[3] * c);
    if (f == 0) a.lse[((long)b * a.Hk * a.G + w.hq) * a.Lq + w.i] = l == 0.f ? -INFINITY : m + fast_log2(l) * LN2;
}

}  // namespace
