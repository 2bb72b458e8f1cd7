// Softmax attention on a band for gfx950, forward and gradient (sinkhorn_attn_layer.h): kernels.
//
// Every kernel is a walk of one side's tiles past a block of the other side's rows, its "owners", 32 to a wavefront:
//
//   forward   owners: queries.  S^T = K Q^T, P = exp(S - m) with the running maximum m, O^T += V^T P^T
//   dQ        owners: queries.  S^T, Z^T = V dO^T, dS = P (Z - delta), dQ^T += K^T dS^T; delta = <dO, O> from the owners' rows
//   dK, dV    owners: keys.     S = Q K^T, Z = dO V^T, dV^T += dO^T P, dK^T += Q^T dS
//
// The walked side is the row dimension of every score tile, so a lane holds 16 scores of one owner: the softmax sums are
// register sums and one exchange between the lane halves, and P in the accumulators' layout is already the operand
// of the second product (whose sum runs over the walked side in any order).  dQ apart from dK and dV means two score
// evaluations (seven products, not five), but no atomics, so that results repeat, and no pass over dQ in fp32.
//
// What bounds them (MI355X, 2 heads, L = 262144, d = 64, W = 256, bf16; products of the band's pairs alone): forward 117 us,
// 589 TFLOP/s; dQ 157 us, 658; dK and dV 205 us, 672.  The forward's HBM traffic is the least possible (200 MB read and 68 written
// by the L2's counters, 2.3 TB/s).  The matrix cores are busy for 29 to 32 % of the cycles: a lone wavefront issues a vector
// instruction every 8 cycles at most, and three wavefronts fit a SIMD's registers (dK, dV: two).  In the forward each lives 20 us,
// of which 3.5 pass until its first tile is there, 12 in the arithmetic of nine tiles, 2.7 waiting for tiles and barriers, 1.9
// storing.
//
// Query heads that share a key head are rows of the same problem: row r of problem (b, key head) is query r / G of head
// r % G of the group, G = Hq / Hk.  Keys are read once for the group, and dK, dV sum over it by themselves.
#pragma once
#include "ska_common.h"

namespace {

// Division of any 32-bit number by a number of the launch: the product with its reciprocal of 33 bits, of which m holds the lower
// 32.  A dozen divisions stand at the start of every workgroup, where a wavefront is alone with their latency.
struct SmDiv {
    unsigned m;
    int s1, s2;
    __host__ static SmDiv by(unsigned d)
    {
        int l = 0;
        while (l < 32 && (1ull << l) < d) ++l;
        return {(unsigned)((((1ull << l) - d) << 32) / d) + 1, l < 1 ? l : 1, l > 1 ? l - 1 : 0};
    }
    __device__ __forceinline__ int operator()(int n) const
    {
        const unsigned t = __umulhi(m, (unsigned)n);
        return (int)((t + (((unsigned)n - t) >> s1)) >> s2);
    }
};
struct SmTensor {
    const void *p;
    long b, h, l;   // elements between items, heads, tokens
};
struct SmArgs {
    SmTensor q, k, v, o, g;        // g: dO
    SmTensor oq, ok, ov;           // forward: oq = O; backward: dQ, dK, dV (written)
    float *lse, *lse2, *delta;     // [B][Hq][Lq]; lse2: LSE log2(e) as dK reads it, inf where there is no row
    const int *start, *len_q, *len_k;
    const unsigned char *mask_q, *mask_k;
    float *part, *part_lse;        // walks in parts: [parts][problems][rows][D] (forward: and their LSE [parts][problems][rows])
    int B, Hk, G, Lq, Lk, W, causal;
    int parts;                     // parts of a walk
    int blocks;                    // blocks of owners per problem
    int total;                     // blocks * parts * problems
    int order;                     // SmOrder
    SmDiv by_g, by_hk, by_n, by_parts, by_blocks;   // G, Hk, problems, parts, blocks * parts
    float c2, cs;                  // log2(e) / (eps sqrt d), 1 / (eps sqrt d)
};

// Order of the workgroups.  Neighbouring blocks of a band walk over the same tiles: a contiguous piece of the problems per XCD
// (workgroups go to the XCDs in turn).  Walks over most of the other side: problems fastest, so that one stays with an XCD
// where they are a multiple of 8 and with few otherwise, and those with the longest walks first.
enum SmOrder { SM_NEIGHBOURS, SM_LAST_FIRST, SM_FIRST_FIRST };

// one block of the grid: problem, block of owners, part of the walk
struct SmPlace { int b, hk, blk, part; };
__device__ __forceinline__ bool sm_place(const SmArgs &a, SmPlace &w)
{
    const int N = a.B * a.Hk;
    int n, x;
    if (a.order != SM_NEIGHBOURS) {
        if ((int)blockIdx.x >= a.total) return false;
        x = a.by_n(blockIdx.x);
        n = blockIdx.x - x * N;
        if (a.order == SM_LAST_FIRST) x = a.blocks * a.parts - 1 - x;
    } else {
        const int per = gridDim.x / 8, at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
        if (at >= a.total) return false;
        n = a.by_blocks(at);
        x = at - n * a.blocks * a.parts;
    }
    w.blk = a.by_parts(x);
    w.part = x - w.blk * a.parts;
    w.b = a.by_hk(n);
    w.hk = n - w.b * a.Hk;
    return true;
}
__device__ __forceinline__ int sm_len(const int *len, int b, int L) { return len ? min(max(len[b], 0), L) : L; }
__device__ __forceinline__ int sm_start(const SmArgs &a, int b) { return a.start ? min(max(a.start[b], 0), 1 << 24) : 0; }

// Tiles: KT walked rows (two score tiles of 32 for narrow bf16 heads, else one), row-major, 16-byte chunks XOR-swizzled
// by the row so that reads of one chunk of many rows, and of one row of many chunks, touch all banks.
template <typename T, int D> struct SmTile {
    static constexpr int KT = sizeof(T) == 2 && D < 128 ? 64 : 32;
    static constexpr int ROWB = D * (int)sizeof(T), CPR = ROWB / 16;
    static constexpr int SUB = 32 * ROWB;      // bytes of one score tile's rows
    static constexpr int BYTES = KT * ROWB;
    static constexpr int RPI = 64 / CPR;       // rows that one load instruction of a wavefront brings (1 KB)
    static __device__ __forceinline__ int swz(int row)
    {
        if constexpr (sizeof(T) == 2) return bf16_swizzle<D>(row);
        else return row & 7;
    }
};

// one such load: 16 bytes a lane from `base` + `at` into `lds` + 16 lane (lds, base uniform: said once more, where a kernel runs
// out of scalar registers)
__device__ __forceinline__ const unsigned char *sm_uniform(const unsigned char *p)
{
    const unsigned long x = (unsigned long)p;
    return reinterpret_cast<const unsigned char *>((unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)x) |
                                                   (unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32);
}
__device__ __forceinline__ void sm_load_pieces(unsigned lds, const unsigned char *base, unsigned at)
{
    // (written out, because the compiler takes every later LDS read for one of these bytes and waits at once; the kernel
    // waits where it needs them.  No register is written.)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(at),
                 "s"(sm_uniform(base))
                 : "memory", "m0");
}

// Tiles come by loads that write LDS directly, KT / RPI instructions a tile dealt to the NW wavefronts: no registers, no
// stores, and the next tile is under way while this one is worked on.
template <typename T, int D, int NW> struct SmLoader {
    using TL = SmTile<T, D>;
    static constexpr int PER = TL::KT / TL::RPI / NW;   // instructions per wavefront and matrix
    static_assert(PER * NW * TL::RPI == TL::KT, "whole instructions");
    int lane, wv, lrow;
    __device__ __forceinline__ SmLoader(int lane, int wv) : lane(lane), wv(wv), lrow(lane / TL::CPR) {}
    // first row of instruction k; this lane's row is lrow below it
    __device__ __forceinline__ int first(int k) const { return (wv + NW * k) * TL::RPI; }
    // byte of a row that this lane brings: its place in LDS is fixed, and the chunk that belongs there depends on the row
    // (the swizzle takes single bits of the row: that of a sum without carries is the exclusive or)
    __device__ __forceinline__ unsigned col(int k) const { return (unsigned)((lane % TL::CPR) ^ TL::swz(lrow) ^ TL::swz(first(k))) * 16; }
    // rows 0 ... rows - 1 of the tile at `base` (uniform), `stride` bytes apart, exist: the others repeat the last one
    __device__ __forceinline__ void load(unsigned lds, const unsigned char *base, long stride, int rows) const
    {
        lds += (unsigned)wv * 1024;
        if (rows >= TL::KT) {
            const unsigned char *at = base + wv * (TL::RPI * stride);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                sm_load_pieces(lds + k * NW * 1024, at, (unsigned)lrow * (unsigned)stride + col(k));
                at += NW * TL::RPI * stride;
            }
        } else {
#pragma unroll 1
            for (int k = 0; k < PER; ++k) {
                const int r = min(first(k), rows - 1), l = min(lrow, rows - 1 - r);
                sm_load_pieces(lds + k * NW * 1024, base + r * stride, (unsigned)l * (unsigned)stride + col(k));
            }
        }
    }
    // after this wavefront's loads have arrived: zeros into those of its rows that do not count
    __device__ __forceinline__ void clear(unsigned char *lds, int rows, unsigned on) const
    {
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (first(k) + lrow >= rows || !(on >> k & 1))
                *reinterpret_cast<uint4 *>(lds + first(k) * TL::ROWB + lane * 16) = make_uint4(0, 0, 0, 0);
    }
};
// Activity of a tile's rows, read beside its loads and looked at when they have arrived: of the rows that this lane's loads
// bring, and of row `lane`; rows beyond the last repeat it.
template <typename T, int D, int NW> struct SmActivity {
    using L = SmLoader<T, D, NW>;
    unsigned char mine[L::PER], lane;
    __device__ __forceinline__ void load(const L &l, const unsigned char *mask, int rows)
    {
#pragma unroll
        for (int k = 0; k < L::PER; ++k) mine[k] = mask[min(l.first(k) + l.lrow, rows - 1)];
        lane = mask[min(l.lane & (SmTile<T, D>::KT - 1), rows - 1)];
    }
    __device__ __forceinline__ unsigned rows() const   // a bit per instruction
    {
        unsigned on = 0;
#pragma unroll
        for (int k = 0; k < L::PER; ++k) on |= (mine[k] ? 1u : 0u) << k;
        return on;
    }
    __device__ __forceinline__ unsigned long long bits() const { return __ballot(lane != 0); }
};
// Waits for this wavefront's loads.  The builtin, not the instruction in text: the compiler must know that the owners' rows have
// come as well, or it waits for them again inside the loop, and with them for the next tile's loads.
__device__ __forceinline__ void sm_arrived()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ unsigned sm_lds(const void *p) { return (unsigned)(size_t)(__attribute__((address_space(3))) const unsigned char *)p; }
// 64 floats at `p` + `at` (bytes, per lane) into LDS
__device__ __forceinline__ void sm_load_words(unsigned lds, const float *p, unsigned at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(at), "s"(p) : "memory", "m0");
}
// the larger of the two lane halves' values, in both
__device__ __forceinline__ float sm_max_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <typename T, int D> __device__ __forceinline__ void sm_frag(OwnerFrag<T, D> &x, const T *row, int h)
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) x.v[s] = *reinterpret_cast<const bf16x8 *>(row + (2 * s + h) * 8);
    } else {
#pragma unroll
        for (int q = 0; q < D / 8; ++q) {
            const float4 z = *reinterpret_cast<const float4 *>(row + h * (D / 2) + 4 * q);
            x.v[4 * q + 0] = z.x; x.v[4 * q + 1] = z.y; x.v[4 * q + 2] = z.z; x.v[4 * q + 3] = z.w;
        }
    }
}
// <x, y> of two rows held as owners' fragments (both lane halves get it)
template <int D> __device__ __forceinline__ float sm_dot(const OwnerFrag<__bf16, D> &x, const OwnerFrag<__bf16, D> &y)
{
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf((float)x.v[k][i], (float)y.v[k][i], s);
    return s + __shfl_xor(s, 32);
}
template <int D> __device__ __forceinline__ float sm_dot(const OwnerFrag<float, D> &x, const OwnerFrag<float, D> &y)
{
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < D / 2; ++k) s = fmaf(x.v[k], y.v[k], s);
    return s + __shfl_xor(s, 32);
}

// Operands of one score tile, read from LDS: rows for the scores, columns (transposed) for the second product.  Reads are asked
// for well before the products that take them (SM_READ_FIRST keeps the compiler from moving them there): a product that
// waits for its own read costs a read's latency, and two or three wavefronts per SIMD do not hide that.  fp32 tiles are read where
// they are used: their products take four times as long.
#define SM_READ_FIRST() __builtin_amdgcn_sched_barrier(0)
template <typename T, int D> struct SmRows {
    bf16x8 a[D / 16];
    __device__ __forceinline__ void read(const unsigned char *tile, int lane)
    {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) a[k] = *reinterpret_cast<const bf16x8 *>(tile + bf16_chunk_off<D>(lane & 31, 2 * k + (lane >> 5)));
    }
};
template <int D> struct SmRows<float, D> {
    const unsigned char *tile;
    __device__ __forceinline__ void read(const unsigned char *t, int) { tile = t; }
};
template <typename T, int D> struct SmCols {
    bf16x8 a[2][D / 32];
    __device__ __forceinline__ void read(const unsigned char *tile, int lane)
    {
        // transposing reads: within 16 lanes, lane i receives element (i & 3) of the 8-byte pieces addressed by lanes
        // (i >> 2) + 4 e, e = 0..3
        typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
        const int row = 4 * (lane >> 5) + ((lane & 15) >> 2), ch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        const unsigned char *sub = tile + (lane & 1) * 8;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int v = 0; v < D / 32; ++v) {
                const bf16x4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4v __attribute__((address_space(3))) *)(
                    sub + bf16_chunk_off<D>(row + 16 * m, ch + 4 * v)));
                const bf16x4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((bf16x4v __attribute__((address_space(3))) *)(
                    sub + bf16_chunk_off<D>(row + 16 * m + 8, ch + 4 * v)));
                a[m][v] = bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            }
    }
};
template <int D> struct SmCols<float, D> {
    const unsigned char *tile;
    __device__ __forceinline__ void read(const unsigned char *t, int) { tile = t; }
};

// s[t, o] = sum_k tile[t][k] own[o][k]
template <typename T, int D>
__device__ __forceinline__ void sm_scores(f32x16 &s, const SmRows<T, D> &rows, const OwnerFrag<T, D> &own, int lane)
{
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows.a[k], own.v[k], s, 0, 0, 0);
    } else {
        using TL = SmTile<T, D>;
        const int t = lane & 31, h = lane >> 5;
#pragma unroll
        for (int q = 0; q < D / 8; ++q) {
            const float4 a = *reinterpret_cast<const float4 *>(rows.tile + t * TL::ROWB + ((h * (D / 8) + q) ^ TL::swz(t)) * 16);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, own.v[4 * q + 0], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, own.v[4 * q + 1], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, own.v[4 * q + 2], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, own.v[4 * q + 3], s, 0, 0, 0);
        }
    }
}
// out[v, o] += sum_t tile[t][v] p[t, o].  bf16: p is rounded to bf16 (half a step, 2^-8), or with EXACT taken as the sum of
// what that gives and of the rest rounded likewise (2^-16).
template <typename T, int D, bool EXACT = false>
__device__ __forceinline__ void sm_accum(f32x16 (&out)[D / 32], const SmCols<T, D> &cols, const float (&p)[16], int lane)
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const bf16x8 pf = pack8(&p[8 * m]);
#pragma unroll
            for (int v = 0; v < D / 32; ++v)
                out[v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cols.a[m][v], pf, out[v], 0, 0, 0);
            if constexpr (EXACT) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = p[8 * m + e] - (float)pf[e];
                const bf16x8 rest = pack8(x);
#pragma unroll
                for (int v = 0; v < D / 32; ++v)
                    out[v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cols.a[m][v], rest, out[v], 0, 0, 0);
            }
        }
    } else {
        using TL = SmTile<T, D>;
        const int c = lane & 31, h = lane >> 5;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = 8 * (r >> 2) + 4 * h + (r & 3);
#pragma unroll
            for (int v = 0; v < D / 32; ++v) {
                const float a = *reinterpret_cast<const float *>(cols.tile + t * TL::ROWB + ((8 * v + (c >> 2)) ^ TL::swz(t)) * 16 + (c & 3) * 4);
                out[v] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[r], out[v], 0, 0, 0);
            }
        }
    }
}

// The rows that a wavefront holds as accumulators (a lane has pieces of 4 features of row lane & 31), times scale, into memory:
// across LDS (32 rows of the wavefront's own), so that a store instruction writes whole rows and not 16 bytes of each of 32.
// row(i): where row i goes, null: nowhere.
template <typename T, int D, typename Row>
__device__ __forceinline__ void sm_store_rows(unsigned char *lds, const f32x16 (&x)[D / 32], float scale, bool live, int lane, Row row)
{
    using TL = SmTile<T, D>;
    const int o = lane & 31, h = lane >> 5;
#pragma unroll
    for (int v = 0; v < D / 32; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = sizeof(T) == 2 ? 4 * v + e : 8 * v + 2 * e + h;   // 16-byte piece of features 32 v + 8 e + 4 h ...
            T *at = reinterpret_cast<T *>(lds + o * TL::ROWB + (c ^ TL::swz(o)) * 16 + (sizeof(T) == 2 ? 8 * h : 0));
            if (live) store4<T>(at, x[v][4 * e] * scale, x[v][4 * e + 1] * scale, x[v][4 * e + 2] * scale, x[v][4 * e + 3] * scale);
            else store4<T>(at, 0.f, 0.f, 0.f, 0.f);
        }
    const int l = lane / TL::CPR, c = lane % TL::CPR;
#pragma unroll
    for (int k = 0; k < 32 / TL::RPI; ++k) {
        const int i = k * TL::RPI + l;
        const uint4 y = *reinterpret_cast<const uint4 *>(lds + i * TL::ROWB + (c ^ TL::swz(i)) * 16);
        T *to = row(i);
        if (to) *reinterpret_cast<uint4 *>(to + c * (16 / (int)sizeof(T))) = y;
    }
}

// A constant of the launch in a vector register: multiply-adds with a scalar operand issue at half the rate of those with
// vector operands alone (4.9 against 2.7 cycles with four wavefronts per SIMD), as maxima, comparisons, selections and
// conversions do; exponentials take 8.9.
__device__ __forceinline__ float sm_vector(float x)
{
    asm("" : "+v"(x));
    return x;
}
// x where bit `bit` of m is set, otherwise `other`
__device__ __forceinline__ float sm_keep(float x, unsigned m, int bit, float other)
{
    const int on = ((int)(m << (31 - bit))) >> 31;
    return __int_as_float((__float_as_int(x) & on) | (~on & __float_as_int(other)));
}
// bits [a, b] of 32 (none where b < a)
__device__ __forceinline__ unsigned sm_bits(int a, int b)
{
    const unsigned hi = b >= 31 ? 0xffffffffu : b < 0 ? 0u : (2u << b) - 1u;
    const unsigned lo = a <= 0 ? 0xffffffffu : a >= 32 ? 0u : ~((1u << a) - 1u);
    return hi & lo;
}

constexpr float SM_NOTHING = -3.402823466e38f;   // LSE of a part whose scores are all -inf (one without keys: -inf)
constexpr float SM_LAZY = 8.f;   // powers of two that a row's maximum may grow by before its sums are scaled to it

enum { SM_FWD, SM_DQ, SM_DKV };

// ------------------------------------------------------------------ queries as owners: forward, dQ
// BWD: dQ instead of O.  NW wavefronts, 32 rows each.
template <typename T, int D, int NW, bool BWD>
__global__ __launch_bounds__(64 * NW, 1) void sm_rows_kernel(const SmArgs a)
{
    using TL = SmTile<T, D>;
    constexpr int KT = TL::KT, NS = KT / 32, BM = 32 * NW;
    __shared__ __align__(1024) unsigned char lds[2][2][TL::BYTES];

    SmPlace w;
    if (!sm_place(a, w)) return;
    const int R = a.Lq * a.G, r0 = w.blk * BM;
    const int lq = sm_len(a.len_q, w.b, a.Lq), lk = sm_len(a.len_k, w.b, a.Lk), start = sm_start(a, w.b);
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const long prob = (long)w.b * a.Hk + w.hk;
    const int up = a.causal ? 0 : a.W;

    const int wr0 = r0 + 32 * wv;   // this wavefront's first row
    // keys that the block's rows, and this wavefront's, can reach
    const int i_last = a.by_g(max(0, min(min(r0 + BM, R), lq * a.G) - 1));   // (lq 0: no row, and no key below)
    int j_lo = max(0, start + a.by_g(r0) - a.W), j_hi = min(lk - 1, start + i_last + up);
    if (lq * a.G <= r0) j_hi = j_lo - 1;
    const int w_first = start + a.by_g(min(wr0, R - 1)), w_last = start + a.by_g(min(wr0 + 31, R - 1));
    const int w_lo = w_first - a.W, w_hi = w_last + up;                        // any of its rows
    const int all_lo = w_last - a.W, all_hi = min(min(w_first + up, lk - 1), j_hi);   // all of them
    int tiles = (j_hi - j_lo + KT) / KT;
    if (a.parts > 1) {
        const int per = a.by_parts(max(0, tiles) + a.parts - 1);
        j_lo += w.part * per * KT;
        tiles = min(per, tiles - w.part * per);
    }

    const unsigned char *kb = reinterpret_cast<const unsigned char *>(reinterpret_cast<const T *>(a.k.p) + w.b * a.k.b + w.hk * a.k.h);
    const unsigned char *vb = reinterpret_cast<const unsigned char *>(reinterpret_cast<const T *>(a.v.p) + w.b * a.v.b + w.hk * a.v.h);
    const long ks = a.k.l * (long)sizeof(T), vs = a.v.l * (long)sizeof(T);
    const unsigned char *mk = a.mask_k ? a.mask_k + (long)w.b * a.Lk : nullptr;
    const SmLoader<T, D, NW> loader(lane, wv);
    const unsigned lds_at = sm_lds(lds);
    SmActivity<T, D, NW> act;
    // (inlined by order: where the compiler called fetch or step, fp32 at d = 128 kept its registers in memory, 661 us instead of 185 for a
    // token of 4 sequences, 8 heads on 2, caches of 65536)
    auto fetch = [&](int j0, int buf) __attribute__((always_inline)) {
        const int rows = j_hi + 1 - j0;
        loader.load(lds_at + buf * 2 * TL::BYTES, kb + j0 * ks, ks, rows);
        loader.load(lds_at + (buf * 2 + 1) * TL::BYTES, vb + j0 * vs, vs, rows);
        if (mk) act.load(loader, mk + j0, rows);
    };
    if (tiles > 0) fetch(j_lo, 0);   // (before the owners' rows: both are under way at a time)

    // this lane's rows
    OwnerFrag<T, D> q, g;
    const int r = wr0 + (lane & 31), rc = min(r, R - 1), i = a.by_g(rc), hq = w.hk * a.G + (rc - i * a.G);
    bool live = r < R && i < lq;
    if (live && a.mask_q) live = a.mask_q[(long)w.b * a.Lq + i] != 0;
    const int my_lo = start + i - a.W, my_hi = min(start + i + up, lk - 1);
    sm_frag<T, D>(q, reinterpret_cast<const T *>(a.q.p) + w.b * a.q.b + hq * a.q.h + i * a.q.l, h);
    float m = -INFINITY, sum = 0.f, delta = 0.f;   // BWD: m = LSE log2(e)
    unsigned keys = 0;                             // forward: not 0 where the row has met a key of its own
    if constexpr (BWD) {
        OwnerFrag<T, D> o;
        sm_frag<T, D>(g, reinterpret_cast<const T *>(a.g.p) + w.b * a.g.b + hq * a.g.h + i * a.g.l, h);
        sm_frag<T, D>(o, reinterpret_cast<const T *>(a.o.p) + w.b * a.o.b + hq * a.o.h + i * a.o.l, h);
        const long at = ((long)w.b * a.G * a.Hk + hq) * a.Lq + i;
        const float lse = a.lse[at];
        live = live && lse != -INFINITY;        // (NaN is a poisoned row's and goes on)
        m = live ? lse * LOG2E : INFINITY;      // (exp2(s - inf) = 0)
        delta = sm_dot<D>(g, o);
        if (!live) delta = 0.f;
        if (w.part == 0 && h == 0 && r < R) {
            a.lse2[at] = m;
            a.delta[at] = delta;
        }
    }

    f32x16 acc[D / 32];
#pragma unroll
    for (int v = 0; v < D / 32; ++v)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[v][e] = 0.f;

    const float c2 = sm_vector(a.c2), none = sm_vector(-INFINITY);
    auto step = [&](auto which, int t) __attribute__((always_inline)) {
        constexpr int buf = decltype(which)::value;   // (a constant: LDS addresses are offsets of the instructions)
        const int j0 = j_lo + t * KT;
        sm_arrived();
        unsigned long long here = ~0ull;   // active keys
        if (j_hi + 1 - j0 < KT || mk) {    // (products with rows that do not count must not meet what they hold)
            unsigned on = ~0u;
            if (mk) {
                on = act.rows();
                here = act.bits();
            }
            loader.clear(lds[buf][0], j_hi + 1 - j0, on);
            loader.clear(lds[buf][1], j_hi + 1 - j0, on);
        }
        __syncthreads();
        if (t + 1 < tiles) fetch(j0 + KT, buf ^ 1);
        if constexpr (!BWD) {
            if (j0 > w_hi || j0 + KT - 1 < w_lo) return;
            const bool whole = j0 >= all_lo && j0 + KT - 1 <= all_hi && here == ~0ull;
            if (whole) keys = 1;
            f32x16 s[NS];
            SmRows<T, D> kr[NS];
            SmCols<T, D> vc[NS];
#pragma unroll
            for (int n = 0; n < NS; ++n) kr[n].read(lds[buf][0] + n * TL::SUB, lane);
            SM_READ_FIRST();
#pragma unroll
            for (int n = 0; n < NS; ++n) sm_scores<T, D>(s[n], kr[n], q, lane);
#pragma unroll
            for (int n = 0; n < NS; ++n) vc[n].read(lds[buf][1] + n * TL::SUB, lane);
            SM_READ_FIRST();
            if (!whole) {
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    const int base = j0 + 32 * n;
                    const unsigned own = sm_bits(my_lo - base, min(my_hi, j_hi) - base) & (unsigned)(here >> (32 * n));
                    const unsigned keep = own >> (4 * h);
                    keys |= own;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[n][e] = sm_keep(s[n][e], keep, 8 * (e >> 2) + (e & 3), none);
                }
            }
            // Running maximum: sums stay relative to an older one until a score exceeds it by 2^SM_LAZY, so that the
            // accumulators are scaled a few times per row and not once per tile; P up to 2^8 loses nothing in either type.
            float top = s[0][0];
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[n][e]);
            top = sm_max_halves(top) * c2;
            if (__any(top > m + SM_LAZY)) {
                const float mn = fmaxf(m, top), x = mn > -INFINITY ? fast_exp2(m - mn) : 1.f;
                sum *= x;
#pragma unroll
                for (int v = 0; v < D / 32; ++v)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[v][e] *= x;
                m = mn;
            }
            const float mu = m > -INFINITY ? m : 0.f;
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                float p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    p[e] = fast_exp2(fmaf(s[n][e], c2, -mu));
                    sum += p[e];
                }
                // bf16: few rows wait for the cache and not for products, so that their P, and in the backward P and dS, need not be
                // rounded: four sequences of one token on caches of 65536, d = 64, 26.0 us against 25.6, and O as near as its type
                // allows (1.7e-3 in the 2-norm); backward of 4 heads, L = 256, d = 64, 18.2 against 17.3.  In sums over few keys a
                // rounding is not averaged.  Many rows pay for it with a fifth to a half of their time, so that theirs are rounded
                // once (O 2.4e-3 off): 2 heads, L = 262144, d = 64, W = 256, forward 109 us, in two parts 155, backward 345, 460;
                // 16 heads on 4, L = 4096, d = 128, causal, backward 312, 382; 8 heads, L = 4096, causal, d = 64, forward 44, 52.
                sm_accum<T, D, NW == 1>(acc, vc[n], p, lane);
            }
        } else {
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const int base = j0 + 32 * n;
                if (base > w_hi || base + 31 < w_lo) continue;
                const bool whole = base >= all_lo && base + 31 <= all_hi && (unsigned)(here >> (32 * n)) == ~0u;
                f32x16 s, z;
                SmRows<T, D> kr, vr;
                SmCols<T, D> kc;
                kr.read(lds[buf][0] + n * TL::SUB, lane);
                vr.read(lds[buf][1] + n * TL::SUB, lane);
                SM_READ_FIRST();
                sm_scores<T, D>(s, kr, q, lane);
                sm_scores<T, D>(z, vr, g, lane);
                kc.read(lds[buf][0] + n * TL::SUB, lane);
                SM_READ_FIRST();
                if (!whole) {
                    const unsigned keep = (sm_bits(my_lo - base, min(my_hi, j_hi) - base) & (unsigned)(here >> (32 * n))) >> (4 * h);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = sm_keep(s[e], keep, 8 * (e >> 2) + (e & 3), none);
                }
                float p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) p[e] = fast_exp2(fmaf(s[e], c2, -m)) * (z[e] - delta);
                sm_accum<T, D, NW == 1>(acc, kc, p, lane);
            }
        }
    };
    for (int t = 0; t < tiles; t += 2) {
        step(std::integral_constant<int, 0>{}, t);
        if (t + 1 < tiles) step(std::integral_constant<int, 1>{}, t + 1);
    }

    __syncthreads();   // (the tiles' LDS is used for the results)
    float scale = a.cs;
    if constexpr (!BWD) {
        // A row without a key is zeros, one that a NaN or an infinite score has poisoned is NaN: no comparison may take the second
        // for the first.  Scores of -inf alone sum to 0 and are 0 / 0 too; in a part of a walk they weigh nothing (SM_NOTHING).
        sum += __shfl_xor(sum, 32);
        live = live && keys != 0;
        const bool nothing = sum == 0.f;
        scale = nothing && a.parts > 1 ? 0.f : 1.f / sum;
        const float lse = !live ? -INFINITY : !nothing ? (m + fast_log2(sum)) * LN2 : a.parts > 1 ? SM_NOTHING : NAN;
        if (h == 0 && r < R) {
            if (a.parts > 1) a.part_lse[((long)w.part * a.B * a.Hk + prob) * R + r] = lse;
            else a.lse[((long)w.b * a.G * a.Hk + hq) * a.Lq + i] = lse;
        }
    }
    if (a.parts > 1) {
        float *out = a.part + (((long)w.part * a.B * a.Hk + prob) * R + r) * D;
        if (r >= R) return;
#pragma unroll
        for (int v = 0; v < D / 32; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<float4 *>(out + 32 * v + 8 * e + 4 * h) =
                    live ? make_float4(acc[v][4 * e] * scale, acc[v][4 * e + 1] * scale, acc[v][4 * e + 2] * scale, acc[v][4 * e + 3] * scale)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
        T *out = reinterpret_cast<T *>(const_cast<void *>(a.oq.p)) + w.b * a.oq.b + (long)w.hk * a.G * a.oq.h;
        sm_store_rows<T, D>(&lds[0][0][0] + wv * TL::SUB, acc, scale, live, lane, [&](int x) -> T * {
            const int rr = wr0 + x, ii = a.by_g(rr);
            return rr < R ? out + (rr - ii * a.G) * a.oq.h + ii * a.oq.l : nullptr;
        });
    }
}

// ------------------------------------------------------------------ keys as owners: dK, dV
// The queries of one head after another: each is a walk of its own over the same positions.
template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW, 1) void sm_keys_kernel(const SmArgs a)
{
    using TL = SmTile<T, D>;
    constexpr int KT = TL::KT, NS = KT / 32, BM = 32 * NW;
    constexpr int NBUF = 4 * TL::BYTES + 1024 <= 65536 ? 2 : 1;   // (fp32, d = 128: one, and other workgroups while it is filled)
    __shared__ __align__(1024) unsigned char lds[NBUF][2][TL::BYTES];
    __shared__ __align__(256) float vec[2][2][64];   // of the tile's rows: LSE log2(e) (inf: no such row), delta

    SmPlace w;
    if (!sm_place(a, w)) return;
    const int k0 = w.blk * BM;
    const int lq = sm_len(a.len_q, w.b, a.Lq), lk = sm_len(a.len_k, w.b, a.Lk), start = sm_start(a, w.b);
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const long prob = (long)w.b * a.Hk + w.hk;
    const int up = a.causal ? 0 : a.W;
    OwnerFrag<T, D> k, v;
    const int w_first = k0 + 32 * wv, w_last = w_first + 31;
    const int jc = min(w_first + (lane & 31), a.Lk - 1);
    sm_frag<T, D>(k, reinterpret_cast<const T *>(a.k.p) + w.b * a.k.b + w.hk * a.k.h + jc * a.k.l, h);
    sm_frag<T, D>(v, reinterpret_cast<const T *>(a.v.p) + w.b * a.v.b + w.hk * a.v.h + jc * a.v.l, h);

    // queries that reach the block's keys: p - W <= j <= p + up
    const int k_last = min(min(k0 + BM, a.Lk), lk) - 1;
    const int i_lo = max(0, k0 - up - start), i_hi = min(lq - 1, k_last + a.W - start);
    const int per_head = k_last < k0 || i_hi < i_lo ? 0 : (i_hi - i_lo + KT) / KT;
    int t0 = 0, t1 = per_head * a.G;
    if (a.parts > 1) {
        const int per = a.by_parts(t1 + a.parts - 1);
        t0 = w.part * per;
        t1 = min(t1, t0 + per);
    }

    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[x][e] = dv[x][e] = 0.f;

    const long head0 = (long)w.b * a.G * a.Hk + w.hk * a.G;
    const T *qb = reinterpret_cast<const T *>(a.q.p) + w.b * a.q.b + (long)w.hk * a.G * a.q.h;
    const T *gb = reinterpret_cast<const T *>(a.g.p) + w.b * a.g.b + (long)w.hk * a.G * a.g.h;
    const long qs = a.q.l * (long)sizeof(T), gs = a.g.l * (long)sizeof(T);
    const unsigned char *mq = a.mask_q ? a.mask_q + (long)w.b * a.Lq : nullptr;
    const SmLoader<T, D, NW> loader(lane, wv);
    const unsigned lds_at = sm_lds(lds), vec_at = sm_lds(vec);
    SmActivity<T, D, NW> act;
    int head = t0 < t1 ? t0 / per_head : 0, at = t0 - head * per_head;   // of the next tile to fetch
    auto fetch = [&](int buf) __attribute__((always_inline)) {
        const int i0 = i_lo + at * KT, rows = i_hi + 1 - i0;
        loader.load(lds_at + buf * 2 * TL::BYTES, reinterpret_cast<const unsigned char *>(qb + head * a.q.h) + i0 * qs, qs, rows);
        loader.load(lds_at + (buf * 2 + 1) * TL::BYTES, reinterpret_cast<const unsigned char *>(gb + head * a.g.h) + i0 * gs, gs, rows);
        if (wv == 0) {   // 64 entries of both vectors: rows beyond the last repeat it
            const long e = (head0 + head) * a.Lq + i0;
            const unsigned o = (unsigned)min(lane, rows - 1) * 4;
            sm_load_words(vec_at + buf * 512, a.lse2 + e, o);
            sm_load_words(vec_at + buf * 512 + 256, a.delta + e, o);
        }
        if (mq) act.load(loader, mq + i0, rows);
        if (++at == per_head) { at = 0; ++head; }
    };
    int i0 = i_lo + at * KT;   // first query of the tile at hand
    const float c2 = sm_vector(a.c2);
    auto step = [&](auto which, int t) __attribute__((always_inline)) {
        constexpr int buf = decltype(which)::value;
        const int rows = i_hi + 1 - i0;
        if (NBUF == 1) {
            if (t > t0) __syncthreads();
            fetch(0);
        }
        sm_arrived();
        if (rows < KT || mq) {
            const unsigned on = mq ? act.rows() : ~0u;
            loader.clear(lds[buf][0], rows, on);
            loader.clear(lds[buf][1], rows, on);
            if (wv == 0 && lane >= rows) {
                vec[buf][0][lane] = INFINITY;
                vec[buf][1][lane] = 0.f;
            }
        }
        __syncthreads();
        const int next = i_lo + at * KT;
        if (NBUF == 2 && t + 1 < t1) fetch(buf ^ 1);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int p_first = start + i0 + 32 * n, p_last = p_first + 31;   // positions of the score tile's rows
            if (p_last + up < w_first || p_first - a.W > w_last || 32 * n >= rows) continue;
            const bool whole = p_first + up >= w_last && p_last - a.W <= w_first;
            f32x16 s, z;
            SmRows<T, D> qr, gr;
            SmCols<T, D> qc, gc;
            qr.read(lds[buf][0] + n * TL::SUB, lane);
            gr.read(lds[buf][1] + n * TL::SUB, lane);
            SM_READ_FIRST();
            sm_scores<T, D>(s, qr, k, lane);
            sm_scores<T, D>(z, gr, v, lane);
            gc.read(lds[buf][1] + n * TL::SUB, lane);
            qc.read(lds[buf][0] + n * TL::SUB, lane);
            SM_READ_FIRST();
            float p[16], ds[16];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 l4 = *reinterpret_cast<const float4 *>(&vec[buf][0][32 * n + 8 * e + 4 * h]);
                const float4 d4 = *reinterpret_cast<const float4 *>(&vec[buf][1][32 * n + 8 * e + 4 * h]);
                const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    p[4 * e + x] = fast_exp2(fmaf(s[4 * e + x], c2, -ls[x]));
                    ds[4 * e + x] = z[4 * e + x] - dl[x];
                }
            }
            if (!whole) {
                // pair (p, j): p - W <= j <= p + up; bits of the tile's rows p_first ...
                const int d = w_first + (lane & 31) - p_first;
                const unsigned keep = sm_bits(d - up, d + a.W) >> (4 * h);
#pragma unroll
                for (int e = 0; e < 16; ++e) p[e] = sm_keep(p[e], keep, 8 * (e >> 2) + (e & 3), 0.f);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) ds[e] *= p[e];
            sm_accum<T, D, NW == 1>(dv, gc, p, lane);   // (rounded as the other kernel's are)
            sm_accum<T, D, NW == 1>(dk, qc, ds, lane);
        }
        i0 = next;
    };
    if (NBUF == 2 && t0 < t1) fetch(0);
    // A key that no query reaches may hold anything, and 0 times its scores or its dP is NaN where it does: such a key is zeros here,
    // once, and is not selected away in every tile (all of the backward of 16 heads on 4, L = 4096, d = 128, causal, 312 us; with dS
    // selected by bits as P is 319)
    if (const int j = w_first + (lane & 31), p0 = start - a.W, p1 = start + lq - 1 + up; __any(j < p0 || j > p1)) {
        if (j < p0 || j > p1) {
            k = OwnerFrag<T, D>{};
            v = OwnerFrag<T, D>{};
        }
    }
    for (int t = t0; t < t1; t += 2) {
        step(std::integral_constant<int, 0>{}, t);
        if (t + 1 < t1) step(std::integral_constant<int, NBUF - 1>{}, t + 1);
    }

    __syncthreads();   // (the tiles' LDS is used for the results)
    const int j = w_first + (lane & 31);
    bool live = j < lk;
    if (live && a.mask_k) live = a.mask_k[(long)w.b * a.Lk + j] != 0;
    if (a.parts > 1) {
        if (j >= a.Lk) return;
        float *out = a.part + (((long)w.part * a.B * a.Hk + prob) * a.Lk + j) * 2 * D;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float *o = out + 32 * x + 8 * e + 4 * h;
                *reinterpret_cast<float4 *>(o) = live ? make_float4(dk[x][4 * e] * a.cs, dk[x][4 * e + 1] * a.cs, dk[x][4 * e + 2] * a.cs, dk[x][4 * e + 3] * a.cs) : make_float4(0.f, 0.f, 0.f, 0.f);
                *reinterpret_cast<float4 *>(o + D) = live ? make_float4(dv[x][4 * e], dv[x][4 * e + 1], dv[x][4 * e + 2], dv[x][4 * e + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
    } else {
        T *ok = reinterpret_cast<T *>(const_cast<void *>(a.ok.p)) + w.b * a.ok.b + w.hk * a.ok.h;
        T *ov = reinterpret_cast<T *>(const_cast<void *>(a.ov.p)) + w.b * a.ov.b + w.hk * a.ov.h;
        // (where one buffer of tiles has not room for all wavefronts' rows: two of them after the other two)
        constexpr bool ROOM = sizeof(lds) >= NW * TL::SUB;
        unsigned char *mine = &lds[0][0][0] + (ROOM ? wv : wv & 1) * TL::SUB;
        for (int turn = 0; turn < (ROOM ? 1 : 2); ++turn) {
            if (ROOM || wv >> 1 == turn) {
                sm_store_rows<T, D>(mine, dk, a.cs, live, lane, [&](int x) -> T * { return w_first + x < a.Lk ? ok + (w_first + x) * a.ok.l : nullptr; });
                sm_store_rows<T, D>(mine, dv, 1.f, live, lane, [&](int x) -> T * { return w_first + x < a.Lk ? ov + (w_first + x) * a.ov.l : nullptr; });
            }
            if (!ROOM) __syncthreads();
        }
    }
}

// ------------------------------------------------------------------ joining the parts of a walk
enum { SM_JOIN_O, SM_JOIN_DQ, SM_JOIN_DKV };
// A thread takes four features of a row over every slices-th part; the slices are joined by LDS in their order.  O: the parts'
// rows weighted by exp(their LSE - the largest); gradients: sums.
template <typename T, int D, int WHAT> __global__ __launch_bounds__(NTHREADS) void sm_join_kernel(const SmArgs a, int slices)
{
    constexpr int F = WHAT == SM_JOIN_DKV ? 2 * D : D, FT = F / 4;   // features of a part's row, threads for them
    __shared__ float4 sx[NTHREADS];
    __shared__ float sm[NTHREADS], sl[NTHREADS];
    const int R = WHAT == SM_JOIN_DKV ? a.Lk : a.Lq * a.G;
    const int f = (threadIdx.x % FT) * 4, rest = threadIdx.x / FT, slice = rest % slices;
    const long rows = (long)a.B * a.Hk * R, row = (long)blockIdx.x * (NTHREADS / FT / slices) + rest / slices;
    const bool have = row < rows;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    if (have) {
#pragma unroll 4
        for (int s = slice; s < a.parts; s += slices) {
            const float4 y = *reinterpret_cast<const float4 *>(a.part + (s * rows + row) * F + f);
            float c = 1.f;
            if constexpr (WHAT == SM_JOIN_O) {
                // (fmaxf passes over a NaN, so that m never is one; c is, and l and x from there on)
                const float lse = a.part_lse[s * rows + row], mn = fmaxf(m, lse);
                const float old = m > -INFINITY ? fast_exp2((m - mn) * LOG2E) : 0.f;
                c = lse != -INFINITY ? fast_exp2((lse - mn) * LOG2E) : 0.f;
                l = fmaf(l, old, c);
                x.x *= old; x.y *= old; x.z *= old; x.w *= old;
                m = mn;
            }
            x.x = fmaf(c, y.x, x.x); x.y = fmaf(c, y.y, x.y); x.z = fmaf(c, y.z, x.z); x.w = fmaf(c, y.w, x.w);
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
            const float4 y = sx[o];
            float c = 1.f, old = 1.f;
            if constexpr (WHAT == SM_JOIN_O) {
                const float mn = fmaxf(m, sm[o]);
                old = m > -INFINITY ? fast_exp2((m - mn) * LOG2E) : 0.f;
                c = sm[o] > -INFINITY ? fast_exp2((sm[o] - mn) * LOG2E) : 0.f;
                l = l * old + sl[o] * c;
                m = mn;
            }
            x.x = x.x * old + y.x * c; x.y = x.y * old + y.y * c; x.z = x.z * old + y.z * c; x.w = x.w * old + y.w * c;
        }
    }
    if (!have) return;
    const int prob = (int)(row / R), r = (int)(row - (long)prob * R), b = a.by_hk(prob), hk = prob - b * a.Hk;
    if constexpr (WHAT == SM_JOIN_DKV) {
        const SmTensor &t = f < D ? a.ok : a.ov;
        T *out = reinterpret_cast<T *>(const_cast<void *>(t.p)) + b * t.b + hk * t.h + r * t.l;
        store4<T>(out + (f < D ? f : f - D), x.x, x.y, x.z, x.w);
    } else {
        const int i = a.by_g(r), hq = hk * a.G + (r - i * a.G);
        if (WHAT == SM_JOIN_O && m == SM_NOTHING) l = NAN;   // (keys, whose scores are all -inf)
        const float c = WHAT == SM_JOIN_O ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        T *out = reinterpret_cast<T *>(const_cast<void *>(a.oq.p)) + b * a.oq.b + hq * a.oq.h + i * a.oq.l;
        store4<T>(out + f, x.x * c, x.y * c, x.z * c, x.w * c);
        if (WHAT == SM_JOIN_O && f == 0) a.lse[((long)b * a.Hk * a.G + hq) * a.Lq + i] = l == 0.f ? -INFINITY : m + fast_log2(l) * LN2;
    }
}

}  // namespace
