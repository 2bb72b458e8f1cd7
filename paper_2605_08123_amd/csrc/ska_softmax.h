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
// Query heads that share a key head are rows of the same problem: row r of problem (b, key head) is query r / G of head
// r % G of the group, G = Hq / Hk.  Keys are read once for the group, and dK, dV sum over it by themselves.
#pragma once
#include "ska_common.h"

namespace {

struct SmTensor {
    const void *p;
    long b, h, l;   // elements between items, heads, tokens
};
struct SmArgs {
    SmTensor q, k, v, o, g;        // g: dO
    SmTensor oq, ok, ov;           // forward: oq = O; backward: dQ, dK, dV (written)
    float *lse, *delta;            // [B][Hq][Lq]
    const int *start, *len_q, *len_k;
    const unsigned char *mask_q, *mask_k;
    float *part, *part_lse;        // walks in parts: [parts][problems][rows][D] (forward: and their LSE [parts][problems][rows])
    int B, Hk, G, Lq, Lk, W, causal;
    int parts;                     // parts of a walk
    int blocks;                    // blocks of owners per problem
    int total;                     // blocks * parts * problems
    int order;                     // SmOrder
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
        x = blockIdx.x / N;
        n = blockIdx.x - x * N;
        if (a.order == SM_LAST_FIRST) x = a.blocks * a.parts - 1 - x;
    } else {
        const int per = gridDim.x / 8, at = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
        if (at >= a.total) return false;
        n = at / (a.blocks * a.parts);
        x = at - n * a.blocks * a.parts;
    }
    w.blk = x / a.parts;
    w.part = x - w.blk * a.parts;
    w.b = n / a.Hk;
    w.hk = n - w.b * a.Hk;
    return true;
}
__device__ __forceinline__ int sm_len(const int *len, int b, int L) { return len ? min(max(len[b], 0), L) : L; }
__device__ __forceinline__ int sm_start(const SmArgs &a, int b) { return a.start ? min(max(a.start[b], 0), 1 << 24) : 0; }

// Tiles: KT walked rows (two score tiles of 32 for bf16, one for fp32: the same bytes)
template <typename T, int D> struct SmTile {
    static constexpr int KT = sizeof(T) == 2 ? 64 : 32;
    static constexpr int CPR = D * (int)sizeof(T) / 16;                      // 16-byte pieces per row
    static constexpr int SUB = Tile<T, D>::RM_BYTES;                         // bytes of 32 rows in LDS
    static constexpr int BYTES = SUB * (KT / 32);
};
// A walked tile of one matrix on its way from memory to LDS, by the NT threads of a workgroup
template <typename T, int D, int NT> struct SmStage {
    using TL = SmTile<T, D>;
    static constexpr int N = TL::KT * TL::CPR / NT;   // pieces per thread
    static_assert(TL::KT * TL::CPR % NT == 0 && NT % TL::CPR == 0, "whole pieces");
    uint4 r[N];
    static __device__ __forceinline__ int row(int c) { return (int)threadIdx.x / TL::CPR + c * (NT / TL::CPR); }
    static __device__ __forceinline__ int chunk() { return (int)threadIdx.x % TL::CPR; }
    __device__ __forceinline__ void load(int c, const T *row_at) { r[c] = *reinterpret_cast<const uint4 *>(row_at + chunk() * (16 / (int)sizeof(T))); }
    __device__ __forceinline__ void store(int c, unsigned char *lds, bool there)
    {
        const uint4 x = there ? r[c] : make_uint4(0, 0, 0, 0);
        const int i = row(c);
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4 *>(lds + bf16_chunk_off<D>(i, chunk())) = x;
        else *reinterpret_cast<uint4 *>(lds + (i * f32_row_floats<D>() + chunk() * 4) * 4) = x;
    }
};
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
// x where bit `bit` of m is set, otherwise -inf
__device__ __forceinline__ float sm_keep(float x, unsigned m, int bit)
{
    const int on = ((int)(m << (31 - bit))) >> 31;
    return __int_as_float((__float_as_int(x) & on) | (~on & (int)0xff800000));
}
// bits [a, b] of 32 (none where b < a)
__device__ __forceinline__ unsigned sm_bits(int a, int b)
{
    const unsigned hi = b >= 31 ? 0xffffffffu : b < 0 ? 0u : (2u << b) - 1u;
    const unsigned lo = a <= 0 ? 0xffffffffu : a >= 32 ? 0u : ~((1u << a) - 1u);
    return hi & lo;
}

constexpr float SM_LAZY = 8.f;   // powers of two that a row's maximum may grow by before its sums are scaled to it

// ------------------------------------------------------------------ queries as owners: forward, dQ
// BWD: dQ instead of O.  NW wavefronts, 32 rows each.
template <typename T, int D, int NW, bool BWD>
__global__ __launch_bounds__(64 * NW) void sm_rows_kernel(const SmArgs a)
{
    using TL = SmTile<T, D>;
    using Stage = SmStage<T, D, 64 * NW>;
    constexpr int KT = TL::KT, NS = KT / 32, BM = 32 * NW;
    constexpr int NBUF = 4 * TL::BYTES <= 65536 ? 2 : 1;
    __shared__ __align__(16) unsigned char lds[NBUF][2][TL::BYTES];

    SmPlace w;
    if (!sm_place(a, w)) return;
    const int R = a.Lq * a.G, r0 = w.blk * BM;
    const int lq = sm_len(a.len_q, w.b, a.Lq), lk = sm_len(a.len_k, w.b, a.Lk), start = sm_start(a, w.b);
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, h = lane >> 5;
    const long prob = (long)w.b * a.Hk + w.hk;

    // this lane's row
    const int r = r0 + 32 * wv + (lane & 31), rc = min(r, R - 1), i = rc / a.G, hq = w.hk * a.G + (rc - i * a.G);
    bool live = r < R && i < lq;
    if (live && a.mask_q) live = a.mask_q[(long)w.b * a.Lq + i] != 0;
    const long head = (long)w.b * a.G * a.Hk + hq;   // of [B][Hq][Lq] vectors
    OwnerFrag<T, D> q, g;
    sm_frag<T, D>(q, reinterpret_cast<const T *>(a.q.p) + w.b * a.q.b + hq * a.q.h + i * a.q.l, h);
    float m = -INFINITY, sum = 0.f, delta = 0.f;   // BWD: m = LSE log2(e)
    if constexpr (BWD) {
        OwnerFrag<T, D> o;
        sm_frag<T, D>(g, reinterpret_cast<const T *>(a.g.p) + w.b * a.g.b + hq * a.g.h + i * a.g.l, h);
        sm_frag<T, D>(o, reinterpret_cast<const T *>(a.o.p) + w.b * a.o.b + hq * a.o.h + i * a.o.l, h);
        const float lse = a.lse[head * a.Lq + i];
        live = live && lse > -INFINITY;
        m = live ? lse * LOG2E : INFINITY;      // (exp2(s - inf) = 0)
        delta = sm_dot<D>(g, o);
        if (!live) delta = 0.f;
        if (w.part == 0 && h == 0 && r < R) a.delta[head * a.Lq + i] = delta;
    }

    // keys that the block's rows, and this wavefront's, can reach
    const int i_last = min(min(r0 + BM, R) - 1, lq * a.G - 1) / a.G;   // (lq 0: no row, and no key below)
    int j_lo = max(0, start + r0 / a.G - a.W), j_hi = min(lk - 1, start + i_last + (a.causal ? 0 : a.W));
    if (lq * a.G <= r0) j_hi = j_lo - 1;
    const int w_first = start + min(r0 + 32 * wv, R - 1) / a.G, w_last = start + min(r0 + 32 * wv + 31, R - 1) / a.G;
    const int up = a.causal ? 0 : a.W;
    const int w_lo = w_first - a.W, w_hi = w_last + up;                  // any of its rows
    const int all_lo = w_last - a.W, all_hi = min(w_first + up, lk - 1); // all of them
    int tiles = (j_hi - j_lo + KT) / KT;
    if (a.parts > 1) {
        const int per = (tiles + a.parts - 1) / a.parts;
        j_lo += w.part * per * KT;
        tiles = min(per, tiles - w.part * per);
    }
    const int my_lo = start + i - a.W, my_hi = min(start + i + up, lk - 1);

    f32x16 acc[D / 32];
#pragma unroll
    for (int v = 0; v < D / 32; ++v)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[v][e] = 0.f;

    const T *kb = reinterpret_cast<const T *>(a.k.p) + w.b * a.k.b + w.hk * a.k.h;
    const T *vb = reinterpret_cast<const T *>(a.v.p) + w.b * a.v.b + w.hk * a.v.h;
    const unsigned char *mk = a.mask_k ? a.mask_k + (long)w.b * a.Lk : nullptr;
    Stage sk, sv;
    unsigned char on = 1, row_on[Stage::N];   // activity of key `lane` of the tile, and of the rows this thread stages
    auto fetch = [&](int j0) {
#pragma unroll
        for (int c = 0; c < Stage::N; ++c) {
            const int j = min(j0 + Stage::row(c), j_hi);
            sk.load(c, kb + j * a.k.l);
            sv.load(c, vb + j * a.v.l);
            row_on[c] = mk ? mk[j] : 1;
        }
        if (mk) on = mk[min(j0 + (lane & (KT - 1)), j_hi)];
    };
    auto put = [&](int j0, int buf) {
#pragma unroll
        for (int c = 0; c < Stage::N; ++c) {
            const bool there = j0 + Stage::row(c) <= j_hi && row_on[c];
            sk.store(c, lds[buf][0], there);
            sv.store(c, lds[buf][1], there);
        }
    };
    if (tiles > 0) fetch(j_lo);
    for (int t = 0; t < tiles; ++t) {
        const int j0 = j_lo + t * KT, buf = NBUF == 2 ? t & 1 : 0;
        if (NBUF == 1 && t) __syncthreads();
        put(j0, buf);
        const unsigned long long active = mk ? __ballot(on != 0) : ~0ull;
        __syncthreads();
        if (t + 1 < tiles) fetch(j0 + KT);
        if (j0 > w_hi || j0 + KT - 1 < w_lo) continue;
        const unsigned char *kt = lds[buf][0], *vt = lds[buf][1];
        f32x16 s[NS], z[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[n][e] = z[n][e] = 0.f;
            s[n] = tile_dot<D>(kt + n * TL::SUB, q, lane, s[n]);
            if constexpr (BWD) z[n] = tile_dot<D>(vt + n * TL::SUB, g, lane, z[n]);
        }
        const bool whole = j0 >= all_lo && j0 + KT - 1 <= all_hi && active == ~0ull;
        if (!whole) {
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const int base = j0 + 32 * n;
                const unsigned keep = (sm_bits(my_lo - base, min(my_hi, j_hi) - base) & (unsigned)(active >> (32 * n))) >> (4 * h);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[n][e] = sm_keep(s[n][e], keep, 8 * (e >> 2) + (e & 3));
            }
        }
        if constexpr (!BWD) {
            // Running maximum: sums stay relative to an older one until a score exceeds it by 2^SM_LAZY, so that the
            // accumulators are scaled a few times per row and not once per tile; P up to 2^8 loses nothing in either type.
            float top = s[0][0];
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, s[n][e]);
            top = fmaxf(top, __shfl_xor(top, 32)) * a.c2;
            if (__any(top > m + SM_LAZY)) {
                const float mn = fmaxf(m, top), f = mn > -INFINITY ? fast_exp2(m - mn) : 1.f;
                sum *= f;
#pragma unroll
                for (int v = 0; v < D / 32; ++v)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[v][e] *= f;
                m = mn;
            }
            const float mu = m > -INFINITY ? m : 0.f;
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                float p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    p[e] = fast_exp2(fmaf(s[n][e], a.c2, -mu));
                    sum += p[e];
                }
                tile_accum<T, D>(acc, vt + n * TL::SUB, p, lane);
            }
        } else {
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                float p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) p[e] = fast_exp2(fmaf(s[n][e], a.c2, -m)) * (z[n][e] - delta);
                tile_accum<T, D>(acc, kt + n * TL::SUB, p, lane);
            }
        }
    }

    float scale = a.cs;
    if constexpr (!BWD) {
        sum += __shfl_xor(sum, 32);
        live = live && sum > 0.f;
        scale = live ? 1.f / sum : 0.f;
        const float lse = live ? (m + fast_log2(sum)) * LN2 : -INFINITY;
        if (h == 0 && r < R) {
            if (a.parts > 1) a.part_lse[((long)w.part * a.B * a.Hk + prob) * R + r] = lse;
            else a.lse[head * a.Lq + i] = lse;
        }
    }
    if (r >= R) return;
    if (a.parts > 1) {
        float *out = a.part + (((long)w.part * a.B * a.Hk + prob) * R + r) * D;
#pragma unroll
        for (int v = 0; v < D / 32; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<float4 *>(out + 32 * v + 8 * e + 4 * h) =
                    live ? make_float4(acc[v][4 * e] * scale, acc[v][4 * e + 1] * scale, acc[v][4 * e + 2] * scale, acc[v][4 * e + 3] * scale)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
        return;
    }
    T *out = reinterpret_cast<T *>(const_cast<void *>(a.oq.p)) + w.b * a.oq.b + hq * a.oq.h + i * a.oq.l;
#pragma unroll
    for (int v = 0; v < D / 32; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            T *at = out + 32 * v + 8 * e + 4 * h;
            if (live) store4<T>(at, acc[v][4 * e] * scale, acc[v][4 * e + 1] * scale, acc[v][4 * e + 2] * scale, acc[v][4 * e + 3] * scale);
            else store4<T>(at, 0.f, 0.f, 0.f, 0.f);
        }
}

// ------------------------------------------------------------------ keys as owners: dK, dV
template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW) void sm_keys_kernel(const SmArgs a)
{
    using TL = SmTile<T, D>;
    using Stage = SmStage<T, D, 64 * NW>;
    constexpr int KT = TL::KT, NS = KT / 32, BM = 32 * NW;
    constexpr int NBUF = 4 * TL::BYTES + 2 * 3 * KT * 4 <= 65536 ? 2 : 1;
    __shared__ __align__(16) unsigned char lds[NBUF][2][TL::BYTES];
    __shared__ __align__(16) float vec[NBUF][3][KT];   // of the tile's rows: LSE log2(e) (inf: no such row), delta, position

    SmPlace w;
    if (!sm_place(a, w)) return;
    const int R = a.Lq * a.G, k0 = w.blk * BM;
    const int lq = sm_len(a.len_q, w.b, a.Lq), lk = sm_len(a.len_k, w.b, a.Lk), start = sm_start(a, w.b);
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, h = lane >> 5;
    const long prob = (long)w.b * a.Hk + w.hk;
    const int j = k0 + 32 * wv + (lane & 31), jc = min(j, a.Lk - 1);
    bool live = j < lk;
    if (live && a.mask_k) live = a.mask_k[(long)w.b * a.Lk + j] != 0;
    OwnerFrag<T, D> k, v;
    sm_frag<T, D>(k, reinterpret_cast<const T *>(a.k.p) + w.b * a.k.b + w.hk * a.k.h + jc * a.k.l, h);
    sm_frag<T, D>(v, reinterpret_cast<const T *>(a.v.p) + w.b * a.v.b + w.hk * a.v.h + jc * a.v.l, h);

    // queries that reach the block's keys, and this wavefront's: p - W <= j <= p + up
    const int up = a.causal ? 0 : a.W;
    const int k_last = min(min(k0 + BM, a.Lk), lk) - 1;
    const int i_lo = max(0, k0 - up - start), i_hi = min(lq - 1, k_last + a.W - start);
    int r_lo = i_lo * a.G, r_hi = i_hi * a.G + a.G - 1;
    if (k_last < k0 || i_hi < i_lo) { r_lo = 0; r_hi = -1; }
    const int w_first = k0 + 32 * wv, w_last = w_first + 31;
    int tiles = (r_hi - r_lo + KT) / KT;
    if (a.parts > 1) {
        const int per = (tiles + a.parts - 1) / a.parts;
        r_lo += w.part * per * KT;
        tiles = min(per, tiles - w.part * per);
    }

    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[x][e] = dv[x][e] = 0.f;

    const long head0 = (long)w.b * a.G * a.Hk + w.hk * a.G;
    const T *qb = reinterpret_cast<const T *>(a.q.p) + w.b * a.q.b + (long)w.hk * a.G * a.q.h;
    const T *gb = reinterpret_cast<const T *>(a.g.p) + w.b * a.g.b + (long)w.hk * a.G * a.g.h;
    const unsigned char *mq = a.mask_q ? a.mask_q + (long)w.b * a.Lq : nullptr;
    Stage sq, sg;
    unsigned char row_on[Stage::N];
    float lse = 0.f, del = 0.f;
    int pos = 0;
    auto fetch = [&](int r0) {
#pragma unroll
        for (int c = 0; c < Stage::N; ++c) {
            const int r = min(r0 + Stage::row(c), r_hi), i = a.G == 1 ? r : r / a.G, hg = r - i * a.G;
            sq.load(c, qb + hg * a.q.h + i * a.q.l);
            sg.load(c, gb + hg * a.g.h + i * a.g.l);
            row_on[c] = mq ? mq[i] : 1;
        }
        if (threadIdx.x < KT) {
            const int r = min(r0 + (int)threadIdx.x, r_hi), i = a.G == 1 ? r : r / a.G, hg = r - i * a.G;
            lse = a.lse[(head0 + hg) * a.Lq + i] * LOG2E;
            del = a.delta[(head0 + hg) * a.Lq + i];
            pos = start + i;
            if (r0 + (int)threadIdx.x > r_hi || !(lse > -INFINITY) || (mq && !mq[i])) { lse = INFINITY; del = 0.f; }
        }
    };
    auto put = [&](int r0, int buf) {
#pragma unroll
        for (int c = 0; c < Stage::N; ++c) {
            const bool there = r0 + Stage::row(c) <= r_hi && row_on[c];
            sq.store(c, lds[buf][0], there);
            sg.store(c, lds[buf][1], there);
        }
        if (threadIdx.x < KT) {
            vec[buf][0][threadIdx.x] = lse;
            vec[buf][1][threadIdx.x] = del;
            vec[buf][2][threadIdx.x] = __int_as_float(pos);
        }
    };
    if (tiles > 0) fetch(r_lo);
    for (int t = 0; t < tiles; ++t) {
        const int r0 = r_lo + t * KT, buf = NBUF == 2 ? t & 1 : 0;
        if (NBUF == 1 && t) __syncthreads();
        put(r0, buf);
        __syncthreads();
        if (t + 1 < tiles) fetch(r0 + KT);
        // positions of the tile's first and last row
        const int p_first = __float_as_int(vec[buf][2][0]), p_last = __float_as_int(vec[buf][2][KT - 1]);
        if (p_last + up < w_first || p_first - a.W > w_last) continue;
        const bool whole = p_first + up >= w_last && p_last - a.W <= w_first;
        const unsigned char *qt = lds[buf][0], *gt = lds[buf][1];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            f32x16 s, z;
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = z[e] = 0.f;
            s = tile_dot<D>(qt + n * TL::SUB, k, lane, s);
            z = tile_dot<D>(gt + n * TL::SUB, v, lane, z);
            float p[16], ds[16];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 l4 = *reinterpret_cast<const float4 *>(&vec[buf][0][32 * n + 8 * e + 4 * h]);
                const float4 d4 = *reinterpret_cast<const float4 *>(&vec[buf][1][32 * n + 8 * e + 4 * h]);
                const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    p[4 * e + x] = fast_exp2(fmaf(s[4 * e + x], a.c2, -ls[x]));
                    ds[4 * e + x] = z[4 * e + x] - dl[x];
                }
            }
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int4 p4 = *reinterpret_cast<const int4 *>(&vec[buf][2][32 * n + 8 * e + 4 * h]);
                    const int ps[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if ((unsigned)(j - ps[x] + a.W) > (unsigned)(a.W + up)) p[4 * e + x] = 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) ds[e] *= p[e];
            tile_accum<T, D>(dv, gt + n * TL::SUB, p, lane);
            tile_accum<T, D>(dk, qt + n * TL::SUB, ds, lane);
        }
    }

    if (j >= a.Lk) return;
    if (a.parts > 1) {
        float *out = a.part + (((long)w.part * a.B * a.Hk + prob) * a.Lk + j) * 2 * D;
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float f = live ? a.cs : 0.f;
                float *at = out + 32 * x + 8 * e + 4 * h;
                *reinterpret_cast<float4 *>(at) = live ? make_float4(dk[x][4 * e] * f, dk[x][4 * e + 1] * f, dk[x][4 * e + 2] * f, dk[x][4 * e + 3] * f) : make_float4(0.f, 0.f, 0.f, 0.f);
                *reinterpret_cast<float4 *>(at + D) = live ? make_float4(dv[x][4 * e], dv[x][4 * e + 1], dv[x][4 * e + 2], dv[x][4 * e + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        return;
    }
    T *ok = reinterpret_cast<T *>(const_cast<void *>(a.ok.p)) + w.b * a.ok.b + w.hk * a.ok.h + j * a.ok.l;
    T *ov = reinterpret_cast<T *>(const_cast<void *>(a.ov.p)) + w.b * a.ov.b + w.hk * a.ov.h + j * a.ov.l;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int f = 32 * x + 8 * e + 4 * h;
            if (live) {
                store4<T>(ok + f, dk[x][4 * e] * a.cs, dk[x][4 * e + 1] * a.cs, dk[x][4 * e + 2] * a.cs, dk[x][4 * e + 3] * a.cs);
                store4<T>(ov + f, dv[x][4 * e], dv[x][4 * e + 1], dv[x][4 * e + 2], dv[x][4 * e + 3]);
            } else {
                store4<T>(ok + f, 0.f, 0.f, 0.f, 0.f);
                store4<T>(ov + f, 0.f, 0.f, 0.f, 0.f);
            }
        }
}

// ------------------------------------------------------------------ joining the parts of a walk
enum { SM_JOIN_O, SM_JOIN_DQ, SM_JOIN_DKV };
// A thread takes four features of a row: O from the parts' rows weighted by exp(their LSE - the row's), gradients as sums.
template <typename T, int D, int WHAT> __global__ __launch_bounds__(NTHREADS) void sm_join_kernel(const SmArgs a)
{
    constexpr int F = WHAT == SM_JOIN_DKV ? 2 * D : D;   // features of a part's row
    const int R = WHAT == SM_JOIN_DKV ? a.Lk : a.Lq * a.G;
    const long rows = (long)a.B * a.Hk * R, at = (long)blockIdx.x * NTHREADS + threadIdx.x;
    const long row = at / (F / 4);
    const int f = (int)(at - row * (F / 4)) * 4;
    if (row >= rows) return;
    const int prob = (int)(row / R), r = (int)(row - (long)prob * R), b = prob / a.Hk, hk = prob - b * a.Hk;
    float x[4] = {0.f, 0.f, 0.f, 0.f}, lse = 0.f, top = -INFINITY;
    if constexpr (WHAT == SM_JOIN_O) {
        for (int s = 0; s < a.parts; ++s) top = fmaxf(top, a.part_lse[s * rows + row]);
        float sum = 0.f;
        if (top > -INFINITY)
            for (int s = 0; s < a.parts; ++s) sum += fast_exp2((a.part_lse[s * rows + row] - top) * LOG2E);
        lse = top > -INFINITY ? top + fast_log2(sum) * LN2 : -INFINITY;
    }
    for (int s = 0; s < a.parts; ++s) {
        const float4 y = *reinterpret_cast<const float4 *>(a.part + (s * rows + row) * F + f);
        float c = 1.f;
        if constexpr (WHAT == SM_JOIN_O) c = top > -INFINITY ? fast_exp2((a.part_lse[s * rows + row] - lse) * LOG2E) : 0.f;
        x[0] = fmaf(c, y.x, x[0]); x[1] = fmaf(c, y.y, x[1]); x[2] = fmaf(c, y.z, x[2]); x[3] = fmaf(c, y.w, x[3]);
    }
    if constexpr (WHAT == SM_JOIN_DKV) {
        const SmTensor &t = f < D ? a.ok : a.ov;
        T *out = reinterpret_cast<T *>(const_cast<void *>(t.p)) + b * t.b + hk * t.h + r * t.l;
        store4<T>(out + (f < D ? f : f - D), x[0], x[1], x[2], x[3]);
    } else {
        const int i = r / a.G, hq = hk * a.G + (r - i * a.G);
        T *out = reinterpret_cast<T *>(const_cast<void *>(a.oq.p)) + b * a.oq.b + hq * a.oq.h + i * a.oq.l;
        store4<T>(out + f, x[0], x[1], x[2], x[3]);
        if (WHAT == SM_JOIN_O && f == 0) a.lse[((long)b * a.Hk * a.G + hq) * a.Lq + i] = lse;
    }
}

}  // namespace
