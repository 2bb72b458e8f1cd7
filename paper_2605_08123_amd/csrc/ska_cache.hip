// Caches in 8 bits (written, read back) and softmax attention on caches and shared prefixes: the host side of the attention
// (sinkhorn_attn_cache.h; kernels in ska_cache.h), and the kernels that write and read.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "sinkhorn_attn_cache.h"
#include "ska_cache_launch.h"
#include "ska_cache_plan.h"

namespace {

int bytes_of(int type) { return type == SKA_F32 ? 4 : type == SKA_BF16 ? 2 : 1; }

// A tensor's pointer and strides; SKA_EINVAL where they cannot be strides, SKA_EUNSUPPORTED where the kernels cannot use them.
int tensor_of(SmTensor &t, const void *p, const ska_strides *s, int B, int H, long L, int d, int type, int align, bool out)
{
    if (!p) return SKA_EINVAL;
    t.p = p;
    if (s) {
        t.b = (long)s->b; t.h = (long)s->h; t.l = (long)s->l;
        if (t.b < 0 || t.h < 0 || t.l < 0) return SKA_EINVAL;
        if (out && ((B > 1 && !t.b) || (H > 1 && !t.h) || (L > 1 && !t.l))) return SKA_EINVAL;
        if (B == 1) t.b = 0;   // (never stepped over, whatever it says)
        if (H == 1) t.h = 0;
        if (L == 1) t.l = 0;
    } else {
        t.l = d; t.h = L * d; t.b = t.h * H;
    }
    const long e = bytes_of(type);
    if (t.l * e >= 1L << 27) return SKA_EUNSUPPORTED;   // (32 tokens lie within 32 bits)
    const unsigned long off = (unsigned long)reinterpret_cast<uintptr_t>(p) | (unsigned long)((t.b | t.h | t.l) * e);
    return off & (unsigned long)(align - 1) ? SKA_EUNSUPPORTED : SKA_OK;
}
struct Scales { const float *p; long b, h; };
int scales_of(Scales &t, const float *p, const ska_scale_strides *s, int B, int H, long L, bool out)
{
    if (!p) return SKA_EINVAL;
    t = {p, s ? (long)s->b : L * H, s ? (long)s->h : L};
    if (t.b < 0 || t.h < 0 || (out && ((B > 1 && !t.b) || (H > 1 && !t.h)))) return SKA_EINVAL;
    if (B == 1) t.b = 0;
    if (H == 1) t.h = 0;
    return reinterpret_cast<uintptr_t>(p) & 3 ? SKA_EUNSUPPORTED : SKA_OK;
}

// ------------------------------------------------------------------ writing and reading
// A thread takes 8 features of a key's row and of the value's: D / 8 threads a row, which compare their largest features in registers.
// Memory bounds both, if only just: the codes are made and read by the conversion instructions, the largest feature of bf16 rows is
// looked for among bit patterns, two at a time (262144 tokens of 2 heads of 64 in bf16 and e4m3, 205 MB each way: written in 42 to 46 us,
// read back in 32, 4.7 and 6.4 TB/s; 20011 of 3 items, 4 heads of 128 in fp32 and int8: one workgroup for keys and values 105 us for both, of
// their own 79).
struct MoveArgs {
    SmTensor k, v, kc, vc;
    Scales ks, vs;
    const int *start, *len;
    int B, Hk, L, Lc;
    int inner;      // heads that follow one another within a token, as a projection leaves them: Hk, or 1
    SmDiv by_hk, by_inner;
};
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// 8 features of a row as they are stored
template <typename T> struct Eight;
template <> struct Eight<__bf16> {
    uint4 w;
    __device__ __forceinline__ void load(const __bf16 *p) { w = *reinterpret_cast<const uint4 *>(p); }
    // bits of the largest magnitude as fp32: as an unsigned number, so that infinities and NaN are the largest
    __device__ __forceinline__ unsigned largest() const
    {
        const unsigned x[4] = {w.x & 0x7fff7fffu, w.y & 0x7fff7fffu, w.z & 0x7fff7fffu, w.w & 0x7fff7fffu};
        u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(__builtin_bit_cast(u16x2, x[0]), __builtin_bit_cast(u16x2, x[1])),
                                            __builtin_elementwise_max(__builtin_bit_cast(u16x2, x[2]), __builtin_bit_cast(u16x2, x[3])));
        return (unsigned)max(m[0], m[1]) << 16;
    }
    __device__ __forceinline__ void floats(float (&f)[8]) const
    {
        const unsigned x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(x[i] << 16), f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    }
    // features 4 i ... 4 i + 3 divided by a power of two, as e4m3 numbers
    __device__ __forceinline__ unsigned e4m3(int i, float scale) const
    {
        const unsigned x[4] = {w.x, w.y, w.z, w.w};
        s16x2 r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, x[2 * i]), scale, false);
        return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2, x[2 * i + 1]), scale, true));
    }
};
template <> struct Eight<float> {
    float f[8];
    __device__ __forceinline__ void load(const float *p)
    {
        load4<float>(p, reinterpret_cast<float(&)[4]>(f[0]));
        load4<float>(p + 4, reinterpret_cast<float(&)[4]>(f[4]));
    }
    __device__ __forceinline__ unsigned largest() const
    {
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ void floats(float (&y)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = f[i];
    }
    __device__ __forceinline__ unsigned e4m3(int i, float scale) const
    {
        s16x2 r = {0, 0};
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[4 * i], f[4 * i + 1], scale, false);
        return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, f[4 * i + 2], f[4 * i + 3], scale, true));
    }
};
// the largest among the N adjacent lanes of a row
template <int N> __device__ __forceinline__ unsigned row_largest(unsigned m)
{
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true));             // lanes 1, 0, 3, 2
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true));             // 2, 3, 0, 1
    if (N > 4) m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true));   // 8 lanes mirrored
    if (N > 8) m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, true));   // 16 lanes mirrored
    return m;
}
// Scale of a row whose largest feature has the bits `a`
template <typename S> __device__ __forceinline__ float move_scale(unsigned a)
{
    if (a >= 0x7f800000u) return NAN;
    if constexpr (std::is_same<S, E4M3>::value)
        // a = 1.m 2^e: 448 = 1.75 2^8, so that the power is e - 8, and one more where 1.m is more than 1.75
        return __uint_as_float((unsigned)max((int)(a >> 23) - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0), 1) << 23);
    else return fminf(fmaxf(__uint_as_float(a) / 127.f, 0x1p-126f), 0x1.020406p+121f);   // (127 times the next number is infinite)
}
// 8 features as codes
template <typename S, typename T> __device__ __forceinline__ uint2 move_codes(const Eight<T> &x, float scale)
{
    if (!(scale > 0.f)) return make_uint2(0, 0);   // (NaN)
    if constexpr (std::is_same<S, E4M3>::value) {
        uint2 w = make_uint2(x.e4m3(0, scale), x.e4m3(1, scale));
        if (scale == 0x1p120f) {   // (256 2^120 would be infinite: codes 0x78 of either sign, and no larger ones, become 240's)
            const auto least = [](unsigned y) {
#pragma unroll
                for (int i = 0; i < 32; i += 8)
                    if ((y >> i & 0x7f) > 0x77) y = (y & ~(0x7fu << i)) | 0x77u << i;
                return y;
            };
            w.x = least(w.x); w.y = least(w.y);
        }
        return w;
    } else {
        // The nearest integer to a product with the rounded reciprocal, in the lower bits of a sum with 1.5 2^23; its remainder, which is exact
        // near a border, says where that was not the quotient's (seldom); doubled against the scale, because half of a scale below 2^-125 is rounded
        constexpr float MAGIC = 12582912.f;
        const float inv = 1.f / scale;
        float f[8], n[8], most = 0.f;
        x.floats(f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] = fmaf(f[i], inv, MAGIC);
            most = fmaxf(most, fabsf(fmaf(MAGIC - n[i], scale, f[i])));
        }
        if (2.f * most >= scale) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float rest = 2.f * fmaf(MAGIC - n[i], scale, f[i]);
                const bool odd = __float_as_uint(n[i]) & 1;
                if (rest > scale || (rest == scale && odd)) n[i] += 1.f;
                else if (rest < -scale || (rest == -scale && odd)) n[i] -= 1.f;
                n[i] = fminf(fmaxf(n[i], MAGIC - 127.f), MAGIC + 127.f);
            }
        }
        unsigned w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned lo = __builtin_amdgcn_perm(__float_as_uint(n[4 * i + 1]), __float_as_uint(n[4 * i]), 0x0c0c0400u);
            const unsigned hi = __builtin_amdgcn_perm(__float_as_uint(n[4 * i + 3]), __float_as_uint(n[4 * i + 2]), 0x0c0c0400u);
            w[i] = lo | hi << 16;
        }
        return make_uint2(w[0], w[1]);
    }
}

// A thread's 8 features: of which item, token and head
template <int D> struct MoveAt {
    int b, h, l, c;
    __device__ __forceinline__ MoveAt(const MoveArgs &a)
    {
        constexpr int TPR = D / 8;
        const int n = blockIdx.y * a.inner, row = blockIdx.x * (NTHREADS / TPR) + threadIdx.x / TPR;
        b = a.by_hk(n);
        l = a.by_inner(row);
        h = n - b * a.Hk + row - l * a.inner;
        c = (threadIdx.x % TPR) * 8;
    }
    template <typename E> __device__ __forceinline__ E *to(const SmTensor &t, long l) const
    {
        return reinterpret_cast<E *>(const_cast<void *>(t.p)) + b * t.b + h * t.h + l * t.l + c;
    }
    __device__ __forceinline__ float *to(const Scales &t, long l) const { return const_cast<float *>(t.p) + b * t.b + h * t.h + l; }
};

template <typename S, typename T, int D> __global__ __launch_bounds__(NTHREADS) void cache_write_kernel(const MoveArgs a)
{
    const MoveAt<D> w(a);
    const long at = (a.start ? a.start[w.b] : 0) + (long)w.l;
    if (w.l >= sm_len(a.len, w.b, a.L) || at < 0 || at >= a.Lc) return;   // (all threads of a row alike)
    const bool values = blockIdx.z;
    Eight<T> x;
    x.load(w.template to<T>(values ? a.v : a.k, w.l));
    const float scale = move_scale<S>(row_largest<D / 8>(x.largest()));
    *reinterpret_cast<uint2 *>(w.template to<unsigned char>(values ? a.vc : a.kc, at)) = move_codes<S>(x, scale);
    if (w.c == 0) *w.to(values ? a.vs : a.ks, at) = scale;
}

template <typename S, typename T, int D> __global__ __launch_bounds__(NTHREADS) void cache_read_kernel(const MoveArgs a)
{
    const MoveAt<D> w(a);
    if (w.l >= a.L) return;
    const bool values = blockIdx.z;
    const long at = (a.start ? a.start[w.b] : 0) + (long)w.l, from = min(max(at, 0L), a.Lc - 1L);   // (loads under a condition are waited for at once)
    const bool on = at >= 0 && at < sm_len(a.len, w.b, a.Lc);
    uint2 x = *reinterpret_cast<const uint2 *>(w.template to<unsigned char>(values ? a.vc : a.kc, from));
    float s = *w.to(values ? a.vs : a.ks, from);
    if (!on) x = make_uint2(0, 0), s = 0.f;
    T *to = w.template to<T>(values ? a.v : a.k, w.l);
    const bf16x8 c = ca_codes<S>(x.x, x.y);
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (float)c[j] * s;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x8 *>(to) = pack8(y);
    else {
        store4<T>(to, y[0], y[1], y[2], y[3]);
        store4<T>(to + 4, y[4], y[5], y[6], y[7]);
    }
}

template <typename S, typename T, int D> int move(bool write, const MoveArgs &a, hipStream_t st)
{
    const long per = NTHREADS / (D / 8);
    const dim3 grid((unsigned)(((long)a.L * a.inner + per - 1) / per), (unsigned)(a.B * a.Hk / a.inner), 2);
    if (write) hipLaunchKernelGGL((cache_write_kernel<S, T, D>), grid, dim3(NTHREADS), 0, st, a);
    else hipLaunchKernelGGL((cache_read_kernel<S, T, D>), grid, dim3(NTHREADS), 0, st, a);
    return hipGetLastError() == hipSuccess ? SKA_OK : SKA_EHIP;
}
template <typename S, typename T> int move(int d, bool write, const MoveArgs &a, hipStream_t st)
{
    return d == 32 ? move<S, T, 32>(write, a, st) : d == 64 ? move<S, T, 64>(write, a, st) : move<S, T, 128>(write, a, st);
}
int move(bool write, const void *K, const ska_strides *k_strides, const void *V, const ska_strides *v_strides, const void *Kc,
         const ska_strides *kc_strides, const float *Ks, const ska_scale_strides *ks_strides, const void *Vc, const ska_strides *vc_strides,
         const float *Vs, const ska_scale_strides *vs_strides, const int *start, const int *len, int B, int Hk, int L, int Lc, int d, int dtype,
         int store, void *stream)
{
    if (B < 1 || Hk < 1 || L < 0 || Lc < 1) return SKA_EINVAL;
    if ((d != 32 && d != 64 && d != 128) || (dtype != SKA_F32 && dtype != SKA_BF16) || !scaled(store)) return SKA_EUNSUPPORTED;
    if (L > 1 << 24 || Lc > 1 << 24 || (long)B * Hk > 65535) return SKA_EUNSUPPORTED;
    MoveArgs a{};
    int rc;
    if ((rc = tensor_of(a.kc, Kc, kc_strides, B, Hk, Lc, d, store, 8, write)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.vc, Vc, vc_strides, B, Hk, Lc, d, store, 8, write)) != SKA_OK) return rc;
    if ((rc = scales_of(a.ks, Ks, ks_strides, B, Hk, Lc, write)) != SKA_OK) return rc;
    if ((rc = scales_of(a.vs, Vs, vs_strides, B, Hk, Lc, write)) != SKA_OK) return rc;
    if (L == 0) return SKA_OK;
    if ((rc = tensor_of(a.k, K, k_strides, B, Hk, L, d, dtype, 16, !write)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.v, V, v_strides, B, Hk, L, d, dtype, 16, !write)) != SKA_OK) return rc;
    a.start = start; a.len = len;
    a.B = B; a.Hk = Hk; a.L = L; a.Lc = Lc;
    a.by_hk = SmDiv::by(Hk);
    a.inner = Hk > 1 && a.k.h == d && (long)L * Hk * (d / 8) < 1L << 31 ? Hk : 1;   // (fewer than 2^32 threads in a dimension)
    a.by_inner = SmDiv::by(a.inner);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (store == SKA_E4M3) return dtype == SKA_F32 ? move<E4M3, float>(d, write, a, st) : move<E4M3, __bf16>(d, write, a, st);
    return dtype == SKA_F32 ? move<INT8, float>(d, write, a, st) : move<INT8, __bf16>(d, write, a, st);
}

// ------------------------------------------------------------------ attention
int check(const CaProblem &p, bool prefix, CaPlan &l)
{
    if (p.B < 1 || p.Hq < 1 || p.Hk < 1 || p.Lq < 1 || p.Lk < 1 || p.W < 0 || p.Hq % p.Hk || (prefix && p.Lp < 1)) return SKA_EINVAL;
    if (p.d != 32 && p.d != 64 && p.d != 128) return SKA_EUNSUPPORTED;
    if (p.dtype != SKA_F32 && p.dtype != SKA_BF16) return SKA_EUNSUPPORTED;
    if (!scaled(p.store) && !(prefix && p.store == p.dtype)) return SKA_EUNSUPPORTED;
    if (p.Lq > 1 << 24 || p.Lk > 1 << 24 || p.Lp > 1 << 24 || (long)p.B * p.Hk > 65535 || p.R() > 1 << 27) return SKA_EUNSUPPORTED;
    if (prefix && p.R() * p.B > 1 << 27) return SKA_EUNSUPPORTED;
    l = ca_plan(p);
    return l.fits() ? SKA_OK : SKA_EUNSUPPORTED;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
size_t ws_lse(const CaProblem &p, int parts) { return up256((size_t)parts * p.rows() * sizeof(float)); }
size_t ws_bytes(const CaProblem &p, int parts) { return parts > 1 ? ws_lse(p, parts) + (size_t)parts * p.rows() * p.d * sizeof(float) : 0; }
size_t ws_need(const CaProblem &p, bool prefix)
{
    CaPlan l;
    return check(p, prefix, l) == SKA_OK ? ws_bytes(p, l.parts) : 0;
}

struct CaKept {   // keys and values of one side as a caller gives them
    const void *K; const ska_strides *ks; const float *Ks; const ska_scale_strides *kss;
    const void *V; const ska_strides *vs; const float *Vs; const ska_scale_strides *vss;
};
int side_of(CaSide &s, const CaKept &c, int B, int Hk, int L, int d, int store)
{
    int rc;
    if ((rc = tensor_of(s.k, c.K, c.ks, B, Hk, L, d, store, 16, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(s.v, c.V, c.vs, B, Hk, L, d, store, 16, false)) != SKA_OK) return rc;
    s.L = L;
    if (!scaled(store)) return c.Ks || c.Vs ? SKA_EINVAL : SKA_OK;
    Scales k, v;
    if ((rc = scales_of(k, c.Ks, c.kss, B, Hk, L, false)) != SKA_OK) return rc;
    if ((rc = scales_of(v, c.Vs, c.vss, B, Hk, L, false)) != SKA_OK) return rc;
    s.ks = k.p; s.ks_b = k.b; s.ks_h = k.h;
    s.vs = v.p; s.vs_b = v.b; s.vs_h = v.h;
    return SKA_OK;
}
void place(CaSide &s, const CaProblem &p, const CaGrid &g, bool prefix)
{
    s.rows = (int)(prefix ? p.R() * p.B : p.R());
    s.problems = prefix ? p.Hk : p.B * p.Hk;
    s.blocks = (int)g.blocks;
    s.parts = g.parts;
    s.order = g.order;
    s.units = (int)(g.units * g.parts);
    s.wgs = (s.units + 7) / 8 * 8;
    s.by_problems = SmDiv::by(s.problems);
    s.by_blocks = SmDiv::by(s.blocks);
    s.by_parts = SmDiv::by(s.parts);
    s.by_span = SmDiv::by(s.parts * CA_WAVES);
}
typedef int (*Launch)(int, bool, const void *, hipStream_t);
#define BY_D(NAME) {NAME##_32, NAME##_64, NAME##_128}
constexpr Launch LAUNCH[6][3] = {BY_D(ska_launch_cache_f32_f32), BY_D(ska_launch_cache_bf16_bf16), BY_D(ska_launch_cache_e4m3_f32),
                                 BY_D(ska_launch_cache_e4m3_bf16), BY_D(ska_launch_cache_int8_f32), BY_D(ska_launch_cache_int8_bf16)};

int attn(const CaProblem &p, const void *Q, const ska_strides *q_strides, const CaKept *prefix, const CaKept &own, void *O, const ska_strides *o_strides,
         float *LSE, const int *len_p, const int *start_q, const int *len_q, const int *len_k, const unsigned char *mask_q,
         const unsigned char *mask_k, const unsigned char *mask_p, float eps, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!LSE || !(eps > 0.f && isfinite(eps))) return SKA_EINVAL;
    CaPlan l;
    int rc = check(p, prefix != nullptr, l);
    if (rc != SKA_OK) return rc;
    CaArgs a{};
    const float cs = 1.f / (eps * sqrtf((float)p.d));
    a.c2 = cs * LOG2E;
    if (!isnormal(cs) || !isnormal(a.c2)) return SKA_EUNSUPPORTED;   // (at 0 a masked score would be 0 times -inf)
    if ((rc = tensor_of(a.q, Q, q_strides, p.B, p.Hq, p.Lq, p.d, p.dtype, 16, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.o, O, o_strides, p.B, p.Hq, p.Lq, p.d, p.dtype, 16, true)) != SKA_OK) return rc;
    if ((rc = side_of(a.side[0], own, p.B, p.Hk, p.Lk, p.d, p.store)) != SKA_OK) return rc;
    if (prefix) {
        CaKept one = *prefix;   // (its strides between items say nothing)
        ska_strides k, v;
        ska_scale_strides ks, vs;
        if (one.ks) k = *one.ks, k.b = 0, one.ks = &k;
        if (one.vs) v = *one.vs, v.b = 0, one.vs = &v;
        if (one.kss) ks = *one.kss, ks.b = 0, one.kss = &ks;
        if (one.vss) vs = *one.vss, vs.b = 0, one.vss = &vs;
        if ((rc = side_of(a.side[1], one, 1, p.Hk, p.Lp, p.d, p.store)) != SKA_OK) return rc;
    }
    a.parts = l.parts;
    const size_t need = ws_bytes(p, l.parts);
    if (need && (!workspace || workspace_bytes < need)) return SKA_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return SKA_EINVAL;
    a.part_lse = static_cast<float *>(workspace);
    a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + ws_lse(p, a.parts));
    a.lse = LSE;
    a.start = start_q; a.len_q = len_q; a.mask_q = mask_q;
    a.side[0].len = len_k; a.side[0].mask = mask_k;
    a.side[1].len = len_p; a.side[1].mask = mask_p;
    a.B = p.B; a.Hk = p.Hk; a.G = p.G(); a.Lq = p.Lq; a.causal = p.causal;
    a.W = std::min(p.W, 1 << 27);   // (positions are below 2^26: this reaches everything, and sums with it stay in 32 bits)
    a.by_g = SmDiv::by(a.G);
    a.by_hk = SmDiv::by(a.Hk);
    a.by_r = SmDiv::by((unsigned)p.R());
    place(a.side[0], p, l.own, false);
    if (l.front.units) place(a.side[1], p, l.front, true);
    const int at = p.store == SKA_F32 ? 0 : p.store == SKA_BF16 ? 1 : (p.store == SKA_E4M3 ? 2 : 4) + (p.dtype == SKA_BF16);
    return LAUNCH[at][p.d == 32 ? 0 : p.d == 64 ? 1 : 2](l.nq, l.both, &a, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

int ska_cache_write(const void *K, const ska_strides *k_strides, const void *V, const ska_strides *v_strides, void *Kc, const ska_strides *kc_strides,
                    float *Ks, const ska_scale_strides *ks_strides, void *Vc, const ska_strides *vc_strides, float *Vs,
                    const ska_scale_strides *vs_strides, const int *start, const int *len_new, int B, int Hk, int L, int Lc, int d, int dtype, int store,
                    void *stream)
{
    return move(true, K, k_strides, V, v_strides, Kc, kc_strides, Ks, ks_strides, Vc, vc_strides, Vs, vs_strides, start, len_new, B, Hk, L, Lc, d, dtype,
                store, stream);
}

int ska_cache_read(const void *Kc, const ska_strides *kc_strides, const float *Ks, const ska_scale_strides *ks_strides, const void *Vc,
                   const ska_strides *vc_strides, const float *Vs, const ska_scale_strides *vs_strides, void *K, const ska_strides *k_strides, void *V,
                   const ska_strides *v_strides, const int *start, const int *len_k, int B, int Hk, int L, int Lc, int d, int dtype, int store, void *stream)
{
    return move(false, K, k_strides, V, v_strides, Kc, kc_strides, Ks, ks_strides, Vc, vc_strides, Vs, vs_strides, start, len_k, B, Hk, L, Lc, d, dtype,
                store, stream);
}

size_t ska_cache_attn_workspace_bytes(int B, int Hq, int Hk, int Lq, int Lc, int d, int W, int causal, int dtype, int store)
{
    const CaProblem p{B, Hq, Hk, Lq, 0, Lc, d, W, causal, dtype, store};
    return ws_need(p, false);
}

int ska_cache_attn_fwd(const void *Q, const ska_strides *q_strides, const void *Kc, const ska_strides *kc_strides, const float *Ks,
                       const ska_scale_strides *ks_strides, const void *Vc, const ska_strides *vc_strides, const float *Vs,
                       const ska_scale_strides *vs_strides, void *O, const ska_strides *o_strides, float *LSE, const int *start_q, const int *len_q,
                       const int *len_k, const unsigned char *mask_q, const unsigned char *mask_k, int B, int Hq, int Hk, int Lq, int Lc, int d, int W,
                       int causal, float eps, int dtype, int store, void *workspace, size_t workspace_bytes, void *stream)
{
    const CaProblem p{B, Hq, Hk, Lq, 0, Lc, d, W, causal, dtype, store};
    return attn(p, Q, q_strides, nullptr, {Kc, kc_strides, Ks, ks_strides, Vc, vc_strides, Vs, vs_strides}, O, o_strides, LSE, nullptr, start_q, len_q,
                len_k, mask_q, mask_k, nullptr, eps, workspace, workspace_bytes, stream);
}

size_t ska_prefix_attn_workspace_bytes(int B, int Hq, int Hk, int Lq, int Lp, int Lk, int d, int W, int causal, int dtype, int store)
{
    const CaProblem p{B, Hq, Hk, Lq, Lp, Lk, d, W, causal, dtype, store};
    return ws_need(p, true);
}

int ska_prefix_attn_fwd(const void *Q, const ska_strides *q_strides, const void *Kp, const ska_strides *kp_strides, const float *Kps,
                        const ska_scale_strides *kps_strides, const void *Vp, const ska_strides *vp_strides, const float *Vps,
                        const ska_scale_strides *vps_strides, const void *K, const ska_strides *k_strides, const float *Ks,
                        const ska_scale_strides *ks_strides, const void *V, const ska_strides *v_strides, const float *Vs,
                        const ska_scale_strides *vs_strides, void *O, const ska_strides *o_strides, float *LSE, const int *len_p, const int *start_q,
                        const int *len_q, const int *len_k, const unsigned char *mask_q, const unsigned char *mask_k, const unsigned char *mask_p, int B,
                        int Hq, int Hk, int Lq, int Lp, int Lk, int d, int W, int causal, float eps, int dtype, int store, void *workspace,
                        size_t workspace_bytes, void *stream)
{
    const CaProblem p{B, Hq, Hk, Lq, Lp, Lk, d, W, causal, dtype, store};
    const CaKept prefix{Kp, kp_strides, Kps, kps_strides, Vp, vp_strides, Vps, vps_strides};
    return attn(p, Q, q_strides, &prefix, {K, k_strides, Ks, ks_strides, V, v_strides, Vs, vs_strides}, O, o_strides, LSE, len_p, start_q, len_q, len_k,
                mask_q, mask_k, mask_p, eps, workspace, workspace_bytes, stream);
}

}  // extern "C"
