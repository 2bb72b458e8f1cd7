// Rotary positions of queries and keys, forward and gradient, in one launch (several beyond 2^32 threads; sinkhorn_attn_layer.h).
//
//   (x1, x2) -> a (x1 cos t - x2 sin t, x2 cos t + x1 sin t),  t = position * freq[k]; the gradient is the same with -t.
// Bound by memory: each feature is read and written once (MI355X: queries and keys of 2 heads, L = 262144, d = 64, bf16, 52 us on
// tensors that no cache holds, 5.1 TB/s, 40 on the same ones again; with one head's pieces asked for at a time 60 and 44).  Single
// pairs and features, where 16 bytes do not fit, take a load and a store each: 4 + 4 heads, L = 100000, d = 64, 18 features turned,
// bf16, 90 us, 2.3 TB/s (with 32 turned, in pieces, 32 us); fp32, L = 92311, d = 128, 34 turned, 175 us, 4.3 TB/s.
// A thread owns one slot of a token (16 bytes of each half, or 16 bytes of adjacent pairs, or 16 bytes that are copied) and
// takes it through several heads, so that an angle's cosine and sine, which cost about 40 instructions a pair, are found once
// for them.  Far positions make angles of 10^5 radians and more, of which fp32 holds two decimals: the product and its
// reduction to a turn are in 64 bits, the rest in fp32.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sinkhorn_attn_layer.h"

namespace {

constexpr int NT = 256;

struct RopeTensor {
    const void *in;
    void *out;
    long ib, ih, il, ob, oh, ol;   // elements between items, heads, tokens
    int H;
};
struct RopeArgs {
    RopeTensor q, k;
    const double *freq;
    const int *start, *pos;
    float amplitude;
    int back, L, d, rot, slots, heads;   // heads a thread takes, of the q.H + k.H
    int l0, l1;                          // tokens of this launch
};
enum { ROPE_ONE = 0, ROPE_HALVES = 1, ROPE_ADJACENT = 2 };   // a slot: one pair or feature; 16 bytes of either half; 16 bytes of pairs

template <typename T, int FORM, bool INTER> __global__ __launch_bounds__(NT) void rope_kernel(const RopeArgs a)
{
    constexpr int V = FORM == ROPE_ONE ? 1 : 16 / (int)sizeof(T);           // features of a load
    constexpr int PAIRS = FORM == ROPE_ADJACENT ? V / 2 : V;                 // pairs of a slot
    typedef T vec __attribute__((ext_vector_type(V)));
    const int b = blockIdx.z;
    const unsigned at = blockIdx.x * NT + threadIdx.x, token = at / (unsigned)a.slots;
    const int l = a.l0 + (int)token, slot = (int)(at - token * (unsigned)a.slots);
    if (l >= a.l1) return;
    const int npair = a.rot / 2 / PAIRS;                                      // slots that are turned
    const bool turned = slot < npair;
    // features of the slot: at f0 and, where a second piece belongs to it, at f1
    int f0, f1;
    if (!turned) f0 = f1 = a.rot + (slot - npair) * V;
    else if (FORM == ROPE_ADJACENT) f0 = f1 = slot * V;
    else if (INTER) { f0 = 2 * slot; f1 = f0 + 1; }
    else { f0 = slot * V; f1 = f0 + a.rot / 2; }
    // heads BATCH at a time: their pieces are all asked for before the first is stored (an output may be its input, so the
    // compiler cannot do that by itself), those of the first ones before the angles are found
    constexpr int BATCH = 4;
    constexpr bool TWO = FORM != ROPE_ADJACENT;   // a turned slot has a second piece
    const int h0 = blockIdx.y * a.heads, h1 = min(h0 + a.heads, a.q.H + a.k.H);
    vec u[BATCH], v[BATCH];
    T *out[BATCH];
    auto ask = [&](int h) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (h + i >= h1) break;
            const bool isq = h + i < a.q.H;
            const RopeTensor &x = isq ? a.q : a.k;
            const int hh = isq ? h + i : h + i - a.q.H;
            const T *in = reinterpret_cast<const T *>(x.in) + b * x.ib + hh * x.ih + l * x.il;
            out[i] = reinterpret_cast<T *>(x.out) + b * x.ob + hh * x.oh + l * x.ol;
            u[i] = *reinterpret_cast<const vec *>(in + f0);
            if (TWO && turned) v[i] = *reinterpret_cast<const vec *>(in + f1);
        }
    };
    ask(h0);
    float c[PAIRS], s[PAIRS];
    if (turned) {
        // (the sum in 64 bits: it may lie beyond 2^31)
        const double p = a.pos ? (double)a.pos[(long)b * a.L + l] : (double)(a.start ? a.start[b] : 0) + (double)l;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            double turns = p * a.freq[slot * PAIRS + i] * 0.15915494309189535;   // 1 / 2 pi
            turns -= rint(turns);
            sincospif(2.f * (float)turns, &s[i], &c[i]);
            c[i] *= a.amplitude;
            s[i] *= a.back ? -a.amplitude : a.amplitude;
        }
    }
    for (int h = h0; h < h1; h += BATCH) {
        if (h > h0) ask(h);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            if (h + j >= h1) break;
            if (turned) {
                // (which product is rounded is said: every form gives the same bits)
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const float x1 = (float)(TWO ? u[j][i] : u[j][2 * i]), x2 = (float)(TWO ? v[j][i] : u[j][2 * i + 1]);
                    const T y1 = (T)fmaf(x1, c[i], -(x2 * s[i])), y2 = (T)fmaf(x2, c[i], x1 * s[i]);
                    if constexpr (TWO) {
                        u[j][i] = y1;
                        v[j][i] = y2;
                    } else {
                        u[j][2 * i] = y1;
                        u[j][2 * i + 1] = y2;
                    }
                }
            }
            *reinterpret_cast<vec *>(out[j] + f0) = u[j];
            if (TWO && turned) *reinterpret_cast<vec *>(out[j] + f1) = v[j];
        }
    }
}

// ------------------------------------------------------------------ host side
bool strides_of(const ska_strides *s, int B, int H, long L, int d, bool out, long &b, long &h, long &l)
{
    if (!s) {
        l = d; h = L * d; b = h * H;
        return true;
    }
    b = (long)s->b; h = (long)s->h; l = (long)s->l;
    if (b < 0 || h < 0 || l < 0) return false;
    if (B == 1) b = 0;   // (never stepped over, whatever it says)
    if (H == 1) h = 0;
    if (L == 1) l = 0;
    return !out || !((B > 1 && !b) || (H > 1 && !h) || (L > 1 && !l));
}
bool tensor_of(RopeTensor &x, const void *in, const ska_strides *is, void *out, const ska_strides *os, int B, int H, int L, int d)
{
    x.in = in; x.out = out; x.H = H;
    return strides_of(is, B, H, L, d, false, x.ib, x.ih, x.il) && strides_of(os, B, H, L, d, true, x.ob, x.oh, x.ol);
}
bool in_pieces(const RopeTensor &x, size_t e)
{
    if (!x.H) return true;
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.in) | reinterpret_cast<uintptr_t>(x.out);
    const unsigned long s = (unsigned long)(x.ib | x.ih | x.il | x.ob | x.oh | x.ol) * e;
    return !((a | s) & 15);
}

template <typename T> int launch_rope(RopeArgs a, int B, int interleaved, hipStream_t st)
{
    constexpr int V = 16 / (int)sizeof(T);
    const bool pieces = in_pieces(a.q, sizeof(T)) && in_pieces(a.k, sizeof(T)) && a.d % V == 0 && a.rot % (interleaved ? V : 2 * V) == 0;
    a.slots = pieces ? a.rot / (interleaved ? V : 2 * V) + (a.d - a.rot) / V : a.rot / 2 + a.d - a.rot;
    // Heads a thread takes: all of them, unless the tokens alone leave the card's 2^19 threads idle.
    const int H = a.q.H + a.k.H;
    const long threads = (long)B * a.L * a.slots;
    a.heads = H;
    while (a.heads > 1 && threads * ((H + a.heads - 1) / a.heads) < (1 << 19)) a.heads = (a.heads + 1) / 2;
    const long most = (0xffffffffL / NT) * NT / a.slots;   // tokens of a launch, which has fewer than 2^32 threads in a dimension
    for (long l0 = 0; l0 < a.L; l0 += most) {
        a.l0 = (int)l0;
        a.l1 = (int)std::min<long>(a.L, l0 + most);
        const dim3 grid((unsigned)(((long)(a.l1 - a.l0) * a.slots + NT - 1) / NT), (H + a.heads - 1) / a.heads, B);
        if (!pieces) {
            if (interleaved) hipLaunchKernelGGL((rope_kernel<T, ROPE_ONE, true>), grid, dim3(NT), 0, st, a);
            else hipLaunchKernelGGL((rope_kernel<T, ROPE_ONE, false>), grid, dim3(NT), 0, st, a);
        } else if (interleaved) hipLaunchKernelGGL((rope_kernel<T, ROPE_ADJACENT, true>), grid, dim3(NT), 0, st, a);
        else hipLaunchKernelGGL((rope_kernel<T, ROPE_HALVES, false>), grid, dim3(NT), 0, st, a);
        if (hipGetLastError() != hipSuccess) return SKA_EHIP;
    }
    return SKA_OK;
}

int rope(int back, const void *Q, const ska_strides *qs, void *Qr, const ska_strides *qrs, const void *K, const ska_strides *ks, void *Kr,
         const ska_strides *krs, const double *freq, float amplitude, const int *start, const int *positions, int B, int Hq, int Hk,
         int L, int d, int rot, int interleaved, int dtype, void *stream)
{
    if (!freq || (start && positions) || B < 1 || Hq < 1 || Hk < 0 || L < 0 || d < 2 || rot < 2 || rot > d || rot % 2 || !isfinite(amplitude)) return SKA_EINVAL;
    if (L > 0 && (!Q || !Qr || (K != nullptr) != (Hk > 0) || (Kr != nullptr) != (Hk > 0))) return SKA_EINVAL;
    if (d > 4096 || B > 65535 || (long)Hq + Hk > 65535 || L > 1 << 24 || (dtype != SKA_F32 && dtype != SKA_BF16)) return SKA_EUNSUPPORTED;
    RopeArgs a{};
    if (!tensor_of(a.q, Q, qs, Qr, qrs, B, Hq, L, d) || (K && !tensor_of(a.k, K, ks, Kr, krs, B, Hk, L, d))) return SKA_EINVAL;
    if (L == 0) return SKA_OK;
    a.freq = freq; a.start = start; a.pos = positions; a.amplitude = amplitude;
    a.back = back; a.L = L; a.d = d; a.rot = rot;
    return dtype == SKA_F32 ? launch_rope<float>(a, B, interleaved, static_cast<hipStream_t>(stream))
                            : launch_rope<__bf16>(a, B, interleaved, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

int ska_rope_frequencies(int rot, double base, int scaling, double factor, int trained_length, double *freq, double *amplitude)
{
    if (!freq || !amplitude || rot < 2 || rot > 4096 || rot % 2 || !(base > 1.0) || !isfinite(base) || !(factor >= 1.0) || !isfinite(factor)) return SKA_EINVAL;
    if (scaling < SKA_ROPE_PLAIN || scaling > SKA_ROPE_YARN || (scaling == SKA_ROPE_YARN && trained_length < 1)) return SKA_EINVAL;
    // by parts: index of the pair that turns n times within the trained length
    const auto pair_of = [&](double n) { return rot * log(trained_length / (n * 2.0 * M_PI)) / (2.0 * log(base)); };
    double lo = 0, hi = 0;
    if (scaling == SKA_ROPE_YARN) {
        lo = fmax(floor(pair_of(32.0)), 0.0);
        hi = fmin(ceil(pair_of(1.0)), rot - 1.0);
        hi = fmax(hi, lo + 1e-3);
    }
    if (scaling == SKA_ROPE_NTK) base *= pow(factor, rot / (rot > 2 ? rot - 2.0 : 1.0));
    for (int k = 0; k < rot / 2; ++k) {
        double f = pow(base, -2.0 * k / rot);
        if (scaling == SKA_ROPE_LINEAR) f /= factor;
        if (scaling == SKA_ROPE_YARN) {
            const double r = fmin(fmax((k - lo) / (hi - lo), 0.0), 1.0);
            f = f * (1.0 - r) + f / factor * r;
        }
        freq[k] = f;
    }
    *amplitude = scaling == SKA_ROPE_YARN && factor > 1.0 ? 0.1 * log(factor) + 1.0 : 1.0;
    return SKA_OK;
}

int ska_rope_fwd(const void *Q, const ska_strides *q_strides, void *Qr, const ska_strides *qr_strides, const void *K,
                 const ska_strides *k_strides, void *Kr, const ska_strides *kr_strides, const double *freq, float amplitude,
                 const int *start, const int *positions, int B, int Hq, int Hk, int L, int d, int rot, int interleaved, int dtype,
                 void *stream)
{
    return rope(0, Q, q_strides, Qr, qr_strides, K, k_strides, Kr, kr_strides, freq, amplitude, start, positions, B, Hq, Hk, L, d, rot,
                interleaved, dtype, stream);
}

int ska_rope_bwd(const void *dQr, const ska_strides *dqr_strides, void *dQ, const ska_strides *dq_strides, const void *dKr,
                 const ska_strides *dkr_strides, void *dK, const ska_strides *dk_strides, const double *freq, float amplitude,
                 const int *start, const int *positions, int B, int Hq, int Hk, int L, int d, int rot, int interleaved, int dtype,
                 void *stream)
{
    return rope(1, dQr, dqr_strides, dQ, dq_strides, dKr, dkr_strides, dK, dk_strides, freq, amplitude, start, positions, B, Hq, Hk, L,
                d, rot, interleaved, dtype, stream);
}

}  // extern "C"
