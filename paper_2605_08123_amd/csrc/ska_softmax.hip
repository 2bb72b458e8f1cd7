// Softmax attention on a band, forward and gradient: the host side (sinkhorn_attn_layer.h; kernels in ska_softmax.h).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "sinkhorn_attn_layer.h"
#include "ska_softmax_launch.h"

namespace {

struct SmProblem {
    int B, Hq, Hk, Lq, Lk, d, W, causal, dtype;
    int G() const { return Hq / Hk; }
    long R() const { return (long)Lq * G(); }
    long N() const { return (long)B * Hk; }
};
int check(const SmProblem &p, bool backward)
{
    if (p.B < 1 || p.Hq < 1 || p.Hk < 1 || p.Lq < 1 || p.Lk < 1 || p.W < 0 || p.Hq % p.Hk) return SKA_EINVAL;
    if (p.d != 32 && p.d != 64 && p.d != 128) return SKA_EUNSUPPORTED;
    if (p.dtype != SKA_F32 && p.dtype != SKA_BF16) return SKA_EUNSUPPORTED;
    if (p.Lq > 1 << 24 || p.Lk > 1 << 24 || p.N() > 65535 || p.R() > 1 << 27) return SKA_EUNSUPPORTED;
    // Two threads a row in whole workgroups of 128 rows, or four times as many of 32: fewer than 2^32 threads with the grid's
    // rounding up to 8 workgroups (a launch is accepted with more, and runs their number modulo 2^32)
    const long owners = backward ? std::max<long>(p.R(), p.Lk) : p.R();
    if ((owners + 127) / 128 * p.N() > (1 << 24) - 8) return SKA_EUNSUPPORTED;
    return SKA_OK;
}

// How one kernel of a call is launched: wavefronts per workgroup, blocks of owners, parts of a walk
struct SmGrid { int nw; long blocks; int parts; };
// Rows of the walked side that a block of `rows` owners can meet, at most (dK, dV: of one head of the group)
long sm_walk(const SmProblem &p, int what, int rows)
{
    const bool keys = what == SM_DKV;
    const long other = keys ? p.Lq : p.Lk, W = std::min<long>(p.W, other), own = keys ? std::min(rows, p.Lk) : std::min(rows / p.G() + 1, p.Lq);
    return std::min(other, own + W + (p.causal ? 0 : W));
}
SmGrid sm_grid(const SmProblem &p, int what)
{
    SmGrid g{4, 0, 1};
    const long owners = what == SM_DKV ? p.Lk : p.R();
    const long problems = p.N(), alone = (owners + 31) / 32 * problems;   // alone: wavefronts, 32 owners each
    const long other = what == SM_DKV ? p.Lq : p.Lk, heads = what == SM_DKV ? p.G() : 1;   // heads: walks of a block
    const bool band = 2L * p.W + 1 < other / 2, triangle = !band && p.causal && p.Lq > p.Lk / 2;
    // One wavefront per workgroup where there are no more rows, or where workgroups of four would leave CUs without any and share
    // little (a band: two problems of 4 heads, L = 701, W = 64, fp32, forward and backward 12.6 and 30.6 us with four, 10.9 and
    // 25.4 with one; all of 8 heads, L = 2000, d = 128, fp32: 176 and 549 with four, 718 and 1290 with one).
    // Two buffers of a pair of fp32 tiles of d = 128 are 64 KB, two workgroups a CU: single wavefronts only where there are half as
    // many as that (8 heads on 4, L = 2000, W = 306, causal, forward and backward 81 and 184 us with one, 50 and 143 with four;
    // 4 heads, L = 2000, W = 20, causal: 19 and 51, 30 and 66).
    const bool large = what != SM_DKV && p.dtype == SKA_F32 && p.d == 128;
    if (owners <= 32 || ((owners + 127) / 128 * problems < 256 && sm_walk(p, what, 128) * heads <= 512 && !(large && alone > 256))) g.nw = 1;
    // dK, dV of a band in fp32 as well: its products take eight times as long as bf16's, and a wavefront of four sits through the
    // tiles that only the other three reach (backward of 8 heads on 2, d = 64, L = 43748, W = 32: 353 us with one, 496 with four;
    // W = 256: 1474, 1621; bf16, 4 on 2, L = 65536, W = 256: 249, 174).  Not where that makes less than one wavefront per
    // SIMD and more than one per two, since at d = 32 a CU has room for eight and takes them: 8 on 2, L = 14400, W = 256: 391, 311.
    if (what == SM_DKV && band && p.dtype == SKA_F32 && (p.d > 32 || alone <= 512 || alone >= 1024)) g.nw = 1;
    const int rows = 32 * g.nw;
    g.blocks = (owners + rows - 1) / rows;
    // Parts where there are fewer wavefronts than SIMDs, to make it one each, but no fewer than two tiles to a part, since parts
    // have to be joined by another launch (4 heads, L = 512, d = 64, causal, backward: one tile 22.4 us, two 21.0, four 22.7); wide
    // fp32 tiles of few rows take longer than that (4 heads on 1, L = 100, backward: d = 128, one tile 35 us, two 50; d = 64, 22, 29;
    // not of many: 4 heads, L = 3000, W = 60, causal, d = 64: 46, 36).
    const long tile = p.dtype == SKA_BF16 && p.d < 128 ? 64 : 32, tiles = (sm_walk(p, what, rows) + tile - 1) / tile * heads;
    const long waves = g.blocks * problems * g.nw;
    const long room = large && g.nw == 1 ? 512 : 1024;   // (4 heads' 8 tokens on a cache of 16384: 33 us, 38 with 1024)
    const auto parts = [&](long each, long least) { return std::max(1L, std::min({room * each / waves, tiles / least, 256L})); };
    g.parts = (int)parts(1, p.dtype == SKA_F32 && p.d >= 64 && waves <= 128 ? 1 : 2);
    if (triangle) {
        // Where a causal mask makes walks of every length, two each, which also evens them out, and where there are up to two
        // anyhow (8 heads, L = 4096, d = 128, forward and backward 69 and 200 us, without 91 and 262; fp32 347 and 1092, without
        // 604 and 1923); in the forward if a part has 512 keys (fp32: 256; 4 heads, L = 2048, d = 64: 19.9 us with parts of 512,
        // 25.0 with 256; fp32 43.7 with 256, 49.6 with 512).
        g.parts = std::max(g.parts, (int)parts(2, what != SM_FWD ? 2 : p.dtype == SKA_F32 ? 8 : 512 / tile));
    } else if (!band) {
        // Two each if that takes less by this count: tiles of a part one after the other, and its start, end and joining, about
        // four tiles' time (fp32: one); two wavefronts of a SIMD take twice as long, or 1.8 times in bf16 at d <= 64, where they
        // fill each other's waits.  Backward, all of it: 16 heads on 4, L = 4096, d = 64, 264 us with two, 298 with one; 8 heads,
        // L = 1400, d = 128, fp32, 331, 370; 8 heads, L = 2048, d = 128, 117, 104; 4 heads, L = 2048, d = 64, 55, 50.  Forward: 6
        // heads on 2, L = 3270, d = 128, 57, 74; four sequences' 64 tokens on caches of 40000, 4 heads, d = 64, 36, 44.
        const auto time = [&](long n) {
            const long each = (waves * n + room - 1) / room, start = p.dtype == SKA_F32 ? 1 : 4;
            return (each == 2 && p.dtype == SKA_BF16 && p.d <= 64 ? 18 : 10 * each) * ((tiles + n - 1) / n + start);
        };
        const long two = parts(2, 2);
        if (time(two) < time(g.parts)) g.parts = (int)two;
    }
    // (joining takes longer than a few tiles where there are many rows: 8 heads' gradient of one query on 2 heads' 8192 keys, d = 128,
    // 27 us, 39 in two parts of two tiles)
    if (p.dtype == SKA_BF16 && tiles < 8 && waves > 128) g.parts = 1;
    const long per = std::max(1L, (tiles + g.parts - 1) / g.parts);
    g.parts = (int)std::max(1L, (tiles + per - 1) / per);   // (none that would be empty)
    return g;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
size_t delta_bytes(const SmProblem &p) { return up256((size_t)p.N() * p.R() * sizeof(float)); }
size_t part_lse_bytes(const SmProblem &p, const SmGrid &g) { return g.parts > 1 ? up256((size_t)g.parts * p.N() * p.R() * sizeof(float)) : 0; }
size_t ws_fwd(const SmProblem &p)
{
    const SmGrid g = sm_grid(p, SM_FWD);
    return g.parts > 1 ? part_lse_bytes(p, g) + (size_t)g.parts * p.N() * p.R() * p.d * sizeof(float) : 0;
}
size_t ws_bwd(const SmProblem &p)
{
    const SmGrid r = sm_grid(p, SM_DQ), k = sm_grid(p, SM_DKV);
    const size_t pr = r.parts > 1 ? (size_t)r.parts * p.N() * p.R() * p.d : 0, pk = k.parts > 1 ? (size_t)k.parts * p.N() * p.Lk * 2 * p.d : 0;
    return 2 * delta_bytes(p) + std::max(pr, pk) * sizeof(float);   // (one after the other)
}

// strides in bytes multiples of 16; SKA_EINVAL where they cannot be strides, SKA_EUNSUPPORTED where the kernels cannot use them
int tensor_of(SmTensor &t, const void *p, const ska_strides *s, int B, int H, long L, int d, int dtype, bool out)
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
    const long e = dtype == SKA_F32 ? 4 : 2;
    if (t.l * e >= 1L << 27) return SKA_EUNSUPPORTED;   // (rows of a load instruction, 16 at most, lie within 32 bits)
    const unsigned long off = (unsigned long)reinterpret_cast<uintptr_t>(p) | (unsigned long)((t.b | t.h | t.l) * e);
    return off & 15 ? SKA_EUNSUPPORTED : SKA_OK;
}

int launch(int what, const SmProblem &p, const SmGrid &g, SmArgs a, hipStream_t st)
{
    a.parts = g.parts;
    a.blocks = (int)g.blocks;
    a.total = (int)(g.blocks * g.parts * p.N());   // (check: below 2^26; parts only where there are few)
    a.by_g = SmDiv::by(a.G);
    a.by_hk = SmDiv::by(a.Hk);
    a.by_n = SmDiv::by(a.B * a.Hk);
    a.by_parts = SmDiv::by(a.parts);
    a.by_blocks = SmDiv::by(a.blocks * a.parts);
    const long other = what == SM_DKV ? p.Lq : p.Lk;
    a.order = 2L * p.W + 1 < other / 2 ? SM_NEIGHBOURS : what == SM_DKV && p.causal ? SM_FIRST_FIRST : SM_LAST_FIRST;
    const auto f = p.dtype == SKA_F32 ? (p.d == 32 ? ska_launch_softmax_f32_32 : p.d == 64 ? ska_launch_softmax_f32_64 : ska_launch_softmax_f32_128)
                                      : (p.d == 32 ? ska_launch_softmax_bf16_32 : p.d == 64 ? ska_launch_softmax_bf16_64 : ska_launch_softmax_bf16_128);
    return f(what, g.nw, &a, st);
}

SmArgs args_of(const SmProblem &p, float eps, float *lse, const int *start_q, const int *len_q, const int *len_k, const unsigned char *mask_q,
               const unsigned char *mask_k)
{
    SmArgs a{};
    a.lse = lse;
    a.start = start_q; a.len_q = len_q; a.len_k = len_k; a.mask_q = mask_q; a.mask_k = mask_k;
    a.B = p.B; a.Hk = p.Hk; a.G = p.G(); a.Lq = p.Lq; a.Lk = p.Lk; a.causal = p.causal;
    a.W = std::min(p.W, 1 << 26);   // (positions are below 2^25: this reaches everything, and sums with it stay in 32 bits)
    a.cs = 1.f / (eps * sqrtf((float)p.d));
    a.c2 = a.cs * LOG2E;
    return a;
}
bool eps_ok(float eps) { return eps > 0.f && isfinite(eps); }
// the scores' factor: at 0 a masked score would be 0 times -inf, at infinity an ordinary one 0 times that
bool scale_ok(const SmArgs &a) { return isnormal(a.cs) && isnormal(a.c2); }

}  // namespace

extern "C" {

size_t ska_softmax_attn_workspace_bytes(int backward, int B, int Hq, int Hk, int Lq, int Lk, int d, int W, int causal, int dtype)
{
    const SmProblem p{B, Hq, Hk, Lq, Lk, d, W, causal, dtype};
    if (check(p, backward) != SKA_OK) return 0;
    return backward ? ws_bwd(p) : ws_fwd(p);
}

int ska_softmax_attn_fwd(const void *Q, const ska_strides *q_strides, const void *K, const ska_strides *k_strides, const void *V,
                         const ska_strides *v_strides, void *O, const ska_strides *o_strides, float *LSE, const int *start_q,
                         const int *len_q, const int *len_k, const unsigned char *mask_q, const unsigned char *mask_k, int B, int Hq,
                         int Hk, int Lq, int Lk, int d, int W, int causal, float eps, int dtype, void *workspace, size_t workspace_bytes,
                         void *stream)
{
    const SmProblem p{B, Hq, Hk, Lq, Lk, d, W, causal, dtype};
    if (!LSE || !eps_ok(eps)) return SKA_EINVAL;
    int rc = check(p, false);
    if (rc != SKA_OK) return rc;
    SmArgs a = args_of(p, eps, LSE, start_q, len_q, len_k, mask_q, mask_k);
    if (!scale_ok(a)) return SKA_EUNSUPPORTED;
    if ((rc = tensor_of(a.q, Q, q_strides, B, Hq, Lq, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.k, K, k_strides, B, Hk, Lk, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.v, V, v_strides, B, Hk, Lk, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.oq, O, o_strides, B, Hq, Lq, d, dtype, true)) != SKA_OK) return rc;
    const size_t need = ws_fwd(p);
    if (need && (!workspace || workspace_bytes < need)) return SKA_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return SKA_EINVAL;
    const SmGrid g = sm_grid(p, SM_FWD);
    a.part_lse = static_cast<float *>(workspace);
    a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + part_lse_bytes(p, g));
    return launch(SM_FWD, p, g, a, static_cast<hipStream_t>(stream));
}

int ska_softmax_attn_bwd(const void *Q, const ska_strides *q_strides, const void *K, const ska_strides *k_strides, const void *V,
                         const ska_strides *v_strides, const void *O, const ska_strides *o_strides, const void *dO,
                         const ska_strides *do_strides, const float *LSE, void *dQ, const ska_strides *dq_strides, void *dK,
                         const ska_strides *dk_strides, void *dV, const ska_strides *dv_strides, const int *start_q, const int *len_q,
                         const int *len_k, const unsigned char *mask_q, const unsigned char *mask_k, int B, int Hq, int Hk, int Lq,
                         int Lk, int d, int W, int causal, float eps, int dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    const SmProblem p{B, Hq, Hk, Lq, Lk, d, W, causal, dtype};
    if (!LSE || !eps_ok(eps)) return SKA_EINVAL;
    int rc = check(p, true);
    if (rc != SKA_OK) return rc;
    SmArgs a = args_of(p, eps, const_cast<float *>(LSE), start_q, len_q, len_k, mask_q, mask_k);
    if (!scale_ok(a)) return SKA_EUNSUPPORTED;
    if ((rc = tensor_of(a.q, Q, q_strides, B, Hq, Lq, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.k, K, k_strides, B, Hk, Lk, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.v, V, v_strides, B, Hk, Lk, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.o, O, o_strides, B, Hq, Lq, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.g, dO, do_strides, B, Hq, Lq, d, dtype, false)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.oq, dQ, dq_strides, B, Hq, Lq, d, dtype, true)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.ok, dK, dk_strides, B, Hk, Lk, d, dtype, true)) != SKA_OK) return rc;
    if ((rc = tensor_of(a.ov, dV, dv_strides, B, Hk, Lk, d, dtype, true)) != SKA_OK) return rc;
    if (!workspace || workspace_bytes < ws_bwd(p)) return SKA_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return SKA_EINVAL;
    a.lse2 = static_cast<float *>(workspace);
    a.delta = a.lse2 + delta_bytes(p) / sizeof(float);
    a.part = a.delta + delta_bytes(p) / sizeof(float);
    hipStream_t st = static_cast<hipStream_t>(stream);
    rc = launch(SM_DQ, p, sm_grid(p, SM_DQ), a, st);   // (writes delta, which dK reads)
    return rc != SKA_OK ? rc : launch(SM_DKV, p, sm_grid(p, SM_DKV), a, st);
}

}  // extern "C"
