/*
 * sinkhorn_attn_cache.h -- C ABI of answering from caches that take fewer bytes: keys and values held in 8 bits (written as
 * they are quantised, read back), softmax attention that reads them, and softmax attention of a batch whose sequences share a
 * prefix, on 8-bit, bf16 and fp32 caches.
 *
 * Conventions are those of sinkhorn_attn_layer.h (ska_strides among them).  For answering: there are no gradients.
 *
 * A cache in 8 bits: codes [B, Hk, Lc, d] by strides, one byte each, and fp32 scales [B, Hk, Lc], one for each token and head,
 * tokens adjacent.  A row of codes c with scale s stands for c s.  Row x is held so, with a = max |x|:
 *   SKA_E4M3  (OCP 8-bit floating point, 4 exponent bits)  s = max(2^ceil(log2(a / 448)), 2^-126), c = the nearest e4m3 number to x / s.
 *             A power of two: no rounding but that of c, half a step of 2^-4 relative (2^-10 s absolute below 2^-6 s).  With
 *             s = 2^120 codes end at 240, so that every value is finite.
 *   SKA_INT8  s = max(a / 127, 2^-126), rounded to fp32 (at most 0x1.020406p+121, so that every value is finite), c = the nearest
 *             integer to x / s, at most 127 in size: within s / 2.
 * Ties go to the even code; the quotient is not rounded before c is.  A row with a NaN or an infinity gets s = NaN and c = 0 and
 * stands for NaN throughout.
 */
#ifndef SINKHORN_ATTN_CACHE_H
#define SINKHORN_ATTN_CACHE_H

#include "sinkhorn_attn_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Further storage types, of caches only (SKA_F32 and SKA_BF16 as everywhere) */
#define SKA_E4M3 2
#define SKA_INT8 3

/* Floats between batch items and heads of the scales; those of a head's tokens lie next to each other.  NULL: contiguous. */
typedef struct { long long b, h; } ska_scale_strides;

/*
 * Quantises L new tokens of each item into its cache: token l < len_new[b] goes to place start[b] + l.
 *   K, V [B,Hk,L,d] of type `dtype` (SKA_F32, SKA_BF16); Kc, Vc [B,Hk,Lc,d] codes of type `store` (SKA_E4M3, SKA_INT8), Ks, Vs
 *   their scales.  All other places of the caches are left as they were, and tokens whose place is not in 0 ... Lc - 1 are not written.
 *   start, len_new: int32 device arrays [B] or NULL (0, L); lengths are clamped to [0, L].
 *   d in {32, 64, 128}; 0 <= L <= 2^24 (0: nothing is read or written, K and V may be NULL), 1 <= Lc <= 2^24, B * Hk <= 65535 (SKA_EUNSUPPORTED otherwise).
 *   Pointers and strides in bytes: of K and V multiples of 16, of Kc and Vc multiples of 8 (SKA_EUNSUPPORTED otherwise).
 */
int ska_cache_write(const void *K, const ska_strides *k_strides, const void *V, const ska_strides *v_strides, void *Kc,
                    const ska_strides *kc_strides, float *Ks, const ska_scale_strides *ks_strides, void *Vc,
                    const ska_strides *vc_strides, float *Vs, const ska_scale_strides *vs_strides, const int *start,
                    const int *len_new, int B, int Hk, int L, int Lc, int d, int dtype, int store, void *stream);

/*
 * The values that places start[b] ... start[b] + L - 1 of a cache stand for, c s in fp32, rounded once to `dtype`; zeros for places
 * that are not in 0 ... len_k[b] - 1, whatever they hold.  K, V [B,Hk,L,d]; what the banded attention or a gradient reads.
 *   start, len_k: int32 device arrays [B] or NULL (0, Lc); lengths are clamped to [0, Lc].  Limits as in ska_cache_write.
 */
int ska_cache_read(const void *Kc, const ska_strides *kc_strides, const float *Ks, const ska_scale_strides *ks_strides,
                   const void *Vc, const ska_strides *vc_strides, const float *Vs, const ska_scale_strides *vs_strides,
                   void *K, const ska_strides *k_strides, void *V, const ska_strides *v_strides, const int *start,
                   const int *len_k, int B, int Hk, int L, int Lc, int d, int dtype, int store, void *stream);

/*
 * Softmax attention (ska_softmax_attn_fwd: band, positions, lengths, masks, rows without a key, NaN) on a cache in 8 bits:
 *   S_ij = <Q_i, c_j> s_j / (eps sqrt d),  LSE_i = log sum_j exp(S_ij),  O_i = sum_j exp(S_ij - LSE_i) s'_j c'_j.
 *   Q, O [B,Hq,Lq,d] of type `dtype`; Kc, Vc [B,Hk,Lc,d] codes of type `store`, Ks, Vs scales; LSE [B,Hq,Lq] fp32.
 *   Codes are exact in bf16 and fp16, products with queries and with probabilities are accumulated in fp32.
 *   fp32 queries are taken as the sum of three bf16 numbers (all their bits), and so is exp(S - LSE) s' (2^-24 relative).
 *   bf16 queries are taken as they are.  exp(S - m), m near the row's largest S, is rounded to fp16 (2^-11 relative; absolute 2^-29
 *   below 2^-18, so that keys with less weight than that add nothing to O).  Values' scales are
 *   fp16 numbers next to a power of two, and their products with it rounded to fp16 again (3 2^-11 in all; absolute 2^-20 of the
 *   value); in 32 tokens with a scale 2^9 times smaller than a value's before, the products are sums of two bf16 numbers (2^-16).
 *   Values 2^100 times smaller than another that is reached may be lost, and so may keys with less than 2^-100 of the largest weight in O.
 *   Values up to 2^127 / (n + 64), n the tokens that a query reaches by position, give finite results: sums over them, not yet divided by those
 *   of exp(S - m), are fp32.
 *   Places of the cache beyond the lengths or inactive may hold anything, and so may those that no query of the item reaches by
 *   position (inactive ones reach as well).  A token that is reached whose value row is not finite is in O of the queries around it too.
 *   Limits, alignment and workspace as ska_softmax_attn_fwd (codes: multiples of 16 bytes); scales on any 4 bytes.  Instead of its
 *   2^24 blocks of 128 rows: fewer than 2^23 - 8 blocks of 64 query rows of a problem (32 on fp32 caches or with d = 128), B Hk problems
 *   of Lq (Hq / Hk) rows (SKA_EUNSUPPORTED otherwise).
 *   The same query can differ by roundings between calls of other sizes; the same call repeats its bits.
 */
size_t ska_cache_attn_workspace_bytes(int B, int Hq, int Hk, int Lq, int Lc, int d, int W, int causal, int dtype, int store);
int ska_cache_attn_fwd(const void *Q, const ska_strides *q_strides, const void *Kc, const ska_strides *kc_strides,
                       const float *Ks, const ska_scale_strides *ks_strides, const void *Vc, const ska_strides *vc_strides,
                       const float *Vs, const ska_scale_strides *vs_strides, void *O, const ska_strides *o_strides,
                       float *LSE, const int *start_q, const int *len_q, const int *len_k, const unsigned char *mask_q,
                       const unsigned char *mask_k, int B, int Hq, int Hk, int Lq, int Lc, int d, int W, int causal,
                       float eps, int dtype, int store, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Softmax attention of a batch behind a prefix that all its items share: the prefix's keys are at positions 0 ... P - 1, key j
 * of item b at P + j, query i at P + start_q[b] + i, P = len_p[0] (int32 on the device, clamped to [0, Lp]) or Lp.  One softmax over
 * both; the prefix is read once for the queries of all items.
 *   Kp, Vp [Hk,Lp,d] (of their strides, h and l count), K, V [B,Hk,Lk,d]: all of type `store`, which is `dtype` (scales NULL) or an
 *   8-bit one (scales Kps, Vps, Ks, Vs).  mask_p [Lp]: uint8, nonzero = active, or NULL.  The other arguments as above.
 *   Places of the prefix beyond P or inactive may hold anything, and so may those that no query of any item reaches by position.
 *   fp32 caches: products in fp32.  bf16: exp(S - m) as the sum of two bf16 numbers (2^-16), from which the row's sum is taken too.  Codes: as above.
 *   1 <= Lp, Lk <= 2^24 (an item without tokens of its own: len_k 0), B * Lq * (Hq / Hk) <= 2^27; the prefix's blocks, of Hk
 *   problems of B Lq (Hq / Hk) rows, count with the items' own (SKA_EUNSUPPORTED otherwise).
 */
size_t ska_prefix_attn_workspace_bytes(int B, int Hq, int Hk, int Lq, int Lp, int Lk, int d, int W, int causal, int dtype,
                                       int store);
int ska_prefix_attn_fwd(const void *Q, const ska_strides *q_strides, const void *Kp, const ska_strides *kp_strides,
                        const float *Kps, const ska_scale_strides *kps_strides, const void *Vp,
                        const ska_strides *vp_strides, const float *Vps, const ska_scale_strides *vps_strides, const void *K,
                        const ska_strides *k_strides, const float *Ks, const ska_scale_strides *ks_strides, const void *V,
                        const ska_strides *v_strides, const float *Vs, const ska_scale_strides *vs_strides, void *O,
                        const ska_strides *o_strides, float *LSE, const int *len_p, const int *start_q, const int *len_q,
                        const int *len_k, const unsigned char *mask_q, const unsigned char *mask_k,
                        const unsigned char *mask_p, int B, int Hq, int Hk, int Lq, int Lp, int Lk, int d, int W, int causal,
                        float eps, int dtype, int store, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SINKHORN_ATTN_CACHE_H */
