/*
 * sinkhorn_attn_layer.h -- C ABI of the operators of an attention layer around the banded Sinkhorn attention: layer norm
 * with its gradient, rotary positions with their gradient, and softmax attention on the same band with its gradient (the
 * ordinary attention that the Sinkhorn operator stands in for, as its comparator in training and for answering).
 *
 * Conventions are those of sinkhorn_attn.h: device pointers owned by the caller, work enqueued on `stream`, asynchronous,
 * nothing allocated, freed or kept; arguments are checked before anything is launched; SKA_OK or a negative ska_status.
 * All kernels of a call run on `stream` itself; the calls take no lock and may be captured into a graph (they record
 * kernels only).  Results are the same bits from call to call.  Sums, statistics and softmax run in fp32; what is rounded to fewer
 * bits on the way is said below.
 */
#ifndef SINKHORN_ATTN_LAYER_H
#define SINKHORN_ATTN_LAYER_H

#include <stddef.h>

#include "sinkhorn_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Elements between batch items, heads and tokens of a [B, H, L, d] tensor; the d features of a token lie next to each
 * other.  A NULL strides argument means a contiguous tensor.  No stride may be negative, and none of an output zero
 * where its dimension has more than one entry (inputs may be broadcast).
 */
typedef struct { long long b, h, l; } ska_strides;

/*
 * Layer norm of N rows of D features, optionally of the sum with a residual:
 *   S = X + R (rounded to the storage type; X itself without R),  mean and variance of S's rows,
 *   Y = (S - mean) rstd weight + bias,  rstd = 1 / sqrt(variance + ln_eps)
 *   X, R, S, Y: rows ldx, ldr, lds, ldy elements apart (>= 0 for inputs, >= D for outputs where N > 1), of type `dtype`.
 *   R and S: both or neither (NULL).  S may be X or R, and Y may be X or R, with the same rows.
 *   weight, bias: [D] of type `wdtype`; NULL: ones, zeros.
 *   stats: [2][N] fp32, the means and the rstds, as the backward needs them; NULL: not wanted.
 *   0 <= N <= 2^31 - 1 (0: nothing is read or written, the rows' pointers may be NULL), 1 <= D <= 65536, ln_eps >= 0 and finite.
 * Any alignment of the elements: rows are read and written in pieces of 16 bytes from their first feature on.
 */
int ska_layer_norm_fwd(const void *X, long long ldx, const void *R, long long ldr, const void *weight,
                       const void *bias, void *S, long long lds, void *Y, long long ldy, float *stats,
                       long long N, int D, float ln_eps, int dtype, int wdtype, void *stream);

/*
 * Its gradient: with h = (S - mean) rstd and g = dY weight (rows),
 *   dX = rstd (g - mean(g) - h mean(g h)) + dS,   dweight = sum over rows of dY h,   dbias = sum over rows of dY.
 *   S, stats: of the forward.  dS: the gradient that reaches S on the residual's way, or NULL.  dX is the gradient of both
 *   X and R, and may be dY or dS.
 *   dweight, dbias: [D] of type `wdtype`, NULL: not wanted.  Overwritten (zeros for N = 0).
 *   workspace: ska_layer_norm_workspace_bytes(N, D) bytes, 16-byte aligned; not needed without dweight and dbias.
 * The sums over rows are taken in a fixed order.
 */
size_t ska_layer_norm_workspace_bytes(long long N, int D);
int ska_layer_norm_bwd(const void *dY, long long lddy, const void *S, long long lds, const void *weight,
                       const float *stats, const void *dS, long long ldds, void *dX, long long lddx, void *dweight,
                       void *dbias, long long N, int D, int dtype, int wdtype, void *workspace,
                       size_t workspace_bytes, void *stream);

/*
 * Frequencies of rotary positions, on the HOST: freq[k], k < rot / 2, radians per position of pair k, and the amplitude
 * that turned features are multiplied by.
 *   SKA_ROPE_PLAIN   base^(-2k / rot)
 *   SKA_ROPE_LINEAR  the same divided by `factor` (positions interpolated)
 *   SKA_ROPE_NTK     base' = base factor^(rot / (rot - 2)): the slowest pair by the factor, the fastest not at all
 *   SKA_ROPE_YARN    by parts: pairs that turn at least 32 times within trained_length stay, those that turn less than once
 *                    are divided by the factor, a linear ramp over the pair's index in between (its ends rounded outwards
 *                    to whole indices); amplitude 0.1 ln(factor) + 1
 * rot even, 2 <= rot <= 4096; base > 1; factor >= 1; trained_length >= 1 (read for SKA_ROPE_YARN only).
 */
#define SKA_ROPE_PLAIN 0
#define SKA_ROPE_LINEAR 1
#define SKA_ROPE_NTK 2
#define SKA_ROPE_YARN 3
int ska_rope_frequencies(int rot, double base, int scaling, double factor, int trained_length, double *freq,
                         double *amplitude);

/*
 * Rotary positions of queries and keys in one launch: the first `rot` features of a token at position p are turned in
 * pairs by p freq[k],
 *   (x1, x2) -> amplitude (x1 cos - x2 sin, x2 cos + x1 sin),
 * pair k being features (k, k + rot/2), or (2k, 2k + 1) where `interleaved` is not 0; the others are copied.
 *   Q [B,Hq,L,d] -> Qr, K [B,Hk,L,d] -> Kr; K and Kr may be NULL (with Hk = 0).  An output may be its input (same strides).
 *   freq: [rot/2] float64 device array.  Angles are formed and reduced in 64 bits, cosine and sine in fp32.
 *   position of token l of item b: positions[b][l] ([B,L] int32), start[b] + l ([B] int32), or l; device arrays, at most one.
 *   2 <= rot <= d <= 4096, rot even; 0 <= L <= 2^24 (0: nothing is read or written, the tensors may be NULL), B <= 65535, Hq + Hk <= 65535.
 * ska_rope_bwd takes the gradients of Qr, Kr to those of Q, K: the transposed map (the angle's sign changed, the same
 * amplitude).
 * 16-byte pieces where pointers, strides, d and the halves of the turned part allow it, single features otherwise.
 */
int ska_rope_fwd(const void *Q, const ska_strides *q_strides, void *Qr, const ska_strides *qr_strides, const void *K,
                 const ska_strides *k_strides, void *Kr, const ska_strides *kr_strides, const double *freq,
                 float amplitude, const int *start, const int *positions, int B, int Hq, int Hk, int L, int d, int rot,
                 int interleaved, int dtype, void *stream);
int ska_rope_bwd(const void *dQr, const ska_strides *dqr_strides, void *dQ, const ska_strides *dq_strides,
                 const void *dKr, const ska_strides *dkr_strides, void *dK, const ska_strides *dk_strides,
                 const double *freq, float amplitude, const int *start, const int *positions, int B, int Hq, int Hk,
                 int L, int d, int rot, int interleaved, int dtype, void *stream);

/*
 * Softmax attention on a band.  Query i of item b stands at position p = start_q[b] + i, key j at position j; they form a
 * pair where |p - j| <= W, j <= p if `causal`, i < len_q[b], j < len_k[b], and mask_q[b][i], mask_k[b][j] are not 0.
 *   S_ij = <Q_i, K_j> / (eps sqrt d),  LSE_i = log sum_j exp(S_ij),  O_i = sum_j exp(S_ij - LSE_i) V_j  over the pairs.
 * A query without any key has O_i = 0 and LSE_i = -inf, and its gradients are zeros.
 * NaN goes on: a query that meets one, in itself or in a key of its pairs, or a score of +inf, or that has keys but scores of -inf
 * alone, has NaN in O_i and LSE_i, and so have the gradients of its pairs.  One in a value is in O_i, and in dQ and dK of its pairs.
 *   Q, O [B,Hq,Lq,d]; K, V [B,Hk,Lk,d]; Hq a multiple of Hk: query head h reads key head h / (Hq / Hk).
 *   LSE [B,Hq,Lq] fp32.
 *   start_q, len_q, len_k: int32 device arrays [B] or NULL (0, Lq, Lk); starts are clamped to [0, 2^24], lengths to
 *   [0, Lq], [0, Lk].  mask_q [B,Lq], mask_k [B,Lk]: uint8 device arrays, nonzero = active, or NULL.
 *   Rows of inactive tokens and beyond the lengths may hold anything, and so may keys that no query, and queries that no key,
 *   of their item reaches by position (|p - j| <= W, j <= p if `causal`, within the lengths; inactive ones reach as well).  An
 *   active token that is reached must be finite to leave the item's others alone: products with a probability of 0 are formed.
 *   W >= 0 (W >= max(Lq, Lk) with starts of 0 is the dense problem); eps > 0 and finite, and 1 / (eps sqrt d) a
 *   normal fp32 number, log2(e) times which is finite (SKA_EUNSUPPORTED otherwise).  Scores are formed in fp32.
 *   d in {32, 64, 128}; 1 <= Lq, Lk <= 2^24; B * Hk <= 65535, Lq * (Hq / Hk) <= 2^27, and at most 2^24 - 8 blocks of
 *   128 rows: B * Hk times Lq * (Hq / Hk) rows, in the gradient also times Lk (SKA_EUNSUPPORTED otherwise).
 *   Pointers and strides in bytes: multiples of 16, tokens less than 128 MiB apart (SKA_EUNSUPPORTED otherwise).
 *   workspace: ska_softmax_attn_workspace_bytes(...) bytes (may be 0: then NULL is fine), 16-byte aligned; scratch.
 * Few queries on many keys (an answer's next token; W >= Lk for a whole cache) are split over the keys, and the parts joined.
 * bf16: scores, maxima, sums and P are fp32; for the product with V, P is rounded to bf16 (2^-8 relative, half a step), or where
 * the call has few rows taken as the sum of two bf16 parts (2^-16): always with Lq * (Hq / Hk) <= 32, else where that launches
 * workgroups of one wavefront, which depends on B * Hk, Lq, Lk and W.  The same query can therefore differ by roundings of P and
 * by the order of its sums between a batch and a call of its own, or between a token's call and the whole sequence's; the same
 * call repeats its bits.
 */
size_t ska_softmax_attn_workspace_bytes(int backward, int B, int Hq, int Hk, int Lq, int Lk, int d, int W, int causal,
                                        int dtype);
int ska_softmax_attn_fwd(const void *Q, const ska_strides *q_strides, const void *K, const ska_strides *k_strides,
                         const void *V, const ska_strides *v_strides, void *O, const ska_strides *o_strides, float *LSE,
                         const int *start_q, const int *len_q, const int *len_k, const unsigned char *mask_q,
                         const unsigned char *mask_k, int B, int Hq, int Hk, int Lq, int Lk, int d, int W, int causal,
                         float eps, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its gradient, from recomputed probabilities P = exp(S - LSE):
 *   delta_i = <dO_i, O_i>,  dS = P (dO V^T - delta),  dV = P^T dO,  dQ = dS K / (eps sqrt d),  dK = dS^T Q / (eps sqrt d),
 * dK and dV summed over the query heads that share a key head, in a fixed order.
 *   O, LSE: of the forward with the same arguments.  Results of keys without any query are zeros.
 * fp32 storage: products in fp32.  bf16: P and dS are rounded to bf16 for the second products (accumulated in fp32), or taken in two
 * parts where the call has few rows, as in the forward (queries for dQ, keys for dK and dV).
 */
int ska_softmax_attn_bwd(const void *Q, const ska_strides *q_strides, const void *K, const ska_strides *k_strides,
                         const void *V, const ska_strides *v_strides, const void *O, const ska_strides *o_strides,
                         const void *dO, const ska_strides *do_strides, const float *LSE, void *dQ,
                         const ska_strides *dq_strides, void *dK, const ska_strides *dk_strides, void *dV,
                         const ska_strides *dv_strides, const int *start_q, const int *len_q, const int *len_k,
                         const unsigned char *mask_q, const unsigned char *mask_k, int B, int Hq, int Hk, int Lq, int Lk,
                         int d, int W, int causal, float eps, int dtype, void *workspace, size_t workspace_bytes,
                         void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SINKHORN_ATTN_LAYER_H */
