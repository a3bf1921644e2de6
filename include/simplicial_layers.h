/*
 * simplicial_layers.h -- C ABI of the operators around 2-simplicial attention, in
 * the same library (libsimplicial_attn.so): what prepares queries and keys
 * (norm and position rotation), the dot-product attention of the layers between
 * the 2-simplicial ones, and the log probabilities of a stack's tokens.
 *
 * Conventions are those of simplicial_attn.h (device pointers, the caller's
 * buffers, no allocation and no state, work enqueued on `stream` without
 * synchronising, SA_OK / SA_ERR_* codes, validation on the host before any HIP
 * call, dtype SA_DTYPE_F32 or SA_DTYPE_BF16), and
 *   Strides  are given in elements where an input may be a view; the innermost
 *            dimension is contiguous. Views of queries, keys and values have
 *            16-byte aligned rows (stride * element size a multiple of 16).
 *            Outputs are contiguous.
 *   Results  are bitwise the same for the same call on the same inputs: no
 *            floating-point atomics are used.
 */
#ifndef SIMPLICIAL_LAYERS_H
#define SIMPLICIAL_LAYERS_H

#include "simplicial_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Norm of each head and position rotation, of up to SA_ROTATE_MAX tensors (q, k,
 * k') in one launch. For every row x[b, n, h, :] of D elements
 *     u = x * r * weight,   r = (mean(x^2) + eps)^(-1/2)     (norm != 0)
 *     u = x                                                  (norm == 0)
 *     y = u with the pairs below turned by the angle a_i = position * freqs[i]:
 *         (u_s, u_t) -> (u_s cos a_i - u_t sin a_i, u_t cos a_i + u_s sin a_i)
 * for i in [0, nfreq). Components of no pair stay u. Pairs (s, t):
 *     SA_ROTATE_HALF   (i, nfreq + i)      nfreq a multiple of 8
 *     SA_ROTATE_PAIRS  (2 i, 2 i + 1)
 *     SA_ROTATE_AXIS   (3 i, 3 i + 1)      about component 3 i + 2 of each
 *         3-component chunk: the determinant logits of simplicial_attn_det_fwd
 *         are then functions of position differences alone
 * nfreq is at most D / 2 (D / 3 for SA_ROTATE_AXIS); 0: no rotation. Angles are
 * reduced in float64, so far positions keep their fraction of a turn. A row of
 * zeros with eps = 0 gives zeros (and zero gradients). Squares and their sum are float32:
 * values past 2^60 may overflow there (the norm is then infinite and the row 0), rows below 2^-60
 * may be taken for zeros where eps = 0.
 *   count       tensors, 1 .. SA_ROTATE_MAX
 *   x[t]        [B, N, heads[t], D], dtype, element strides
 *               strides[3 t .. 3 t + 2] of (batch, position, head)
 *   weight[t]   [D] of wdtype, or NULL (ones); `weight` itself may be NULL
 *   y[t]        [B, N, heads[t], D] contiguous, dtype, fully overwritten
 *   positions   [B, N] int64 with batch stride pos_stride (0: shared by the
 *               batch) and unit position stride, or NULL: start + n
 *   freqs       nfreq doubles in HOST memory (read during the call)
 *   D           16, 32, 64 or 128
 */
#define SA_ROTATE_MAX 3
#define SA_ROTATE_HALF 0
#define SA_ROTATE_PAIRS 1
#define SA_ROTATE_AXIS 2
int simplicial_norm_rotate_fwd(int32_t count, const void* const* x, const int64_t* strides,
                               const void* const* weight, void* const* y, const int32_t* heads,
                               const int64_t* positions, int64_t pos_stride, int64_t start, int64_t B,
                               int64_t N, int64_t D, int32_t norm, float eps, int32_t layout,
                               const double* freqs, int32_t nfreq, int32_t dtype, int32_t wdtype,
                               void* stream);

/*
 * Its backward: with g = dy turned back by the same angles,
 *     dweight = sum over b, n, h of g * x * r
 *     dx = r * (g * weight - x * r^2 * mean(g * weight * x))
 *   x, strides, weight, ...  as in the forward
 *   dy[t], dx[t]   [B, N, heads[t], D] contiguous, dtype
 *   dweight[t]     [D], wdtype, or NULL; fully overwritten
 *   workspace      at least simplicial_norm_rotate_bwd_workspace_size() bytes (0
 *                  where no dweight is asked for: the pointer may then be NULL)
 */
size_t simplicial_norm_rotate_bwd_workspace_size(int32_t count, int64_t B, int64_t N, int64_t D);
int simplicial_norm_rotate_bwd(int32_t count, const void* const* x, const int64_t* strides,
                               const void* const* weight, const void* const* dy, void* const* dx,
                               void* const* dweight, const int32_t* heads, const int64_t* positions,
                               int64_t pos_stride, int64_t start, void* workspace,
                               size_t workspace_bytes, int64_t B, int64_t N, int64_t D, int32_t norm,
                               float eps, int32_t layout, const double* freqs, int32_t nfreq,
                               int32_t dtype, int32_t wdtype, void* stream);

/*
 * Dot-product attention. The Nq queries are the last of a sequence of L keys
 * (L = k_lens[b], clamped to [0, Nk], or Nk): query i has position p = L - Nq + i.
 *     s[i,j] = scale * <q_i, k_j>
 *     a[i,j] = softcap * tanh(s / softcap) (softcap > 0; else s) - slopes[h] * |p - j|
 *     O_i    = sum_j softmax_j(a)[i,j] v_j,   LSE_i = log sum_j exp(a[i,j])
 * over the keys j < L that query i sees: those with
 *     (j <= p if causal) and (|p - j| < window if window > 0), or j < prefix[b],
 * and, with documents, documents[b, p] == documents[b, j] >= 0 (a negative number
 * marks padding, which sees nothing and is not seen). Document numbers may come
 * in any order. A query that sees no key (p < 0 among them) has O = 0 and LSE =
 * -inf. Values outside what a query sees do not reach it, infinities and NaN
 * included. Query head h reads head h / (H / Hkv) of k and v. Scores, statistics and sums are
 * float32; SA_DTYPE_BF16 rounds P (and the backward P and dS) to bf16 for its products with V (K, Q
 * and dO), SA_DTYPE_F32 rounds nothing below float32.
 *   q           [B, Nq, H, D], strides q_sb, q_sn, q_sh (batch, position, head)
 *   k, v        [B, Nk, Hkv, D], strides likewise
 *   out         [B, Nq, H, D] contiguous, dtype;  lse [B, H, Nq] float32
 *   out_lo      as out, or NULL: what its rounding took, rounded likewise (out + out_lo
 *               has twice the digits), for the backward. SA_DTYPE_BF16 only.
 *   slopes      [H] float32, documents [B, Nk] int32, prefix [B] int32, k_lens
 *               [B] int32, each contiguous or NULL
 *   workspace   simplicial_dot_attn_fwd_workspace_size() bytes (0: may be NULL):
 *               partial results of the parts a long key axis is split into where
 *               there are few queries, and the ranges of document numbers
 *   scale, softcap  finite, with normal float32 numbers as their quotient and 1 / softcap
 *   D           16, 32, 64 or 128;  1 <= Nq <= Nk
 */
size_t simplicial_dot_attn_fwd_workspace_size(int64_t B, int64_t Nq, int64_t Nk, int64_t H,
                                              int64_t Hkv, int64_t D, int32_t causal, int32_t window,
                                              int32_t has_documents, int32_t dtype);
int simplicial_dot_attn_fwd(const void* q, const void* k, const void* v, void* out, void* out_lo,
                            float* lse, void* workspace, size_t workspace_bytes, int64_t B, int64_t Nq, int64_t Nk,
                            int64_t H, int64_t Hkv, int64_t D, int64_t q_sb, int64_t q_sn, int64_t q_sh,
                            int64_t k_sb, int64_t k_sn, int64_t k_sh, int64_t v_sb, int64_t v_sn,
                            int64_t v_sh, float scale, float softcap, int32_t causal, int32_t window,
                            const float* slopes, const int32_t* documents, const int32_t* prefix,
                            const int32_t* k_lens, int32_t dtype, void* stream);

/*
 * Its backward:
 *     dA = P * (<dO_i, v_j> - Delta_i),  Delta_i = <dO_i, O_i>,  P = exp(a - LSE_i)
 *     dS = dA * (1 - tanh^2(s / softcap))
 *     dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
 * dK and dV of a head shared by several query heads are sums over them in
 * float32, rounded once. The slopes get no gradient. P carries the rounding of LSE to
 * float32, 2^-24 |LSE|: gradients of scores past 2^20 or so mean little.
 *   out, lse, dout   of the forward, contiguous
 *   out_lo           of the forward, or NULL: Delta of the rounded output, whose error (bf16
 *                    2^-8 of |dO| |O|) all of a row's gradients share;  dq [B, Nq, H, D], dk and dv
 *                    [B, Nk, Hkv, D] contiguous, fully overwritten (rows that no
 *                    query sees with zeros)
 *   workspace        simplicial_dot_attn_bwd_workspace_size() bytes
 */
size_t simplicial_dot_attn_bwd_workspace_size(int64_t B, int64_t Nq, int64_t Nk, int64_t H,
                                              int64_t Hkv, int64_t D, int32_t causal, int32_t window,
                                              int32_t has_documents, int32_t dtype);
int simplicial_dot_attn_bwd(const void* q, const void* k, const void* v, const void* out,
                            const void* out_lo, const void* dout, const float* lse, void* dq, void* dk, void* dv,
                            void* workspace, size_t workspace_bytes, int64_t B, int64_t Nq, int64_t Nk,
                            int64_t H, int64_t Hkv, int64_t D, int64_t q_sb, int64_t q_sn, int64_t q_sh,
                            int64_t k_sb, int64_t k_sn, int64_t k_sh, int64_t v_sb, int64_t v_sn,
                            int64_t v_sh, float scale, float softcap, int32_t causal, int32_t window,
                            const float* slopes, const int32_t* documents, const int32_t* prefix,
                            const int32_t* k_lens, int32_t dtype, void* stream);

/*
 * Log probabilities of given tokens, the entropy of every row's distribution and
 * its most probable tokens, in one pass over the logits:
 *     lse = log sum_j exp(x_j),  logprob = x[target] - lse,
 *     entropy = -sum_j p_j log p_j,  p_j = exp(x_j - lse)
 *     top_index, top_logprob: the `top` largest logits in descending order, equal
 *     ones by ascending index
 * A negative target leaves the row's logprob out (0, and no gradient through
 * it); one past the vocabulary gives NaN. Logits of -inf are tokens without
 * probability; a row of nothing else has lse = logprob = -inf (0 where the target is
 * left out) and entropy 0. A row with NaN or +inf has NaN everywhere; its
 * top_index holds distinct tokens.
 *   logits       [R, V], dtype, row stride row_stride >= V elements, aligned to
 *                its element; V at most 4000000
 *   targets      [R] int64
 *   logprob, entropy, lse   [R] float32
 *   top          0 .. min(V, SA_LOGPROBS_MAX_TOP)
 *   top_logprob  [R, top] float32, top_index [R, top] int64 (NULL for top = 0)
 *   workspace    simplicial_logprobs_fwd_workspace_size() bytes (0: may be NULL):
 *                partial results of long or few rows, which several workgroups share
 *   dtype        with SA_LOGPROBS_LSE_LO added, lse is [2, R]: behind lse what its rounding to
 *                float32 took (their sum has twice the digits), for the backward
 */
#define SA_LOGPROBS_MAX_TOP 32
#define SA_LOGPROBS_LSE_LO 0x100
size_t simplicial_logprobs_fwd_workspace_size(int64_t R, int64_t V, int32_t top, int32_t dtype);
int simplicial_logprobs_fwd(const void* logits, const int64_t* targets, float* logprob,
                            float* entropy, float* lse, float* top_logprob, int64_t* top_index,
                            void* workspace, size_t workspace_bytes, int64_t R, int64_t V,
                            int64_t row_stride, int32_t top, int32_t dtype, void* stream);

/*
 * Its backward, from the gradients of logprob, entropy and lse ([R] float32 each,
 * any of them NULL: zeros):
 *     dx_j = p_j (d_lse - d_logprob - d_entropy (log p_j + entropy)) + d_logprob [j = target]
 * A row without any probability gets zeros. The top tokens carry no gradient. p_j is
 * formed from lse: with SA_LOGPROBS_LSE_LO added to dtype and lse [2, R] of the forward a
 * constant added to a row's logits changes nothing; without it p_j carries the rounding of
 * lse to float32, 2^-24 |lse| of itself.
 *   dlogits   [R, V] contiguous, dtype, fully overwritten
 */
int simplicial_logprobs_bwd(const void* logits, const int64_t* targets, const float* lse,
                            const float* entropy, const float* d_logprob, const float* d_entropy,
                            const float* d_lse, void* dlogits, int64_t R, int64_t V,
                            int64_t row_stride, int32_t dtype, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SIMPLICIAL_LAYERS_H */
