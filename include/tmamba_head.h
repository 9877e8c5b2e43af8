/*
 * tmamba_head.h — the ends of a training step around the blocks: the loss of the
 * head over a large vocabulary, with a teacher's top logits, and the block's norm,
 * with their gradients.  Conventions, status codes and stream semantics are those
 * of tmamba.h; workspaces as in tmamba_seq.h, the head's of the size that is asked for
 * with the call's device current.  Results are deterministic.
 */
#ifndef TMAMBA_HEAD_H
#define TMAMBA_HEAD_H

#include "tmamba.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * tm_head_loss — the training objective (paper Eq. 1) of every token, from the
 * head's input, without keeping the logits z = h W^T:
 *   CE = ln sum_v e^{z_v} - z_y
 *   q = softmax of t_k / tau over the teacher's kept words, s = softmax(z / tau),
 *   KL = sum_k q_k (ln q_k - ln s[id_k]),
 *   loss = (1 - alpha) CE + alpha tau^2 KL;  without a teacher: CE.
 * A token whose label lies outside 0 .. V - 1 has no CE, one whose teacher keeps
 * no word no KL; neither: loss 0, and its row of h is not read.  A teacher's word is
 * kept if it lies in 0 .. V - 1 and its logit is not -infinity; words may come
 * twice (their shares add).  Infinities and NaN of a row of h that has a loss make its
 * loss NaN or infinite, those of W every loss's; a kept logit of +infinity or NaN makes its token's
 * loss NaN.
 *   type       of h and W: 1 bfloat16, 2 float16
 *   h          [T, D], W [V, D] (16-byte aligned); D % 8 == 0
 *   labels     int32 (labels_i64 = 0) or int64 (1) [T]
 *   top_ids    int32 (ids_i64 = 0) or int64 (1) [T, K], top [T, K] float32
 *              (top_type 0), bfloat16 (1) or float16 (2); both NULL with K = 0: no teacher
 *   alpha      0 .. 1, tau 2^-10 .. 2^10 (beyond, float32 holds too little of z / tau or of
 *              tau^2 KL); both ignored without a teacher
 *   loss       float32 [T]
 *   stats      float32 [T (4 + K)]: what tm_head_loss_bwd needs of this call
 *   T 1 .. 2^23, V 1 .. 2^23, D 8 .. 2^16, K 0 .. 1024, T (K + 1) < 2^31
 * Products of h and W are exact, sums and softmax statistics float32.
 */
tm_status tm_head_loss(const void* h, const void* W, int32_t type, int64_t T, int64_t V, int64_t D,
                       const void* labels, int32_t labels_i64, const void* top_ids,
                       int32_t ids_i64, const void* top, int32_t top_type, int32_t K, float alpha,
                       float tau, float* loss, float* stats, void* workspace,
                       int64_t workspace_bytes, tm_stream stream);
int64_t tm_head_loss_workspace(int64_t T, int64_t V, int64_t D); /* -1: sizes out of range */

/*
 * tm_head_loss_bwd — its gradients, dloss float32 [T] being the losses':
 *   dz_v = dloss ((1 - alpha) (p_v - 1[v = y]) + alpha tau (s_v - sum_k q_k 1[id_k = v])),
 *   dh = dz W,  dW = dz^T h.
 * The other arguments as they were in the forward call that wrote stats.  The
 * logits are made again, a piece of the vocabulary at a time; a logit's gradient is
 * rounded once to h's type (by 2^-8 of it in bfloat16, 2^-11 in float16, at a scale of its
 * own in every row) before the two products, whose sums are float32.  dW's product takes h
 * times its token's dloss, in h's type against the largest: exact in bfloat16 down to
 * 2^-126 of it, in float16 where such a value is above 2^-28 of the largest one of the call, and
 * off by at most 2^-39 of that below (one token's huge dloss hides others' small ones there).
 * Tokens without
 * a loss, or whose dloss is 0, have rows of zeros in dh and no part in dW,
 * whatever their rows of h hold.
 *   dh         [T, D], h's type (16-byte aligned), or NULL: not wanted
 *   dW         [V, D] (16-byte aligned) or NULL (not both); dW_type 0 float32 or h's
 *              type; accumulate 1 (float32 only): dW += the gradient
 */
tm_status tm_head_loss_bwd(const void* h, const void* W, int32_t type, int64_t T, int64_t V,
                           int64_t D, const void* labels, int32_t labels_i64, const void* top_ids,
                           int32_t ids_i64, int32_t K, float alpha, float tau, const float* stats,
                           const float* dloss, void* dh, void* dW, int32_t dW_type,
                           int32_t accumulate, void* workspace, int64_t workspace_bytes,
                           tm_stream stream);
int64_t tm_head_loss_bwd_workspace(int64_t T, int64_t V, int64_t D);

/*
 * tm_block_norm — the pre-norm of a block, or the final one, for training:
 *   r = residual + y  (y NULL: residual),
 *   x = bf16(r / sqrt(mean(r^2) + eps) * w).
 *   residual, y    float32 [T, D]
 *   residual_out   float32 [T, D]: r; may be residual; NULL only without y
 *   w float32 [D]; x bfloat16 [T, D]; eps finite, >= 0
 *   T 1 .. 2^23, D 1 .. 2^20; arrays aligned to their element
 */
tm_status tm_block_norm(const float* residual, const float* y, int64_t T, int64_t D, const float* w,
                        float eps, float* residual_out, uint16_t* x, tm_stream stream);

/*
 * tm_block_norm_bwd — its gradients: with rho = 1 / sqrt(mean(r^2) + eps), a = w dx,
 *   dr = dresidual + rho a - r rho^3 mean(a r)   (of residual and of y)
 *   dw = sum_t dx r rho.
 *   r           float32 [T, D]: residual_out of the forward call
 *   dx          bfloat16 [T, D]
 *   dresidual   float32 [T, D] or NULL (zeros): the gradient of residual_out
 *   dr          float32 [T, D]; may be dresidual.  dw float32 [D]
 */
tm_status tm_block_norm_bwd(const float* r, int64_t T, int64_t D, const float* w, float eps,
                            const uint16_t* dx, const float* dresidual, float* dr, float* dw,
                            void* workspace, int64_t workspace_bytes, tm_stream stream);
int64_t tm_block_norm_bwd_workspace(int64_t T, int64_t D);

#ifdef __cplusplus
}
#endif

#endif /* TMAMBA_HEAD_H */
