/*
 * tmamba_seq.h — the Mamba-2 mixer over whole sequences (prompts, training)
 * and the embedding: what tm_mixer_step does for one token, for packed
 * sequences, with the gradients.  Conventions, status codes and stream
 * semantics are those of tmamba.h.
 *
 * A layer of H = nheads heads has d = 64 H channels, 128 states and one group
 * of B and C; cd = d + 256, Z = 2 d + 256 + H.  zxbcdt [T, Z] holds in_proj's
 * output of T tokens, z | x | B | C | dt, bfloat16 (z_f32 = 0) or float32
 * (z_f32 = 1).  T 1 .. 2^23, H 1 .. 4096.
 *
 * Sequences are packed along the tokens: offsets, int32 [nseq + 1] in device
 * memory (4-byte aligned), not descending, from 0 to at most T; sequence i is
 * tokens offsets[i] .. offsets[i + 1] - 1 and may be empty.  NULL with nseq = 1:
 * one sequence of all T tokens.  nseq 1 .. 65535.  Tokens outside the sequences
 * (behind the last offset) are read by nothing that is written, and their
 * outputs are left as they were.  Being device data, the offsets are not
 * checked; whatever they hold, no call accesses memory outside its arrays.
 * Infinities and NaN reach what depends on them, by their own token or a later
 * one of the same sequence (where tm_mixer_step would give an infinity, it may be
 * NaN).  In the gradients they may reach any token of their own sequence.
 *
 * u, y, their gradients and the outputs are bfloat16 (16-byte aligned),
 * parameters and their gradients float32 (4-byte aligned), zxbcdt and its
 * gradient aligned to their element.  dzxbcdt [T, Z] has zxbcdt's type; each
 * backward call writes its own columns of it and no others.  Results are
 * deterministic.  Workspaces are device memory owned by the caller, 256-byte
 * aligned, of at least the bytes that the call's _workspace function says (0:
 * may be NULL); nothing need be set before a call and nothing is kept after
 * it.  Calls that share a workspace must not run concurrently.
 */
#ifndef TMAMBA_SEQ_H
#define TMAMBA_SEQ_H

#include "tmamba.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * tm_mixer_conv — the causal depthwise convolution with SiLU:
 *   a[t, c] = conv_b[c] + sum_{k < 4} conv_w[c, 3 - k] xBC[t - k, c],
 *   u[t, c] = bf16(a / (1 + e^-a)),
 * xBC = columns d .. d + cd - 1 of zxbcdt.
 *   conv_w float32 [cd, 4] (oldest tap first), conv_b [cd]
 *   ring_in   float16 [nseq, cd, 4] or NULL (zeros): the inputs before each
 *             sequence, decode's conv_state
 *   ring_pos  int32 [1]: slot (pos + j) % 4 of a ring holds the j-th oldest
 *             input (with either ring; it is not moved)
 *   ring_out  float16 [nseq, cd, 4] or NULL: the last four inputs of ring_in
 *             and the sequence, in the same slots; may be ring_in, no other
 *             overlap.  8-byte aligned, as ring_in.
 *   u         bf16 [T, cd]
 */
tm_status tm_mixer_conv(const void* zxbcdt, int32_t z_f32, int64_t T, int32_t nseq, int32_t nheads,
                        const int32_t* offsets, const float* conv_w, const float* conv_b,
                        const uint16_t* ring_in, const int32_t* ring_pos, uint16_t* ring_out,
                        uint16_t* u, tm_stream stream);

/*
 * tm_mixer_conv_bwd — its gradients, sequences beginning with zeros (no ring):
 * with da = du SiLU'(a), columns xBC of dzxbcdt get sum_k conv_w[c, 3 - k]
 * da[t + k, c] over the tokens t + k of the same sequence; dconv_w [cd, 4] and
 * dconv_b [cd] the sums over the sequences' tokens (float32).
 *   du bf16 [T, cd]
 */
tm_status tm_mixer_conv_bwd(const void* zxbcdt, int32_t z_f32, int64_t T, int32_t nseq,
                            int32_t nheads, const int32_t* offsets, const float* conv_w,
                            const float* conv_b, const uint16_t* du, void* dzxbcdt, float* dconv_w,
                            float* dconv_b, void* workspace, int64_t workspace_bytes,
                            tm_stream stream);
int64_t tm_mixer_conv_bwd_workspace(int64_t T, int32_t nheads); /* -1: sizes out of range */

/*
 * tm_mixer_scan — the selective state space scan: per head, with x, B, C the
 * columns of u, dt' = softplus(dt + dt_bias) and dt of zxbcdt,
 *   S_t = e^{-dt'_t e^A_log} S_{t-1} + dt'_t x_t B_t^T,  y_t = S_t C_t + D x_t.
 *   u         bf16 [T, cd] (tm_mixer_conv's)
 *   dt_bias, A_log, D  float32 [H]
 *   ssm_in    float16 [nseq, H, 64, 128] or NULL (zeros): the states before
 *             the sequences, decode's ssm_state (16-byte aligned)
 *   ssm_out   the same shape or NULL: the states after them, float32 within the
 *             call and rounded once; may be ssm_in, no other overlap
 *   y         bf16 [T, d]
 */
tm_status tm_mixer_scan(const uint16_t* u, const void* zxbcdt, int32_t z_f32, int64_t T,
                        int32_t nseq, int32_t nheads, const int32_t* offsets, const float* dt_bias,
                        const float* A_log, const float* D, const uint16_t* ssm_in,
                        uint16_t* ssm_out, uint16_t* y, void* workspace, int64_t workspace_bytes,
                        tm_stream stream);
int64_t tm_mixer_scan_workspace(int64_t T, int32_t nseq, int32_t nheads);

/*
 * tm_mixer_scan_bwd — its gradients, sequences beginning with zero states: of
 * u (du bf16 [T, cd]; dB and dC the sums over the heads), of dt (columns dt of
 * dzxbcdt), and ddt_bias, dA_log, dD [H] (float32).
 *   dy bf16 [T, d]
 */
tm_status tm_mixer_scan_bwd(const uint16_t* u, const void* zxbcdt, int32_t z_f32, int64_t T,
                            int32_t nseq, int32_t nheads, const int32_t* offsets,
                            const float* dt_bias, const float* A_log, const float* D,
                            const uint16_t* dy, void* dzxbcdt, uint16_t* du, float* ddt_bias,
                            float* dA_log, float* dD, void* workspace, int64_t workspace_bytes,
                            tm_stream stream);
int64_t tm_mixer_scan_bwd_workspace(int64_t T, int32_t nseq, int32_t nheads);

/*
 * tm_mixer_norm — the gated RMS norm of every row: g = y z / (1 + e^-z),
 *   out = bf16(g / sqrt(mean(g^2) + eps) * norm_w),
 * z = columns 0 .. d - 1 of zxbcdt.  y, out bf16 [T, d]; norm_w float32 [d];
 * eps finite, >= 0.  Every row by itself; the offsets only say which rows there
 * are.
 */
tm_status tm_mixer_norm(const uint16_t* y, const void* zxbcdt, int32_t z_f32, int64_t T,
                        int32_t nseq, int32_t nheads, const int32_t* offsets, const float* norm_w,
                        float eps, uint16_t* out, tm_stream stream);

/*
 * tm_mixer_norm_bwd — its gradients: dy bf16 [T, d], columns z of dzxbcdt,
 * dnorm_w float32 [d].  dout bf16 [T, d].
 */
tm_status tm_mixer_norm_bwd(const uint16_t* y, const void* zxbcdt, int32_t z_f32, int64_t T,
                            int32_t nseq, int32_t nheads, const int32_t* offsets,
                            const float* norm_w, float eps, const uint16_t* dout, void* dzxbcdt,
                            uint16_t* dy, float* dnorm_w, void* workspace,
                            int64_t workspace_bytes, tm_stream stream);
int64_t tm_mixer_norm_bwd_workspace(int64_t T, int32_t nheads);

/*
 * tm_embed — rows of an embedding: out[t] = scale * weight[ids[t]].
 *   ids     int32 (ids_i64 = 0) or int64 (1) [T]; an id outside 0 .. V - 1
 *           gives a row of zeros (padding)
 *   weight  [V, D], w_type 0 float32, 1 bfloat16, 2 float16; aligned to its
 *           element
 *   out     float32 [T, D] (4-byte aligned): the residual stream
 *   T 1 .. 2^23, V 1 .. 2^23, D 1 .. 2^30; scale finite
 */
tm_status tm_embed(const void* ids, int32_t ids_i64, int64_t T, const void* weight, int32_t w_type,
                   int64_t V, int64_t D, float scale, float* out, tm_stream stream);

/*
 * tm_embed_bwd — the gradient of its weight: dW[v] = scale * the sum of dout[t]
 * over the tokens t with id v, in ascending order of t (in float32; beyond 64
 * tokens, sums of 64 each are added up, to 4096 tokens of a batch in float32, in
 * longer ones in float64); accumulate 1: dW += that.
 *   dout float32 [T, D], dW float32 [V, D] (4-byte aligned)
 */
tm_status tm_embed_bwd(const void* ids, int32_t ids_i64, int64_t T, const float* dout, int64_t V,
                       int64_t D, float scale, float* dW, int32_t accumulate, void* workspace,
                       int64_t workspace_bytes, tm_stream stream);
int64_t tm_embed_bwd_workspace(int64_t T, int64_t V, int64_t D);

#ifdef __cplusplus
}
#endif

#endif /* TMAMBA_SEQ_H */
