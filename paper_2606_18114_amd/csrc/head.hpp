// The head's loss and the block norm (tmamba_head.h): sizes, workspaces and what the kernels of
// head_gemm.hip and head_loss.hip hand each other.  Arguments are checked by
// the caller (abi_head.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tmk {

// rows of h with a loss, their labels and teacher, the weight
struct HeadIn {
  const uint16_t* h;  // [T, D]
  const uint16_t* w;  // [V, D]
  bool f16;           // else bfloat16
  int64_t T, V;
  int D;
  const void* targets;  // [T], int32 or int64
  const void* ids;      // [T, K] or NULL, int32 or int64
  bool targets64, ids64;
  int K;
  float alpha, tau;  // (0, 1 without a teacher)
};

// `stats`: four planes [T], log2 of the sum of exponentials, the same at the temperature,
// which terms a token has (1: cross entropy, 2: divergence) and, in float16, how large its row of h
// is, the logit gradient (of the loss over head_unit) at its label; then [T, K], that gradient at
// the teacher's words.
enum HeadStat { kStatLse, kStatLseT, kStatTerms, kStatLabel, kStatPlanes };
// the third plane: terms + 4 (25 + exponent of the row's largest value, -25 .. 15), 0 without terms
inline __device__ float head_stat_terms(int terms, int exponent) {
  return (float)(terms + 4 * (25 + exponent));
}
inline __device__ int head_terms(float stat) { return (int)stat & 3; }
inline __device__ int head_exponent(float stat) { return ((int)stat >> 2) - 25; }
inline __host__ __device__ int64_t head_stats_floats(int64_t T, int64_t K) {
  return (kStatPlanes + K) * T;
}

// |gradient of a logit| <= head_unit * |dloss|; the gradient over it is what
// is held in 16 bits
inline __host__ __device__ float head_unit(float alpha, float tau) {
  return (1.0f - alpha) + alpha * tau;
}

// A row of the backward pass: the exponents' offsets and the factors of the
// two softmaxes, 16 bytes.  Where there is one softmax, lse_t holds the bits of the label's
// word and c2 its dlogit; word -1: a teacher's words and the label are stored by a
// launch of their own.
struct HeadRow {
  float lse, lse_t, c1, c2;
};

// dlogits in 16 bits are (gradient over head_unit and a power of two) times
// 2^kHeadShift: float16 then holds probabilities down to 2^-27 with 11 bits;
// bfloat16 has the exponents anyway
template <bool F16>
constexpr int kHeadShift = F16 ? 13 : 0;

// Pieces of the vocabulary in the backward pass, and how products are cut
struct HeadPlan {
  int64_t piece = 0, pieces = 0;  // words (a multiple of 256) of a piece; their number
  int parts_h = 1, per_h = 0;     // dh's contraction (words of a piece), stages of 32
  int nst_h = 0;                  // all of them
  int parts_w = 1, per_w = 0;     // dW's contraction (tokens)
  int last_w = 1, last_per = 0;   // the same of the last piece
};
HeadPlan head_plan(int64_t T, int64_t V, int64_t D);

// How dh's contraction of nst stages is cut for the n rows in use of T: as planned for T, or,
// where the tiles of n times those parts leave some of P workgroups idle, into as many more as
// fill them and as the parts' place, parts T rows, has room for, in fours of stages (3001 tokens
// of 32003 x 768, a third without a loss: 124 us as planned, 95 to 101 so).
struct HeadCut {
  int parts, per;
};
inline __device__ HeadCut head_cut(HeadCut plan, int nst, int64_t T, int n, int D, int P) {
  const int tiles = (n + 255) / 256 * ((D + 255) / 256);
  if (tiles == 0 || tiles * plan.parts >= P) return plan;
  const int room = (int)(plan.parts * T / n), fill = P / tiles;
  const int k = room < fill ? room : fill;
  if (k <= plan.parts) return plan;
  const int per = ((nst + k - 1) / k + 3) / 4 * 4;
  return HeadCut{(nst + per - 1) / per, per};
}

int64_t head_loss_bytes(int64_t T, int64_t V, int64_t D);
hipError_t launch_head_loss(const HeadIn& in, const void* top, int top_type, float* loss,
                            float* stats, void* workspace, hipStream_t stream);
int64_t head_loss_bwd_bytes(int64_t T, int64_t V, int64_t D);
// dh or dw may be NULL; dw_type 0 float32, 1 h's type; accumulate only with float32
hipError_t launch_head_loss_bwd(const HeadIn& in, const float* stats, const float* dloss,
                                uint16_t* dh, void* dw, int dw_type, bool accumulate,
                                void* workspace, hipStream_t stream);

hipError_t launch_block_norm(const float* residual, const float* y, int64_t T, int d,
                             const float* w, float eps, float* residual_out, uint16_t* x,
                             hipStream_t stream);
int64_t block_norm_bwd_bytes(int64_t T, int64_t d);
hipError_t launch_block_norm_bwd(const float* r, int64_t T, int d, const float* w, float eps,
                                 const uint16_t* dx, const float* dres, float* dr, float* dw,
                                 void* workspace, hipStream_t stream);

// ---- products (head_gemm.hip); `count` [1]: rows in use, on the device
// ht [D rounded up to 128, head_padded(T)]: the transposed rows in use, zeros around them.
inline int64_t head_padded(int64_t T) { return (T + 255) / 256 * 256; }
// partial softmax sums of the rows: part[(wg + tile)][half][token][pair], see head_loss.hip
int64_t head_part_floats(int64_t T, int64_t words);
int head_tile_tokens(int64_t T, int64_t words, bool stats);       // tokens of a tile
int head_logits_grid(int64_t T, int64_t words, int tile);         // workgroups
hipError_t launch_head_logits(const HeadIn& in, const uint16_t* ht, const int* count, float* part,
                              hipStream_t stream);
// dlogits over *mantissa (a float's bits) of words w0 .. w0 + n - 1 to G [rows rounded up to 256, ld], ld >= n rounded up to
// 256, with zeros past the rows and words
hipError_t launch_head_dlogits(const HeadIn& in, const uint16_t* ht, const int* count,
                               const HeadRow* rows, const int* mantissa, int64_t w0, int64_t n,
                               uint16_t* G, int64_t ld,
                               hipStream_t stream);
// part_h[s][row][D] (+)= the s-th part of G . W[w0 ..], cut by head_cut; *used: the parts
hipError_t launch_head_dh(const HeadIn& in, const int* count, const uint16_t* G, int64_t ld,
                          int64_t w0, int64_t n, HeadCut plan, int nst, bool add, float* part_h,
                          int* used, hipStream_t stream);
// dW[w0 ..] (+)= 2^exp[0] (float at exp[2]) G^T . hs, whole, or into part_w[s][n][D] and from there
hipError_t launch_head_dw(const HeadIn& in, const int* count, const uint16_t* G, int64_t ld,
                          const uint16_t* hs, int64_t w0, int64_t n, int parts, int per,
                          const int* exp, void* dw, int dw_type, bool accumulate, float* part_w,
                          hipStream_t stream);

}  // namespace tmk
