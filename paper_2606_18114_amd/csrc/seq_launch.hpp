// Launchers of the kernels over packed sequences, and the sizes of their
// workspaces.  Arguments are checked by the callers (abi_seq.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tmk {

// in_proj's output and where the sequences lie in it
struct SeqIn {
  const void* zx;      // [T, 2 d + 256 + nheads], float32 or bfloat16
  bool f32;
  int T, nseq, nheads;
  const int* offsets;  // [nseq + 1] or NULL
};

hipError_t launch_seq_conv(const SeqIn& in, const float* conv_w, const float* conv_b,
                           const uint16_t* ring_in, const int* ring_pos, uint16_t* ring_out,
                           uint16_t* u, hipStream_t stream);
int64_t seq_conv_bwd_bytes(int64_t T, int64_t nheads);
hipError_t launch_seq_conv_bwd(const SeqIn& in, const float* conv_w, const float* conv_b,
                               const uint16_t* du, void* dzx, float* dconv_w, float* dconv_b,
                               void* workspace, hipStream_t stream);

hipError_t launch_seq_norm(const SeqIn& in, const uint16_t* y, const float* norm_w, float eps,
                           uint16_t* out, hipStream_t stream);
int64_t seq_norm_bwd_bytes(int64_t T, int64_t nheads);
hipError_t launch_seq_norm_bwd(const SeqIn& in, const uint16_t* y, const float* norm_w, float eps,
                               const uint16_t* dout, void* dzx, uint16_t* dy, float* dnorm_w,
                               void* workspace, hipStream_t stream);

int64_t seq_scan_bytes(int64_t T, int64_t nheads);
hipError_t launch_seq_scan(const SeqIn& in, const uint16_t* u, const float* dt_bias,
                           const float* A_log, const float* D, const uint16_t* ssm_in,
                           uint16_t* ssm_out, uint16_t* y, void* workspace, hipStream_t stream);
// float32 states behind the chunks of the backward pass that another one follows
// (rev: their gradients): state [T / 128 + 1][nheads][64 * 128], with scratch decay
// [T / 128 + 1][nheads] (places: seq_scan_dev.hpp)
hipError_t launch_chunk_states(const SeqIn& in, const uint16_t* u, const uint16_t* dy, bool rev,
                               const float* dt_bias, const float* A_log, float* state,
                               float* decay, hipStream_t stream);
int64_t seq_scan_bwd_bytes(int64_t T, int64_t nseq, int64_t nheads);
hipError_t launch_seq_scan_bwd(const SeqIn& in, const uint16_t* u, const float* dt_bias,
                               const float* A_log, const float* D, const uint16_t* dy, void* dzx,
                               uint16_t* du, float* ddt_bias, float* dA_log, float* dD,
                               void* workspace, hipStream_t stream);

// ids int32 or int64; weight float32 (0), bfloat16 (1) or float16 (2)
hipError_t launch_embed(const void* ids, bool ids64, int64_t T, const void* weight, int type,
                        int64_t V, int64_t D, float scale, float* out, hipStream_t stream);
int64_t embed_bwd_bytes(int64_t T, int64_t V, int64_t D);
hipError_t launch_embed_bwd(const void* ids, bool ids64, int64_t T, const float* dout, int64_t V,
                            int64_t D, float scale, float* dW, bool accumulate, void* workspace,
                            hipStream_t stream);

// out[c] = sum over r < rows of part[r * stride + c], c < cols, in 16 or 64 interleaved
// chains of rows, as there are more or fewer columns
hipError_t launch_sum_rows(const float* part, int64_t rows, int64_t cols, int64_t stride,
                           float* out, hipStream_t stream);

}  // namespace tmk
