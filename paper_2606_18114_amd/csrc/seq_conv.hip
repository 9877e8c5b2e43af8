// The mixer's short causal convolution over packed sequences and its
// gradients:
//   a[t, c] = b[c] + sum_{k < 4} w[c, 3 - k] x[t - k, c],  u = bf16(a sigmoid(a)),
// x = the xBC columns of zxbcdt; inputs from before a sequence come from its
// float16 ring (decode's convolution state), or are zero.  With da = du
// SiLU'(a):
//   dx[t] = sum_k w[3 - k] da[t + k]  (t + k in the same sequence),
//   dw[c, j] = sum_t da[t] x[t - 3 + j],  db = sum_t da.
//
// Bound by memory: a thread owns 8 channels (16 bytes of bfloat16; 4 backward)
// and walks a run of tokens with the last three inputs in registers, so an input
// is read once but for the three before each run.  16384 tokens of 64 heads in
// bfloat16: 61 us (4.7 TB/s, a copy reaches 5.1), the gradients 114 + 6 us (3.8).
#include "seq.hpp"
#include "seq_launch.hpp"

namespace tmk {

constexpr int kCvCh = 8;       // channels of a thread
constexpr int kCvBatch = 8;    // tokens whose loads are issued together
constexpr int kCvBwdCh = 4;    // its channels a thread: with 8 the sums leave two waves a SIMD
constexpr int kCvBwdBatch = 8;
constexpr int kCvSimds = 1024;  // 256 CUs

// grid (runs, ceil(cd / 512)), one wave each.  ring_out: not ring, or NULL
template <bool F32>
__global__ __launch_bounds__(64) void seq_conv_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int T, int nheads, const int* __restrict__ off,
    int nseq, int run, const float* __restrict__ conv_w, const float* __restrict__ conv_b,
    const uint16_t* ring, const int* __restrict__ ring_pos, uint16_t* ring_out,
    uint16_t* __restrict__ u) {
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int c = ((int)blockIdx.y * 64 + (int)threadIdx.x) * kCvCh;
  if (c >= cd) return;
  const int t0 = (int)blockIdx.x * run, t1 = min(T, t0 + run);
  const typename Zx<F32>::T* x = zx + d + c;
  float w[kSqTaps][kCvCh], b[kCvCh];
#pragma unroll
  for (int i = 0; i < kCvCh; ++i) {
    b[i] = conv_b[c + i];
#pragma unroll
    for (int j = 0; j < kSqTaps; ++j) w[j][i] = conv_w[(int64_t)(c + i) * kSqTaps + j];
  }
  const int pos = ring_pos ? ring_pos[0] & 3 : 0;
  if (ring_out)  // empty sequences keep their rings
    for (int i = blockIdx.x; i < nseq; i += gridDim.x) {
      const int a = off ? off[i] : 0, e = off ? min(off[i + 1], T) : T;
      if (a >= 0 && e > a) continue;
      const u32x2 zero = {0, 0};
      const int64_t at = ((int64_t)i * cd + c) * kSqTaps;
#pragma unroll
      for (int k = 0; k < kCvCh; ++k)
        *(u32x2*)(ring_out + at + k * kSqTaps) =
            ring ? *(const u32x2*)(ring + at + k * kSqTaps) : zero;
    }
  SeqAt sq = seq_find(off, nseq, T, t0);
  float h[3][kCvCh];  // the three inputs before the token, oldest first
  auto past = [&](int t) {
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int tj = t - 3 + j;
      if (tj >= sq.st) {
        Zx<F32>::ld8(x + tj * Z, h[j]);
      } else {
#pragma unroll
        for (int i = 0; i < kCvCh; ++i) h[j][i] = 0.f;
        if (ring && sq.i >= 0) {
          const int slot = (pos + 4 + tj - sq.st) & 3;
          const uint16_t* r = ring + ((int64_t)sq.i * cd + c) * kSqTaps;
#pragma unroll
          for (int i = 0; i < kCvCh; ++i) {  // a channel's four slots are 8 bytes
            const uint64_t q = *(const uint64_t*)(r + i * kSqTaps);
            h[j][i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(q >> (16 * slot)));
          }
        }
      }
    }
  };
  past(t0);
  for (int tb = t0; tb < t1; tb += kCvBatch) {
    float v[kCvBatch][kCvCh];
#pragma unroll
    for (int q = 0; q < kCvBatch; ++q) Zx<F32>::ld8(x + min(tb + q, T - 1) * Z, v[q]);
#pragma unroll
    for (int q = 0; q < kCvBatch; ++q) {
      const int t = tb + q;
      if (t >= t1) break;
      if (t >= sq.en) {
        sq = seq_find(off, nseq, T, t);
        past(t);
      }
      if (ring_out && t == sq.en - 1 && sq.i >= 0) {  // the last four inputs
        uint64_t* r = (uint64_t*)(ring_out + ((int64_t)sq.i * cd + c) * kSqTaps);
#pragma unroll
        for (int i = 0; i < kCvCh; ++i) {
          auto h16 = [](float f) { return (uint64_t)__builtin_bit_cast(uint16_t, (_Float16)f); };
          const uint64_t n = h16(h[0][i]) | h16(h[1][i]) << 16 | h16(h[2][i]) << 32 |
                             h16(v[q][i]) << 48;
          r[i] = pos ? n << (16 * pos) | n >> (64 - 16 * pos) : n;  // the oldest into slot pos
        }
      }
      float o[kCvCh];
#pragma unroll
      for (int i = 0; i < kCvCh; ++i) {
        float a = __builtin_fmaf(h[0][i], w[0][i], b[i]);
        a = __builtin_fmaf(h[1][i], w[1][i], a);
        a = __builtin_fmaf(h[2][i], w[2][i], a);
        a = __builtin_fmaf(v[q][i], w[3][i], a);
        o[i] = a * sq_sigmoid(a);
        h[0][i] = h[1][i], h[1][i] = h[2][i], h[2][i] = v[q][i];
      }
      if (sq.i >= 0) {
        u32x4 p = {bf_pack(o[0], o[1]), bf_pack(o[2], o[3]), bf_pack(o[4], o[5]),
                   bf_pack(o[6], o[7])};
        st16(u + (int64_t)t * cd + c, p);
      }
    }
  }
}

// The ring after the sequences where it is updated in place, a launch of its own:
// other workgroups of the convolution may still read the old one.  grid (ceil(cd /
// 256), nseq); a thread takes one channel: its last four inputs, of the ring
// where the sequence is shorter than that.
template <bool F32>
__global__ __launch_bounds__(256) void seq_ring_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int T, int nheads, const int* __restrict__ off,
    const int* __restrict__ ring_pos, uint16_t* __restrict__ ring) {
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int c = (int)(blockIdx.x * 256 + threadIdx.x), i = (int)blockIdx.y;
  if (c >= cd) return;
  const int st = off ? off[i] : 0, en = off ? min(off[i + 1], T) : T;
  const int len = st >= 0 && en > st ? en - st : 0;
  if (len == 0) return;
  const int pos = ring_pos[0] & 3;
  uint16_t* r = ring + ((int64_t)i * cd + c) * kSqTaps;
  uint16_t old[kSqTaps], now[kSqTaps];
#pragma unroll
  for (int j = 0; j < kSqTaps; ++j) old[j] = r[(pos + j) & 3];
#pragma unroll
  for (int j = 0; j < kSqTaps; ++j) {
    const int k = len + j - kSqTaps;  // the input's place in the sequence
    if (k >= 0) {
      now[j] = __builtin_bit_cast(uint16_t, (_Float16)Zx<F32>::at(zx + (int64_t)(st + k) * Z + d + c));
    } else {
      now[j] = 0;
#pragma unroll
      for (int q = 0; q < kSqTaps; ++q)
        if (q == k + kSqTaps) now[j] = old[q];
    }
  }
#pragma unroll
  for (int j = 0; j < kSqTaps; ++j) r[(pos + j) & 3] = now[j];
}

// Backward, a run of tokens (conv_bwd_run): da of the run's tokens and of the three
// behind it (which only feed dx of the run's last ones).  dx[t] is complete
// once da[t + 3] is known or the sequence has ended.  part [run][5][cd]: the
// run's sums for w (4) and b.
template <bool F32>
__global__ __launch_bounds__(64) void seq_conv_bwd_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int T, int nheads, const int* __restrict__ off,
    int nseq, int run, const float* __restrict__ conv_w, const float* __restrict__ conv_b,
    const uint16_t* __restrict__ du, typename Zx<F32>::T* __restrict__ dzx,
    float* __restrict__ part) {
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int c = ((int)blockIdx.y * 64 + (int)threadIdx.x) * kCvBwdCh;
  if (c >= cd) return;
  const int t0 = (int)blockIdx.x * run, t1 = min(T, t0 + run);
  const typename Zx<F32>::T* x = zx + d + c;
  typename Zx<F32>::T* dx = dzx + d + c;
  float w[kSqTaps][kCvBwdCh], b[kCvBwdCh];
#pragma unroll
  for (int i = 0; i < kCvBwdCh; ++i) {
    b[i] = conv_b[c + i];
#pragma unroll
    for (int j = 0; j < kSqTaps; ++j) w[j][i] = conv_w[(int64_t)(c + i) * kSqTaps + j];
  }
  SeqAt sq = seq_find(off, nseq, T, t0);
  float h[3][kCvBwdCh], acc[3][kCvBwdCh], dw[kSqTaps][kCvBwdCh], db[kCvBwdCh];
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const int tj = t0 - 3 + j;
    if (tj >= sq.st) {
      Zx<F32>::ld4(x + tj * Z, h[j]);
    } else {
#pragma unroll
      for (int i = 0; i < kCvBwdCh; ++i) h[j][i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < kCvBwdCh; ++i) acc[j][i] = 0.f;  // dx of t - 3, t - 2, t - 1 so far
  }
#pragma unroll
  for (int i = 0; i < kCvBwdCh; ++i) {
    db[i] = 0.f;
#pragma unroll
    for (int j = 0; j < kSqTaps; ++j) dw[j][i] = 0.f;
  }
  // stores dx of token t (in the run, in a sequence that began at st)
  auto emit = [&](int t, int st, const float(&v)[kCvBwdCh]) {
    if (t >= t0 && t < t1 && t >= st) Zx<F32>::st4(dx + t * Z, v);
  };
  const int te = min(T, t1 + 3);
  int t = t0;
  bool open = sq.i >= 0;
  for (int tb = t0; tb < te; tb += kCvBwdBatch) {
    float v[kCvBwdBatch][kCvBwdCh], g[kCvBwdBatch][kCvBwdCh];
#pragma unroll
    for (int q = 0; q < kCvBwdBatch; ++q) {
      const int64_t tq = min(tb + q, T - 1);
      Zx<F32>::ld4(x + tq * Z, v[q]);
      Zx<false>::ld4(du + tq * cd + c, g[q]);
    }
#pragma unroll
    for (int q = 0; q < kCvBwdBatch; ++q) {
      t = tb + q;
      if (t >= te) break;
      if (t >= sq.en) {  // the sequence ended: its last three dx are complete
        if (open) {
          emit(t - 3, sq.st, acc[0]);
          emit(t - 2, sq.st, acc[1]);
          emit(t - 1, sq.st, acc[2]);
        }
        sq = seq_find(off, nseq, T, t);
        open = sq.i >= 0;
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
          for (int i = 0; i < kCvBwdCh; ++i) h[j][i] = acc[j][i] = 0.f;
      }
      float now[kCvBwdCh], first[kCvBwdCh];
#pragma unroll
      for (int i = 0; i < kCvBwdCh; ++i) {
        float a = __builtin_fmaf(h[0][i], w[0][i], b[i]);
        a = __builtin_fmaf(h[1][i], w[1][i], a);
        a = __builtin_fmaf(h[2][i], w[2][i], a);
        a = __builtin_fmaf(v[q][i], w[3][i], a);
        const float s = sq_sigmoid(a);
        const float da = g[q][i] * s * __builtin_fmaf(a, 1.f - s, 1.f);
        if (t < t1 && open) {  // a token of this run: the parameters' sums
          db[i] += da;
          dw[0][i] = __builtin_fmaf(da, h[0][i], dw[0][i]);
          dw[1][i] = __builtin_fmaf(da, h[1][i], dw[1][i]);
          dw[2][i] = __builtin_fmaf(da, h[2][i], dw[2][i]);
          dw[3][i] = __builtin_fmaf(da, v[q][i], dw[3][i]);
        }
        first[i] = __builtin_fmaf(w[0][i], da, acc[0][i]);
        acc[0][i] = __builtin_fmaf(w[1][i], da, acc[1][i]);
        acc[1][i] = __builtin_fmaf(w[2][i], da, acc[2][i]);
        acc[2][i] = w[3][i] * da;
        now[i] = v[q][i];
      }
      if (open) emit(t - 3, sq.st, first);
#pragma unroll
      for (int i = 0; i < kCvBwdCh; ++i) h[0][i] = h[1][i], h[1][i] = h[2][i], h[2][i] = now[i];
    }
  }
  // what is left: tokens te - 3 .. te - 1 (of the run only where T ended it)
  if (open) {
    emit(te - 3, sq.st, acc[0]);
    emit(te - 2, sq.st, acc[1]);
    emit(te - 1, sq.st, acc[2]);
  }
  float* p = part + (int64_t)blockIdx.x * 5 * cd + c;
#pragma unroll
  for (int j = 0; j < kSqTaps; ++j)
    *reinterpret_cast<f32x4*>(p + (int64_t)j * cd) = f32x4{dw[j][0], dw[j][1], dw[j][2], dw[j][3]};
  *reinterpret_cast<f32x4*>(p + (int64_t)4 * cd) = f32x4{db[0], db[1], db[2], db[3]};
}

// out[c] = sum_r part[r][c]: COLS columns a workgroup, 1024 / COLS chains of rows
// added in their order, the chains in LDS.  64 columns where that makes a
// workgroup for every CU (21760 columns of 256 rows: 8 us, 11 with 16), else 16
// (4096 of 1024: 8 us, 21 with 64).  With ntap != 0 column q * cd + c goes to
// out[c * ntap + q] for q < ntap, to out2[c] for q == ntap.
template <int COLS>
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float* __restrict__ part,
                                                        int64_t rows, int64_t cols,
                                                        int64_t stride, float* __restrict__ out,
                                                        int ntap, int64_t cd,
                                                        float* __restrict__ out2) {
  constexpr int kChains = 1024 / COLS;
  __shared__ float s[kChains][COLS];
  const int lane = threadIdx.x % COLS, chain = threadIdx.x / COLS;
  const int64_t col = (int64_t)blockIdx.x * COLS + lane;
  float v = 0.f;
  if (col < cols) {
#pragma unroll 4
    for (int64_t r = chain; r < rows; r += kChains) v += part[r * stride + col];
  }
  s[chain][lane] = v;
  __syncthreads();
  if (chain != 0 || col >= cols) return;
#pragma unroll 8
  for (int k = 1; k < kChains; ++k) v += s[k][lane];
  if (ntap == 0) {
    out[col] = v;
  } else {
    const int64_t q = col / cd, ch = col - q * cd;
    if (q < ntap) out[ch * ntap + q] = v;
    else out2[ch] = v;
  }
}

static hipError_t sum_rows(const float* part, int64_t rows, int64_t cols, int64_t stride,
                           float* out, int ntap, int64_t cd, float* out2, hipStream_t stream) {
  if (cols >= 256 * 64)
    hipLaunchKernelGGL(sum_rows_kernel<64>, dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0,
                       stream, part, rows, cols, stride, out, ntap, cd, out2);
  else
    hipLaunchKernelGGL(sum_rows_kernel<16>, dim3((unsigned)((cols + 15) / 16)), dim3(1024), 0,
                       stream, part, rows, cols, stride, out, ntap, cd, out2);
  return hipGetLastError();
}

hipError_t launch_sum_rows(const float* part, int64_t rows, int64_t cols, int64_t stride,
                           float* out, hipStream_t stream) {
  return sum_rows(part, rows, cols, stride, out, 0, 1, nullptr, stream);
}

template <bool F32>
static hipError_t conv_go(const SeqIn& in, const float* conv_w, const float* conv_b,
                          const uint16_t* ring_in, const int* ring_pos, uint16_t* ring_out,
                          uint16_t* u, hipStream_t stream) {
  typedef typename Zx<F32>::T E;
  const int cd = in.nheads * kSqP + 2 * kSqN;
  const int cblk = (cd / kCvCh + 63) / 64;
  // runs as long as two waves a SIMD are left, at most 16 tokens
  int run = (int)((int64_t)in.T * cblk / (2 * kCvSimds));
  run = run < 1 ? 1 : run > 16 ? 16 : run;
  hipLaunchKernelGGL(seq_conv_kernel<F32>, dim3((unsigned)((in.T + run - 1) / run), (unsigned)cblk),
                     dim3(64), 0, stream, (const E*)in.zx, in.T, in.nheads, in.offsets, in.nseq,
                     run, conv_w, conv_b, ring_in, ring_pos,
                     ring_out == ring_in ? nullptr : ring_out, u);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || ring_out == nullptr || ring_out != ring_in) return e;
  hipLaunchKernelGGL(seq_ring_kernel<F32>, dim3((unsigned)((cd + 255) / 256), (unsigned)in.nseq),
                     dim3(256), 0, stream, (const E*)in.zx, in.T, in.nheads, in.offsets, ring_pos,
                     ring_out);
  return hipGetLastError();
}

hipError_t launch_seq_conv(const SeqIn& in, const float* conv_w, const float* conv_b,
                           const uint16_t* ring_in, const int* ring_pos, uint16_t* ring_out,
                           uint16_t* u, hipStream_t stream) {
  return in.f32 ? conv_go<true>(in, conv_w, conv_b, ring_in, ring_pos, ring_out, u, stream)
                : conv_go<false>(in, conv_w, conv_b, ring_in, ring_pos, ring_out, u, stream);
}

// Tokens of a backward run: as long as three waves a SIMD are left, for the run's
// sums are written and added up, and 8 to 64: with few tokens it is a run's walk
// that takes the time (1000 tokens of 64 heads: 18 us, 32 in runs of 64; 16384: 115).
static int conv_bwd_run(int64_t T, int64_t nheads) {
  const int64_t cblk = ((nheads * kSqP + 2 * kSqN) / kCvBwdCh + 63) / 64;
  const int64_t run = T * cblk / (3 * kCvSimds) / 8 * 8;
  return (int)(run < 8 ? 8 : run > 64 ? 64 : run);
}

int64_t seq_conv_bwd_bytes(int64_t T, int64_t nheads) {
  const int run = conv_bwd_run(T, nheads);
  return (T + run - 1) / run * 5 * (nheads * kSqP + 2 * kSqN) * 4;
}

template <bool F32>
static hipError_t conv_bwd_go(const SeqIn& in, const float* conv_w, const float* conv_b,
                              const uint16_t* du, void* dzx, float* dconv_w, float* dconv_b,
                              void* workspace, hipStream_t stream) {
  typedef typename Zx<F32>::T E;
  const int cd = in.nheads * kSqP + 2 * kSqN;
  const int run = conv_bwd_run(in.T, in.nheads), runs = (in.T + run - 1) / run;
  float* part = (float*)workspace;
  hipLaunchKernelGGL(seq_conv_bwd_kernel<F32>,
                     dim3((unsigned)runs, (unsigned)((cd / kCvBwdCh + 63) / 64)), dim3(64), 0, stream,
                     (const E*)in.zx, in.T, in.nheads, in.offsets, in.nseq, run, conv_w, conv_b,
                     du, (E*)dzx, part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t cols = (int64_t)5 * cd;
  return sum_rows(part, runs, cols, cols, dconv_w, kSqTaps, cd, dconv_b, stream);
}

hipError_t launch_seq_conv_bwd(const SeqIn& in, const float* conv_w, const float* conv_b,
                               const uint16_t* du, void* dzx, float* dconv_w, float* dconv_b,
                               void* workspace, hipStream_t stream) {
  return in.f32 ? conv_bwd_go<true>(in, conv_w, conv_b, du, dzx, dconv_w, dconv_b, workspace, stream)
                : conv_bwd_go<false>(in, conv_w, conv_b, du, dzx, dconv_w, dconv_b, workspace, stream);
}

}  // namespace tmk
