// The gated RMS norm before out_proj over the rows of a batch, and its
// gradients:  g = y SiLU(z);  r = 1 / sqrt(mean(g^2) + eps);  out = bf16(g r w).
// With q = dout w and m = mean(q g):  dg = r q - g r^3 m;  dy = bf16(dg SiLU(z)),
// dz = dg y SiLU'(z), dw = sum_t dout g r.
//
// Bound by memory: a workgroup (a wave where a row has at most 1024 channels)
// takes a row, 8 channels a thread at a time, and keeps the row's values in
// registers between the sum of squares and the output (rows up to 16384
// channels; longer ones are read twice).  16384 rows of 4096 in bfloat16: 77 us
// (5.2 TB/s, a copy's rate), the gradients 145 + 8 us (4.6 TB/s).
#include "seq.hpp"
#include "seq_launch.hpp"

namespace tmk {

constexpr int kNmBwdGroups = 1024;  // row groups of the backward's partial sums of dw

// sum over the workgroup's L threads, in every thread
template <int L>
__device__ __forceinline__ float nm_sum(float v, float* lds) {
  v = wave_sum(v);
  if constexpr (L == 64) {
    return v;
  } else {
    __syncthreads();  // the previous sum has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float a = (lds[0] + lds[1]) + (lds[2] + lds[3]);
    if constexpr (L == 512) a += (lds[4] + lds[5]) + (lds[6] + lds[7]);
    return a;
  }
}

// rows outside the sequences (tokens before the first offset, behind the last)
// are nobody's: not read, not written, in no sum
__device__ __forceinline__ bool nm_outside(const int* __restrict__ off, int nseq, int64_t t) {
  return off != nullptr && (t < off[0] || t >= off[nseq]);
}

// grid (T), L threads; NV vectors of 8 channels a thread in registers (0: the
// row is read again for the output)
template <bool F32, int L, int NV>
__global__ __launch_bounds__(L) void seq_norm_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int64_t Z, int d, const uint16_t* __restrict__ y,
    const float* __restrict__ w, float eps, const int* __restrict__ off, int nseq,
    uint16_t* __restrict__ out) {
  __shared__ float lds[8];
  const int64_t t = blockIdx.x;
  if (nm_outside(off, nseq, t)) return;
  const typename Zx<F32>::T* zr = zx + t * Z;
  const uint16_t* yr = y + t * d;
  uint16_t* o = out + t * d;
  auto gate = [&](int c, float (&g)[8]) {
    float z[8];
    Zx<F32>::ld8(zr + c, z);
    Zx<false>::ld8(yr + c, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] *= z[i] * sq_sigmoid(z[i]);
  };
  auto put = [&](int c, const float (&g)[8], float r) {
    float v[8];
    Zx<true>::ld8(w + c, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = g[i] * r * v[i];
    st16(o + c, u32x4{bf_pack(v[0], v[1]), bf_pack(v[2], v[3]), bf_pack(v[4], v[5]),
                      bf_pack(v[6], v[7])});
  };
  float sq = 0.f;
  if constexpr (NV > 0) {
    float g[NV][8];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = ((int)threadIdx.x + k * L) * 8;
      if (c < d) {
        gate(c, g[k]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[k][i] = 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = __builtin_fmaf(g[k][i], g[k][i], sq);
    const float r = 1.f / sqrtf(nm_sum<L>(sq, lds) / (float)d + eps);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = ((int)threadIdx.x + k * L) * 8;
      if (c < d) put(c, g[k], r);
    }
  } else {
    float g[8];
    for (int c = (int)threadIdx.x * 8; c < d; c += 8 * L) {
      gate(c, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = __builtin_fmaf(g[i], g[i], sq);
    }
    const float r = 1.f / sqrtf(nm_sum<L>(sq, lds) / (float)d + eps);
    for (int c = (int)threadIdx.x * 8; c < d; c += 8 * L) {
      gate(c, g);
      put(c, g, r);
    }
  }
}

// grid (groups): rows blockIdx.x, + gridDim.x, ...; part [groups][d]: the
// group's sums of dout g r (NV == 0: added up in memory, column by column)
template <bool F32, int L, int NV>
__global__ __launch_bounds__(L) void seq_norm_bwd_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int64_t Z, int d, int T,
    const uint16_t* __restrict__ y, const float* __restrict__ w, float eps,
    const int* __restrict__ off, int nseq, const uint16_t* __restrict__ dout, typename Zx<F32>::T* __restrict__ dzx,
    uint16_t* __restrict__ dy, float* __restrict__ part) {
  __shared__ float lds[8];
  constexpr int kV = NV > 0 ? NV : 1;
  float dw[kV][8], wv[kV][8];
  float* prow = part + (int64_t)blockIdx.x * d;
#pragma unroll
  for (int k = 0; k < kV; ++k) {
    const int c = ((int)threadIdx.x + k * L) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[k][i] = wv[k][i] = 0.f;
    if (NV > 0 && c < d) Zx<true>::ld8(w + c, wv[k]);
  }
  const float inv = 1.f / (float)d;
  // the row's gradients from its values and the two sums
  auto grads = [&](int64_t t, int c, const float (&yv)[8], const float (&z)[8],
                   const float (&q)[8], float r, float m) {
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = sq_sigmoid(z[i]), si = z[i] * s, g = yv[i] * si;
      const float dg = r * (q[i] - g * m);
      a[i] = dg * si;
      b[i] = dg * yv[i] * s * __builtin_fmaf(z[i], 1.f - s, 1.f);
    }
    Zx<false>::st8(dy + t * d + c, a);
    Zx<F32>::st8(dzx + t * Z + c, b);
  };
  bool first = true;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    if (nm_outside(off, nseq, t)) continue;
    const typename Zx<F32>::T* zr = zx + t * Z;
    float sq = 0.f, sg = 0.f;
    if constexpr (NV > 0) {
      float yv[NV][8], z[NV][8], o[NV][8];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = ((int)threadIdx.x + k * L) * 8;
        if (c < d) {
          Zx<F32>::ld8(zr + c, z[k]);
          Zx<false>::ld8(y + t * d + c, yv[k]);
          Zx<false>::ld8(dout + t * d + c, o[k]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) yv[k][i] = z[k][i] = o[k][i] = 0.f;
        }
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = yv[k][i] * z[k][i] * sq_sigmoid(z[k][i]);
          sq = __builtin_fmaf(g, g, sq);
          sg = __builtin_fmaf(o[k][i] * wv[k][i], g, sg);
        }
      const float r = 1.f / sqrtf(nm_sum<L>(sq, lds) * inv + eps);
      const float m = nm_sum<L>(sg, lds) * inv * r * r;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = ((int)threadIdx.x + k * L) * 8;
        if (c >= d) continue;
        float q[8];
        if constexpr (NV == 4) {  // the sums' SiLUs are made again: kept, they spill
#pragma unroll
          for (int i = 0; i < 8; ++i) asm("" : "+v"(z[k][i]));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = yv[k][i] * z[k][i] * sq_sigmoid(z[k][i]);
          dw[k][i] = __builtin_fmaf(o[k][i], g * r, dw[k][i]);
          q[i] = o[k][i] * wv[k][i];
        }
        grads(t, c, yv[k], z[k], q, r, m);
      }
    } else {
      float yv[8], z[8], o[8], wq[8];
      auto load = [&](int c) {
        Zx<F32>::ld8(zr + c, z);
        Zx<false>::ld8(y + t * d + c, yv);
        Zx<false>::ld8(dout + t * d + c, o);
        Zx<true>::ld8(w + c, wq);
      };
      for (int c = (int)threadIdx.x * 8; c < d; c += 8 * L) {
        load(c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = yv[i] * z[i] * sq_sigmoid(z[i]);
          sq = __builtin_fmaf(g, g, sq);
          sg = __builtin_fmaf(o[i] * wq[i], g, sg);
        }
      }
      const float r = 1.f / sqrtf(nm_sum<L>(sq, lds) * inv + eps);
      const float m = nm_sum<L>(sg, lds) * inv * r * r;
      for (int c = (int)threadIdx.x * 8; c < d; c += 8 * L) {
        load(c);
        float p[8], q[8];
        if (!first) Zx<true>::ld8(prow + c, p);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float g = yv[i] * z[i] * sq_sigmoid(z[i]);
          p[i] = __builtin_fmaf(o[i], g * r, first ? 0.f : p[i]);
          q[i] = o[i] * wq[i];
        }
        Zx<true>::st8(prow + c, p);
        grads(t, c, yv, z, q, r, m);
      }
      first = false;
    }
  }
  if constexpr (NV == 0) {
    const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (first)
      for (int c = (int)threadIdx.x * 8; c < d; c += 8 * L) Zx<true>::st8(prow + c, none);
  } else {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = ((int)threadIdx.x + k * L) * 8;
      if (c < d) Zx<true>::st8(prow + c, dw[k]);
    }
  }
}

// Calls f with the row's thread count and vectors a thread.  Backward a thread also
// holds the weight, dout and the sums of dw: above 4096 channels 512 threads share a
// row (8192 rows of 8192 channels 152 us, 201 with 256 threads, whose 276 registers
// leave a wave a SIMD; of 16384 300, 574 with spills; in float32 202, 219; 387, 582).
// From 16385 on the row is read twice.
template <bool BWD, typename Fn>
static void norm_form(int d, Fn&& f) {
  using std::integral_constant;
  constexpr int kWide = BWD ? 512 : 256;
  if (d <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (d <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (d <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (d <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (d <= 8192) f(integral_constant<int, kWide>{}, integral_constant<int, 1024 / kWide>{});
  else if (d <= 16384) f(integral_constant<int, kWide>{}, integral_constant<int, 2048 / kWide>{});
  else f(integral_constant<int, 256>{}, integral_constant<int, 0>{});
}

hipError_t launch_seq_norm(const SeqIn& in, const uint16_t* y, const float* norm_w, float eps,
                           uint16_t* out, hipStream_t stream) {
  const int d = in.nheads * kSqP;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + in.nheads;
  norm_form<false>(d, [&](auto l, auto nv) {
    if (in.f32)
      hipLaunchKernelGGL((seq_norm_kernel<true, l(), nv()>), dim3((unsigned)in.T), dim3(l()), 0,
                         stream, (const float*)in.zx, Z, d, y, norm_w, eps,
                         in.offsets, in.nseq, out);
    else
      hipLaunchKernelGGL((seq_norm_kernel<false, l(), nv()>), dim3((unsigned)in.T), dim3(l()), 0,
                         stream, (const uint16_t*)in.zx, Z, d, y, norm_w, eps,
                         in.offsets, in.nseq, out);
  });
  return hipGetLastError();
}

static int64_t norm_groups(int64_t T) { return T < kNmBwdGroups ? T : kNmBwdGroups; }

int64_t seq_norm_bwd_bytes(int64_t T, int64_t nheads) {
  return norm_groups(T) * nheads * kSqP * 4;
}

hipError_t launch_seq_norm_bwd(const SeqIn& in, const uint16_t* y, const float* norm_w, float eps,
                               const uint16_t* dout, void* dzx, uint16_t* dy, float* dnorm_w,
                               void* workspace, hipStream_t stream) {
  const int d = in.nheads * kSqP;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + in.nheads;
  const int64_t groups = norm_groups(in.T);
  float* part = (float*)workspace;
  norm_form<true>(d, [&](auto l, auto nv) {
    if (in.f32)
      hipLaunchKernelGGL((seq_norm_bwd_kernel<true, l(), nv()>), dim3((unsigned)groups), dim3(l()),
                         0, stream, (const float*)in.zx, Z, d, in.T, y, norm_w, eps,
                         in.offsets, in.nseq, dout, (float*)dzx, dy, part);
    else
      hipLaunchKernelGGL((seq_norm_bwd_kernel<false, l(), nv()>), dim3((unsigned)groups),
                         dim3(l()), 0, stream, (const uint16_t*)in.zx, Z, d, in.T, y, norm_w, eps,
                         in.offsets, in.nseq, dout, (uint16_t*)dzx, dy, part);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_sum_rows(part, groups, d, d, dnorm_w, stream);
}

}  // namespace tmk
