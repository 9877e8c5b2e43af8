// The pre-norm of a block over many rows, and its gradients:
//   r = residual + y;  rho = 1 / sqrt(mean(r^2) + eps);  x = bf16(r rho w);
//   a = w dx;  dr = dresidual + rho (a - r rho^2 mean(a r));  dw = sum_t dx r rho.
//
// Bound by memory: 14 bytes an element forward (6 without y) and backward (10 without
// dresidual).  A workgroup (a wave up to 512 columns) takes a row and keeps it in
// registers between the sum and the output, up to 8192 columns; wider rows are
// read twice.  Columns are taken four at a time, whatever a row's alignment: the
// hardware takes vectors at any multiple of their element.
#include <type_traits>

#include "common.hpp"
#include "head.hpp"
#include "seq_launch.hpp"

namespace tmk {

namespace {

constexpr int kBnGroups = 1024;  // row groups of the backward's partial sums of dw
constexpr int64_t kBnRows = int64_t(1) << 22;  // of a launch's first dimension, forward

struct __attribute__((packed, aligned(4))) F4 {
  float v[4];
};
struct __attribute__((packed, aligned(2))) H4 {
  uint16_t v[4];
};

// columns c .. c + 3 of a row of d, zeros past its end
__device__ __forceinline__ void ld4(const float* p, int c, int d, float (&v)[4]) {
  if (c + 4 <= d) {
    const F4 x = *reinterpret_cast<const F4*>(p + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < d ? p[c + i] : 0.f;
  }
}
__device__ __forceinline__ void ld4(const uint16_t* p, int c, int d, float (&v)[4]) {
  H4 x;
  if (c + 4 <= d) {
    x = *reinterpret_cast<const H4*>(p + c);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = c + i < d ? p[c + i] : 0;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float((uint32_t)x.v[i] << 16);
}
__device__ __forceinline__ void st4(float* p, int c, int d, const float (&v)[4]) {
  if (c + 4 <= d) {
    F4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = v[i];
    *reinterpret_cast<F4*>(p + c) = x;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < d) p[c + i] = v[i];
  }
}
__device__ __forceinline__ void st4(uint16_t* p, int c, int d, const float (&v)[4]) {
  H4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.v[i] = __builtin_bit_cast(uint16_t, (__bf16)v[i]);
  if (c + 4 <= d) {
    *reinterpret_cast<H4*>(p + c) = x;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < d) p[c + i] = x.v[i];
  }
}

// sum over the workgroup's L threads, in every thread
template <int L>
__device__ __forceinline__ float row_sum(float v, float* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
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

// grid (x, y) of at least T, L threads; NV vectors a thread in registers (0: the row is read again)
template <int L, int NV>
__global__ __launch_bounds__(L) void block_norm_kernel(const float* residual, const float* y,
                                                       int64_t T, int d,
                                                       const float* __restrict__ w, float eps,
                                                       float* residual_out,
                                                       uint16_t* __restrict__ x) {
  __shared__ float lds[8];
  const int64_t t = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (t >= T) return;
  const int64_t at = t * d;
  auto load = [&](int c, float (&r)[4]) {
    ld4(residual + at, c, d, r);
    if (y) {
      float v[4];
      ld4(y + at, c, d, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] += v[i];
    }
  };
  auto put = [&](int c, const float (&r)[4], float rho) {
    float v[4], o[4];
    ld4(w, c, d, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = r[i] * rho * v[i];
    st4(x + at, c, d, o);
  };
  const bool write = residual_out && (residual_out != residual || y);
  float sq = 0.f;
  if constexpr (NV > 0) {
    float r[NV][4];
#pragma unroll
    for (int k = 0; k < NV; ++k) load(((int)threadIdx.x + k * L) * 4, r[k]);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) sq = __builtin_fmaf(r[k][i], r[k][i], sq);
    if (write) {
#pragma unroll
      for (int k = 0; k < NV; ++k) st4(residual_out + at, ((int)threadIdx.x + k * L) * 4, d, r[k]);
    }
    const float rho = 1.f / sqrtf(row_sum<L>(sq, lds) / (float)d + eps);
#pragma unroll
    for (int k = 0; k < NV; ++k) put(((int)threadIdx.x + k * L) * 4, r[k], rho);
  } else {
    float r[4];
    for (int c = (int)threadIdx.x * 4; c < d; c += 4 * L) {
      load(c, r);
#pragma unroll
      for (int i = 0; i < 4; ++i) sq = __builtin_fmaf(r[i], r[i], sq);
      if (write) st4(residual_out + at, c, d, r);
    }
    const float rho = 1.f / sqrtf(row_sum<L>(sq, lds) / (float)d + eps);
    for (int c = (int)threadIdx.x * 4; c < d; c += 4 * L) {
      ld4((write ? residual_out : residual) + at, c, d, r);  // (this thread's own)
      put(c, r, rho);
    }
  }
}

// grid (groups): rows blockIdx.x, + gridDim.x, ...; part [groups][d]: the group's sums of dx r rho
// (NV == 0: added up in memory, column by column)
template <int L, int NV>
__global__ __launch_bounds__(L) void block_norm_bwd_kernel(
    const float* __restrict__ r_in, int64_t T, int d, const float* __restrict__ w, float eps,
    const uint16_t* __restrict__ dx, const float* dres, float* dr, float* __restrict__ part) {
  __shared__ float lds[8];
  constexpr int kV = NV > 0 ? NV : 1;
  float dw[kV][4], wv[kV][4];
  float* prow = part + (int64_t)blockIdx.x * d;
#pragma unroll
  for (int k = 0; k < kV; ++k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[k][i] = 0.f;
    if constexpr (NV > 0) ld4(w, ((int)threadIdx.x + k * L) * 4, d, wv[k]);
  }
  const float inv = 1.f / (float)d;
  auto grads = [&](int64_t at, int c, const float (&r)[4], const float (&a)[4], float rho,
                   float m) {
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    if (dres) ld4(dres + at, c, d, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += rho * (a[i] - r[i] * m);
    st4(dr + at, c, d, o);
  };
  bool first = true;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const int64_t at = t * d;
    float sq = 0.f, sa = 0.f;
    if constexpr (NV > 0) {
      float r[NV][4], o[NV][4];
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = ((int)threadIdx.x + k * L) * 4;
        ld4(r_in + at, c, d, r[k]);
        ld4(dx + at, c, d, o[k]);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sq = __builtin_fmaf(r[k][i], r[k][i], sq);
          sa = __builtin_fmaf(o[k][i] * wv[k][i], r[k][i], sa);
        }
      const float rho = 1.f / sqrtf(row_sum<L>(sq, lds) * inv + eps);
      const float m = row_sum<L>(sa, lds) * inv * rho * rho;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          dw[k][i] = __builtin_fmaf(o[k][i], r[k][i] * rho, dw[k][i]);
          a[i] = o[k][i] * wv[k][i];
        }
        grads(at, ((int)threadIdx.x + k * L) * 4, r[k], a, rho, m);
      }
    } else {
      float r[4], o[4], q[4];
      auto load = [&](int c) {
        ld4(r_in + at, c, d, r);
        ld4(dx + at, c, d, o);
        ld4(w, c, d, q);
      };
      for (int c = (int)threadIdx.x * 4; c < d; c += 4 * L) {
        load(c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sq = __builtin_fmaf(r[i], r[i], sq);
          sa = __builtin_fmaf(o[i] * q[i], r[i], sa);
        }
      }
      const float rho = 1.f / sqrtf(row_sum<L>(sq, lds) * inv + eps);
      const float m = row_sum<L>(sa, lds) * inv * rho * rho;
      for (int c = (int)threadIdx.x * 4; c < d; c += 4 * L) {
        load(c);
        float p[4] = {0.f, 0.f, 0.f, 0.f};
        if (!first) ld4(prow, c, d, p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = __builtin_fmaf(o[i], r[i] * rho, p[i]);
          q[i] *= o[i];
        }
        st4(prow, c, d, p);
        grads(at, c, r, q, rho, m);
      }
      first = false;
    }
  }
  if constexpr (NV > 0)
#pragma unroll
    for (int k = 0; k < NV; ++k) st4(prow, ((int)threadIdx.x + k * L) * 4, d, dw[k]);
}

// calls f with a row's threads and the vectors of four a thread
template <typename Fn>
void bn_form(int d, Fn&& f) {
  using std::integral_constant;
  if (d <= 256) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (d <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (d <= 1024) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (d <= 2048) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (d <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (d <= 8192) f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  else f(integral_constant<int, 256>{}, integral_constant<int, 0>{});
}

int64_t bn_groups(int64_t T) { return T < kBnGroups ? T : kBnGroups; }

}  // namespace

hipError_t launch_block_norm(const float* residual, const float* y, int64_t T, int d,
                             const float* w, float eps, float* residual_out, uint16_t* x,
                             hipStream_t stream) {
  // a dimension of a launch has less than 2^32 threads, here 512 a row at most
  const int64_t ny = (T + kBnRows - 1) / kBnRows, nx = (T + ny - 1) / ny;
  bn_form(d, [&](auto l, auto nv) {
    hipLaunchKernelGGL((block_norm_kernel<l(), nv()>), dim3((unsigned)nx, (unsigned)ny), dim3(l()),
                       0, stream, residual, y, T, d, w, eps, residual_out, x);
  });
  return hipGetLastError();
}

int64_t block_norm_bwd_bytes(int64_t T, int64_t d) { return bn_groups(T) * d * 4; }

hipError_t launch_block_norm_bwd(const float* r, int64_t T, int d, const float* w, float eps,
                                 const uint16_t* dx, const float* dres, float* dr, float* dw,
                                 void* workspace, hipStream_t stream) {
  float* part = static_cast<float*>(workspace);
  const int64_t groups = bn_groups(T);
  bn_form(d, [&](auto l, auto nv) {
    hipLaunchKernelGGL((block_norm_bwd_kernel<l(), nv()>), dim3((unsigned)groups), dim3(l()), 0,
                       stream, r, T, d, w, eps, dx, dres, dr, part);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_sum_rows(part, groups, d, d, dw, stream);
}

}  // namespace tmk
