// Shared pieces of the kernels over packed sequences (the mixer's convolution,
// scan and gated norm, and the embedding): launcher declarations, sequence
// lookup, element loads and SiLU.
//
// Sequences are packed one after another along the tokens: sequence i holds
// tokens offsets[i] .. offsets[i + 1] - 1 (offsets NULL: one sequence of all T
// tokens).  The offsets are device memory, so nothing on the host has checked
// them: every kernel takes a token only from its own grid (0 .. T - 1) and a
// sequence index only from the search below (0 .. nseq - 1), which keeps every
// access in bounds whatever the offsets hold.
#pragma once

#include <hip/hip_runtime.h>

#include "common.hpp"

namespace tmk {

constexpr int kSqP = 64;     // channels of a head
constexpr int kSqN = 128;    // states
constexpr int kSqTaps = 4;   // convolution taps

// a 16-byte access at any element boundary (a row of zxbcdt begins at a
// multiple of 16 bytes only if nheads is a multiple of 8)
typedef u32x4 __attribute__((aligned(2))) u32x4_u2;
typedef u32x2 __attribute__((aligned(2))) u32x2_u2;
typedef f32x4 __attribute__((aligned(4))) f32x4_u4;

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// round to nearest even; a NaN stays one (its payload is not kept)
__device__ __forceinline__ uint16_t bf_rne(float f) {
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}
// two values at once: one v_cvt_pk_bf16_f32
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// zxbcdt's element types
template <bool F32>
struct Zx;
template <>
struct Zx<false> {
  typedef uint16_t T;
  static __device__ __forceinline__ float at(const T* p) {
    return __uint_as_float((uint32_t)*p << 16);
  }
  static __device__ __forceinline__ void put(T* p, float v) { *p = bf_rne(v); }
  static __device__ __forceinline__ void ld8(const T* p, float (&v)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4_u2*>(p);
    v[0] = bf_lo(w.x), v[1] = bf_hi(w.x), v[2] = bf_lo(w.y), v[3] = bf_hi(w.y);
    v[4] = bf_lo(w.z), v[5] = bf_hi(w.z), v[6] = bf_lo(w.w), v[7] = bf_hi(w.w);
  }
  static __device__ __forceinline__ void ld4(const T* p, float (&v)[4]) {
    const u32x2 w = *reinterpret_cast<const u32x2_u2*>(p);
    v[0] = bf_lo(w.x), v[1] = bf_hi(w.x), v[2] = bf_lo(w.y), v[3] = bf_hi(w.y);
  }
  static __device__ __forceinline__ void st4(T* p, const float (&v)[4]) {
    *reinterpret_cast<u32x2_u2*>(p) = u32x2{bf_pack(v[0], v[1]), bf_pack(v[2], v[3])};
  }
  static __device__ __forceinline__ void st8(T* p, const float (&v)[8]) {
    *reinterpret_cast<u32x4_u2*>(p) = u32x4{bf_pack(v[0], v[1]), bf_pack(v[2], v[3]),
                                            bf_pack(v[4], v[5]), bf_pack(v[6], v[7])};
  }
};
template <>
struct Zx<true> {
  typedef float T;
  static __device__ __forceinline__ float at(const T* p) { return *p; }
  static __device__ __forceinline__ void put(T* p, float v) { *p = v; }
  static __device__ __forceinline__ void ld8(const T* p, float (&v)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4_u4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4_u4*>(p + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  static __device__ __forceinline__ void ld4(const T* p, float (&v)[4]) {
    const f32x4 a = *reinterpret_cast<const f32x4_u4*>(p);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
  }
  static __device__ __forceinline__ void st4(T* p, const float (&v)[4]) {
    *reinterpret_cast<f32x4_u4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  }
  static __device__ __forceinline__ void st8(T* p, const float (&v)[8]) {
    *reinterpret_cast<f32x4_u4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_u4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};

// the sequence that token t lies in: its index and its tokens [st, en);
// i = -1 where there is none (before the first offset, behind the last)
struct SeqAt {
  int i, st, en;
};
__device__ __forceinline__ SeqAt seq_find(const int* __restrict__ off, int nseq, int T, int t) {
  if (off == nullptr) return SeqAt{0, 0, T};
  int lo = 0, hi = nseq;  // the last i with off[i] <= t is the one that is not empty there
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int st = off[lo], en = min(off[lo + 1], T);
  if (st < 0 || st > t || en <= t) return SeqAt{-1, t, t + 1};
  return SeqAt{lo, st, en};
}

// 1 / (1 + e^-a): v_exp_f32 and v_rcp_f32 are good to one unit in the last
// place, the product's rounding before the exponential adds |a| 2^-24
__device__ __forceinline__ float sq_sigmoid(float a) {
  return __builtin_amdgcn_rcpf(1.f + __expf(-a));
}

// sum over the 64 lanes, in every lane
__device__ __forceinline__ float wave_sum(float v) {
  v += __uint_as_float(lane_xchg<1>(__float_as_uint(v)));
  v += __uint_as_float(lane_xchg<2>(__float_as_uint(v)));
  v += __uint_as_float(lane_xchg<4>(__float_as_uint(v)));
  v += __uint_as_float(lane_xchg<8>(__float_as_uint(v)));
  v += __uint_as_float(lane_xchg<16>(__float_as_uint(v)));
  v += __uint_as_float(lane_xchg<32>(__float_as_uint(v)));
  return v;
}

}  // namespace tmk
