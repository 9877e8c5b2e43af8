// Device pieces of the selective scan's kernels: where a workgroup's tokens
// lie, the decays of a tile, matrix operands from LDS, values split into
// bfloat16 terms.
//
// Mathematics (a head; dt' = softplus(dt + dt_bias), l_t = -dt'_t e^A_log):
//   S_t = e^{l_t} S_{t-1} + dt'_t x_t B_t^T,   y_t = S_t C_t + D x_t.
// Over a tile of Q tokens with c_t = l_1 + .. + l_t and S0 the state before it
//   y_t = sum_{s <= t} e^{c_t - c_s} dt'_s (C_t . B_s) x_s + e^{c_t} S0 C_t + D x_t,
//   S_Q = e^{c_Q} S0 + sum_s e^{c_Q - c_s} dt'_s x_s B_s^T,
// products for the matrix cores.  Every exponent is at most 0.
//
// Operands: x, B, C and dy are bfloat16 and enter as they are; a float32
// operand (a state, the decayed C . B) enters as a sum of bfloat16 terms, two
// (2^-17 of the value) where a bfloat16 output is made of it, three (2^-25)
// where a float32 gradient is.
#pragma once

#include "mixer_dev.hpp"
#include "seq.hpp"
#include "seq_launch.hpp"

namespace tmk {

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kScQ = 64;           // tokens of a tile of the walking kernels
constexpr int kScChunk = 128;      // tokens of a chunk of the backward pass
constexpr int kScState = kSqP * kSqN;
// LDS rows in bytes: what transpose reads take has 32 bytes more than the data
// (the 32-byte pieces of four rows then lie in different banks), what only row
// reads take 16 more (the 16-byte pieces of eight rows)
constexpr int kScRowN = 2 * kSqN + 32;  // 128 states, transpose reads
constexpr int kScRowP = 2 * kSqP + 32;  // 64 channels, transpose reads
constexpr int kScRowS = 2 * kSqN + 16;  // 128 states, row reads

// Slot sl of the segments of segT tokens that the sequences are cut into.
// Sequence i's segment k has slot off[i] / segT + i + k, which leaves every
// sequence at least as many slots as it has segments without adding lengths
// up; T / segT + nseq slots in all.  t0 >= t1: no tokens.
//
// States that segments hand on lie at sl - i = off[i] / segT + k, for the segments
// k that another one of their sequence follows: those have off[i] + (k + 1) segT <
// off[i + 1], so that the places of later sequences are higher, and the last place
// is at most (T - 1) / segT, however many sequences there are.
struct Slot {
  int i, k, t0, t1;  // sequence, segment, the segment's tokens
  int st, en;        // the sequence's tokens
};
__device__ __forceinline__ int slot_off(const int* off, int T, int i) {
  const int o = off[i];
  return o < 0 ? 0 : o > T ? T : o;
}
__device__ __forceinline__ Slot slot_find(const int* __restrict__ off, int nseq, int T, int segT,
                                          int sl) {
  Slot s;
  if (off == nullptr) {
    s.i = 0, s.st = 0, s.en = T, s.k = sl;
  } else {
    int lo = 0, hi = nseq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (slot_off(off, T, mid) / segT + mid <= sl) lo = mid;
      else hi = mid;
    }
    s.i = lo;
    s.st = slot_off(off, T, lo);
    s.en = slot_off(off, T, lo + 1);
    s.k = sl - (s.st / segT + lo);
  }
  const int64_t a = (int64_t)s.st + (int64_t)s.k * segT;
  if (s.k < 0 || a >= s.en) {
    s.t0 = s.t1 = s.en;
  } else {
    s.t0 = (int)a;
    s.t1 = (int)min((int64_t)s.en, a + segT);
  }
  return s;
}
inline __host__ __device__ int64_t slot_count(int64_t T, int64_t nseq, int64_t segT) {
  return T / segT + nseq;
}
inline __host__ __device__ int64_t state_count(int64_t T, int64_t segT) { return T / segT + 1; }

// e^A_log, held finite: with an infinite rate the exponents of tokens that are
// not there would be NaN (0 times it); any step that is longer than 2^-115 ends
// every state at this one as well
__device__ __forceinline__ float sc_rate(float A_log) {
  const float r = expf(A_log);
  return r > 3.402823466e38f ? 3.402823466e38f : r;
}
// A token's exponent of 2 at least: nothing that float32 holds is left of a state
// that decays by 2^-4096, and a chunk's sum of such exponents has an exact hi
constexpr double kScLeast = -4096.0;

// A tile's token values in LDS.  The exponents c (base 2) are held as hi, a
// multiple of 1/16 (at most 2^19 of them are 128 tokens': exact in float32), and
// the rest lo: differences of two hi are exact, so that c_t - c_s keeps 2^-29 of
// near tokens even where c itself is in the hundreds.  (Aligned: hi, lo and dt are read
// four at a time.)
template <int Q>
struct alignas(16) Toks {
  float hi[Q], lo[Q];  // c_t log2(e)
  float dt[Q];         // dt'
  float ec[Q];         // e^{c_t}
  float eq[Q];         // e^{c_Q - c_t}
  float last;          // e^{c_Q}
};

template <bool F32>
__device__ __forceinline__ float tok_raw(const typename Zx<F32>::T* zx, int64_t Z, int nheads,
                                         int h, int t) {
  return Zx<F32>::at(zx + t * Z + (Z - nheads) + h);
}

// inclusive sums over the lanes by DPP moves (shifts inside 16 lanes, then the
// broadcasts of lane 15 and lane 31): a tenth of the latency of going through LDS
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, true);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double lanes_before_and_own_f64(double v) {
  v += dpp_f64<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8: zeros come in
  v += dpp_f64<0x112, 0xF>(v);
  v += dpp_f64<0x114, 0xF>(v);
  v += dpp_f64<0x118, 0xF>(v);
  v += dpp_f64<0x142, 0xA>(v);  // lane 15 of a row to the next row (rows 1 and 3)
  v += dpp_f64<0x143, 0xC>(v);  // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ double last_lane_f64(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 63);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

// 2^c, c <= 0: the integer part into the exponent, so that what is rounded to
// float32 before v_exp_f32 is at most 1/2 (a rounded c of -20 would be off by
// 2^-20, and these factors stand on whole states)
__device__ __forceinline__ float exp2_f64(double c) {
  const double n = __builtin_rint(c);
  return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f((float)(c - n)), n < -200.0 ? -200 : (int)n);
}

// one wave: Q / 64 consecutive tokens a lane, raw[] their dt + dt_bias;
// tokens from n on do nothing (dt' = 0)
template <int Q>
__device__ __forceinline__ void toks_make(Toks<Q>& k, const float (&raw)[Q / 64], int n,
                                          float rate) {
  constexpr int R = Q / 64;
  const int lane = threadIdx.x & 63;
  const double r2 = -(double)rate * 1.4426950408889634;
  double c[R], sum = 0.0;
  float dt[R];
#pragma unroll
  for (int q = 0; q < R; ++q) {
    dt[q] = lane * R + q < n ? mx_softplus(raw[q]) : 0.f;
    const double l = r2 * (double)dt[q];
    sum += l < kScLeast ? kScLeast : l;
    c[q] = sum;
  }
  const double inc = lanes_before_and_own_f64(sum);
  const double before = inc - sum, total = last_lane_f64(inc);
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int s = lane * R + q;
    const double cc = before + c[q];
    const float hi = (float)(__builtin_rint(cc * 16.0) * 0.0625);
    k.hi[s] = hi;
    k.lo[s] = (float)(cc - (double)hi);
    k.dt[s] = dt[q];
    k.ec[s] = exp2_f64(cc);
    k.eq[s] = exp2_f64(total - cc);
  }
  if (lane == 0) k.last = exp2_f64(total);
}

// eight values as bfloat16 terms (two at a time: three instructions a value and
// term, the pairs left where the matrix operand wants them)
template <int NT>
__device__ __forceinline__ void split8(const float (&v)[8], bf16x8 (&t)[NT]) {
  u32x4 w[NT];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int q = 0; q < NT; ++q) {
      const uint32_t p = bf_pack(a, b);
      w[q][i] = p;
      if (q + 1 < NT) a -= bf_lo(p), b -= bf_hi(p);
    }
  }
#pragma unroll
  for (int q = 0; q < NT; ++q) t[q] = as_bf16x8(w[q]);
}

// Operand of 16 columns (lane & 15) by 32 tokens out of token-major LDS rows,
// by two transpose reads: in each group of 16 lanes, lane j passes the address
// of 4 columns (4 (j % 4)) of row j / 4 and lane i receives column i of the
// four rows.  ra, rb: the rows of the lane group's first and second four.
__device__ __forceinline__ bf16x8 tr_op(const uint8_t* tile, int row_bytes, int ra, int rb,
                                        int col) {
  const int j = threadIdx.x & 15;
  const uint8_t* p = tile + 2 * (col + 4 * (j & 3));
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4*)(p + (ra + (j >> 2)) * row_bytes));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_s16x4*)(p + (rb + (j >> 2)) * row_bytes));
  bf16x8 r;
  const u32x2 ua = __builtin_bit_cast(u32x2, a), ub = __builtin_bit_cast(u32x2, b);
  r = __builtin_bit_cast(bf16x8, u32x4{ua.x, ua.y, ub.x, ub.y});
  return r;
}
// Operand of 16 rows (lane & 15) by 32 contiguous columns
__device__ __forceinline__ bf16x8 row_op(const uint8_t* tile, int row_bytes, int row, int col) {
  const int lane = threadIdx.x & 63;
  return as_bf16x8(ld16(tile + (row + (lane & 15)) * row_bytes + 2 * (col + 8 * (lane >> 4))));
}

}  // namespace tmk
