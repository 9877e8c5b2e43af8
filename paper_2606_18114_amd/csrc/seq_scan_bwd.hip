// Gradients of the selective scan (formulas of the scan: seq_scan_dev.hpp).
//
// With E the gradient that reaches the state at a chunk's end from later
// tokens, S0 the state before the chunk, m[t, s] = dy_t . x_s, g = C_t . B_s and
// L = e^{c_t - c_s} (s <= t):
//   dx_s = dt'_s (sum_t g L dy_t + e^{c_Q - c_s} E B_s) + D dy_s,
//   dB_s = sum_heads dt'_s (sum_t m L C_t + e^{c_Q - c_s} E^T x_s),
//   dC_t = sum_heads (sum_s m L dt'_s B_s + e^{c_t} S0^T dy_t),
//   E before the chunk = e^{c_Q} E + sum_t e^{c_t} dy_t C_t^T.
// The decay's exponent l_s lies on every path from a token before s to one at
// or behind it.  With the paths by where they begin and end,
//   qi_t = sum_{s < t} g L dt'_s m,  ki_s = dt'_s sum_{t > s} g L m  (inside the
//                                       chunk; s = t is on no l's path),
//   qo_t = e^{c_t} dy_t . S0 C_t,  ko_s = dt'_s e^{c_Q - c_s} x_s . E B_s,
//   pa = e^{c_Q} <E, S0>                                     (through it),
//   dl_s = sum_{t >= s} (qi_t - ki_t + qo_t) + sum_{s' < s} ko_s' + pa,
//   ddt'_s = g_ss m_ss + (ki_s + ko_s) / dt'_s - e^A_log dl_s,  dA_log = sum_s l_s dl_s.
// No sum runs over more than a chunk, so nothing cancels over a long sequence.
//
// Chunks of 128 tokens: S0 and E of every chunk and head come first
// (launch_scan_states, float32).  Then a workgroup of eight waves takes a chunk
// and a group of heads, so that dB and dC, which all heads share, add up in
// registers: scan_bwd_off_kernel everything with S0 and E that reaches a
// float32 gradient (three bfloat16 terms), scan_bwd_in_kernel what is inside
// the chunk, and dx.  scan_bwd_fin_kernel makes dt's gradient of the sums above.
#include "seq_scan_dev.hpp"

namespace tmk {

constexpr int kSbQ = 128;       // tokens of a chunk
constexpr int kSbThreads = 512;

// rows t0 .. t0 + 127 of 64 channels, two vectors of 16 bytes a thread
__device__ __forceinline__ void sb_load(u32x4 (&r)[2], const uint16_t* src, int64_t ld, int t0,
                                        int t1) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int t = t0 + q * 64 + ((int)threadIdx.x >> 3);
    r[q] = t < t1 ? ld16(src + t * ld + (threadIdx.x & 7) * 8) : u32x4{0, 0, 0, 0};
  }
}
__device__ __forceinline__ void sb_store(const u32x4 (&r)[2], uint8_t* dst) {
#pragma unroll
  for (int q = 0; q < 2; ++q)
    st16(dst + (q * 64 + ((int)threadIdx.x >> 3)) * kScRowP + (threadIdx.x & 7) * 16, r[q]);
}

// the heads of group blockIdx.y
__device__ __forceinline__ void sb_heads(int nheads, int& h0, int& h1) {
  const int per = (nheads + (int)gridDim.y - 1) / (int)gridDim.y;
  h0 = (int)blockIdx.y * per;
  h1 = min(nheads, h0 + per);
}

// The part of the chunk's outside.  Wave w owns states 16 w .. + 15: its slices
// of S0 and E go from memory straight to registers; dC^T and dB^T (rows states,
// columns tokens) add up over the heads in registers.
// part [groups][T][256] (dB, dC), qo, ko [slots][nheads][128] (ko without dt'),
// pa [slots][nheads]
template <bool F32>
__global__ __launch_bounds__(kSbThreads) void scan_bwd_off_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u,
    const uint16_t* __restrict__ dy, int T, int nheads, const int* __restrict__ off, int nseq,
    const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    const float* __restrict__ S0, const float* __restrict__ E, float* __restrict__ part,
    float* __restrict__ qo, float* __restrict__ ko, float* __restrict__ pa) {
  __shared__ __attribute__((aligned(16))) uint8_t xs[kSbQ * kScRowP], ys[kSbQ * kScRowP];
  __shared__ Toks<kSbQ> tk;
  __shared__ float qp[8][kSbQ], kp[8][kSbQ], pp[8];
  const int sl = blockIdx.x;
  const Slot s = slot_find(off, nseq, T, kSbQ, sl);
  if (s.t0 >= s.t1) return;
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
  const bool first = s.k == 0, last = s.t1 == s.en;
  int h0, h1;
  sb_heads(nheads, h0, h1);
  f32x4 dC[8], dB[8];
  u32x2 Cv[8], Bv[8];  // C and B of token 16 b + col, states 16 wave + 4 g .. + 3
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    dC[b] = dB[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int t = s.t0 + 16 * b + col;
    const uint16_t* p = u + (int64_t)t * cd + d + 16 * wave + 4 * g;
    Bv[b] = t < s.t1 ? *(const u32x2*)p : u32x2{0, 0};
    Cv[b] = t < s.t1 ? *(const u32x2*)(p + kSqN) : u32x2{0, 0};
  }
  auto dot4 = [](const f32x4& a, u32x2 w) {
    float v = a.x * bf_lo(w.x);
    v = __builtin_fmaf(a.y, bf_hi(w.x), v);
    v = __builtin_fmaf(a.z, bf_lo(w.y), v);
    return __builtin_fmaf(a.w, bf_hi(w.y), v);
  };
  auto over_g = [](float v) {  // over the four lane groups
    v += __uint_as_float(lane_xchg<16>(__float_as_uint(v)));
    return v + __uint_as_float(lane_xchg<32>(__float_as_uint(v)));
  };
  for (int h = h0; h < h1; ++h) {
    const int64_t sh = (int64_t)sl * nheads + h;
    u32x4 rx[2], ry[2];
    sb_load(rx, u + h * kSqP, cd, s.t0, s.t1);
    sb_load(ry, dy + h * kSqP, d, s.t0, s.t1);
    float a[2][8], e[2][8];  // S0 and E, channels 32 k + 8 g + j, state 16 wave + col
    const int64_t at = sh * kScState + 8 * g * kSqN + 16 * wave + col;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        a[k][j] = first ? 0.f : S0[at + (32 * k + j) * kSqN];
        e[k][j] = last ? 0.f : E[at + (32 * k + j) * kSqN];
      }
    if (wave == 0) {
      float raw[2];
#pragma unroll
      for (int q = 0; q < 2; ++q)
        raw[q] = tok_raw<F32>(zx, Z, nheads, h, min(s.t0 + 2 * lane + q, T - 1)) + dt_bias[h];
      toks_make<kSbQ>(tk, raw, s.t1 - s.t0, expf(A_log[h]));
    }
    sb_store(rx, xs);
    sb_store(ry, ys);
    float pv = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) pv = __builtin_fmaf(a[k][j], e[k][j], pv);
    pv = wave_sum(pv);
    if (lane == 0) pp[wave] = pv;
    bf16x8 as[2][3], es[2][3];
#pragma unroll
    for (int k = 0; k < 2; ++k) split8<3>(a[k], as[k]), split8<3>(e[k], es[k]);
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const int t = 16 * b + col;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (!first) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bf16x8 yo = row_op(ys, kScRowP, 16 * b, 32 * k);
#pragma unroll
          for (int q = 2; q >= 0; --q) v = mfma16(as[k][q], yo, v);
        }
        v *= tk.ec[t];
        dC[b] += v;
      }
      const float qv = over_g(dot4(v, Cv[b]));
      if (g == 0) qp[wave][t] = qv;
      v = f32x4{0.f, 0.f, 0.f, 0.f};
      if (!last) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const bf16x8 xo = row_op(xs, kScRowP, 16 * b, 32 * k);
#pragma unroll
          for (int q = 2; q >= 0; --q) v = mfma16(es[k][q], xo, v);
        }
        v *= tk.eq[t];
        dB[b] += v * tk.dt[t];
      }
      const float kv = over_g(dot4(v, Bv[b]));
      if (g == 0) kp[wave][t] = kv;
    }
    __syncthreads();
    if (threadIdx.x < 2 * kSbQ) {
      const int t = threadIdx.x & (kSbQ - 1);
      const float(*p)[kSbQ] = threadIdx.x < kSbQ ? qp : kp;
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += p[k][t];
      (threadIdx.x < kSbQ ? qo : ko)[sh * kSbQ + t] = v;
    } else if (threadIdx.x == 2 * kSbQ) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += pp[k];
      pa[sh] = v * tk.last;
    }
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const int t = s.t0 + 16 * b + col;
    if (t >= s.t1) continue;
    float* p = part + ((int64_t)blockIdx.y * T + t) * (2 * kSqN) + 16 * wave + 4 * g;
    *(f32x4*)p = dB[b];
    *(f32x4*)(p + kSqN) = dC[b];
  }
}

// The part inside the chunk, and dx.  Wave w makes, for tokens t = 16 w .. + 15
// with the s up to them, dC^T (rows states), and for tokens s = 16 w .. + 15 with
// the t from them on, dB^T and dx^T: nine blocks of 16 x 16 for every wave.  The
// blocks of m are made in both orientations, so that the lanes of a product hold
// what the next one takes of it.
template <bool F32>
__global__ __launch_bounds__(kSbThreads) void scan_bwd_in_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u,
    const uint16_t* __restrict__ dy, int T, int nheads, const int* __restrict__ off, int nseq,
    const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    const float* __restrict__ Dp, const float* __restrict__ E, float* __restrict__ part,
    float* __restrict__ qi, float* __restrict__ ki, float* __restrict__ kd,
    float* __restrict__ dd, uint16_t* __restrict__ du) {
  __shared__ __attribute__((aligned(16))) uint8_t Bs[kSbQ * kScRowN], Cs[kSbQ * kScRowN];
  __shared__ __attribute__((aligned(16))) uint8_t xs[kSbQ * kScRowP], ys[kSbQ * kScRowP];
  __shared__ __attribute__((aligned(16))) uint8_t El[2][kSqP * kScRowN];
  __shared__ Toks<kSbQ> tk;
  __shared__ float ddp[8];
  const int sl = blockIdx.x;
  const Slot s = slot_find(off, nseq, T, kSbQ, sl);
  if (s.t0 >= s.t1) return;
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, col = lane & 15;
  const bool last = s.t1 == s.en;
  int h0, h1;
  sb_heads(nheads, h0, h1);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = q * 32 + (tid >> 4), t = s.t0 + row;
    const uint16_t* p = u + (int64_t)t * cd + d + (tid & 15) * 8;
    st16(Bs + row * kScRowN + (tid & 15) * 16, t < s.t1 ? ld16(p) : u32x4{0, 0, 0, 0});
    st16(Cs + row * kScRowN + (tid & 15) * 16, t < s.t1 ? ld16(p + kSqN) : u32x4{0, 0, 0, 0});
  }
  f32x4 dC[8], dB[8];
#pragma unroll
  for (int b = 0; b < 8; ++b) dC[b] = dB[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int me = 16 * wave + col;  // this lane's token, as t and as s
  for (int h = h0; h < h1; ++h) {
    const int64_t sh = (int64_t)sl * nheads + h;
    u32x4 rx[2], ry[2];
    f32x4 re[4];
    sb_load(rx, u + h * kSqP, cd, s.t0, s.t1);
    sb_load(ry, dy + h * kSqP, d, s.t0, s.t1);
    if (!last)
#pragma unroll
      for (int q = 0; q < 4; ++q) re[q] = *(const f32x4*)(E + sh * kScState + (q * kSbThreads + tid) * 4);
    if (wave == 0) {
      float raw[2];
#pragma unroll
      for (int q = 0; q < 2; ++q)
        raw[q] = tok_raw<F32>(zx, Z, nheads, h, min(s.t0 + 2 * lane + q, T - 1)) + dt_bias[h];
      toks_make<kSbQ>(tk, raw, s.t1 - s.t0, expf(A_log[h]));
    }
    sb_store(rx, xs);
    sb_store(ry, ys);
    if (!last)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = (q * kSbThreads + tid) * 4;
        uint8_t* p = El[0] + (e / kSqN) * kScRowN + 2 * (e % kSqN);
        const uint32_t a0 = bf_pack(re[q].x, re[q].y), a1 = bf_pack(re[q].z, re[q].w);
        *(u32x2*)p = u32x2{a0, a1};
        *(u32x2*)(p + kSqP * kScRowN) = u32x2{bf_pack(re[q].x - bf_lo(a0), re[q].y - bf_hi(a0)),
                                              bf_pack(re[q].z - bf_lo(a1), re[q].w - bf_hi(a1))};
      }
    __syncthreads();
    const float mhi = tk.hi[me], mlo = tk.lo[me], mdt = tk.dt[me];
    // ---- tokens t = 16 wave + col, rows s ----
    {
      bf16x8 yo[2], co[4];
#pragma unroll
      for (int k = 0; k < 2; ++k) yo[k] = row_op(ys, kScRowP, 16 * wave, 32 * k);
#pragma unroll
      for (int k = 0; k < 4; ++k) co[k] = row_op(Cs, kScRowN, 16 * wave, 32 * k);
      float q = 0.f;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        if (2 * kb > wave) break;
        float v[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int sb = 2 * kb + half, s0 = 16 * sb + 4 * g;
          f32x4 m = {0.f, 0.f, 0.f, 0.f}, gg = m;
          if (sb <= wave) {
#pragma unroll
            for (int k = 0; k < 2; ++k) m = mfma16(row_op(xs, kScRowP, 16 * sb, 32 * k), yo[k], m);
#pragma unroll
            for (int k = 0; k < 4; ++k) gg = mfma16(row_op(Bs, kScRowN, 16 * sb, 32 * k), co[k], gg);
          }
          const f32x4 shi = *(const f32x4*)(tk.hi + s0), slo = *(const f32x4*)(tk.lo + s0),
                      sdt = *(const f32x4*)(tk.dt + s0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e = __builtin_amdgcn_exp2f((mhi - shi[i]) + (mlo - slo[i]));
            const float w = s0 + i <= me ? m[i] * e * sdt[i] : 0.f;
            v[4 * half + i] = w;
            q = __builtin_fmaf(gg[i], s0 + i < me ? w : 0.f, q);
          }
        }
        bf16x8 vt[2];
        split8<2>(v, vt);
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) {
          const bf16x8 bo = tr_op(Bs, kScRowN, 32 * kb + 4 * g, 32 * kb + 16 + 4 * g, 16 * nb);
          dC[nb] = mfma16(bo, vt[1], dC[nb]);
          dC[nb] = mfma16(bo, vt[0], dC[nb]);
        }
      }
      q += __uint_as_float(lane_xchg<16>(__float_as_uint(q)));
      q += __uint_as_float(lane_xchg<32>(__float_as_uint(q)));
      if (g == 0) qi[sh * kSbQ + me] = q;
    }
    // ---- tokens s = 16 wave + col, rows t ----
    {
      bf16x8 xo[2], bo[4];
#pragma unroll
      for (int k = 0; k < 2; ++k) xo[k] = row_op(xs, kScRowP, 16 * wave, 32 * k);
#pragma unroll
      for (int k = 0; k < 4; ++k) bo[k] = row_op(Bs, kScRowN, 16 * wave, 32 * k);
      f32x4 dx[4];
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        dx[pb] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!last) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            dx[pb] = mfma16(row_op(El[1], kScRowN, 16 * pb, 32 * k), bo[k], dx[pb]);
            dx[pb] = mfma16(row_op(El[0], kScRowN, 16 * pb, 32 * k), bo[k], dx[pb]);
          }
          dx[pb] *= tk.eq[me];
        }
      }
      float kk = 0.f, diag = 0.f, own = 0.f;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        if (2 * kb + 1 < wave) continue;
        float v[8], w[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int tb = 2 * kb + half, r0 = 16 * tb + 4 * g;
          f32x4 m = {0.f, 0.f, 0.f, 0.f}, gg = m;
          if (tb >= wave) {
#pragma unroll
            for (int k = 0; k < 2; ++k) m = mfma16(row_op(ys, kScRowP, 16 * tb, 32 * k), xo[k], m);
#pragma unroll
            for (int k = 0; k < 4; ++k) gg = mfma16(row_op(Cs, kScRowN, 16 * tb, 32 * k), bo[k], gg);
          }
          const f32x4 thi = *(const f32x4*)(tk.hi + r0), tlo = *(const f32x4*)(tk.lo + r0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float e = __builtin_amdgcn_exp2f((thi[i] - mhi) + (tlo[i] - mlo));
            const float ge = r0 + i >= me ? gg[i] * e : 0.f;
            w[4 * half + i] = ge;
            v[4 * half + i] = r0 + i >= me ? m[i] * e * mdt : 0.f;
            kk = __builtin_fmaf(r0 + i > me ? ge : 0.f, m[i], kk);
            if (r0 + i == me) diag = m[i], own = gg[i] * m[i];
          }
        }
        bf16x8 vt[2], wt[2];
        split8<2>(v, vt);
        split8<2>(w, wt);
        const int ra = 32 * kb + 4 * g, rb = ra + 16;
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) {
          const bf16x8 co = tr_op(Cs, kScRowN, ra, rb, 16 * nb);
          dB[nb] = mfma16(co, vt[1], dB[nb]);
          dB[nb] = mfma16(co, vt[0], dB[nb]);
        }
#pragma unroll
        for (int pb = 0; pb < 4; ++pb) {
          const bf16x8 yo = tr_op(ys, kScRowP, ra, rb, 16 * pb);
          dx[pb] = mfma16(yo, wt[1], dx[pb]);
          dx[pb] = mfma16(yo, wt[0], dx[pb]);
        }
      }
      kk += __uint_as_float(lane_xchg<16>(__float_as_uint(kk)));
      kk += __uint_as_float(lane_xchg<32>(__float_as_uint(kk)));
      if (g == 0) ki[sh * kSbQ + me] = kk;
      if (g == (col >> 2)) kd[sh * kSbQ + me] = own;
      diag = wave_sum(diag);
      if (lane == 0) ddp[wave] = diag;
      if (s.t0 + me < s.t1) {
        const float skip = Dp[h];
        uint16_t* o = du + (int64_t)(s.t0 + me) * cd + h * kSqP + 4 * g;
#pragma unroll
        for (int pb = 0; pb < 4; ++pb) {
          const u32x2 yw = *(const u32x2*)(ys + me * kScRowP + 2 * (16 * pb + 4 * g));
          const f32x4 a = dx[pb] * mdt;
          *(u32x2*)(o + 16 * pb) =
              u32x2{bf_pack(__builtin_fmaf(skip, bf_lo(yw.x), a.x), __builtin_fmaf(skip, bf_hi(yw.x), a.y)),
                    bf_pack(__builtin_fmaf(skip, bf_lo(yw.y), a.z), __builtin_fmaf(skip, bf_hi(yw.y), a.w))};
        }
      }
    }
    __syncthreads();
    if (tid == 0) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += ddp[k];
      dd[sh] = v;
    }
    // (ddp is written again behind the next head's first barrier)
  }
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    if (s.t0 + me >= s.t1) break;
    float* p = part + ((int64_t)blockIdx.y * T + s.t0 + me) * (2 * kSqN) + 16 * b + 4 * g;
    *(f32x4*)p = dB[b];
    *(f32x4*)(p + kSqN) = dC[b];
  }
}

// du's B and C columns: the sums over the head groups (both kernels'), in a
// fixed order.  grid (T), 256 threads
__global__ __launch_bounds__(256) void scan_bwd_bc_kernel(const float* __restrict__ part,
                                                          int groups, int T, int nheads,
                                                          const int* __restrict__ off, int nseq,
                                                          uint16_t* __restrict__ du) {
  const int t = blockIdx.x;
  if (seq_find(off, nseq, T, t).i < 0) return;
  float v = 0.f;
  for (int k = 0; k < groups; ++k) v += part[((int64_t)k * T + t) * (2 * kSqN) + threadIdx.x];
  const int d = nheads * kSqP;
  du[(int64_t)t * (d + 2 * kSqN) + d + threadIdx.x] = bf_rne(v);
}

// A wave a chunk and head, two tokens a lane: dl, dt's gradient, and the
// chunk's sums for dt_bias, A_log and D (sums [slots][3][nheads]).
// grid (slots, ceil(nheads / 4)), 256 threads
template <bool F32>
__global__ __launch_bounds__(256) void scan_bwd_fin_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int T, int nheads, const int* __restrict__ off,
    int nseq, const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    const float* __restrict__ qi, const float* __restrict__ ki, const float* __restrict__ kd,
    const float* __restrict__ qo, const float* __restrict__ ko, const float* __restrict__ pa, const float* __restrict__ dd,
    typename Zx<F32>::T* __restrict__ dzx, float* __restrict__ sums) {
  const int sl = blockIdx.x, h = (int)blockIdx.y * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (h >= nheads) return;
  const Slot s = slot_find(off, nseq, T, kSbQ, sl);
  float* o = sums + (int64_t)sl * 3 * nheads + h;
  if (s.t0 >= s.t1) {
    if (lane < 3) o[lane * nheads] = 0.f;
    return;
  }
  const int d = nheads * kSqP;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads, sh = (int64_t)sl * nheads + h;
  const float rate = expf(A_log[h]), bias = dt_bias[h];
  float raw[2], dt[2], kin[2], kout[2], own[2];
  double a[2], b[2];  // what the sums over t >= s and over s' < s take
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int i = 2 * lane + q;
    const bool in = s.t0 + i < s.t1;
    raw[q] = tok_raw<F32>(zx, Z, nheads, h, min(s.t0 + i, T - 1)) + bias;
    dt[q] = in ? mx_softplus(raw[q]) : 0.f;
    kin[q] = in ? ki[sh * kSbQ + i] : 0.f;
    kout[q] = in ? ko[sh * kSbQ + i] : 0.f;
    own[q] = in ? kd[sh * kSbQ + i] : 0.f;
    a[q] = in ? (double)qi[sh * kSbQ + i] - (double)dt[q] * kin[q] + (double)qo[sh * kSbQ + i] : 0.0;
    b[q] = (double)dt[q] * kout[q];
  }
  double ai = a[0] + a[1], bi = b[0] + b[1];  // from this lane up, up to this lane
  const double a2 = ai, b2 = bi;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const double x = __shfl_down(ai, k, 64), y = __shfl_up(bi, k, 64);
    if (lane + k < 64) ai += x;
    if (lane >= k) bi += y;
  }
  const double above = ai - a2, before = bi - b2, through = pa[sh];
  const double dl[2] = {above + a[1] + a[0] + before + through,
                        above + a[1] + before + b[0] + through};
  float sb = 0.f, sa = 0.f;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int t = s.t0 + 2 * lane + q;
    if (t >= s.t1) break;
    const float ds = (float)((double)own[q] + kin[q] + kout[q] - (double)rate * dl[q]);
    const float v = ds / (1.f + expf(-raw[q]));
    Zx<F32>::put(dzx + t * Z + (Z - nheads) + h, v);
    sb += v;
    sa -= dt[q] * rate * (float)dl[q];
  }
  sb = wave_sum(sb);
  sa = wave_sum(sa);
  if (lane == 0) {
    o[0] = sb;
    o[nheads] = sa;
    o[2 * nheads] = dd[sh];
  }
}

// column c of sums [rows][3 nheads] over the rows, 16 chains, to the three outputs
__global__ __launch_bounds__(1024) void scan_bwd_sum_kernel(const float* __restrict__ sums,
                                                            int64_t rows, int nheads,
                                                            float* __restrict__ ddt_bias,
                                                            float* __restrict__ dA_log,
                                                            float* __restrict__ dD) {
  __shared__ float p[16][64];
  const int lane = threadIdx.x & 63, chain = threadIdx.x >> 6;
  const int64_t cols = (int64_t)3 * nheads, c = (int64_t)blockIdx.x * 64 + lane;
  float v = 0.f;
  if (c < cols)
    for (int64_t r = chain; r < rows; r += 16) v += sums[r * cols + c];
  p[chain][lane] = v;
  __syncthreads();
  if (chain != 0 || c >= cols) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) v += p[k][lane];
  const int q = (int)(c / nheads), h = (int)(c - (int64_t)q * nheads);
  (q == 0 ? ddt_bias : q == 1 ? dA_log : dD)[h] = v;
}

// groups of heads: two rounds of workgroups over the chip's CUs, more only
// makes more partial sums of dB and dC (1 KiB a token and group, twice)
static int sb_groups(int64_t slots, int64_t nheads) {
  const int64_t n = (512 + slots - 1) / slots;
  return (int)(n > nheads ? nheads : n);
}

struct ScanBwdWs {
  float *S0, *E, *dec0, *dec1, *qi, *ki, *kd, *qo, *ko, *pa, *dd, *sums, *part;
  int64_t bytes;
};
static ScanBwdWs sb_ws(void* p, int64_t T, int64_t nseq, int64_t nheads) {
  const int64_t slots = slot_count(T, nseq, kSbQ), sh = slots * nheads;
  ScanBwdWs w;
  float* f = (float*)p;
  auto take = [&](int64_t n) {
    float* r = f;
    f += (n + 63) / 64 * 64;
    return r;
  };
  w.S0 = take(sh * kScState);
  w.E = take(sh * kScState);
  w.dec0 = take(sh), w.dec1 = take(sh);
  w.qi = take(sh * kSbQ), w.ki = take(sh * kSbQ), w.kd = take(sh * kSbQ), w.qo = take(sh * kSbQ), w.ko = take(sh * kSbQ);
  w.pa = take(sh), w.dd = take(sh);
  w.sums = take(3 * sh);
  w.part = take(2 * sb_groups(slots, nheads) * T * 2 * kSqN);
  w.bytes = (int64_t)((uintptr_t)f - (uintptr_t)p);
  return w;
}

int64_t seq_scan_bwd_bytes(int64_t T, int64_t nseq, int64_t nheads) {
  return sb_ws(nullptr, T, nseq, nheads).bytes;
}

template <bool F32>
static hipError_t scan_bwd_go(const SeqIn& in, const uint16_t* u, const float* dt_bias,
                              const float* A_log, const float* D, const uint16_t* dy, void* dzx,
                              uint16_t* du, float* ddt_bias, float* dA_log, float* dD,
                              void* workspace, hipStream_t stream) {
  typedef typename Zx<F32>::T X;
  const X* zx = (const X*)in.zx;
  const ScanBwdWs w = sb_ws(workspace, in.T, in.nseq, in.nheads);
  const int64_t slots = slot_count(in.T, in.nseq, kSbQ);
  const int groups = sb_groups(slots, in.nheads);
  hipError_t e = launch_scan_states(in, u, nullptr, false, 3, kSbQ, dt_bias, A_log, nullptr, w.S0,
                                    w.dec0, stream);
  if (e != hipSuccess) return e;
  e = launch_scan_states(in, u, dy, true, 3, kSbQ, dt_bias, A_log, nullptr, w.E, w.dec1, stream);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)slots, (unsigned)groups);
  float* part2 = w.part + (int64_t)groups * in.T * 2 * kSqN;
  hipLaunchKernelGGL(scan_bwd_off_kernel<F32>, grid, dim3(kSbThreads), 0, stream, zx, u, dy, in.T,
                     in.nheads, in.offsets, in.nseq, dt_bias, A_log, w.S0, w.E, w.part, w.qo, w.ko,
                     w.pa);
  hipLaunchKernelGGL(scan_bwd_in_kernel<F32>, grid, dim3(kSbThreads), 0, stream, zx, u, dy, in.T,
                     in.nheads, in.offsets, in.nseq, dt_bias, A_log, D, w.E, part2, w.qi, w.ki,
                     w.kd, w.dd, du);
  hipLaunchKernelGGL(scan_bwd_bc_kernel, dim3((unsigned)in.T), dim3(256), 0, stream, w.part,
                     2 * groups, in.T, in.nheads, in.offsets, in.nseq, du);
  hipLaunchKernelGGL(scan_bwd_fin_kernel<F32>, dim3((unsigned)slots, (unsigned)((in.nheads + 3) / 4)),
                     dim3(256), 0, stream, zx, in.T, in.nheads, in.offsets, in.nseq, dt_bias,
                     A_log, w.qi, w.ki, w.kd, w.qo, w.ko, w.pa, w.dd, (X*)dzx, w.sums);
  hipLaunchKernelGGL(scan_bwd_sum_kernel, dim3((unsigned)((3 * in.nheads + 63) / 64)), dim3(1024),
                     0, stream, w.sums, slots, in.nheads, ddt_bias, dA_log, dD);
  return hipGetLastError();
}

hipError_t launch_seq_scan_bwd(const SeqIn& in, const uint16_t* u, const float* dt_bias,
                               const float* A_log, const float* D, const uint16_t* dy, void* dzx,
                               uint16_t* du, float* ddt_bias, float* dA_log, float* dD,
                               void* workspace, hipStream_t stream) {
  return in.f32 ? scan_bwd_go<true>(in, u, dt_bias, A_log, D, dy, dzx, du, ddt_bias, dA_log, dD,
                                    workspace, stream)
                : scan_bwd_go<false>(in, u, dt_bias, A_log, D, dy, dzx, du, ddt_bias, dA_log, dD,
                                     workspace, stream);
}

}  // namespace tmk
