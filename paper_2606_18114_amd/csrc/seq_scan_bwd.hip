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
//   qi_t = sum_s g L m dt'_s,  ki_s = sum_t g L m dt'_s      (inside the chunk),
//   qo_t = e^{c_t} dy_t . S0 C_t,  ko_s = dt'_s e^{c_Q - c_s} x_s . E B_s,
//   pa = e^{c_Q} <E, S0>                                     (through it),
//   dl_s = sum_{t >= s} (qi_t - ki_t + qo_t) + sum_{s' < s} ko_s' + pa,
//   ddt'_s = sum_t g L m + ko_s / dt'_s - e^A_log dl_s,  dA_log = sum_s l_s dl_s.
// No sum runs over more than a chunk, so nothing cancels over a long sequence.
// Inside the chunk the pairs with s and t on the same side of l cancel between
// qi and ki: both are sums, in float64, of the same float32 numbers g (m L dt'_s)
// (with each sum's own float32 roundings dA_log and ddt_bias, sums of many
// dl, were off by 2 to 3e-6).
//
// Chunks of 128 tokens: S0 and E of every chunk and head come first
// (launch_chunk_states, float32).  Then a workgroup takes a chunk and a group of
// heads, so that dB and dC, which all heads share, add up in registers:
// scan_bwd_off_kernel everything with S0 and E that reaches a float32 gradient
// (three bfloat16 terms), scan_bwd_to_kernel and scan_bwd_from_kernel what is
// inside the chunk, for its targets t and its sources s (with dx).  Blocks of m
// are made in both orientations, so that the lanes of a product hold what the
// next one takes of it.  scan_bwd_fin_kernel makes dt's gradient of the sums above.
//
// 16384 tokens of 64 heads, eight sequences: states 102 + 77 us each way (0.94 GB
// written, read and written again), off 325 (1.1 to 1.4 GB), to 180, from 270
// (0.7 GB), bc 37, fin 21.  The float32 states of the chunks, half a gigabyte, are
// most of the traffic; shorter ones would be more of it, longer ones more work
// inside the chunk, which grows with its length.
#include "seq_scan_dev.hpp"

namespace tmk {

constexpr int kSbQ = kScChunk;
constexpr int kSbThreads = 512;

// rows t0 .. t0 + 127 of 64 channels in 16-byte vectors, 1024 / THREADS a thread.
// No load here is under a condition (the compiler would wait for every one before
// it): behind the last token it is read again, and zeros are put in its place.
template <int THREADS>
struct SbTile {
  u32x4 r[1024 / THREADS];
  __device__ __forceinline__ void load(const uint16_t* src, int64_t ld, int t0, int t1) {
#pragma unroll
    for (int q = 0; q < 1024 / THREADS; ++q) {
      const int t = min(t0 + q * (THREADS / 8) + ((int)threadIdx.x >> 3), t1 - 1);
      r[q] = ld16(src + t * ld + (threadIdx.x & 7) * 8);
    }
  }
  __device__ __forceinline__ void store(uint8_t* dst, int n) const {  // n: tokens
    const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 1024 / THREADS; ++q) {
      const int row = q * (THREADS / 8) + ((int)threadIdx.x >> 3);
      st16(dst + row * kScRowP + (threadIdx.x & 7) * 16, row < n ? r[q] : zero);
    }
  }
};
// the chunk's B or C rows (128 states) into LDS, by kSbThreads threads
__device__ __forceinline__ void sb_rows(const uint16_t* src, int64_t ld, int t0, int t1,
                                        uint8_t* dst) {
  u32x4 r[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t t = min(t0 + q * 32 + ((int)threadIdx.x >> 4), t1 - 1);
    r[q] = ld16(src + t * ld + (threadIdx.x & 15) * 8);
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = q * 32 + ((int)threadIdx.x >> 4);
    st16(dst + row * kScRowN + (threadIdx.x & 15) * 16,
         t0 + row < t1 ? r[q] : u32x4{0, 0, 0, 0});
  }
}
// operands of one token a lane, straight from memory: K of 32 columns
template <int K>
__device__ __forceinline__ void sb_own(bf16x8 (&o)[K], const uint16_t* row) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int k = 0; k < K; ++k) o[k] = as_bf16x8(ld16(row + 32 * k + 8 * g));
}
// a chunk's token values, by one wave; raw loaded a head earlier
template <bool F32>
struct SbToks {
  float raw[2], rate;
  __device__ __forceinline__ void load(const typename Zx<F32>::T* zx, int64_t Z, int nheads, int h,
                                       int t0, int T, const float* dt_bias, const float* A_log) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      raw[q] = tok_raw<F32>(zx, Z, nheads, h, min(t0 + 2 * lane + q, T - 1)) + dt_bias[h];
    rate = sc_rate(A_log[h]);
  }
  __device__ __forceinline__ void make(Toks<kSbQ>& tk, int n) const {
    toks_make<kSbQ>(tk, raw, n, rate);
  }
};

// the heads of a group
__device__ __forceinline__ void sb_heads(int nheads, int group, int groups, int& h0, int& h1) {
  const int per = (nheads + groups - 1) / groups;
  h0 = group * per;
  h1 = min(nheads, h0 + per);
}
// 16-token block of wave w: the blocks of the two waves of a SIMD (w and w + 4)
// add up to the same work
__device__ __forceinline__ int sb_block(int w) { return w < 4 ? w : 11 - w; }
__device__ __forceinline__ float over_groups(float v) {
  v += __uint_as_float(lane_xchg<16>(__float_as_uint(v)));
  return v + __uint_as_float(lane_xchg<32>(__float_as_uint(v)));
}

// The part of the chunk's outside, a quarter a workgroup of four waves: side 0
// makes dC and qo of S0 and dy, 1 dB and ko of E and x, for one half of the
// states, 16 a wave.  The quarters of a chunk and head group read the same values
// and run on one XCD, next to each other.  A wave's slice of S0 or E goes
// from memory straight to registers; dC^T or dB^T (rows states, columns tokens)
// add up over the heads there.  The next head's values are on their way
// meanwhile, and wave 0 makes its token values.
// part [groups][T][256] (dB, dC); dots [2 halves][2: qo, ko without dt'][nheads][T],
// pa [2 halves][slots][nheads]
template <bool F32>
__global__ __launch_bounds__(256, 2) void scan_bwd_off_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u,
    const uint16_t* __restrict__ dy, int T, int nheads, const int* __restrict__ off, int nseq,
    const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    const float* __restrict__ S0, const float* __restrict__ E, float* __restrict__ part,
    float* __restrict__ dots, float* __restrict__ pa, int slots, int groups) {
  __shared__ __attribute__((aligned(16))) uint8_t vs[kSbQ * kScRowP];  // dy or x
  __shared__ Toks<kSbQ> tks[2];
  __shared__ float dw[4][kSbQ], pp[4];
  // workgroup i runs on XCD i % 8
  const uint32_t pair = (blockIdx.x >> 5) * 8 + (blockIdx.x & 7);  // slot and group
  if (pair >= (uint32_t)slots * groups) return;
  const int side = (blockIdx.x >> 3) & 1, half = (blockIdx.x >> 4) & 1;
  const int grp = (int)(pair / (uint32_t)slots), sl = (int)(pair - (uint32_t)grp * slots);
  const Slot s = slot_find(off, nseq, T, kSbQ, sl);
  if (s.t0 >= s.t1) return;
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = 64 * half + 16 * wave;  // the wave's states
  const bool first = s.k == 0, last = s.t1 == s.en;
  const bool none = side ? last : first;  // the slice is zero
  int h0, h1;
  sb_heads(nheads, grp, groups, h0, h1);
  f32x4 acc[8];
  u32x2 dv[8];  // C or B of token 16 b + col, states n0 + 4 g .. + 3
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t t = min(s.t0 + 16 * b + col, s.t1 - 1);
    dv[b] = *(const u32x2*)(u + t * cd + d + (side ? 0 : kSqN) + n0 + 4 * g);
  }
  const uint16_t* vec = side ? u : dy;
  const int64_t ldv = side ? cd : d;
  const float* slice = side ? E : S0;
  SbTile<256> tile;
  float a[2][8];  // the slice: channels 32 k + 8 g + j, state n0 + col
  SbToks<F32> st;
  const int at = 8 * g * kSqN + n0 + col;
  // the places of the states before and behind the chunk
  const int64_t behind = sl - s.i, before = max(sl - s.i - 1, 0);
  auto load = [&](int h) {
    tile.load(vec + h * kSqP, ldv, s.t0, s.t1);
    // (a slice that is zero has no place; what is loaded is not used)
    const float* p = slice + ((side ? behind : before) * nheads + h) * kScState;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) a[k][j] = p[at + (32 * k + j) * kSqN];
  };
  auto toks = [&](int h) { st.load(zx, Z, nheads, h, s.t0, T, dt_bias, A_log); };
  if (h0 < h1) {
    load(h0);
    if (wave == 0) {
      toks(h0);
      st.make(tks[0], s.t1 - s.t0);
      if (h0 + 1 < h1) toks(h0 + 1);
    }
  }
  int buf = 0;
  for (int h = h0; h < h1; ++h, buf ^= 1) {
    const int64_t sh = (int64_t)sl * nheads + h;
    tile.store(vs, s.t1 - s.t0);
    if (side == 0) {  // <E, S0> of the slice
      float pv = 0.f;
      if (!first && !last) {
        const float* e = E + (behind * nheads + h) * kScState;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < 8; ++j) pv = __builtin_fmaf(a[k][j], e[at + (32 * k + j) * kSqN], pv);
        pv = wave_sum(pv);
      }
      if (lane == 0) pp[wave] = pv;
    }
    bf16x8 as[2][3];
#pragma unroll
    for (int k = 0; k < 2; ++k) split8<3>(a[k], as[k]);
    __syncthreads();
    const Toks<kSbQ>& tk = tks[buf];
    if (h + 1 < h1) {
      load(h + 1);
      if (wave == 0) {
        st.make(tks[buf ^ 1], s.t1 - s.t0);
        if (h + 2 < h1) toks(h + 2);
      }
    }
    if (none) {
#pragma unroll
      for (int b = 0; b < 8; ++b)
        if (g == 0) dw[wave][16 * b + col] = 0.f;
    } else {
      bf16x8 vo[2][4];  // two blocks of tokens, two steps of 32 channels
      auto fetch = [&](int bb) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          vo[bb & 1][q] = row_op(vs, kScRowP, 32 * bb + 16 * (q >> 1), 32 * (q & 1));
      };
      fetch(0);
#pragma unroll
      for (int bb = 0; bb < 4; ++bb) {
        if (bb < 3) fetch(bb + 1);
        __builtin_amdgcn_sched_barrier(0);
        f32x4 v[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int q = 2; q >= 0; --q)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] = mfma16(as[k][q], vo[bb & 1][2 * i + k], v[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int b = 2 * bb + i, t = 16 * b + col;
          const float f = side ? tk.eq[t] : tk.ec[t];
          v[i] *= f;
          if (side) acc[b] += v[i] * tk.dt[t];
          else acc[b] += v[i];
          float x = v[i].x * bf_lo(dv[b].x);
          x = __builtin_fmaf(v[i].y, bf_hi(dv[b].x), x);
          x = __builtin_fmaf(v[i].z, bf_lo(dv[b].y), x);
          x = over_groups(__builtin_fmaf(v[i].w, bf_hi(dv[b].y), x));
          if (g == 0) dw[wave][t] = x;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();
    if (threadIdx.x < kSbQ) {
      const int t = threadIdx.x;
      if (s.t0 + t < s.t1)
        dots[((int64_t)(half * 2 + side) * nheads + h) * T + s.t0 + t] =
            (dw[0][t] + dw[1][t]) + (dw[2][t] + dw[3][t]);
    } else if (threadIdx.x == kSbQ && side == 0) {
      pa[(int64_t)half * slots * nheads + sh] = ((pp[0] + pp[1]) + (pp[2] + pp[3])) * tk.last;
    }
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const int t = s.t0 + 16 * b + col;
    if (t < s.t1)
      *(f32x4*)(part + ((int64_t)grp * T + t) * (2 * kSqN) + (side ? 0 : kSqN) + n0 + 4 * g) =
          acc[b];
  }
}

// Inside the chunk, by target: wave w makes dC^T (rows states) and qi of the
// tokens t of its block with the s up to them.
template <bool F32>
__global__ __launch_bounds__(kSbThreads, 4) void scan_bwd_to_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u,
    const uint16_t* __restrict__ dy, int T, int nheads, const int* __restrict__ off, int nseq,
    const float* __restrict__ dt_bias, const float* __restrict__ A_log, float* __restrict__ part,
    double* __restrict__ qi) {
  __shared__ __attribute__((aligned(16))) uint8_t Bs[kSbQ * kScRowN], xs[kSbQ * kScRowP];
  __shared__ Toks<kSbQ> tks[2];
  const int sl = blockIdx.x;
  const Slot s = slot_find(off, nseq, T, kSbQ, sl);
  if (s.t0 >= s.t1) return;
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wb = sb_block(w);
  int h0, h1;
  sb_heads(nheads, blockIdx.y, gridDim.y, h0, h1);
  const int me = 16 * wb + col, tm = s.t0 + me;  // this lane's token
  // (behind the chunk's last one it works on that one's values, and stores nothing)
  const int64_t tc = min(tm, s.t1 - 1);
  sb_rows(u + d, cd, s.t0, s.t1, Bs);
  bf16x8 co[4];
  sb_own<4>(co, u + tc * cd + d + kSqN);
  f32x4 acc[8];
#pragma unroll
  for (int b = 0; b < 8; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  SbToks<F32> st;
  auto toks = [&](int h) { st.load(zx, Z, nheads, h, s.t0, T, dt_bias, A_log); };
  if (w == 0 && h0 < h1) {
    toks(h0);
    st.make(tks[0], s.t1 - s.t0);
    if (h0 + 1 < h1) toks(h0 + 1);
  }
  int buf = 0;
  for (int h = h0; h < h1; ++h, buf ^= 1) {
    // (no values ahead of the head: two workgroups share a CU, 128 registers a lane)
    bf16x8 yo[2];
    SbTile<kSbThreads> tile;
    tile.load(u + h * kSqP, cd, s.t0, s.t1);
    sb_own<2>(yo, dy + tc * d + h * kSqP);
    tile.store(xs, s.t1 - s.t0);
    __syncthreads();
    const Toks<kSbQ>& tk = tks[buf];
    if (w == 0 && h + 1 < h1) {
      st.make(tks[buf ^ 1], s.t1 - s.t0);
      if (h + 2 < h1) toks(h + 2);
    }
    const float mhi = tk.hi[me], mlo = tk.lo[me];
    double q = 0.0;
    // (not unrolled: its four steps' addresses would not stay in registers)
#pragma clang loop unroll(disable)
    for (int kb = 0; 2 * kb <= wb; ++kb) {
      float v[8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int sb = 2 * kb + half, s0 = 16 * sb + 4 * g;
        f32x4 m = {0.f, 0.f, 0.f, 0.f}, gg = m;
        if (sb <= wb) {
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
          const float a = s0 + i <= me ? m[i] * e * sdt[i] : 0.f;
          v[4 * half + i] = a;
          q += (double)(gg[i] * a);
        }
      }
      bf16x8 vt[2];
      split8<2>(v, vt);
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) {
        const bf16x8 bo = tr_op(Bs, kScRowN, 32 * kb + 4 * g, 32 * kb + 16 + 4 * g, 16 * nb);
        acc[nb] = mfma16(bo, vt[1], acc[nb]);
        acc[nb] = mfma16(bo, vt[0], acc[nb]);
      }
    }
    q += lane_xchg_f64<16>(q);
    q += lane_xchg_f64<32>(q);
    if (g == 0 && tm < s.t1) qi[(int64_t)h * T + tm] = q;
    __syncthreads();
  }
  if (tm < s.t1) {
    float* p = part + ((int64_t)blockIdx.y * T + tm) * (2 * kSqN) + kSqN + 4 * g;
#pragma unroll
    for (int b = 0; b < 8; ++b) *(f32x4*)(p + 16 * b) = acc[b];
  }
}

// Inside the chunk, by source: wave w makes dB^T, dx^T (with E's part) and ki of
// the tokens s of its block with the t from them on.
template <bool F32>
__global__ __launch_bounds__(kSbThreads, 2) void scan_bwd_from_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u,
    const uint16_t* __restrict__ dy, int T, int nheads, const int* __restrict__ off, int nseq,
    const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    const float* __restrict__ Dp, const float* __restrict__ E, float* __restrict__ part,
    double* __restrict__ ki, float* __restrict__ kd, float* __restrict__ dd,
    uint16_t* __restrict__ du) {
  __shared__ __attribute__((aligned(16))) uint8_t Cs[kSbQ * kScRowN], ys[kSbQ * kScRowP];
  __shared__ __attribute__((aligned(16))) uint8_t El[2][kSqP * kScRowS];
  __shared__ Toks<kSbQ> tks[2];
  __shared__ float ddp[8];
  const int sl = blockIdx.x;
  const Slot s = slot_find(off, nseq, T, kSbQ, sl);
  if (s.t0 >= s.t1) return;
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, col = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wb = sb_block(w);
  const bool last = s.t1 == s.en;
  int h0, h1;
  sb_heads(nheads, blockIdx.y, gridDim.y, h0, h1);
  const int me = 16 * wb + col, tm = s.t0 + me;  // this lane's token
  // (behind the chunk's last one it works on that one's values, and stores nothing)
  const int64_t tc = min(tm, s.t1 - 1);
  sb_rows(u + d + kSqN, cd, s.t0, s.t1, Cs);
  bf16x8 bo[4], xn[2];
  sb_own<4>(bo, u + tc * cd + d);
  f32x4 acc[8];
#pragma unroll
  for (int b = 0; b < 8; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  SbTile<kSbThreads> tile;
  f32x4 re[4];
  SbToks<F32> st;
  auto load = [&](int h) {
    tile.load(dy + h * kSqP, d, s.t0, s.t1);
    sb_own<2>(xn, u + tc * cd + h * kSqP);
    if (!last)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        re[q] = *(const f32x4*)(E + ((int64_t)(sl - s.i) * nheads + h) * kScState +
                                (q * kSbThreads + tid) * 4);
  };
  auto toks = [&](int h) { st.load(zx, Z, nheads, h, s.t0, T, dt_bias, A_log); };
  constexpr int kTokWave = 4;  // block 7: one block of t
  if (h0 < h1) {
    load(h0);
    if (w == kTokWave) {
      toks(h0);
      st.make(tks[0], s.t1 - s.t0);
      if (h0 + 1 < h1) toks(h0 + 1);
    }
  }
  int buf = 0;
  for (int h = h0; h < h1; ++h, buf ^= 1) {
    const int64_t sh = (int64_t)sl * nheads + h;
    tile.store(ys, s.t1 - s.t0);
    const bf16x8 xo[2] = {xn[0], xn[1]};
    if (!last)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = (q * kSbThreads + tid) * 4;
        uint8_t* p = El[0] + (e / kSqN) * kScRowS + 2 * (e % kSqN);
        const uint32_t a0 = bf_pack(re[q].x, re[q].y), a1 = bf_pack(re[q].z, re[q].w);
        *(u32x2*)p = u32x2{a0, a1};
        *(u32x2*)(p + kSqP * kScRowS) = u32x2{bf_pack(re[q].x - bf_lo(a0), re[q].y - bf_hi(a0)),
                                              bf_pack(re[q].z - bf_lo(a1), re[q].w - bf_hi(a1))};
      }
    __syncthreads();
    const Toks<kSbQ>& tk = tks[buf];
    if (h + 1 < h1) {
      load(h + 1);
      if (w == kTokWave) {
        st.make(tks[buf ^ 1], s.t1 - s.t0);
        if (h + 2 < h1) toks(h + 2);
      }
    }
    const float mhi = tk.hi[me], mlo = tk.lo[me], mdt = tk.dt[me];
    f32x4 dx[4];
#pragma unroll
    for (int pb = 0; pb < 4; ++pb) dx[pb] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!last) {
      bf16x8 ef[2][4][2];
      auto fetch = [&](int k) {
#pragma unroll
        for (int pb = 0; pb < 4; ++pb)
#pragma unroll
          for (int q = 0; q < 2; ++q) ef[k & 1][pb][q] = row_op(El[q], kScRowS, 16 * pb, 32 * k);
      };
      fetch(0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k < 3) fetch(k + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 1; q >= 0; --q)
#pragma unroll
          for (int pb = 0; pb < 4; ++pb) dx[pb] = mfma16(ef[k & 1][pb][q], bo[k], dx[pb]);
        __builtin_amdgcn_sched_barrier(0);
      }
      const float eq = tk.eq[me];
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) dx[pb] *= eq;
    }
    double kk = 0.0;
    float diag = 0.f, own = 0.f;
#pragma clang loop unroll(disable)
    for (int kb = wb >> 1; kb < 4; ++kb) {
      f32x4 m[2], gg[2];
      {
        bf16x8 yo[2][2], co[2][4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int k = 0; k < 2; ++k) yo[half][k] = row_op(ys, kScRowP, 32 * kb + 16 * half, 32 * k);
#pragma unroll
          for (int k = 0; k < 4; ++k) co[half][k] = row_op(Cs, kScRowN, 32 * kb + 16 * half, 32 * k);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int half = 0; half < 2; ++half) m[half] = gg[half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int half = 0; half < 2; ++half) m[half] = mfma16(yo[half][k], xo[k], m[half]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int half = 0; half < 2; ++half) gg[half] = mfma16(co[half][k], bo[k], gg[half]);
      }
      const int ra = 32 * kb + 4 * g, rb = ra + 16;
      bf16x8 yt[4], ct[8];
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) yt[pb] = tr_op(ys, kScRowP, ra, rb, 16 * pb);
#pragma unroll
      for (int nb = 0; nb < 8; ++nb) ct[nb] = tr_op(Cs, kScRowN, ra, rb, 16 * nb);
      __builtin_amdgcn_sched_barrier(0);
      float v[8], wv[8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int tb = 2 * kb + half, r0 = 16 * tb + 4 * g;
        const f32x4 thi = *(const f32x4*)(tk.hi + r0), tlo = *(const f32x4*)(tk.lo + r0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f((thi[i] - mhi) + (tlo[i] - mlo));
          const float a = r0 + i >= me ? m[half][i] * e * mdt : 0.f;
          const float b = r0 + i >= me ? gg[half][i] * e : 0.f;
          v[4 * half + i] = a;
          wv[4 * half + i] = b;
          kk += (double)(gg[half][i] * a);
          own = __builtin_fmaf(b, m[half][i], own);
        }
        if (tb == wb)
#pragma unroll
          for (int i = 0; i < 4; ++i) diag += r0 + i == me ? m[half][i] : 0.f;
      }
      bf16x8 vt[2], wt[2];
      split8<2>(wv, wt);
      split8<2>(v, vt);
#pragma unroll
      for (int r = 1; r >= 0; --r)
#pragma unroll
        for (int pb = 0; pb < 4; ++pb) dx[pb] = mfma16(yt[pb], wt[r], dx[pb]);
#pragma unroll
      for (int r = 1; r >= 0; --r)
#pragma unroll
        for (int nb = 0; nb < 8; ++nb) acc[nb] = mfma16(ct[nb], vt[r], acc[nb]);
    }
    kk += lane_xchg_f64<16>(kk);
    kk += lane_xchg_f64<32>(kk);
    if (g == 0 && tm < s.t1) ki[(int64_t)h * T + tm] = kk;
    own = over_groups(own);
    if (g == 0 && tm < s.t1) kd[(int64_t)h * T + tm] = own;
    diag = wave_sum(diag);
    if (lane == 0) ddp[w] = diag;
    if (tm < s.t1) {
      const float skip = Dp[h];
      uint16_t* o = du + (int64_t)tm * cd + h * kSqP + 4 * g;
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        const u32x2 yw = *(const u32x2*)(ys + me * kScRowP + 2 * (16 * pb + 4 * g));
        const f32x4 a = dx[pb] * mdt;
        *(u32x2*)(o + 16 * pb) =
            u32x2{bf_pack(__builtin_fmaf(skip, bf_lo(yw.x), a.x), __builtin_fmaf(skip, bf_hi(yw.x), a.y)),
                  bf_pack(__builtin_fmaf(skip, bf_lo(yw.y), a.z), __builtin_fmaf(skip, bf_hi(yw.y), a.w))};
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
  if (tm < s.t1) {
    float* p = part + ((int64_t)blockIdx.y * T + tm) * (2 * kSqN) + 4 * g;
#pragma unroll
    for (int b = 0; b < 8; ++b) *(f32x4*)(p + 16 * b) = acc[b];
  }
}

// du's B and C columns: the sums over the head groups (of what lies outside the
// chunks, and inside), in a fixed order.  grid (ceil(T / 4)), 256 threads: a wave a token, four columns a lane
__global__ __launch_bounds__(256) void scan_bwd_bc_kernel(const float* __restrict__ part,
                                                          int groups, int T, int nheads,
                                                          const int* __restrict__ off, int nseq,
                                                          uint16_t* __restrict__ du) {
  const int t = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (threadIdx.x & 63) * 4;
  if (t >= T || seq_find(off, nseq, T, t).i < 0) return;
  const float* p = part + (int64_t)t * (2 * kSqN) + c;
  const int64_t step = (int64_t)T * (2 * kSqN);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  int k = 0;
  for (; k + 8 <= groups; k += 8) {
    f32x4 x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = *(const f32x4*)(p + (k + q) * step);
#pragma unroll
    for (int q = 0; q < 8; ++q) v += x[q];
  }
  for (; k < groups; ++k) v += *(const f32x4*)(p + k * step);
  const int d = nheads * kSqP;
  *(u32x2*)(du + (int64_t)t * (d + 2 * kSqN) + d + c) =
      u32x2{bf_pack(v.x, v.y), bf_pack(v.z, v.w)};
}

// A wave a chunk and head, two tokens a lane: dl, dt's gradient, and the
// chunk's sums for dt_bias, A_log and D (sums [slots][3][nheads]).  dots, pa NULL:
// nothing from outside the chunks.  grid (slots, ceil(nheads / 4)), 256 threads
template <bool F32>
__global__ __launch_bounds__(256) void scan_bwd_fin_kernel(
    const typename Zx<F32>::T* __restrict__ zx, int T, int nheads, const int* __restrict__ off,
    int nseq, const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    const double* __restrict__ qi, const double* __restrict__ ki, const float* __restrict__ kd,
    const float* __restrict__ dots, const float* __restrict__ pa, const float* __restrict__ dd,
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
  const float rate = sc_rate(A_log[h]), bias = dt_bias[h];
  const int64_t per = (int64_t)nheads * T, ht = (int64_t)h * T + s.t0;
  float raw[2], dt[2], kout[2], own[2];
  double a[2], b[2];  // what the sums over t >= s and over s' < s take
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int i = 2 * lane + q;
    const bool in = s.t0 + i < s.t1;
    raw[q] = tok_raw<F32>(zx, Z, nheads, h, min(s.t0 + i, T - 1)) + bias;
    dt[q] = in ? mx_softplus(raw[q]) : 0.f;
    float qout = 0.f;  // the halves of the states
    kout[q] = 0.f;
    if (in && dots) {
      const float* p = dots + ht + i;
      qout = p[0] + p[2 * per];
      kout[q] = p[per] + p[3 * per];
    }
    own[q] = in ? kd[ht + i] : 0.f;
    a[q] = in ? qi[ht + i] - ki[ht + i] + (double)qout : 0.0;
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
  const double above = ai - a2, before = bi - b2,
               through = pa ? (double)pa[sh] + (double)pa[(int64_t)gridDim.x * nheads + sh] : 0.0;
  const double dl[2] = {above + a[1] + a[0] + before + through,
                        above + a[1] + before + b[0] + through};
  double sb = 0.0, sa = 0.0;  // (many small terms of either sign)
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int t = s.t0 + 2 * lane + q;
    if (t >= s.t1) break;
    const float ds = (float)((double)own[q] + (double)kout[q] - (double)rate * dl[q]);
    const float v = ds / (1.f + expf(-raw[q]));
    Zx<F32>::put(dzx + t * Z + (Z - nheads) + h, v);
    sb += v;
    sa -= (double)dt[q] * rate * dl[q];
  }
  sb = group_sum_f64<64>(sb);
  sa = group_sum_f64<64>(sa);
  if (lane == 0) {
    o[0] = (float)sb;
    o[nheads] = (float)sa;
    o[2 * nheads] = dd[sh];
  }
}

// column c of sums [rows][3 nheads] over the rows, 16 chains, to the three outputs
__global__ __launch_bounds__(1024) void scan_bwd_sum_kernel(const float* __restrict__ sums,
                                                            int64_t rows, int nheads,
                                                            float* __restrict__ ddt_bias,
                                                            float* __restrict__ dA_log,
                                                            float* __restrict__ dD) {
  __shared__ double p[16][64];
  const int lane = threadIdx.x & 63, chain = threadIdx.x >> 6;
  const int64_t cols = (int64_t)3 * nheads, c = (int64_t)blockIdx.x * 64 + lane;
  double v = 0.0;
  if (c < cols)
    for (int64_t r = chain; r < rows; r += 16) v += sums[r * cols + c];
  p[chain][lane] = v;
  __syncthreads();
  if (chain != 0 || c >= cols) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) v += p[k][lane];
  const int q = (int)(c / nheads), h = (int)(c - (int64_t)q * nheads);
  (q == 0 ? ddt_bias : q == 1 ? dA_log : dD)[h] = (float)v;
}

// Groups of heads: 640 workgroups of a chunk and group.  16384 tokens of 64 heads
// (136 slots): off + to + from + bc 838 us in 5 groups; 865 in 4, which leaves
// scan_bwd_to_kernel's second workgroup a CU unused, 882 in 8, where the partial
// sums of dB and dC (1 KiB a token and group, written and read twice) cost more.
static int sb_groups(int64_t slots, int64_t nheads) {
  int64_t n = (640 + slots - 1) / slots;
  n = n > nheads ? nheads : n;
  const int64_t per = (nheads + n - 1) / n;
  return (int)((nheads + per - 1) / per);
}

// Whether there may be states between chunks: up to 128 tokens a sequence is one
// chunk, and the launches for what lies outside of one are left out (four sequences
// of 64 heads in 128 tokens: 41 us, 55 with the launch by chunks; in 129: 65)
static bool sb_states(int64_t T) { return T > kSbQ; }

struct ScanBwdWs {
  double *qi, *ki;
  float *S0, *E, *dec, *kd, *dots, *pa, *dd, *sums, *part;
  int64_t bytes;
};
static ScanBwdWs sb_ws(void* p, int64_t T, int64_t nseq, int64_t nheads) {
  const int64_t slots = slot_count(T, nseq, kSbQ), sh = slots * nheads, th = T * nheads;
  const int64_t states = state_count(T, kSbQ) * nheads;
  ScanBwdWs w;
  float* f = (float*)p;
  auto take = [&](int64_t n) {
    float* r = f;
    f += (n + 63) / 64 * 64;
    return r;
  };
  w.S0 = w.E = w.dec = w.dots = w.pa = nullptr;
  if (sb_states(T)) {
    w.S0 = take(states * kScState);
    w.E = take(states * kScState);
    w.dec = take(states);
    w.dots = take(4 * th), w.pa = take(2 * sh);
  }
  w.qi = (double*)take(2 * th), w.ki = (double*)take(2 * th);
  w.kd = take(th), w.dd = take(sh);
  w.sums = take(3 * sh);
  w.part = take((sb_states(T) ? 2 : 1) * sb_groups(slots, nheads) * T * 2 * kSqN);
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
  const dim3 grid((unsigned)slots, (unsigned)groups);
  float* inside = w.part;  // the partial sums of dB and dC from inside the chunks
  int parts = groups;
  if (sb_states(in.T)) {
    hipError_t e = launch_chunk_states(in, u, nullptr, false, dt_bias, A_log, w.S0, w.dec, stream);
    if (e != hipSuccess) return e;
    e = launch_chunk_states(in, u, dy, true, dt_bias, A_log, w.E, w.dec, stream);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(scan_bwd_off_kernel<F32>, dim3((unsigned)((slots * groups + 7) / 8 * 32)),
                       dim3(256), 0, stream, zx, u, dy, in.T, in.nheads, in.offsets, in.nseq,
                       dt_bias, A_log, w.S0, w.E, w.part, w.dots, w.pa, (int)slots, groups);
    inside += (int64_t)groups * in.T * 2 * kSqN;
    parts += groups;
  }
  hipLaunchKernelGGL(scan_bwd_to_kernel<F32>, grid, dim3(kSbThreads), 0, stream, zx, u, dy, in.T,
                     in.nheads, in.offsets, in.nseq, dt_bias, A_log, inside, w.qi);
  hipLaunchKernelGGL(scan_bwd_from_kernel<F32>, grid, dim3(kSbThreads), 0, stream, zx, u, dy, in.T,
                     in.nheads, in.offsets, in.nseq, dt_bias, A_log, D, w.E, inside, w.ki, w.kd,
                     w.dd, du);
  hipLaunchKernelGGL(scan_bwd_bc_kernel, dim3((unsigned)((in.T + 3) / 4)), dim3(256), 0, stream, w.part,
                     parts, in.T, in.nheads, in.offsets, in.nseq, du);
  hipLaunchKernelGGL(scan_bwd_fin_kernel<F32>, dim3((unsigned)slots, (unsigned)((in.nheads + 3) / 4)),
                     dim3(256), 0, stream, zx, in.T, in.nheads, in.offsets, in.nseq, dt_bias,
                     A_log, w.qi, w.ki, w.kd, w.dots, w.pa, w.dd, (X*)dzx, w.sums);
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
