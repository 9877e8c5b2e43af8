// The head's loss around its products (tmamba_head.h): which rows take part,
// the loss from the softmax sums, the sparse part of the dlogits, and dh.
//
//   z = h W^T;  CE = ln sum e^z - z[y];  with a teacher's words id_k, logits t_k:
//   q = softmax over the kept k of t_k / tau,  s = softmax(z / tau),
//   KL = sum_k q_k (ln q_k - ln s[id_k]),  loss = (1 - alpha) CE + alpha tau^2 KL,
//   dz_v = g ((1 - alpha)(p_v - 1[v = y]) + alpha tau (s_v - sum_k q_k 1[id_k = v])).
//
// Forward: rows with a loss are listed (rows_kernel), the products leave a few
// partial sums a row, and one workgroup or wave a row joins them, takes the
// logits at its label and the teacher's words by their own dot products (float32;
// exact products) and computes the loss.  It also writes the gradient at those
// words, everything summed in float32, so that backward's sparse part is a
// store over the dense part, whatever words coincide.
//
// Backward, per piece of the vocabulary: dlogits (dense), the sparse stores, dh and
// dW.  A row's gradient is g = m 2^e, 1 <= m < 2; the dlogits hold m times the unit
// gradient (16 bits, rounded once: by 2^-8 of each in bfloat16, 2^-11 in float16), h is
// copied times 2^(e - largest e) (exact but for what falls under the type's
// smallest number), and dh and dW are multiplied by powers of two at the end: the
// roundings do not depend on how the loss is scaled.
#include "common.hpp"
#include "head.hpp"
#include "launchers.hpp"

namespace tmk {

namespace {

constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

inline __host__ __device__ int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
inline __host__ __device__ int64_t up128(int64_t v) { return (v + 127) / 128 * 128; }

__device__ __forceinline__ int64_t id_at(const void* p, bool i64, int64_t i) {
  return i64 ? static_cast<const int64_t*>(p)[i] : (int64_t)static_cast<const int*>(p)[i];
}

__device__ __forceinline__ float lo16(uint32_t x, bool f16) {
  if (f16) return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
  return __uint_as_float(x << 16);
}

// 8 elements as float32
template <bool F16>
__device__ __forceinline__ void widen(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = lo16(v[i] & 0xFFFFu, F16);
    x[2 * i + 1] = F16 ? lo16(v[i] >> 16, true) : __uint_as_float(v[i] & 0xFFFF0000u);
  }
}

template <bool F16>
__device__ __forceinline__ uint16_t narrow(float v) {
  if constexpr (F16)
    return __builtin_bit_cast(uint16_t, (_Float16)v);
  else
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

__device__ __forceinline__ float top_at(const void* p, int type, int64_t i) {
  if (type == 0) return static_cast<const float*>(p)[i];
  return lo16(static_cast<const uint16_t*>(p)[i], type == 2);
}

// exponent of a row's gradient (0 where it is not finite)
__device__ __forceinline__ int exp_of(float g) {
  const bool fin = fabsf(g) < __builtin_inff();
  return fin ? ilogbf(g) : 0;
}

struct Rows {
  int* count;  // [1]
  int* idx;    // [T]: the token of a row
  int* pos;    // [T]: the row of a token, or -1
  int* exps;   // [2]: the largest exponent, and that without the dlogits' shift (backward)
  HeadRow* row;  // [T] (backward)
  uint8_t* terms;  // [T]: 1 label, 2 teacher (forward)
};

// terms[t]: a label in the vocabulary; a kept word of the teacher.  A wave a token.
__global__ __launch_bounds__(256) void terms_kernel(HeadIn in, const void* __restrict__ top,
                                                    int top_type, uint8_t* __restrict__ terms) {
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (t >= in.T) return;
  bool some = false;
  for (int k = lane; k < in.K; k += 64) {
    const int64_t id = id_at(in.ids, in.ids64, t * in.K + k);
    if (id >= 0 && id < in.V && top_at(top, top_type, t * in.K + k) != -__builtin_inff())
      some = true;
  }
  const bool kl = __any(some);
  const int64_t y = id_at(in.targets, in.targets64, t);
  if (lane == 0) terms[t] = (uint8_t)((y >= 0 && y < in.V ? 1 : 0) | (kl ? 2 : 0));
}

// Lists the rows in the tokens' order.  A workgroup has `per` tokens (a multiple of
// 1024); it counts the rows before them by itself, then lists its own, 1024 at a time.
// At most 64 workgroups, so that counting again costs 32 reads a token at most.
// BWD: rows whose loss has a gradient, with their factors.
template <bool BWD>
__global__ __launch_bounds__(1024) void rows_kernel(HeadIn in, const float* __restrict__ stats,
                                                    const float* __restrict__ dloss, int shift,
                                                    int64_t per, Rows out) {
  __shared__ int sums[16];
  __shared__ int maxs[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t T = in.T, t0 = blockIdx.x * per, t1 = t0 + per < T ? t0 + per : T;
  auto has = [&](int64_t t) {
    if constexpr (BWD) {
      return stats[kStatTerms * T + t] != 0.f && !(dloss[t] == 0.f);
    } else {
      if (in.K > 0) return out.terms[t] != 0;
      const int64_t y = id_at(in.targets, in.targets64, t);
      return y >= 0 && y < in.V;
    }
  };
  const float unit = head_unit(in.alpha, in.tau);
  int n = 0, e = -1000;
  // the first workgroup looks at all gradients for the largest
#pragma unroll 4
  for (int64_t t = tid; t < (BWD && blockIdx.x == 0 ? T : t0); t += 1024) {
    const bool yes = has(t);
    if (t < t0) n += yes;
    if constexpr (BWD) {
      const float g = dloss[t] * unit;
      if (yes && fabsf(g) < __builtin_inff() && g != 0.f) e = max(e, ilogbf(g));
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    n += __shfl_xor(n, o, 64);
    e = max(e, __shfl_xor(e, o, 64));
  }
  if (lane == 0) {
    sums[wave] = n;
    maxs[wave] = e;
  }
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    base += sums[w];
    e = max(e, maxs[w]);
  }
  if (BWD && blockIdx.x == 0 && tid == 0) {
    out.exps[0] = e == -1000 ? 0 : e;
    out.exps[1] = out.exps[0] - shift;
  }
  for (int64_t c = t0; c < t1; c += 1024) {
    const int64_t t = c + tid;
    const bool yes = t < t1 && has(t);
    const uint64_t mask = __ballot(yes);
    __syncthreads();  // the previous sums have been read
    if (lane == 0) sums[wave] = __popcll(mask);
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      before += w < wave ? sums[w] : 0;
      all += sums[w];
    }
    const int r = base + before + __popcll(mask & ((uint64_t(1) << lane) - 1));
    base += all;
    if (t < t1) out.pos[t] = yes ? r : -1;
    if (yes) {
      out.idx[r] = (int)t;
      if constexpr (BWD) {
        const float g = dloss[t] * unit;
        const float m = ldexpf(g, shift - exp_of(g));
        const int terms = (int)stats[kStatTerms * T + t];
        float c1 = terms & 1 ? (1.0f - in.alpha) / unit * m : 0.f;
        float c2 = terms & 2 ? in.alpha * in.tau / unit * m : 0.f;
        if (in.tau == 1.0f) {  // one softmax
          c1 += c2;
          c2 = 0.f;
        }
        out.row[r] = HeadRow{stats[kStatLse * T + t], stats[kStatLseT * T + t], c1, c2};
      }
    }
  }
  if (t1 == T && tid == 0) *out.count = base;
}

// The loss and the stats of a token, a wave (WAVES 0: no teacher) or a workgroup a
// token, of sixteen waves where tokens are few (1 token, 64 words: XX us, YY of four).  Bound: the dot products' rows of W, from the caches for
// frequent words.
struct Finish {
  HeadIn in;
  const void* top;
  int top_type;
  const float* part;
  int tile, grid;  // tokens of a tile and workgroups of the logits' launch
  Rows rows;
  float* loss;
  float* stats;
};

// h[t] . W[v] over the lanes of a wave, in every lane
template <bool F16>
__device__ __forceinline__ float row_dot(const uint16_t* h, const uint16_t* w, int D, int lane) {
  float s = 0.f;
  for (int d = lane * 8; d < D; d += 512) {
    float x[8], y[8];
    widen<F16>(ld16(h + d), x);
    widen<F16>(ld16(w + d), y);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(x[i], y[i], s);
  }
  return wave_sum(s);
}

// the softmax sums of row r: the parts of its token tile's workgroups, joined.  m: the largest
// logit; s: sum of 2^(log2e (z - m)); sT the same at the temperature (TEMP)
template <bool TEMP>
__device__ __forceinline__ void join(const float* part, int r, int n, int64_t V, int tile, int grid, float k2,
                                     int lane, float& m, float& s, float& sT) {
  constexpr int E = TEMP ? 3 : 2;
  const int64_t nt = (n + tile - 1) / tile, nv = (V + 255) / 256, N = nt * nv;
  const int64_t P = N < grid ? N : grid;
  const int64_t j = r / tile;
  // the workgroups whose runs hold the tile's first and last item
  const int64_t w0 = ((j * nv + 1) * P - 1) / N, w1 = (((j + 1) * nv) * P - 1) / N;
  const int cnt = (int)(w1 - w0 + 1) * 2;
  auto at = [&](int i) { return part + (((w0 + j) * 2 + i) * 256 + r % tile) * E; };
  float mm = -__builtin_inff();
  for (int i = lane; i < cnt; i += 64) mm = fmaxf(mm, at(i)[0]);
  m = wave_max(mm);
  const float ref = m == -__builtin_inff() ? 0.f : m;
  float a = 0.f, b = 0.f;
  for (int i = lane; i < cnt; i += 64) {
    const float* p = at(i);
    a += p[1] * __builtin_amdgcn_exp2f((p[0] - ref) * kLog2e);
    if constexpr (TEMP) b += p[2] * __builtin_amdgcn_exp2f((p[0] - ref) * k2);
  }
  s = wave_sum(a);
  sT = TEMP ? wave_sum(b) : s;
}

template <bool F16, bool TEMP, int WAVES>
__global__ __launch_bounds__(WAVES ? 64 * WAVES : 256) void finish_kernel(Finish f) {
  constexpr bool TEACH = WAVES > 0;
  constexpr int L = WAVES * 64;
  extern __shared__ float sh[];  // TEACH: z[K], q[K], id[K]
  __shared__ float red[TEACH ? WAVES : 1];
  const HeadIn& in = f.in;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = TEACH ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  if (t >= in.T) return;
  float* st = f.stats + t;  // the token's place in each plane
  float* st_top = f.stats + kStatPlanes * in.T + t * in.K;
  const int64_t y = id_at(in.targets, in.targets64, t);
  const bool ce = y >= 0 && y < in.V;
  const int terms = TEACH ? f.rows.terms[t] : (ce ? 1 : 0);
  const int first = TEACH ? threadIdx.x : lane;
  if (terms == 0) {  // no loss
    if (first < kStatPlanes) st[first * in.T] = 0.f;
    for (int i = first; i < in.K; i += L) st_top[i] = 0.f;
    if (first == 0) f.loss[t] = 0.f;
    return;
  }
  const int n = *f.rows.count;
  const float it = 1.0f / in.tau, k2 = kLog2e * it;
  float m, s, sT;
  join<TEMP>(f.part, f.rows.pos[t], n, in.V, f.tile, f.grid, k2, lane, m, s, sT);
  const float mf = m == -__builtin_inff() ? 0.f : m;  // (as the sums took it)
  const float lse2 = __builtin_fmaf(mf, kLog2e, __builtin_amdgcn_logf(s));
  const float lseT2 = __builtin_fmaf(mf, k2, __builtin_amdgcn_logf(sT));
  const uint16_t* h = in.h + t * in.D;
  const float unit = head_unit(in.alpha, in.tau);
  const float c1 = terms & 1 ? (1.0f - in.alpha) / unit : 0.f;
  const float c2 = terms & 2 ? in.alpha * in.tau / unit : 0.f;
  // gradient over the unit at a word with logit z; hit: its share of the label and the teacher
  auto grad = [&](float z, float hit) {
    return c1 * __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -lse2)) +
           c2 * __builtin_amdgcn_exp2f(__builtin_fmaf(z, k2, -lseT2)) - hit;
  };
  const float zy = ce ? row_dot<F16>(h, in.w + y * in.D, in.D, lane) : 0.f;
  const float ce_loss = ce ? __builtin_amdgcn_logf(s) * kLn2 + (mf - zy) : 0.f;
  if constexpr (!TEACH) {
    if (lane == 0) {
      f.loss[t] = ce_loss;
      st[kStatLse * in.T] = lse2;
      st[kStatLseT * in.T] = lse2;
      st[kStatTerms * in.T] = 1.f;
      st[kStatLabel * in.T] = grad(zy, 1.0f);
    }
    return;
  }
  const int K = in.K;
  float* z = sh;
  float* q = sh + K;
  int* id = reinterpret_cast<int*>(sh + 2 * K);
  // the teacher's softmax over its kept words; 2^(log2e / tau t)
  float tm = -__builtin_inff();
  for (int k = threadIdx.x; k < K; k += L) {
    const int64_t v = id_at(in.ids, in.ids64, t * K + k);
    const bool in_v = v >= 0 && v < in.V;
    id[k] = in_v ? (int)v : -1;
    q[k] = in_v ? top_at(f.top, f.top_type, t * K + k) * it : -__builtin_inff();
    tm = fmaxf(tm, q[k]);
  }
  auto block = [&](float v, bool sum) {
    v = sum ? wave_sum(v) : wave_max(v);
    __syncthreads();
    if (lane == 0) red[wave] = v;
    __syncthreads();
    float all = red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) all = sum ? all + red[w] : fmaxf(all, red[w]);
    return all;
  };
  tm = block(tm, false);
  float ts = 0.f;
  for (int k = threadIdx.x; k < K; k += L)
    if (q[k] != -__builtin_inff()) ts += __builtin_amdgcn_exp2f((q[k] - tm) * kLog2e);
  ts = block(ts, true);
  const float tl = __builtin_amdgcn_logf(ts) * kLn2;
  // four words a wave at a time: their loads overlap
  for (int k0 = 4 * wave; k0 < K; k0 += 4 * WAVES) {
    float d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = k0 + i < K ? k0 + i : K - 1;
      const int v = id[k] >= 0 ? id[k] : 0;
      d[i] = row_dot<F16>(h, in.w + (int64_t)v * in.D, in.D, lane);
    }
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k0 + i < K) z[k0 + i] = d[i];
  }
  __syncthreads();
  float kl = 0.f;
  if (terms & 2) {
    for (int k = threadIdx.x; k < K; k += L) {
      const float a = q[k];
      if (a == -__builtin_inff()) {
        q[k] = 0.f;
        continue;
      }
      const float lq = (a - tm) - tl;  // ln q
      const float p = __builtin_amdgcn_exp2f(lq * kLog2e);
      q[k] = p;
      // ln s = (z - m) / tau - ln of the sum
      if (p != 0.f) kl += p * (lq - ((z[k] - mf) * it - __builtin_amdgcn_logf(sT) * kLn2));
    }
    kl = block(kl, true);
  } else {
    for (int k = threadIdx.x; k < K; k += L) q[k] = 0.f;
  }
  __syncthreads();
  auto hits = [&](int64_t v) {
    float x = 0.f;
    for (int j = 0; j < K; ++j)
      if (id[j] == v) x += q[j];
    return c2 * x + (v == y ? c1 : 0.f);
  };
  for (int k = threadIdx.x; k < K; k += L)
    st_top[k] = id[k] >= 0 ? grad(id[k] == y ? zy : z[k], hits(id[k])) : 0.f;
  if (threadIdx.x == 0) {
    f.loss[t] = (terms & 1 ? (1.0f - in.alpha) * ce_loss : 0.f) +
                (terms & 2 ? in.alpha * in.tau * in.tau * kl : 0.f);
    st[kStatLse * in.T] = lse2;
    st[kStatLseT * in.T] = lseT2;
    st[kStatTerms * in.T] = (float)terms;
    st[kStatLabel * in.T] = ce ? grad(zy, hits(y)) : 0.f;
  }
}

// ht[d][r] = h[idx[r]][d]: the logits' second operand, with zeros up to a multiple of 128
// columns d and of 256 rows r.  64 x 64 a workgroup, through LDS.
__global__ __launch_bounds__(256) void rows_transpose_kernel(HeadIn in, Rows rows, int64_t tp,
                                                             uint16_t* __restrict__ ht) {
  __shared__ uint16_t s[64][72];
  const int n = *rows.count;
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  const int d0 = blockIdx.y * 64, q = threadIdx.x >> 3, c = 8 * (threadIdx.x & 7);
  if (r0 >= up256(n)) return;
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    u32x4 v = {0, 0, 0, 0};
    if (r0 + q + i < n && d0 + c < in.D)
      v = ld16(in.h + (int64_t)rows.idx[r0 + q + i] * in.D + d0 + c);
    st16(&s[q + i][c], v);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = (uint32_t)s[c + 2 * j][q + i] | (uint32_t)s[c + 2 * j + 1][q + i] << 16;
    st16(ht + (int64_t)(d0 + q + i) * tp + r0 + c, v);
  }
}

// hs[r] = h[idx[r]] times 2^(e - emax): the rows dW contracts, one after another
template <bool F16>
__global__ __launch_bounds__(256) void rows_copy_kernel(HeadIn in, const float* __restrict__ dloss,
                                                        Rows rows, uint16_t* __restrict__ hs) {
  const int64_t r = blockIdx.x;
  if (r >= *rows.count) return;
  const int64_t t = rows.idx[r];
  const int e = exp_of(dloss[t] * head_unit(in.alpha, in.tau)) - rows.exps[0];
  const uint16_t* src = in.h + t * in.D;
  uint16_t* dst = hs + r * in.D;
  for (int d = threadIdx.x * 8; d < in.D; d += 2048) {
    u32x4 v = ld16(src + d);
    if (e != 0) {
      float x[8];
      widen<F16>(v, x);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = (uint32_t)narrow<F16>(ldexpf(x[2 * i], e)) |
               (uint32_t)narrow<F16>(ldexpf(x[2 * i + 1], e)) << 16;
    }
    st16(dst + d, v);
  }
}

// The label's and the teacher's words of the piece, over the dense dlogits.
// Words that coincide carry the same value, so their order does not matter.
template <bool F16>
__global__ __launch_bounds__(256) void sparse_kernel(HeadIn in, const float* __restrict__ stats,
                                                     const float* __restrict__ dloss, Rows rows,
                                                     int64_t w0, int64_t n, uint16_t* __restrict__ G,
                                                     int64_t ld) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = i / (in.K + 1);
  const int e = (int)(i % (in.K + 1));
  if (r >= *rows.count) return;
  const int64_t t = rows.idx[r];
  const int terms = (int)stats[kStatTerms * in.T + t];
  if (!(terms & (e == 0 ? 1 : 2))) return;
  const int64_t v =
      (e == 0 ? id_at(in.targets, in.targets64, t) : id_at(in.ids, in.ids64, t * in.K + e - 1)) -
      w0;
  if (v < 0 || v >= n) return;
  const float g = dloss[t] * head_unit(in.alpha, in.tau);
  const float x = stats[e == 0 ? kStatLabel * in.T + t : kStatPlanes * in.T + t * in.K + e - 1];
  G[r * ld + v] = narrow<F16>(x * ldexpf(g, kHeadShift<F16> - exp_of(g)));
}

// dh[t] = 2^(e - shift) times the sum of the row's parts; zeros for a token without a row
template <bool F16>
__global__ __launch_bounds__(256) void dh_out_kernel(HeadIn in, const float* __restrict__ dloss,
                                                     Rows rows, const float* __restrict__ part,
                                                     int parts, uint16_t* __restrict__ dh) {
  const int64_t t = blockIdx.x;
  const int r = rows.pos[t];
  uint16_t* dst = dh + t * in.D;
  const int e = exp_of(dloss[t] * head_unit(in.alpha, in.tau)) - kHeadShift<F16>;
  for (int d = threadIdx.x * 8; d < in.D; d += 2048) {
    u32x4 o = {0, 0, 0, 0};
    if (r >= 0) {
      f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll 4
      for (int s = 0; s < parts; ++s) {
        const float* p = part + ((int64_t)s * in.T + r) * in.D + d;
        a += *reinterpret_cast<const f32x4*>(p);
        b += *reinterpret_cast<const f32x4*>(p + 4);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        o[i] = (uint32_t)narrow<F16>(ldexpf(a[2 * i], e)) |
               (uint32_t)narrow<F16>(ldexpf(a[2 * i + 1], e)) << 16;
        o[2 + i] = (uint32_t)narrow<F16>(ldexpf(b[2 * i], e)) |
                   (uint32_t)narrow<F16>(ldexpf(b[2 * i + 1], e)) << 16;
      }
    }
    st16(dst + d, o);
  }
}

// Parts of a contraction of nst stages of `tiles` tiles on P workgroups: the
// fewest rounds times stages, against 0.5 us for writing and reading a tile's
// part (256 KiB each way).  A stage takes 0.8 us a workgroup; parts are a multiple of
// `unit` stages, the ring's.
void cut(int64_t tiles, int64_t nst, int64_t P, int unit, int* parts, int* per) {
  double best = 0;
  for (int64_t k = 1; k <= nst && k <= 64 && (k == 1 || tiles * k <= 4 * P); ++k) {
    const int64_t len = ((nst + k - 1) / k + unit - 1) / unit * unit;
    if ((nst + len - 1) / len != k) continue;  // an empty part
    const int64_t rounds = (tiles * k + P - 1) / P;
    const double us = (double)rounds * ((double)len * 0.8 + 3.0) +
                      (k > 1 ? 0.1 * (double)(tiles * k) + 3.0 : 0.0);
    if (k == 1 || us < best) {
      best = us;
      *parts = (int)k;
      *per = (int)len;
    }
  }
}

}  // namespace

// A piece holds at most 2^28 dlogits (512 MiB: with dh's float32 sums read
// and written once a piece, a quarter of it adds a tenth to the time of dh),
// or 4096 words where tokens are many.  Where there are several pieces, dW's tiles of all but
// the last one fill whole rounds of the workgroups.
HeadPlan head_plan(int64_t T, int64_t V, int64_t D) {
  HeadPlan p;
  const int64_t P = current_cu_count();
  int64_t most = (int64_t(1) << 28) / up256(T) / 256 * 256;
  if (most < 4096) most = 4096;
  p.pieces = (up256(V) + most - 1) / most;
  p.piece = up256((V + p.pieces - 1) / p.pieces);
  if (p.pieces > 1) {
    const int64_t round = P / ((D + 255) / 256) * 256;  // words of a round
    if (round > 0 && round <= most) p.piece = most / round * round;
  }
  p.pieces = (V + p.piece - 1) / p.piece;
  const int64_t nd = (D + 255) / 256, nt = (T + 255) / 256, nv = p.piece / 256;
  const int64_t words = p.pieces == 1 ? V : p.piece;
  cut(nt * nd, (words + 31) / 32, P, 4, &p.parts_h, &p.per_h);
  cut(nv * nd, (T + 31) / 32, P, 4, &p.parts_w, &p.per_w);
  const int64_t rest = V - (p.pieces - 1) * p.piece;
  cut((rest + 255) / 256 * nd, (T + 31) / 32, P, 4, &p.last_w, &p.last_per);
  return p;
}

namespace {

struct Layout {
  Rows rows;
  float* part;
  uint16_t *ht, *hs, *G;
  float *part_h, *part_w;
  int64_t bytes;
};

template <typename T>
void take(T** p, uint8_t* base, int64_t* at, int64_t bytes) {
  *p = reinterpret_cast<T*>(base + *at);
  *at += up256(bytes);
}

Layout forward_layout(int64_t T, int64_t V, int64_t D, void* ws) {
  Layout l{};
  uint8_t* b = static_cast<uint8_t*>(ws);
  take(&l.rows.count, b, &l.bytes, 4);
  take(&l.rows.idx, b, &l.bytes, 4 * T);
  take(&l.rows.pos, b, &l.bytes, 4 * T);
  take(&l.rows.terms, b, &l.bytes, T);
  take(&l.ht, b, &l.bytes, 2 * head_padded(T) * up128(D));
  take(&l.part, b, &l.bytes, 4 * head_part_floats(T, V));
  return l;
}

Layout backward_layout(int64_t T, int64_t V, int64_t D, const HeadPlan& p, void* ws) {
  Layout l{};
  uint8_t* b = static_cast<uint8_t*>(ws);
  take(&l.rows.count, b, &l.bytes, 4);
  take(&l.rows.exps, b, &l.bytes, 8);
  take(&l.rows.idx, b, &l.bytes, 4 * T);
  take(&l.rows.pos, b, &l.bytes, 4 * T);
  take(&l.rows.row, b, &l.bytes, (int64_t)sizeof(HeadRow) * T);
  take(&l.ht, b, &l.bytes, 2 * head_padded(T) * up128(D));
  take(&l.hs, b, &l.bytes, 2 * T * D);
  take(&l.G, b, &l.bytes, 2 * up256(T) * p.piece);  // (tiles are written whole)
  take(&l.part_h, b, &l.bytes, 4 * p.parts_h * T * D);
  const int64_t rest = V - (p.pieces - 1) * p.piece;
  const int64_t full = p.pieces > 1 && p.parts_w > 1 ? p.parts_w * p.piece : 0;
  const int64_t end = p.last_w > 1 ? p.last_w * rest : 0;
  take(&l.part_w, b, &l.bytes, 4 * D * (full > end ? full : end));
  return l;
}

}  // namespace

int64_t head_loss_bytes(int64_t T, int64_t V, int64_t D) {
  return forward_layout(T, V, D, nullptr).bytes;
}

int64_t head_loss_bwd_bytes(int64_t T, int64_t V, int64_t D) {
  return backward_layout(T, V, D, head_plan(T, V, D), nullptr).bytes;
}

#define TM_RET(expr)                     \
  do {                                   \
    const hipError_t e_ = (expr);        \
    if (e_ != hipSuccess) return e_;     \
  } while (0)

static int64_t rows_per_group(int64_t T) {
  const int64_t per = (T + 63) / 64;
  return (per + 1023) / 1024 * 1024;
}

static hipError_t transpose(const HeadIn& in, const Layout& l, hipStream_t stream) {
  hipLaunchKernelGGL(rows_transpose_kernel,
                     dim3((unsigned)(head_padded(in.T) / 64), (unsigned)(up128(in.D) / 64)), dim3(256), 0,
                     stream, in, l.rows, head_padded(in.T), l.ht);
  return hipGetLastError();
}

template <bool F16, int WAVES>
static hipError_t run_finish_of(const Finish& f, hipStream_t stream) {
  const dim3 grid((unsigned)(WAVES ? f.in.T : (f.in.T + 3) / 4)), block(WAVES ? 64 * WAVES : 256);
  if (WAVES && f.in.tau != 1.0f)
    hipLaunchKernelGGL((finish_kernel<F16, true, WAVES>), grid, block, (unsigned)(12 * f.in.K),
                       stream, f);
  else
    hipLaunchKernelGGL((finish_kernel<F16, false, WAVES>), grid, block, (unsigned)(12 * f.in.K),
                       stream, f);
  return hipGetLastError();
}

template <bool F16>
static hipError_t run_finish(const Finish& f, hipStream_t stream) {
  if (f.in.K == 0) return run_finish_of<F16, 0>(f, stream);
  if (f.in.T <= 512 && f.in.K > 16) return run_finish_of<F16, 16>(f, stream);
  return run_finish_of<F16, 4>(f, stream);
}

hipError_t launch_head_loss(const HeadIn& in, const void* top, int top_type, float* loss,
                            float* stats, void* workspace, hipStream_t stream) {
  const Layout l = forward_layout(in.T, in.V, in.D, workspace);
  if (in.K > 0) {
    hipLaunchKernelGGL(terms_kernel, dim3((unsigned)((in.T + 3) / 4)), dim3(256), 0, stream, in,
                       top, top_type, l.rows.terms);
    TM_RET(hipGetLastError());
  }
  const int64_t per = rows_per_group(in.T);
  hipLaunchKernelGGL(rows_kernel<false>, dim3((unsigned)((in.T + per - 1) / per)), dim3(1024), 0,
                     stream, in, nullptr, nullptr, 0, per, l.rows);
  TM_RET(hipGetLastError());
  TM_RET(transpose(in, l, stream));
  TM_RET(launch_head_logits(in, l.ht, l.rows.count, l.part, stream));
  const int tile = head_tile_tokens(in.T, in.V, true);
  const Finish f{in, top, top_type, l.part, tile, head_logits_grid(in.T, in.V, tile), l.rows, loss, stats};
  return in.f16 ? run_finish<true>(f, stream) : run_finish<false>(f, stream);
}

template <bool F16>
static hipError_t run_bwd(const HeadIn& in, const float* stats, const float* dloss, uint16_t* dh,
                          void* dw, int dw_type, bool accumulate, void* workspace,
                          hipStream_t stream) {
  const HeadPlan p = head_plan(in.T, in.V, in.D);
  const Layout l = backward_layout(in.T, in.V, in.D, p, workspace);
  const int64_t per = rows_per_group(in.T);
  hipLaunchKernelGGL(rows_kernel<true>, dim3((unsigned)((in.T + per - 1) / per)), dim3(1024), 0,
                     stream, in, stats, dloss, kHeadShift<F16>, per, l.rows);
  TM_RET(hipGetLastError());
  if (dw) {
    hipLaunchKernelGGL(rows_copy_kernel<F16>, dim3((unsigned)in.T), dim3(256), 0, stream, in, dloss,
                       l.rows, l.hs);
    TM_RET(hipGetLastError());
  }
  TM_RET(transpose(in, l, stream));
  for (int64_t i = 0; i < p.pieces; ++i) {
    const int64_t w0 = i * p.piece, n = in.V - w0 < p.piece ? in.V - w0 : p.piece;
    TM_RET(launch_head_dlogits(in, l.ht, l.rows.count, l.rows.row, w0, n, l.G, p.piece,
                               stream));
    hipLaunchKernelGGL(sparse_kernel<F16>, dim3((unsigned)((in.T * (in.K + 1) + 255) / 256)),
                       dim3(256), 0, stream, in, stats, dloss, l.rows, w0, n, l.G, p.piece);
    TM_RET(hipGetLastError());
    if (dh)
      TM_RET(launch_head_dh(in, l.rows.count, l.G, p.piece, w0, n, p.parts_h, p.per_h, i > 0,
                          l.part_h, stream));
    const bool last = i == p.pieces - 1;
    if (dw)
      TM_RET(launch_head_dw(in, l.rows.count, l.G, p.piece, l.hs, w0, n, last ? p.last_w : p.parts_w,
                          last ? p.last_per : p.per_w, l.rows.exps + 1, dw, dw_type, accumulate, l.part_w, stream));
  }
  if (dh)
    hipLaunchKernelGGL(dh_out_kernel<F16>, dim3((unsigned)in.T), dim3(256), 0, stream, in, dloss,
                       l.rows, l.part_h, p.parts_h, dh);
  return hipGetLastError();
}

hipError_t launch_head_loss_bwd(const HeadIn& in, const float* stats, const float* dloss,
                                uint16_t* dh, void* dw, int dw_type, bool accumulate,
                                void* workspace, hipStream_t stream) {
  return in.f16
             ? run_bwd<true>(in, stats, dloss, dh, dw, dw_type, accumulate, workspace, stream)
             : run_bwd<false>(in, stats, dloss, dh, dw, dw_type, accumulate, workspace, stream);
}

}  // namespace tmk
