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
// dW.  A row's gradient is g = m 2^e, 1 <= m < 2, that of the largest M 2^E; the dlogits hold
// m / M times the unit gradient (16 bits, rounded once: by 2^-8 of each in bfloat16, 2^-11 in
// float16), h is copied times 2^e over a power of two that all rows share, and dh and dW are
// multiplied by M and powers of two at the end: the roundings do not depend on how the loss is
// scaled, and where all gradients are equal (a mean) a label's dlogit, close to -1, is close to
// exact.  The copy of h is exact but for what falls under the type's smallest numbers.  In bfloat16
// the power is 2^E: h times its gradient's share of the largest keeps its bits down to 2^-126.  In
// float16 it is the one that brings the largest h 2^e to float16's own largest numbers (the forward
// pass leaves each row's exponent in `stats`): a value keeps its 11 bits where it is, times its
// gradient, above 2^-28 of the largest such product, and is off by at most 2^-39 of that product
// below.
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

template <bool F16>
__device__ __forceinline__ f32x4 mfma_16(u32x4 a, u32x4 b, f32x4 c) {
  typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return mfma16(as_bf16x8(a), as_bf16x8(b), c);
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

// exponent of a row's gradient (0 where it is not finite; of a zero, which is left of a gradient
// times a small unit, one so low that h times it is zero)
__device__ __forceinline__ int exp_of(float g) {
  if (g == 0.f) return -1000;
  return fabsf(g) < __builtin_inff() ? ilogbf(g) : 0;
}

struct Rows {
  int* count;  // [1]
  int* idx;    // [T]: the token of a row
  int* pos;    // [T]: the row of a token, or -1
  // backward: the exponent that h's copy is over, that without the dlogits' shift, the parts of
  // dh, the bits of the largest gradient's mantissa
  int* exps;
  HeadRow* row;  // [T] (backward)
  uint8_t* terms;  // [T]: 1 label, 2 teacher (forward)
};

// What the list of rows is made from: forward the labels, or with a teacher `terms`; backward
// the stats and the gradients of the losses.
struct Of {
  const void* top;  // forward, with a teacher
  int top_type;
  const float* stats;  // backward
  const float* dloss;
  int shift;
};

__device__ __forceinline__ bool in_vocabulary(const HeadIn& in, int64_t v) {
  return v >= 0 && v < in.V;
}

// which terms a token has, in every lane of a wave: 1 a label in the vocabulary, 2 a kept word of
// the teacher
__device__ __forceinline__ int terms_of(const HeadIn& in, const Of& of, int64_t t, int lane) {
  bool some = false;
  for (int k = lane; k < in.K; k += 64)
    if (in_vocabulary(in, id_at(in.ids, in.ids64, t * in.K + k)) &&
        top_at(of.top, of.top_type, t * in.K + k) != -__builtin_inff())
      some = true;
  return (in_vocabulary(in, id_at(in.targets, in.targets64, t)) ? 1 : 0) | (__any(some) ? 2 : 0);
}

// a wave a token
__global__ __launch_bounds__(256) void terms_kernel(HeadIn in, Of of, uint8_t* __restrict__ terms) {
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= in.T) return;
  const int v = terms_of(in, of, t, threadIdx.x & 63);
  if ((threadIdx.x & 63) == 0) terms[t] = (uint8_t)v;
}

// whether token t has a row: a loss; backward, one whose gradient is not zero
template <bool BWD>
__device__ __forceinline__ bool has_row(const HeadIn& in, const Of& of, const uint8_t* terms,
                                        int64_t t) {
  if constexpr (BWD)
    return head_terms(of.stats[kStatTerms * in.T + t]) != 0 && !(of.dloss[t] == 0.f);
  else
    return in.K > 0 ? terms[t] != 0
                    : in_vocabulary(in, id_at(in.targets, in.targets64, t));
}

// token t's gradient's size as bits (their order is the floats'), 0 where it has none
__device__ __forceinline__ int row_size(const HeadIn& in, const Of& of, int64_t t) {
  const float g = fabsf(of.dloss[t] * head_unit(in.alpha, in.tau));
  return g < __builtin_inff() ? __float_as_int(g) : 0;
}

// exponent of the largest value of token t's row of h times that of its gradient, kNowhere where
// it has none
constexpr int kNowhere = -100000;
__device__ __forceinline__ int row_reach(const HeadIn& in, const Of& of, int64_t t) {
  const float g = fabsf(of.dloss[t] * head_unit(in.alpha, in.tau));
  return g > 0.f && g < __builtin_inff()
             ? ilogbf(g) + head_exponent(of.stats[kStatTerms * in.T + t])
             : kNowhere;
}

// token t's row r
template <bool BWD>
__device__ __forceinline__ void put_row(const HeadIn& in, const Of& of, const Rows& out, int64_t t,
                                        int r) {
  out.idx[r] = (int)t;
  if constexpr (BWD) {
    const int64_t T = in.T;
    const float unit = head_unit(in.alpha, in.tau), g = of.dloss[t] * unit;
    const float m = ldexpf(g, of.shift - exp_of(g));
    const int terms = head_terms(of.stats[kStatTerms * T + t]);
    float c1 = terms & 1 ? (1.0f - in.alpha) / unit * m : 0.f;
    float c2 = terms & 2 ? in.alpha * in.tau / unit * m : 0.f;
    float lse_t = of.stats[kStatLseT * T + t];
    if (in.tau == 1.0f) {  // one softmax
      c1 += c2;
      lse_t = __int_as_float(in.K > 0 ? -1 : (int)id_at(in.targets, in.targets64, t));
      c2 = of.stats[kStatLabel * T + t] * m;
    }
    out.row[r] = HeadRow{of.stats[kStatLse * T + t], lse_t, c1, c2};
  }
}

// size: the largest of row_size; reach: of row_reach
__device__ __forceinline__ int exp_of_size(int size) {
  return size == 0 ? 0 : ilogbf(__int_as_float(size));
}
// exponent that h's copy is over: the largest gradient's, or in float16 the one that leaves the
// largest product with an exponent of 15, float16's largest
__device__ __forceinline__ int copy_exp(bool f16, int size, int reach) {
  if (!f16) return exp_of_size(size);
  return reach == kNowhere ? 0 : reach - 15;
}
__device__ __forceinline__ void put_exps(const HeadIn& in, const Of& of, const Rows& out, int size,
                                         int reach) {
  const int e = copy_exp(in.f16, size, reach);
  out.exps[0] = e;
  out.exps[1] = e - of.shift;
  out.exps[3] = __float_as_int(
      size == 0 ? 1.0f : ldexpf(__int_as_float(size), -exp_of_size(size)));
}

// Lists the rows in the tokens' order, where tokens are many.  A workgroup has `per` tokens (a
// multiple of 1024); it counts the rows before them by itself, then lists its own, 1024 at a time.
// At most 64 workgroups, so that counting again costs 32 reads a token at most.
template <bool BWD>
__global__ __launch_bounds__(1024) void rows_kernel(HeadIn in, Of of, int64_t per, Rows out) {
  __shared__ int sums[16];
  __shared__ int maxs[16], reaches[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t T = in.T, t0 = blockIdx.x * per, t1 = t0 + per < T ? t0 + per : T;
  int n = 0, e = 0, reach = kNowhere;
  // the first workgroup looks at all gradients for the largest
#pragma unroll 4
  for (int64_t t = tid; t < (BWD && blockIdx.x == 0 ? T : t0); t += 1024) {
    const bool yes = has_row<BWD>(in, of, out.terms, t);
    if (t < t0) n += yes;
    if constexpr (BWD)
      if (yes) {
        e = max(e, row_size(in, of, t));
        reach = max(reach, row_reach(in, of, t));
      }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    n += __shfl_xor(n, o, 64);
    if constexpr (BWD) {
      e = max(e, __shfl_xor(e, o, 64));
      reach = max(reach, __shfl_xor(reach, o, 64));
    }
  }
  if (lane == 0) {
    sums[wave] = n;
    maxs[wave] = e;
    reaches[wave] = reach;
  }
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    base += sums[w];
    e = max(e, maxs[w]);
    reach = max(reach, reaches[w]);
  }
  if constexpr (BWD)
    if (blockIdx.x == 0 && tid == 0) put_exps(in, of, out, e, reach);
  for (int64_t c = t0; c < t1; c += 1024) {
    const int64_t t = c + tid;
    const bool yes = t < t1 && has_row<BWD>(in, of, out.terms, t);
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
    if (yes) put_row<BWD>(in, of, out, t, r);
  }
  if (t1 == T && tid == 0) *out.count = base;
}

// The rows as the products read them, 64 rows x 64 columns a workgroup, through LDS:
//   ht[d][r] = h[idx[r]][d], the logits' second operand, with zeros up to a multiple of 128
//   columns d and of 256 rows r;
//   backward, hs[r] = h[idx[r]] times 2^(e - exps[0]), what dW contracts (NULL: not wanted).
// LIST (up to kListTokens tokens): every workgroup lists the rows by itself and the first one
// writes the list, which saves a launch (3 us).
constexpr int kListTokens = 1024;

template <bool F16, bool BWD, bool LIST>
__global__ __launch_bounds__(256) void gather_kernel(HeadIn in, Of of, Rows rows, int64_t tp,
                                                     uint16_t* __restrict__ ht,
                                                     uint16_t* __restrict__ hs) {
  __shared__ uint16_t s[64][72];
  __shared__ int list[LIST ? kListTokens : 1];
  __shared__ int sums[4][4], maxs[4], reaches[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int n, over = 0;
  if constexpr (LIST) {
    const bool first = blockIdx.x == 0 && blockIdx.y == 0;
    const int T = (int)in.T;
    bool yes[4];
    uint64_t mask[4];
    int e = 0, reach = kNowhere;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int t = 256 * c + tid;
      yes[c] = t < T && has_row<BWD>(in, of, rows.terms, t);
      if constexpr (BWD)
        if (yes[c]) {
          e = max(e, row_size(in, of, t));
          if constexpr (F16) reach = max(reach, row_reach(in, of, t));
        }
      mask[c] = __ballot(yes[c]);
      if (lane == 0) sums[c][wave] = __popcll(mask[c]);
    }
    if constexpr (BWD) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        e = max(e, __shfl_xor(e, o, 64));
        if constexpr (F16) reach = max(reach, __shfl_xor(reach, o, 64));
      }
      if (lane == 0) {
        maxs[wave] = e;
        reaches[wave] = reach;
      }
    }
    __syncthreads();
    n = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      int r = n + __popcll(mask[c] & ((uint64_t(1) << lane) - 1));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        r += w < wave ? sums[c][w] : 0;
        n += sums[c][w];
      }
      const int t = 256 * c + tid;
      if (yes[c]) list[r] = t;
      if (first && t < T) {
        rows.pos[t] = yes[c] ? r : -1;
        if (yes[c]) put_row<BWD>(in, of, rows, t, r);
      }
    }
    if constexpr (BWD) {
      e = max(max(maxs[0], maxs[1]), max(maxs[2], maxs[3]));
      reach = max(max(reaches[0], reaches[1]), max(reaches[2], reaches[3]));
      over = copy_exp(F16, e, reach);
      if (first && tid == 0) put_exps(in, of, rows, e, reach);
    }
    if (first && tid == 0) *rows.count = n;
    __syncthreads();
  } else {
    n = *rows.count;
    if constexpr (BWD) over = rows.exps[0];
  }
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  if (r0 >= up256(n)) return;
  const int d0 = blockIdx.y * 64, q = tid >> 3, c = 8 * (tid & 7);
#pragma unroll
  for (int i = 0; i < 64; i += 32) {
    const int64_t r = r0 + q + i;
    u32x4 v = {0, 0, 0, 0};
    if (r < n && d0 + c < in.D) {
      const int64_t t = LIST ? list[r] : rows.idx[r];
      v = ld16(in.h + t * in.D + d0 + c);
      if constexpr (BWD)
        if (hs) {
          const int e = exp_of(of.dloss[t] * head_unit(in.alpha, in.tau)) - over;
          u32x4 o = v;
          if (e != 0) {
            float x[8];
            widen<F16>(v, x);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              o[j] = (uint32_t)narrow<F16>(ldexpf(x[2 * j], e)) |
                     (uint32_t)narrow<F16>(ldexpf(x[2 * j + 1], e)) << 16;
          }
          st16(hs + r * in.D + d0 + c, o);
        }
    }
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

// (few_kernel) tokens whose kept words every workgroup looks up by itself, for a launch less
constexpr int kListTeach = 16;

// Softmax sums of up to 64 tokens, 16 NT: a read of W.  Every wave has a run of V / waves words to
// itself, 64 at a time as four blocks of 16 x 16 x 32 matrix products with the tokens; W goes
// from memory to registers (no other wave wants it), four steps of 64 columns ahead, 32 KiB a
// wave, h from LDS, kCols columns at a time.  Every workgroup lists the rows by itself, the
// first one writes the list.  part as the logits' kernel leaves it, one tile of tokens and a tile
// of words a workgroup.
// Bound: HBM (50000 x 2048, W in memory, the call: 1 token 46 us, 16 50, 64 60; by tiles of 64
// tokens 62, 64 and 66; 5000 words: 28, 47 by tiles).  R = 8 and so twice the loads in flight:
// 53 us; R = 2: 49, but 32 for 5000 words.
template <bool F16, bool TEMP, int NT>
__global__ __launch_bounds__(256) void few_kernel(HeadIn in, Of of, Rows rows,
                                                  float* __restrict__ part) {
  constexpr int E = TEMP ? 3 : 2, NB = 4, R = 4;
  constexpr int kCols = 4096 / NT, kPitch = 2 * kCols + 16;
  __shared__ __attribute__((aligned(16))) uint8_t hl[16 * NT * kPitch];
  __shared__ float sums[4][16 * NT][3];
  __shared__ int list[64];
  __shared__ int found;
  __shared__ uint8_t few[kListTeach];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = (int)in.T, D = in.D, V = (int)in.V;
  const int waves = 4 * gridDim.x, wv = 4 * blockIdx.x + wave;
  const int v_beg = (int)((int64_t)wv * V / waves), v_end = (int)((int64_t)(wv + 1) * V / waves);
  const int blocks = ((V + waves - 1) / waves + 16 * NB - 1) / (16 * NB);  // of every wave's run
  const int nit = (D + 63) / 64;
  // A wave takes a chunk's columns from a place of its own on, and a workgroup the chunks, where
  // 64 tokens make them short and all are whole: rows are often a power of two apart, and waves
  // in step would ask the same memory channels (50000 x 2048, 16 tokens: 50 us, 59 in step; 64
  // tokens: 60, 66 with the chunks in step).
  constexpr int C = kCols / 64;
  const int chunks = (nit + C - 1) / C, last = (chunks - 1) * C, c_last = nit - last;
  const int turn = NT == 4 && c_last == C ? blockIdx.x % chunks : 0;
  const int rot = (wv * 5) % C, rot_last = (wv * 5) % c_last;
  auto chunk = [&](int i) {  // the first step of the i-th step's chunk
    if constexpr (NT < 4) return i >= last ? last : i / C * C;
    const int p = i / C + turn;
    return (p >= chunks ? p - chunks : p) * C;
  };
  auto step = [&](int i) {  // the i-th step's columns, in 64s
    const int base = chunk(i), c = base == last ? c_last : C;
    const int k = i % C + (base == last ? rot_last : rot);
    return base + (k >= c ? k - c : k);
  };
  int words = 0;  // of the block that the loads are for
  const uint16_t* w[NB];
  u32x4 a[R][NB][2];
  auto load = [&](u32x4 (&to)[NB][2], int i) {
    const int k = 64 * step(i < nit ? i : nit - 1) + 8 * g;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int x = 0; x < 2; ++x) to[b][x] = ld16(w[b] + (k + 32 * x < D ? k + 32 * x : D - 8));
  };
  auto begin = [&](int blk) {
    const int v0 = v_beg + (int)((int64_t)(v_end - v_beg) * blk / blocks);
    words = v_beg + (int)((int64_t)(v_end - v_beg) * (blk + 1) / blocks) - v0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {  // (rows past the block's: its last one)
      const int r = 16 * b + l16 < words ? 16 * b + l16 : words > 0 ? words - 1 : 0;
      w[b] = in.w + (int64_t)(v0 + r < V ? v0 + r : V - 1) * D;
    }
#pragma unroll
    for (int j = 0; j < R; ++j) load(a[j], j);
  };
  begin(0);  // W's first columns are under way while the rows are listed and h is copied
  __builtin_amdgcn_sched_barrier(0);

  const bool first = blockIdx.x == 0;
  const uint8_t* terms = rows.terms;
  if (in.K > 0 && T <= kListTeach) {
    for (int t = wave; t < T; t += 4) {
      const int v = terms_of(in, of, t, lane);
      if (lane == 0) {
        few[t] = (uint8_t)v;
        if (first) rows.terms[t] = (uint8_t)v;
      }
    }
    __syncthreads();
    terms = few;
  }
  if (wave == 0) {
    const bool yes = lane < T && has_row<false>(in, of, terms, lane);
    const uint64_t mask = __ballot(yes);
    const int r = __popcll(mask & ((uint64_t(1) << lane) - 1));
    if (yes) list[r] = lane;
    if (lane == 0) found = __popcll(mask);
    if (first) {
      if (lane < T) rows.pos[lane] = yes ? r : -1;
      if (lane == 0) *rows.count = __popcll(mask);
    }
  }
  __syncthreads();
  const int n = __builtin_amdgcn_readfirstlane(found);
  if (n == 0) return;

  auto fill = [&](int base) {  // h's columns from 64 base on, 4096 pieces of 8 at once
    const int per = 8 * (nit - base < C ? nit - base : C);  // pieces of a row
    const int dr = 256 / per, dc = 256 - dr * per;
    int r = tid / per, c = tid - r * per;
    while (__any(r < n)) {
      u32x4 v[16];
      int at[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int col = 64 * base + 8 * c;
        at[j] = r < n ? r * kPitch + 16 * c : -1;
        v[j] = ld16(in.h + (int64_t)list[r < n ? r : 0] * D + (col < D ? col : 0));
        if (col >= D) v[j] = u32x4{0, 0, 0, 0};
        r += dr;
        c += dc;
        if (c >= per) {
          c -= per;
          ++r;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (at[j] >= 0) st16(hl + at[j], v[j]);
    }
  };

  const float k1 = kLog2e, k2 = kLog2e / in.tau;
  float mx[NT], sm[NT], st[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    mx[t] = -__builtin_inff();
    sm[t] = st[t] = 0.f;
  }
  for (int blk = 0; blk < blocks; ++blk) {
    f32x4 acc[NB][NT];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < nit; i0 += R) {
      if (i0 % C == 0 && (nit > C || blk == 0)) {
        __syncthreads();  // the columns before have been read
        fill(chunk(i0));
        __syncthreads();
      }
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if (i0 + j < nit) {
          const int at = step(i0 + j), k = 64 * at + 8 * g;
          const uint8_t* hp = hl + l16 * kPitch + 128 * (at % C) + 16 * g;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const bool in_row = k + 32 * x < D;
            u32x4 wf[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b)
              wf[b] = in_row ? a[j][b][x] : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const u32x4 hf = *reinterpret_cast<const u32x4*>(hp + 16 * t * kPitch + 64 * x);
#pragma unroll
              for (int b = 0; b < NB; ++b) acc[b][t] = mfma_16<F16>(wf[b], hf, acc[b][t]);
            }
          }
        }
        load(a[j], i0 + j + R);
      }
    }
    // a lane: token 16 t + l16, words 16 b + 4 g + i
    const int left = words;
    if (blk + 1 < blocks) begin(blk + 1);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float m = mx[t];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (16 * b + 4 * g + i >= left) acc[b][t][i] = -__builtin_inff();
          m = fmaxf(m, acc[b][t][i]);
        }
      const float ref = m == -__builtin_inff() ? 0.f : m;
      float s = sm[t] * __builtin_amdgcn_exp2f((mx[t] - ref) * k1);
      float sT = TEMP ? st[t] * __builtin_amdgcn_exp2f((mx[t] - ref) * k2) : 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s += __builtin_amdgcn_exp2f((acc[b][t][i] - ref) * k1);
          if constexpr (TEMP) sT += __builtin_amdgcn_exp2f((acc[b][t][i] - ref) * k2);
        }
      mx[t] = m;
      sm[t] = s;
      st[t] = sT;
    }
  }
  // (m, s, sT) of two runs of words
  auto both = [&](float& m, float& s, float& sT, float om, float os, float oT) {
    const float top = fmaxf(m, om), ref = top == -__builtin_inff() ? 0.f : top;
    s = s * __builtin_amdgcn_exp2f((m - ref) * k1) + os * __builtin_amdgcn_exp2f((om - ref) * k1);
    if constexpr (TEMP)
      sT = sT * __builtin_amdgcn_exp2f((m - ref) * k2) +
           oT * __builtin_amdgcn_exp2f((om - ref) * k2);
    m = top;
  };
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int o = 16; o < 64; o <<= 1)
      both(mx[t], sm[t], st[t], __shfl_xor(mx[t], o, 64), __shfl_xor(sm[t], o, 64),
           TEMP ? __shfl_xor(st[t], o, 64) : 0.f);
    if (g == 0) {
      float* p = sums[wave][16 * t + l16];
      p[0] = mx[t];
      p[1] = sm[t];
      p[2] = st[t];
    }
  }
  __syncthreads();
  const int e = tid >> 6;
  if (e < 2 && lane < n) {
    const float *x = sums[2 * e][lane], *y = sums[2 * e + 1][lane];
    float m = x[0], s = x[1], sT = x[2];
    both(m, s, sT, y[0], y[1], y[2]);
    float* p = part + ((int64_t)(2 * blockIdx.x + e) * 256 + lane) * E;
    p[0] = m;
    p[1] = s;
    if constexpr (TEMP) p[2] = sT;
  }
}

// What the losses are made from
struct Finish {
  HeadIn in;
  const void* top;
  int top_type;
  const float* part;
  int tile, grid;  // tokens of a tile and workgroups of the logits' launch
  int64_t nv;      // its tiles of words
  Rows rows;
  float* loss;
  float* stats;
};

// h . w[i] for N rows w over the lanes of a wave, in every lane; UNROLL steps of 512
// columns under way at once.  Returns the size of the largest of the lane's values of h, where F16
// (0 else).
template <bool F16, int N, int UNROLL>
__device__ __forceinline__ float row_dots(const uint16_t* h, const uint16_t* const* w, int D,
                                          int lane, float (&s)[N]) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = 0.f;
#pragma unroll UNROLL
  for (int d = lane * 8; d < D; d += 512) {
    float x[8], y[8];
    widen<F16>(ld16(h + d), x);
    if constexpr (F16) {
#pragma unroll
      for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[j]));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      widen<F16>(ld16(w[i] + d), y);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i] = __builtin_fmaf(x[j], y[j], s[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
  return most;
}

// the exponent of a row's largest value, from what row_dots left in the lanes (an infinity's: 15)
template <bool F16>
__device__ __forceinline__ int row_exponent(float most) {
  if constexpr (!F16) return -25;
  const float m = wave_max(most);
  return m == 0.f ? -25 : m < 65536.f ? ilogbf(m) : 15;
}

// the softmax sums of row r: the parts of its token tile's workgroups, joined.  m: the largest
// logit; s: sum of 2^(log2e (z - m)); sT the same at the temperature (TEMP)
template <bool TEMP>
__device__ __forceinline__ void join(const float* part, int r, int n, int64_t nv, int tile,
                                     int grid, float k2, int lane, float& m, float& s, float& sT) {
  constexpr int E = TEMP ? 3 : 2, N = 8;
  const int64_t nt = (n + tile - 1) / tile, all = nt * nv;
  const int64_t P = all < grid ? all : grid;
  const int64_t j = r / tile;
  // the workgroups whose runs hold the tile's first and last item
  const int64_t w0 = ((j * nv + 1) * P - 1) / all, w1 = (((j + 1) * nv) * P - 1) / all;
  const int cnt = (int)(w1 - w0 + 1) * 2;
  const float* at = part + ((w0 + j) * 512 + r % tile) * E;
  float a = 0.f, b = 0.f;
  m = -__builtin_inff();
  for (int i0 = 0; i0 < cnt; i0 += 64 * N) {  // N at once: their loads overlap
    float pm[N], ps[N], pt[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = i0 + 64 * k + lane;
      const float* p = at + (int64_t)(i < cnt ? i : 0) * 256 * E;
      pm[k] = i < cnt ? p[0] : -__builtin_inff();
      ps[k] = i < cnt ? p[1] : 0.f;
      if constexpr (TEMP) pt[k] = i < cnt ? p[2] : 0.f;
    }
    const float old = m;
#pragma unroll
    for (int k = 0; k < N; ++k) m = fmaxf(m, pm[k]);
    const float ref = m == -__builtin_inff() ? 0.f : m;
    a *= __builtin_amdgcn_exp2f((old - ref) * kLog2e);
    if constexpr (TEMP) b *= __builtin_amdgcn_exp2f((old - ref) * k2);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      a += ps[k] * __builtin_amdgcn_exp2f((pm[k] - ref) * kLog2e);
      if constexpr (TEMP) b += pt[k] * __builtin_amdgcn_exp2f((pm[k] - ref) * k2);
    }
  }
  const float mine = m;
  m = wave_max(m);
  const float ref = m == -__builtin_inff() ? 0.f : m;
  s = wave_sum(a * __builtin_amdgcn_exp2f((mine - ref) * kLog2e));
  sT = TEMP ? wave_sum(b * __builtin_amdgcn_exp2f((mine - ref) * k2)) : s;
}

// A row's softmax: the largest logit (0 for a row without one), log2 of the sums, the sums'
// logarithms, and the factors of the two gradients over the unit
struct Softmax {
  float m, lse, lse_t, ln, ln_t, c1, c2, k2;
  // gradient over the unit at a word with logit z; hit: its share of the label and the teacher
  __device__ __forceinline__ float grad(float z, float hit) const {
    return c1 * __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -lse)) +
           c2 * __builtin_amdgcn_exp2f(__builtin_fmaf(z, k2, -lse_t)) - hit;
  }
};

template <bool TEMP>
__device__ __forceinline__ Softmax softmax_of(const Finish& f, int64_t t, int terms, int lane) {
  const HeadIn& in = f.in;
  Softmax x;
  x.k2 = kLog2e / in.tau;
  float m, s, sT;
  join<TEMP>(f.part, f.rows.pos[t], *f.rows.count, f.nv, f.tile, f.grid, x.k2, lane, m, s, sT);
  x.m = m == -__builtin_inff() ? 0.f : m;  // (as the sums took it)
  const float l = __builtin_amdgcn_logf(s), lT = __builtin_amdgcn_logf(sT);
  x.lse = __builtin_fmaf(x.m, kLog2e, l);
  x.lse_t = __builtin_fmaf(x.m, x.k2, lT);
  x.ln = l * kLn2;
  x.ln_t = lT * kLn2;
  const float unit = head_unit(in.alpha, in.tau);
  x.c1 = terms & 1 ? (1.0f - in.alpha) / unit : 0.f;
  x.c2 = terms & 2 ? in.alpha * in.tau / unit : 0.f;
  return x;
}

__device__ __forceinline__ void put_stats(const Finish& f, int64_t t, float loss, float lse,
                                          float lse_t, float terms, float label) {
  float* st = f.stats + t;  // the token's place in each plane
  f.loss[t] = loss;
  st[kStatLse * f.in.T] = lse;
  st[kStatLseT * f.in.T] = lse_t;
  st[kStatTerms * f.in.T] = terms;
  st[kStatLabel * f.in.T] = label;
}

// The cross entropy and the stats of a token, a wave a token
template <bool F16>
__global__ __launch_bounds__(256) void finish_kernel(Finish f) {
  const HeadIn& in = f.in;
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= in.T) return;
  const int64_t y = id_at(in.targets, in.targets64, t);
  if (!in_vocabulary(in, y)) {
    if (lane == 0) put_stats(f, t, 0.f, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  float z[1];
  const uint16_t* const w[1] = {in.w + y * in.D};
  const float most = row_dots<F16, 1, 4>(in.h + t * in.D, w, in.D, lane, z);
  const float terms = head_stat_terms(1, row_exponent<F16>(most));
  const Softmax x = softmax_of<false>(f, t, 1, lane);
  if (lane == 0) put_stats(f, t, x.ln + (x.m - z[0]), x.lse, x.lse, terms, x.grad(z[0], 1.0f));
}

// The same with a teacher, a workgroup of WAVES waves a token: four, or sixteen where tokens
// are few and their words many (run_finish).  Entry 0 is the label, the others
// the teacher's words: their logits are dealt over the waves, four or five at a time; of four
// waves each makes the softmaxes by itself.  Bound: the words' rows of W from the caches (16384 tokens of
// 64 words of 2048 columns, 4.3 GB: 330 us).
template <bool F16, bool TEMP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void teach_kernel(Finish f) {
  constexpr int L = 64 * WAVES;
  // sixteen waves: the last one makes the softmaxes while the others make the logits
  constexpr bool SPLIT = WAVES == 16;
  constexpr int DOTS = SPLIT ? WAVES - 1 : WAVES, N = SPLIT ? 5 : 4;
  extern __shared__ float sh[];  // K + 1 each: logits; teacher's logits, probabilities; words
  // (the teacher's logits as they are, -infinity: not kept; over tau only what is left of them once
  // their largest is taken off, or float32's lowest value, a usual mask, would leave its range)
  __shared__ Softmax shared_x;
  __shared__ float shared_t[2];
  const HeadIn& in = f.in;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const int n = in.K + 1;
  float* st_top = f.stats + kStatPlanes * in.T + t * in.K;
  const int terms = f.rows.terms[t];
  if (terms == 0) {  // no loss
    for (int i = tid; i < in.K; i += L) st_top[i] = 0.f;
    if (tid == 0) put_stats(f, t, 0.f, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  float *z = sh, *q = sh + n, *p = sh + 2 * n;
  int* id = reinterpret_cast<int*>(sh + 3 * n);
  const float it = 1.0f / in.tau;
  for (int e = tid; e < n; e += L) {
    const int64_t v = e == 0 ? id_at(in.targets, in.targets64, t)
                             : id_at(in.ids, in.ids64, t * in.K + e - 1);
    const bool ok = in_vocabulary(in, v);
    id[e] = ok ? (int)v : -1;
    q[e] = ok && e > 0 ? top_at(f.top, f.top_type, t * in.K + e - 1) : -__builtin_inff();
  }
  __syncthreads();
  const uint16_t* h = in.h + t * in.D;
  float most = 0.f;
  if (wave < DOTS)
    for (int e0 = N * wave; e0 < n; e0 += N * DOTS) {
      float d[N];
      const uint16_t* w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = e0 + i < n ? e0 + i : n - 1;
        w[i] = in.w + (int64_t)(id[e] >= 0 ? id[e] : 0) * in.D;
      }
      most = row_dots<F16, N, SPLIT ? 4 : 1>(h, w, in.D, lane, d);
      if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (e0 + i < n) z[e0 + i] = d[i];
    }
  Softmax x;
  float tm = -__builtin_inff(), tl = 0.f;
  if (!SPLIT || wave == DOTS) {
    x = softmax_of<TEMP>(f, t, terms, lane);
    // the teacher's softmax over its kept words
    float ts = 0.f;
    for (int e = lane; e < n; e += 64) tm = fmaxf(tm, q[e]);
    tm = wave_max(tm);
    for (int e = lane; e < n; e += 64)
      if (q[e] != -__builtin_inff()) ts += __builtin_amdgcn_exp2f((q[e] - tm) * it * kLog2e);
    tl = __builtin_amdgcn_logf(wave_sum(ts)) * kLn2;
    for (int e = SPLIT ? lane : tid; e < n; e += SPLIT ? 64 : L)
      p[e] = q[e] != -__builtin_inff()
                 ? __builtin_amdgcn_exp2f(((q[e] - tm) * it - tl) * kLog2e)
                 : 0.f;
    if (SPLIT && lane == 0) {
      shared_x = x;
      shared_t[0] = tm;
      shared_t[1] = tl;
    }
  }
  __syncthreads();
  if constexpr (SPLIT) {
    x = shared_x;
    tm = shared_t[0];
    tl = shared_t[1];
  }
  if (wave == 0) {
    float kl = 0.f;
    for (int e = lane; e < n; e += 64)  // ln q - ln s, s = e^((z - m) / tau) / sum
      if (p[e] != 0.f) kl += p[e] * (((q[e] - tm) * it - tl) - ((z[e] - x.m) * it - x.ln_t));
    kl = wave_sum(kl);
    if (lane == 0)
      f.loss[t] = (terms & 1 ? (1.0f - in.alpha) * (x.ln + (x.m - z[0])) : 0.f) +
                  (terms & 2 ? in.alpha * in.tau * in.tau * kl : 0.f);
  }
  const int y = id[0], exponent = row_exponent<F16>(most);  // (the first wave's counts)
  for (int e = tid; e < n; e += L) {
    const int v = id[e];
    float hit = 0.f;
#pragma unroll 8
    for (int j = 1; j < n; ++j) hit += id[j] == v ? p[j] : 0.f;
    const float g = v >= 0 ? x.grad(z[e], x.c2 * hit + (v == y ? x.c1 : 0.f)) : 0.f;
    if (e == 0) {
      float* st = f.stats + t;
      st[kStatLse * in.T] = x.lse;
      st[kStatLseT * in.T] = x.lse_t;
      st[kStatTerms * in.T] = head_stat_terms(terms, exponent);
      st[kStatLabel * in.T] = g;
    } else {
      st_top[e - 1] = g;
    }
  }
}

// With a teacher: the label's and its words of the piece, over the dense dlogits.  (A label
// alone is stored with its tile: a launch less, 5 us.)
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
  const int terms = head_terms(stats[kStatTerms * in.T + t]);
  if (!(terms & (e == 0 ? 1 : 2))) return;
  const int64_t v =
      (e == 0 ? id_at(in.targets, in.targets64, t) : id_at(in.ids, in.ids64, t * in.K + e - 1)) -
      w0;
  if (v < 0 || v >= n) return;
  const float g = dloss[t] * head_unit(in.alpha, in.tau);
  const float x = stats[e == 0 ? kStatLabel * in.T + t : kStatPlanes * in.T + t * in.K + e - 1];
  const float m = ldexpf(g, kHeadShift<F16> - exp_of(g)) / __int_as_float(rows.exps[3]);
  G[r * ld + v] = narrow<F16>(x * m);
}

// dh[t] = 2^(e - shift) times the sum of the row's parts; zeros for a token without a row.
// A wave has 512 columns.
template <bool F16>
__global__ __launch_bounds__(64) void dh_out_kernel(HeadIn in, const float* __restrict__ dloss,
                                                    Rows rows, const float* __restrict__ part,
                                                    uint16_t* __restrict__ dh) {
  const int64_t t = blockIdx.x;
  const int d = (blockIdx.y * 64 + threadIdx.x) * 8;
  if (d >= in.D) return;
  const int r = rows.pos[t];
  const int e = exp_of(dloss[t] * head_unit(in.alpha, in.tau)) - kHeadShift<F16>;
  u32x4 o = {0, 0, 0, 0};
  if (r >= 0) {
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    const float* p = part + (int64_t)r * in.D + d;
    const float m = __int_as_float(rows.exps[3]);
    const int n = *rows.count, parts = rows.exps[2];
#pragma unroll 8
    for (int s = 0; s < parts; ++s) {
      a += *reinterpret_cast<const f32x4*>(p);
      b += *reinterpret_cast<const f32x4*>(p + 4);
      p += (int64_t)n * in.D;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o[i] = (uint32_t)narrow<F16>(ldexpf(m * a[2 * i], e)) |
             (uint32_t)narrow<F16>(ldexpf(m * a[2 * i + 1], e)) << 16;
      o[2 + i] = (uint32_t)narrow<F16>(ldexpf(m * b[2 * i], e)) |
                 (uint32_t)narrow<F16>(ldexpf(m * b[2 * i + 1], e)) << 16;
    }
  }
  st16(dh + t * in.D + d, o);
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
  p.nst_h = (int)((words + 127) / 128 * 4);
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
  take(&l.rows.exps, b, &l.bytes, 16);
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

// Softmax sums of up to kFewTokens tokens, without gather's copies
constexpr int kFewTokens = 64;

static int few_grid(int64_t V) {
  const int64_t cus = current_cu_count(), n = (V + 15) / 16;
  return (int)(n < cus ? n : cus);
}

template <bool F16>
static hipError_t run_few(const HeadIn& in, const Of& of, const Layout& l, hipStream_t stream) {
  if (in.K > 0 && in.T > kListTeach) {
    hipLaunchKernelGGL(terms_kernel, dim3((unsigned)((in.T + 3) / 4)), dim3(256), 0, stream, in, of,
                       l.rows.terms);
    TM_RET(hipGetLastError());
  }
  const dim3 grid((unsigned)few_grid(in.V));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, in, of, l.rows, l.part);
    return hipGetLastError();
  };
  const bool temp = in.K > 0 && in.tau != 1.0f;
  if (in.T <= 16) return temp ? go(few_kernel<F16, true, 1>) : go(few_kernel<F16, false, 1>);
  if (in.T <= 32) return temp ? go(few_kernel<F16, true, 2>) : go(few_kernel<F16, false, 2>);
  return temp ? go(few_kernel<F16, true, 4>) : go(few_kernel<F16, false, 4>);
}

// the rows, their list and their copies
template <bool F16, bool BWD>
static hipError_t gather(const HeadIn& in, const Of& of, const Layout& l, uint16_t* hs,
                         hipStream_t stream) {
  const bool list = in.T <= kListTokens;
  if (!BWD && in.K > 0) {
    hipLaunchKernelGGL(terms_kernel, dim3((unsigned)((in.T + 3) / 4)), dim3(256), 0, stream, in, of,
                       l.rows.terms);
    TM_RET(hipGetLastError());
  }
  const dim3 grid((unsigned)(head_padded(in.T) / 64), (unsigned)(up128(in.D) / 64));
  if (list) {
    hipLaunchKernelGGL((gather_kernel<F16, BWD, true>), grid, dim3(256), 0, stream, in, of, l.rows,
                       head_padded(in.T), l.ht, hs);
    return hipGetLastError();
  }
  const int64_t per = ((in.T + 63) / 64 + 1023) / 1024 * 1024;
  hipLaunchKernelGGL(rows_kernel<BWD>, dim3((unsigned)((in.T + per - 1) / per)), dim3(1024), 0,
                     stream, in, of, per, l.rows);
  TM_RET(hipGetLastError());
  hipLaunchKernelGGL((gather_kernel<F16, BWD, false>), grid, dim3(256), 0, stream, in, of, l.rows,
                     head_padded(in.T), l.ht, hs);
  return hipGetLastError();
}

template <bool F16, int WAVES>
static hipError_t run_teach(const Finish& f, hipStream_t stream) {
  const dim3 grid((unsigned)f.in.T), block(64 * WAVES);
  const unsigned lds = 16 * (f.in.K + 1);
  if (f.in.tau != 1.0f)
    hipLaunchKernelGGL((teach_kernel<F16, true, WAVES>), grid, block, lds, stream, f);
  else
    hipLaunchKernelGGL((teach_kernel<F16, false, WAVES>), grid, block, lds, stream, f);
  return hipGetLastError();
}

template <bool F16>
static hipError_t run_finish(const Finish& f, hipStream_t stream) {
  // Sixteen waves while every token's workgroup finds a CU of its own, and from 28 words on (50000
  // x 2048, sixteen and four waves: 1 token of 24 words 12.0 and 11.8 us, of 32 12.5 and 14.1, of 64
  // 15.0 and 20.5; 256 tokens of 24 words 14.0 and 13.6, of 32 14.8 and 16.0, of 64 19.0 and 23.5;
  // 257 tokens of 64 words 26.5 and 22.6).
  if (f.in.K > 0)
    return f.in.T <= current_cu_count() && f.in.K >= 28 ? run_teach<F16, 16>(f, stream)
                                         : run_teach<F16, 4>(f, stream);
  hipLaunchKernelGGL(finish_kernel<F16>, dim3((unsigned)((f.in.T + 3) / 4)), dim3(256), 0, stream,
                     f);
  return hipGetLastError();
}

hipError_t launch_head_loss(const HeadIn& in, const void* top, int top_type, float* loss,
                            float* stats, void* workspace, hipStream_t stream) {
  const Layout l = forward_layout(in.T, in.V, in.D, workspace);
  const Of of{top, top_type, nullptr, nullptr, 0};
  Finish f{in, top, top_type, l.part, kFewTokens, 0, 0, l.rows, loss, stats};
  if (in.T <= kFewTokens) {
    f.nv = f.grid = few_grid(in.V);
    TM_RET(in.f16 ? run_few<true>(in, of, l, stream) : run_few<false>(in, of, l, stream));
  } else {
    f.tile = head_tile_tokens(in.T, in.V, true);
    f.grid = head_logits_grid(in.T, in.V, f.tile);
    f.nv = (in.V + 255) / 256;
    TM_RET(in.f16 ? (gather<true, false>(in, of, l, nullptr, stream))
                  : (gather<false, false>(in, of, l, nullptr, stream)));
    TM_RET(launch_head_logits(in, l.ht, l.rows.count, l.part, stream));
  }
  return in.f16 ? run_finish<true>(f, stream) : run_finish<false>(f, stream);
}

template <bool F16>
static hipError_t run_bwd(const HeadIn& in, const float* stats, const float* dloss, uint16_t* dh,
                          void* dw, int dw_type, bool accumulate, void* workspace,
                          hipStream_t stream) {
  const HeadPlan p = head_plan(in.T, in.V, in.D);
  const Layout l = backward_layout(in.T, in.V, in.D, p, workspace);
  const Of of{nullptr, 0, stats, dloss, kHeadShift<F16>};
  TM_RET((gather<F16, true>(in, of, l, dw ? l.hs : nullptr, stream)));
  for (int64_t i = 0; i < p.pieces; ++i) {
    const int64_t w0 = i * p.piece, n = in.V - w0 < p.piece ? in.V - w0 : p.piece;
    TM_RET(launch_head_dlogits(in, l.ht, l.rows.count, l.rows.row, l.rows.exps + 3, w0, n, l.G, p.piece,
                               stream));
    if (in.K > 0) {
      hipLaunchKernelGGL(sparse_kernel<F16>, dim3((unsigned)((in.T * (in.K + 1) + 255) / 256)),
                         dim3(256), 0, stream, in, stats, dloss, l.rows, w0, n, l.G, p.piece);
      TM_RET(hipGetLastError());
    }
    if (dh)
      TM_RET(launch_head_dh(in, l.rows.count, l.G, p.piece, w0, n, HeadCut{p.parts_h, p.per_h},
                            p.nst_h, i > 0, l.part_h, l.rows.exps + 2, stream));
    const bool last = i == p.pieces - 1;
    if (dw)
      TM_RET(launch_head_dw(in, l.rows.count, l.G, p.piece, l.hs, w0, n, last ? p.last_w : p.parts_w,
                          last ? p.last_per : p.per_w, l.rows.exps + 1, dw, dw_type, accumulate, l.part_w, stream));
  }
  if (dh)
    hipLaunchKernelGGL(dh_out_kernel<F16>, dim3((unsigned)in.T, (unsigned)((in.D + 511) / 512)),
                       dim3(64), 0, stream, in, dloss, l.rows, l.part_h, dh);
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
