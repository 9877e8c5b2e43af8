// Rows of an embedding, e[t] = scale W[id_t] (float32, the residual stream's
// type), and the gradient of its weight, dW[v] = scale sum_{t: id_t = v} de[t],
// the tokens of a row in ascending order, so that repeated calls give the same
// bits.  An id outside [0, V) gives a row of zeros and no gradient.
//
// The gradient is bound by writing dW's V rows.  Few tokens are found by going
// through the ids (embed_direct_kernel, embed_first_kernel).  Many are sorted by id
// into segments: a count per id, a place per segment (whichever: only the order
// inside a segment shows in the sums), and the positions, in any order, which the
// workgroup of a row brings into ascending order.  An id of more than
// kEmPiece tokens (the most frequent one of a text is a tenth of it) is cut
// into pieces of that many, whose sums meet in the row's workgroup; a piece
// finds its tokens by going through the ids, which are few bytes.  16384 tokens,
// 50000 ids of 2048 columns: 149 us, 100 of them for the rows (4.8 TB/s).
#include "seq.hpp"
#include "seq_launch.hpp"

namespace tmk {

constexpr int kEmPiece = 64;    // tokens of a piece
// Tokens that a row's workgroup goes through by itself: one launch (256 tokens, 1000
// ids of 512: 7 us).
constexpr int kEmDirect = 256, kEmDirectV = 16384;
// Tokens that a token's workgroup does; from there on the sort's launches are less
// than T workgroups that each read T ids (4000 tokens, 10000 ids of 1024: 29 us, 37
// sorted).
constexpr int kEmScan = 4096;

template <typename I>
__device__ __forceinline__ int64_t em_id(const I* ids, int64_t t, int64_t V) {
  const int64_t v = (int64_t)ids[t];
  return v >= 0 && v < V ? v : -1;
}

// TYPE 0 float32, 1 bfloat16, 2 float16
template <int TYPE>
__device__ __forceinline__ void em_ld8(const void* w, int64_t at, float (&v)[8]) {
  if constexpr (TYPE == 0) {
    Zx<true>::ld8((const float*)w + at, v);
  } else if constexpr (TYPE == 1) {
    Zx<false>::ld8((const uint16_t*)w + at, v);
  } else {
    typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
    const f16x8 h = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(
        (const u32x4_u2*)((const uint16_t*)w + at)));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
  }
}
template <int TYPE>
__device__ __forceinline__ float em_ld(const void* w, int64_t at) {
  if constexpr (TYPE == 0) return ((const float*)w)[at];
  else if constexpr (TYPE == 1) return __uint_as_float((uint32_t)((const uint16_t*)w)[at] << 16);
  else return (float)__builtin_bit_cast(_Float16, ((const uint16_t*)w)[at]);
}

// grid (T), 256 threads
template <int TYPE, typename I>
__global__ __launch_bounds__(256) void embed_kernel(const I* __restrict__ ids, int64_t V,
                                                    int64_t D, const void* __restrict__ w,
                                                    float scale, float* __restrict__ out) {
  const int64_t t = blockIdx.x;
  const int64_t v = em_id(ids, t, V);
  float* o = out + t * D;
  const int64_t D8 = D & ~(int64_t)7;
  for (int64_t c = (int64_t)threadIdx.x * 8; c < D8; c += 256 * 8) {
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (v >= 0) {
      em_ld8<TYPE>(w, v * D + c, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= scale;
    }
    Zx<true>::st8(o + c, x);
  }
  const int64_t c = D8 + threadIdx.x;
  if (c < D) o[c] = v >= 0 ? em_ld<TYPE>(w, v * D + c) * scale : 0.f;
}

// the workspace: count, place (the first piece's number where an id is in
// pieces), filled [V] each; cursors [2] (of tokens, of pieces); sorted [T]; a
// piece's id and its number in its row [pieces] each; pieces' sums [pieces][D]
struct EmbedWs {
  int *count, *place, *filled, *cursor, *sorted, *pid, *pno;
  float* psum;
};
static int64_t em_pieces(int64_t T) { return 2 * (T / kEmPiece) + 1; }
static int64_t em_ints(int64_t T, int64_t V) {
  return (3 * V + 2 + T + 2 * em_pieces(T) + 63) / 64 * 64;
}
static EmbedWs em_ws(void* p, int64_t T, int64_t V) {
  EmbedWs w;
  int* i = (int*)p;
  w.count = i, w.place = i + V, w.filled = i + 2 * V, w.cursor = i + 3 * V;
  w.sorted = w.cursor + 2;
  w.pid = w.sorted + T;
  w.pno = w.pid + em_pieces(T);
  w.psum = (float*)(i + em_ints(T, V));
  return w;
}
int64_t embed_bwd_bytes(int64_t T, int64_t V, int64_t D) {
  if (T <= kEmScan) return 0;
  return em_ints(T, V) * 4 + em_pieces(T) * D * 4;
}

__global__ __launch_bounds__(256) void embed_clear_kernel(EmbedWs w, int64_t V) {
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (v < V) w.count[v] = w.filled[v] = 0;
  if (v < 2) w.cursor[v] = 0;
}

// (a wave adds an id's tokens at once, as those of a frequent one would queue up at
// its address: 16384 tokens of 50000 ids as a text has them 149 us in all, 155
// token by token; all of one id 157, 339; hardly any twice 125, 122)
template <typename I>
__global__ __launch_bounds__(256) void embed_count_kernel(const I* __restrict__ ids, int64_t T,
                                                          int64_t V, EmbedWs w) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int v = t < T ? (int)em_id(ids, t, V) : -1;
  int n = 0;  // in the id's first lane
  for (uint64_t left = __ballot(v >= 0); left != 0;) {
    const int first = __builtin_ctzll(left);
    const uint64_t same = __ballot(v == __builtin_amdgcn_readlane(v, first));
    if ((int)(threadIdx.x & 63) == first) n = __popcll(same);
    left &= ~same;
  }
  if (n) atomicAdd(&w.count[v], n);
}

// with few ids their counts queue up at few addresses: each workgroup counts its
// 1024 tokens in LDS first (16000 tokens of 100 ids: 37 us in all, 72 otherwise)
constexpr int kEmCountV = 16384;

template <typename I>
__global__ __launch_bounds__(1024) void embed_count_lds_kernel(const I* __restrict__ ids,
                                                               int64_t T, int V, EmbedWs w) {
  __shared__ int cnt[kEmCountV];
  const int tid = threadIdx.x;
  for (int k = tid; k < V; k += 1024) cnt[k] = 0;
  __syncthreads();
  const int64_t t = (int64_t)blockIdx.x * 1024 + tid;
  const int64_t v = t < T ? em_id(ids, t, V) : -1;
  if (v >= 0) atomicAdd(&cnt[v], 1);
  __syncthreads();
  for (int k = tid; k < V; k += 1024)
    if (cnt[k]) atomicAdd(&w.count[k], cnt[k]);
}

// a place for every segment, and the pieces of the long ones
__global__ __launch_bounds__(256) void embed_place_kernel(int64_t V, EmbedWs w) {
  __shared__ int sum[2][256], base[2];
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int i = threadIdx.x;
  const int n = v < V ? w.count[v] : 0;
  const int np = n > kEmPiece ? (n + kEmPiece - 1) / kEmPiece : 0;
  int a = n, b = np;  // inclusive sums over the workgroup
  sum[0][i] = a, sum[1][i] = b;
  for (int o = 1; o < 256; o <<= 1) {
    __syncthreads();
    const int pa = i >= o ? sum[0][i - o] : 0, pb = i >= o ? sum[1][i - o] : 0;
    __syncthreads();
    sum[0][i] = a += pa, sum[1][i] = b += pb;
  }
  if (i == 255) {
    base[0] = atomicAdd(&w.cursor[0], a);
    base[1] = atomicAdd(&w.cursor[1], b);
  }
  __syncthreads();
  if (v >= V) return;
  const int first = base[1] + b - np;
  w.place[v] = np ? first : base[0] + a - n;
  for (int k = 0; k < np; ++k) w.pid[first + k] = (int)v, w.pno[first + k] = k;
}

template <typename I>
__global__ __launch_bounds__(256) void embed_sort_kernel(const I* __restrict__ ids, int64_t T,
                                                         int64_t V, EmbedWs w) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= T) return;
  const int64_t v = em_id(ids, t, V);
  if (v < 0 || w.count[v] > kEmPiece) return;  // the pieces find their own
  w.sorted[w.place[v] + atomicAdd(&w.filled[v], 1)] = (int)t;
}

// sum of the rows list[0 .. n) of de, columns c .. c + 3 (all below D)
__device__ __forceinline__ f32x4 em_sum4(const float* __restrict__ de, int64_t D, const int* list,
                                         int n, int64_t c) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  int k = 0;
  for (; k + 8 <= n; k += 8) {
    f32x4 x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = *(const f32x4_u4*)(de + (int64_t)list[k + q] * D + c);
#pragma unroll
    for (int q = 0; q < 8; ++q) s += x[q];
  }
  for (; k < n; ++k) s += *(const f32x4_u4*)(de + (int64_t)list[k] * D + c);
  return s;
}

// grid (pieces at most): a piece's tokens, the kEmPiece occurrences of its id
// from number kEmPiece pno on, then their sum.  The ids are gone through 4096 at
// a time, four a thread, so that their loads overlap and few barriers remain.
template <typename I>
__global__ __launch_bounds__(1024) void embed_piece_kernel(const I* __restrict__ ids, int64_t T,
                                                           const float* __restrict__ de, int64_t D,
                                                           EmbedWs w) {
  constexpr int kPer = 4, kWaves = 16;
  __shared__ int list[kEmPiece], wave_n[2][kWaves];
  if ((int)blockIdx.x >= w.cursor[1]) return;
  const int v = w.pid[blockIdx.x];
  const int lo = w.pno[blockIdx.x] * kEmPiece;
  const int total = w.count[v] - lo, n = total < kEmPiece ? total : kEmPiece;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int seen = 0;
  for (int64_t tb = 0, step = 0; tb < T && seen < lo + n; tb += 1024 * kPer, ++step) {
    // a wave goes through 64 kPer consecutive ids, 64 at a time
    const int64_t t0 = tb + wave * 64 * kPer + lane;
    bool hit[kPer];
    int before[kPer], mine = 0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int64_t t = t0 + 64 * q;
      hit[q] = t < T && (int64_t)ids[t < T ? t : T - 1] == v;
    }
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const uint64_t m = __ballot(hit[q]);
      before[q] = mine + __popcll(m & ((1ull << lane) - 1));
      mine += __popcll(m);
    }
    int* wn = wave_n[step & 1];  // (the other half may still be read)
    if (lane == 0) wn[wave] = mine;
    __syncthreads();
    int base = seen;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const int c = wn[k];
      base += k < wave ? c : 0;
      seen += c;
    }
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int at = base + before[q] - lo;
      if (hit[q] && at >= 0 && at < n) list[at] = (int)(t0 + 64 * q);
    }
  }
  __syncthreads();
  float* o = w.psum + (int64_t)blockIdx.x * D;
  const int64_t D4 = D & ~(int64_t)3;
  for (int64_t c = (int64_t)threadIdx.x * 4; c < D4; c += 4096)
    *(f32x4_u4*)(o + c) = em_sum4(de, D, list, n, c);
  for (int64_t c = D4 + threadIdx.x; c < D; c += 1024) {
    float s = 0.f;
    for (int k = 0; k < n; ++k) s += de[(int64_t)list[k] * D + c];
    o[c] = s;
  }
}

// Few tokens (at most kEmDirect): a row's workgroup finds its own among the ids.
// grid (V), kEmDirect threads

template <typename I, bool ACC>
__global__ __launch_bounds__(kEmDirect) void embed_direct_kernel(const I* __restrict__ ids, int T,
                                                                 const float* __restrict__ de,
                                                                 int64_t D, float scale,
                                                                 float* __restrict__ dW) {
  __shared__ int list[kEmDirect], wave_n[4];
  const int64_t v = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool hit = (int64_t)ids[min(tid, T - 1)] == v && tid < T;
  const uint64_t m = __ballot(hit);
  if (lane == 0) wave_n[wave] = __popcll(m);
  __syncthreads();
  const int n = wave_n[0] + wave_n[1] + wave_n[2] + wave_n[3];
  if (ACC && n == 0) return;
  int at = __popcll(m & ((1ull << lane) - 1));
  for (int k = 0; k < wave; ++k) at += wave_n[k];
  if (hit) list[at] = tid;  // ascending
  __syncthreads();
  float* o = dW + v * D;
  const int64_t D4 = D & ~(int64_t)3;
  for (int64_t c = (int64_t)tid * 4; c < D4; c += 4 * kEmDirect) {
    f32x4 s = em_sum4(de, D, list, n, c) * scale;
    if (ACC) s += *(const f32x4_u4*)(o + c);
    *(f32x4_u4*)(o + c) = s;
  }
  for (int64_t c = D4 + tid; c < D; c += kEmDirect) {
    float s = 0.f;
    for (int k = 0; k < n; ++k) s += de[(int64_t)list[k] * D + c];
    o[c] = ACC ? o[c] + s * scale : s * scale;
  }
}

// Up to kEmScan tokens: dW is cleared by a launch of its own, and a workgroup a
// token goes through all ids; the one of an id's first token adds up all of them:
// four quarters of its threads take pieces of kEmPiece tokens in turn, whose sums
// meet in LDS.  No sort and no workspace.  grid (T), 1024 threads
__global__ __launch_bounds__(256) void embed_zero_kernel(float* __restrict__ p, int64_t n) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i + 4 <= n) *(f32x4_u4*)(p + i) = f32x4{0.f, 0.f, 0.f, 0.f};
  else
    for (int64_t j = i; j < n; ++j) p[j] = 0.f;
}

template <typename I, bool ACC>
__global__ __launch_bounds__(1024) void embed_first_kernel(const I* __restrict__ ids, int T,
                                                           int64_t V,
                                                           const float* __restrict__ de,
                                                           int64_t D, float scale,
                                                           float* __restrict__ dW) {
  constexpr int kPer = kEmScan / 1024;
  __shared__ int list[kEmScan], wave_n[16], before;
  __shared__ __attribute__((aligned(16))) float part[3][1024];
  const int t0 = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t v = em_id(ids, t0, V);
  if (v < 0) return;
  if (tid == 0) before = 0;
  // a wave goes through 64 kPer consecutive ids, 64 at a time
  const int tw = wave * 64 * kPer + lane;
  bool hit[kPer];
#pragma unroll
  for (int q = 0; q < kPer; ++q)
    hit[q] = (int64_t)ids[min(tw + 64 * q, T - 1)] == v && tw + 64 * q < T;
  int at[kPer], mine = 0;
  bool earlier = false;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const uint64_t m = __ballot(hit[q]);
    at[q] = mine + __popcll(m & ((1ull << lane) - 1));
    mine += __popcll(m);
    earlier |= hit[q] && tw + 64 * q < t0;
  }
  __syncthreads();
  if (lane == 0) wave_n[wave] = mine;
  if (earlier) before = 1;
  __syncthreads();
  if (before) return;  // not the first
  int base = 0, n = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    base += k < wave ? wave_n[k] : 0;
    n += wave_n[k];
  }
#pragma unroll
  for (int q = 0; q < kPer; ++q)
    if (hit[q]) list[base + at[q]] = tw + 64 * q;
  __syncthreads();
  float* o = dW + v * D;
  const int quarter = tid >> 8, lc = tid & 255;
  // all threads stay in step: a column range ends for all at once
  for (int64_t c0 = 0; c0 < D; c0 += 1024) {
    const int64_t c = c0 + 4 * lc;
    const bool whole = c + 4 <= D;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int k = quarter * kEmPiece; k < n; k += 4 * kEmPiece) {
      const int m = min(kEmPiece, n - k);
      if (whole) {
        s += em_sum4(de, D, list + k, m, c);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < m && c + i < D; ++j) s[i] += de[(int64_t)list[k + j] * D + c + i];
      }
    }
    if (n > kEmPiece) {  // (else the first quarter has it all)
      if (quarter) *(f32x4*)(part[quarter - 1] + 4 * lc) = s;
      __syncthreads();
      if (quarter == 0)
#pragma unroll
        for (int q = 0; q < 3; ++q) s += *(const f32x4*)(part[q] + 4 * lc);
    }
    if (quarter == 0) {
      s *= scale;
      if (whole) {
        if (ACC) s += *(const f32x4_u4*)(o + c);
        *(f32x4_u4*)(o + c) = s;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < D) o[c + i] = ACC ? o[c + i] + s[i] : s[i];
      }
    }
    if (n > kEmPiece) __syncthreads();
  }
}

// grid (V): row v, zeros where no token has it
template <bool ACC>
__global__ __launch_bounds__(256) void embed_row_kernel(const float* __restrict__ de, int64_t D,
                                                        float scale, float* __restrict__ dW,
                                                        EmbedWs w) {
  __shared__ int list[kEmPiece];
  const int64_t v = blockIdx.x;
  int n = w.count[v];
  if (ACC && n == 0) return;
  const float* src = de;
  if (n > kEmPiece) {  // the pieces' sums instead of tokens
    src = w.psum + (int64_t)w.place[v] * D;
    n = (n + kEmPiece - 1) / kEmPiece;
  } else if (n > 0) {
    // the tokens in ascending order: each goes where as many are smaller
    const int i = threadIdx.x;
    const int* seg = w.sorted + w.place[v];
    if (i < n) {
      const int t = seg[i];
      int at = 0;
      for (int k = 0; k < n; ++k) at += seg[k] < t;
      list[at] = t;
    }
    __syncthreads();
  }
  const bool pieces = src != de;
  float* o = dW + v * D;
  const int64_t D4 = D & ~(int64_t)3;
  for (int64_t c = (int64_t)threadIdx.x * 4; c < D4; c += 1024) {
    f32x4 s;
    if (pieces) {
      s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (int k = 0; k < n; ++k) s += *(const f32x4_u4*)(src + (int64_t)k * D + c);
    } else {
      s = em_sum4(src, D, list, n, c);
    }
    s *= scale;
    if (ACC) s += *(const f32x4_u4*)(o + c);
    *(f32x4_u4*)(o + c) = s;
  }
  for (int64_t c = D4 + threadIdx.x; c < D; c += 256) {
    float s = 0.f;
    for (int k = 0; k < n; ++k) s += src[(int64_t)(pieces ? k : list[k]) * D + c];
    o[c] = ACC ? o[c] + s * scale : s * scale;
  }
}

template <int TYPE>
static void embed_go(const void* ids, bool ids64, int64_t T, const void* w, int64_t V, int64_t D,
                     float scale, float* out, hipStream_t stream) {
  if (ids64)
    hipLaunchKernelGGL((embed_kernel<TYPE, int64_t>), dim3((unsigned)T), dim3(256), 0, stream,
                       (const int64_t*)ids, V, D, w, scale, out);
  else
    hipLaunchKernelGGL((embed_kernel<TYPE, int32_t>), dim3((unsigned)T), dim3(256), 0, stream,
                       (const int32_t*)ids, V, D, w, scale, out);
}

hipError_t launch_embed(const void* ids, bool ids64, int64_t T, const void* weight, int type,
                        int64_t V, int64_t D, float scale, float* out, hipStream_t stream) {
  if (type == 0) embed_go<0>(ids, ids64, T, weight, V, D, scale, out, stream);
  else if (type == 1) embed_go<1>(ids, ids64, T, weight, V, D, scale, out, stream);
  else embed_go<2>(ids, ids64, T, weight, V, D, scale, out, stream);
  return hipGetLastError();
}

template <typename I>
static hipError_t embed_bwd_go(const I* ids, int64_t T, const float* de, int64_t V, int64_t D,
                               float scale, float* dW, bool accumulate, void* workspace,
                               hipStream_t stream) {
  if (T <= kEmDirect && V <= kEmDirectV) {
    if (accumulate)
      hipLaunchKernelGGL((embed_direct_kernel<I, true>), dim3((unsigned)V), dim3(kEmDirect), 0,
                         stream, ids, (int)T, de, D, scale, dW);
    else
      hipLaunchKernelGGL((embed_direct_kernel<I, false>), dim3((unsigned)V), dim3(kEmDirect), 0,
                         stream, ids, (int)T, de, D, scale, dW);
    return hipGetLastError();
  }
  if (T <= kEmScan) {
    if (accumulate) {
      hipLaunchKernelGGL((embed_first_kernel<I, true>), dim3((unsigned)T), dim3(1024), 0, stream,
                         ids, (int)T, V, de, D, scale, dW);
    } else {
      const int64_t n = V * D;
      // 2^31 threads at most a launch
      for (int64_t i = 0; i < n; i += int64_t(1) << 32) {
        const int64_t m = n - i < (int64_t(1) << 32) ? n - i : int64_t(1) << 32;
        hipLaunchKernelGGL(embed_zero_kernel, dim3((unsigned)((m + 1023) / 1024)), dim3(256), 0,
                           stream, dW + i, m);
      }
      hipLaunchKernelGGL((embed_first_kernel<I, false>), dim3((unsigned)T), dim3(1024), 0, stream,
                         ids, (int)T, V, de, D, scale, dW);
    }
    return hipGetLastError();
  }
  const EmbedWs w = em_ws(workspace, T, V);
  const unsigned vb = (unsigned)((V + 255) / 256), tb = (unsigned)((T + 255) / 256);
  hipLaunchKernelGGL(embed_clear_kernel, dim3(vb), dim3(256), 0, stream, w, V);
  if (V <= kEmCountV)
    hipLaunchKernelGGL(embed_count_lds_kernel<I>, dim3((unsigned)((T + 1023) / 1024)), dim3(1024),
                       0, stream, ids, T, (int)V, w);
  else
    hipLaunchKernelGGL(embed_count_kernel<I>, dim3(tb), dim3(256), 0, stream, ids, T, V, w);
  hipLaunchKernelGGL(embed_place_kernel, dim3(vb), dim3(256), 0, stream, V, w);
  hipLaunchKernelGGL(embed_sort_kernel<I>, dim3(tb), dim3(256), 0, stream, ids, T, V, w);
  hipLaunchKernelGGL(embed_piece_kernel<I>, dim3((unsigned)em_pieces(T)), dim3(1024), 0, stream,
                     ids, T, de, D, w);
  if (accumulate)
    hipLaunchKernelGGL(embed_row_kernel<true>, dim3((unsigned)V), dim3(256), 0, stream, de, D,
                       scale, dW, w);
  else
    hipLaunchKernelGGL(embed_row_kernel<false>, dim3((unsigned)V), dim3(256), 0, stream, de, D,
                       scale, dW, w);
  return hipGetLastError();
}

hipError_t launch_embed_bwd(const void* ids, bool ids64, int64_t T, const float* dout, int64_t V,
                            int64_t D, float scale, float* dW, bool accumulate, void* workspace,
                            hipStream_t stream) {
  return ids64 ? embed_bwd_go((const int64_t*)ids, T, dout, V, D, scale, dW, accumulate,
                              workspace, stream)
               : embed_bwd_go((const int32_t*)ids, T, dout, V, D, scale, dW, accumulate,
                              workspace, stream);
}

}  // namespace tmk
