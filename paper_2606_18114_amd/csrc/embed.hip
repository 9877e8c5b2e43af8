// Rows of an embedding, e[t] = scale W[id_t] (float32, the residual stream's
// type), and the gradient of its weight, dW[v] = scale sum_{t: id_t = v} de[t],
// the tokens of a row in ascending order, so that repeated calls give the same
// bits.  An id outside [0, V) gives a row of zeros and no gradient.
//
// The gradient is bound by writing dW's V rows.  Few tokens are found by going
// through the ids (embed_direct_kernel, embed_first_kernel).  More are sorted by id
// into segments: a count per id, a place per segment (whichever: only the order
// inside a segment shows in the sums), and the positions, in any order, which the
// workgroup of a row brings into ascending order.  An id of more than
// kEmPiece tokens (the most frequent one of a text is a tenth of it) is cut
// into pieces of that many, whose sums meet, in float64, in the row's workgroup; a
// piece finds its tokens by going through the ids, which are few bytes.  16384 tokens,
// 50000 ids of 2048 columns: 149 us, 100 of them for the rows (4.8 TB/s).
//
// That search grows with the square of the tokens: above kEmSearch of them the sort
// is a stable one by digits of the id (embed_digit_*), which leaves every
// segment ascending, so that a piece takes its tokens from where they lie, and 64
// pieces' sums are added up by a workgroup of their own (embed_fold_kernel).
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
// Tokens up to which pieces search for their own.  98304 tokens of 50000 ids of 2048
// columns, as a text has them: 349 us so, 334 with the sort by digits; all of one id
// 648, 342; hardly any twice 260, 279.  65536: 252, 276; 448, 275; 209, 231.  2^20
// of 512 columns: 15.4 ms, 0.54; 18.3, 0.56; 0.57, 0.52.
constexpr int64_t kEmSearch = 98304;
constexpr int kEmDigit = 8;         // bits of a digit
constexpr int kEmBlock = 4096;      // tokens of a workgroup that places them
constexpr int kEmTotals = 3 << kEmDigit;  // of the digits of the (at most 3) passes

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
// pieces), filled (sorted by digits: where its segment begins) [V] each; cursors
// [2] (of tokens, of pieces); sorted [T]; a piece's id and its number in its row
// [pieces] each; pieces' sums [pieces][D].  Sorted by digits also: the other
// positions and two arrays of ids [T] each, digits' counts [passes][2^kEmDigit], and of
// a pass by block [2^kEmDigit][blocks]
struct EmbedWs {
  int *count, *place, *filled, *cursor, *sorted, *pid, *pno, *other, *key[2], *total, *digits;
  float* psum;
  int fold;  // sums that a piece's stands for in a row of more pieces than that
};
static int64_t em_pieces(int64_t T) { return 2 * (T / kEmPiece) + 1; }
static int64_t em_blocks(int64_t T) { return (T + kEmBlock - 1) / kEmBlock; }
static int64_t em_ints(int64_t T, int64_t V) {
  const int64_t n = 3 * V + 2 + T + 2 * em_pieces(T) +
                    (T > kEmSearch ? 3 * T + kEmTotals + (em_blocks(T) << kEmDigit) : 0);
  return (n + 63) / 64 * 64;
}
static EmbedWs em_ws(void* p, int64_t T, int64_t V) {
  EmbedWs w = {};
  int* i = (int*)p;
  w.count = i, w.place = i + V, w.filled = i + 2 * V, w.cursor = i + 3 * V;
  w.sorted = w.cursor + 2;
  w.pid = w.sorted + T;
  w.pno = w.pid + em_pieces(T);
  w.fold = 1;
  if (T > kEmSearch) {
    w.other = w.pno + em_pieces(T);
    w.key[0] = w.other + T, w.key[1] = w.key[0] + T;
    w.total = w.key[1] + T;
    w.digits = w.total + kEmTotals;
    w.fold = kEmPiece;
  }
  w.psum = (float*)(i + em_ints(T, V));
  return w;
}
int64_t embed_bwd_bytes(int64_t T, int64_t V, int64_t D) {
  return T <= kEmScan ? 0 : em_ints(T, V) * 4 + em_pieces(T) * D * 4;
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

// ---- more than kEmSearch tokens: a stable sort by the ids' digits --------------
// A pass: the digits' counts of every block of kEmBlock tokens, the places that
// follow from them (digit by digit, block by block), and the tokens to their
// places.  An id without a row is sorted as V, behind the others.

__global__ __launch_bounds__(256) void embed_digit_clear_kernel(EmbedWs w, int64_t V,
                                                                int64_t pieces) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < V) w.filled[i] = w.place[i] = 0;
  if (i < pieces) w.pid[i] = -1;
  if (i < kEmTotals) w.total[i] = 0;
}

// FIRST: of the ids; else of key, with positions pos
template <typename I, bool FIRST>
__device__ __forceinline__ int em_key(const I* __restrict__ ids, const int* __restrict__ key,
                                      int64_t t, int64_t V) {
  if constexpr (FIRST) {
    const int64_t v = em_id(ids, t, V);
    return (int)(v < 0 ? V : v);
  } else {
    return key[t];
  }
}

// grid (blocks), 1024 threads
template <typename I, bool FIRST>
__global__ __launch_bounds__(1024) void embed_digit_count_kernel(
    const I* __restrict__ ids, const int* __restrict__ key, int64_t T, int64_t V, int shift,
    int* __restrict__ digits, int* __restrict__ total) {
  __shared__ int cnt[1 << kEmDigit];
  const int tid = threadIdx.x;
  if (tid < 1 << kEmDigit) cnt[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kEmBlock / 1024; ++q) {
    const int64_t t = (int64_t)blockIdx.x * kEmBlock + q * 1024 + tid;
    if (t < T)
      atomicAdd(&cnt[em_key<I, FIRST>(ids, key, t, V) >> shift & ((1 << kEmDigit) - 1)], 1);
  }
  __syncthreads();
  if (tid < 1 << kEmDigit) {
    digits[(int64_t)tid * gridDim.x + blockIdx.x] = cnt[tid];
    if (cnt[tid]) atomicAdd(&total[tid], cnt[tid]);
  }
}

// Places, in place: a digit's workgroup adds up what lies before it, all of the lower
// digits (total) and the blocks before.  grid (2^kEmDigit), 256 threads, each of which
// takes blocks / 256 of them in a row
__global__ __launch_bounds__(256) void embed_digit_scan_kernel(int* __restrict__ digits,
                                                               const int* __restrict__ total,
                                                               int blocks) {
  __shared__ int sum[256];
  const int i = threadIdx.x, per = (blocks + 255) / 256;
  const int lo = min(blocks, i * per), hi = min(blocks, lo + per);
  int* row = digits + (int64_t)blockIdx.x * blocks;
  auto sums = [&](int a) {  // up to this thread's and with it
    sum[i] = a;
    for (int o = 1; o < 256; o <<= 1) {
      __syncthreads();
      const int p = i >= o ? sum[i - o] : 0;
      __syncthreads();
      sum[i] = a += p;
    }
    __syncthreads();
    return a;
  };
  sums(i < (int)blockIdx.x ? total[i] : 0);
  const int below = sum[255];
  __syncthreads();
  int own = 0;
  for (int k = lo; k < hi; ++k) own += row[k];
  int a = below + sums(own) - own;
  for (int k = lo; k < hi; ++k) {
    const int d = row[k];
    row[k] = a;
    a += d;
  }
}

// grid (blocks), 1024 threads: a wave takes kEmBlock / 16 tokens in a row, 64 at a
// time.  A token's place: its digit's in the block, the waves before, the wave's
// earlier ones (cnt so far), the lanes below with the same digit.
template <typename I, bool FIRST>
__global__ __launch_bounds__(1024) void embed_digit_place_kernel(
    const I* __restrict__ ids, const int* __restrict__ key, const int* __restrict__ pos, int64_t T,
    int64_t V, int shift, const int* __restrict__ digits, int* __restrict__ key_out,
    int* __restrict__ pos_out) {
  constexpr int kPer = kEmBlock / 1024, kDig = 1 << kEmDigit;
  __shared__ int cnt[16][kDig];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int k = tid; k < 16 * kDig; k += 1024) cnt[k / kDig][k % kDig] = 0;
  int v[kPer], at[kPer];
  bool in[kPer];
  const int64_t t0 = (int64_t)blockIdx.x * kEmBlock + wave * 64 * kPer + lane;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int64_t t = t0 + 64 * q;
    in[q] = t < T;
    v[q] = em_key<I, FIRST>(ids, key, t < T ? t : T - 1, V);
  }
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    __syncthreads();  // cnt is clear; the step before has been counted
    const int dig = v[q] >> shift & (kDig - 1);
    uint64_t same = __ballot(in[q]);
#pragma unroll
    for (int b = 0; b < kEmDigit; ++b) {
      const uint64_t set = __ballot(dig >> b & 1);
      same &= dig >> b & 1 ? set : ~set;
    }
    at[q] = cnt[wave][dig] + __popcll(same & ((1ull << lane) - 1));
    __syncthreads();
    if (in[q] && lane == __builtin_ctzll(same)) cnt[wave][dig] += __popcll(same);
  }
  __syncthreads();
  if (tid < kDig) {  // what lies before every wave's
    int a = digits[(int64_t)tid * gridDim.x + blockIdx.x];
    for (int k = 0; k < 16; ++k) {
      const int n = cnt[k][tid];
      cnt[k][tid] = a;
      a += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    if (!in[q]) continue;
    const int p = cnt[wave][v[q] >> shift & (kDig - 1)] + at[q];
    key_out[p] = v[q];
    pos_out[p] = FIRST ? (int)(t0 + 64 * q) : pos[t0 + 64 * q];
  }
}

// where the segments begin (filled) and end (place)
__global__ __launch_bounds__(256) void embed_digit_ends_kernel(const int* __restrict__ key,
                                                               int64_t T, int64_t V, EmbedWs w) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= T) return;
  const int v = key[i];
  if (v >= V) return;
  if (i == 0 || key[i - 1] != v) w.filled[v] = (int)i;
  if (i == T - 1 || key[i + 1] != v) w.place[v] = (int)i + 1;
}

// A segment's count and place.  Pieces: from number 2 (begin / kEmPiece) on.  One
// of n > kEmPiece tokens has np >= 2 of them; the next one begins n > kEmPiece (np -
// 1) tokens later, so at a number higher by 2 (np - 1) >= np; the last number is at most
// 2 (T / kEmPiece).
__global__ __launch_bounds__(256) void embed_digit_rows_kernel(int64_t V, EmbedWs w) {
  const int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (v >= V) return;
  const int begin = w.filled[v], n = w.place[v] - begin;
  w.count[v] = n;
  w.place[v] = n > kEmPiece ? 2 * (begin / kEmPiece) : begin;
}

// which pieces there are
__global__ __launch_bounds__(256) void embed_digit_pieces_kernel(const int* __restrict__ key,
                                                                 int64_t T, int64_t V, EmbedWs w) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= T) return;
  const int v = key[i];
  if (v >= V || w.count[v] <= kEmPiece) return;
  const int k = (int)i - w.filled[v];
  if (k % kEmPiece) return;
  const int p = w.place[v] + k / kEmPiece;
  w.pid[p] = v, w.pno[p] = k / kEmPiece;
}

// grid (pieces at most), 256 threads: a piece's sum
__global__ __launch_bounds__(256) void embed_digit_sum_kernel(const float* __restrict__ de,
                                                              int64_t D, EmbedWs w) {
  __shared__ int list[kEmPiece];
  const int v = w.pid[blockIdx.x];
  if (v < 0) return;
  const int lo = w.pno[blockIdx.x] * kEmPiece, n = min(kEmPiece, w.count[v] - lo);
  if ((int)threadIdx.x < n) list[threadIdx.x] = w.sorted[w.filled[v] + lo + threadIdx.x];
  __syncthreads();
  float* o = w.psum + (int64_t)blockIdx.x * D;
  const int64_t D4 = D & ~(int64_t)3;
  for (int64_t c = (int64_t)threadIdx.x * 4; c < D4; c += 1024)
    *(f32x4_u4*)(o + c) = em_sum4(de, D, list, n, c);
  for (int64_t c = D4 + threadIdx.x; c < D; c += 256) {
    float s = 0.f;
    for (int k = 0; k < n; ++k) s += de[(int64_t)list[k] * D + c];
    o[c] = s;
  }
}

// grid (pieces at most), 256 threads: where a row has more than kEmPiece pieces, the
// sums of as many into the first one's
__global__ __launch_bounds__(256) void embed_fold_kernel(int64_t D, EmbedWs w) {
  const int v = w.pid[blockIdx.x];
  if (v < 0) return;
  const int k = w.pno[blockIdx.x], np = (w.count[v] + kEmPiece - 1) / kEmPiece;
  if (k % kEmPiece || np <= kEmPiece) return;
  const int n = min(kEmPiece, np - k);
  float* o = w.psum + (int64_t)blockIdx.x * D;
  for (int64_t c = threadIdx.x; c < D; c += 256) {
    double a = 0.0;
#pragma unroll 16
    for (int q = 0; q < n; ++q) a += (double)o[q * D + c];
    o[c] = (float)a;
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
  int64_t step = D;
  if (n > kEmPiece) {  // the pieces' sums instead of tokens
    src = w.psum + (int64_t)w.place[v] * D;
    n = (n + kEmPiece - 1) / kEmPiece;
    if (w.fold > 1 && n > w.fold) n = (n + w.fold - 1) / w.fold, step = w.fold * D;
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
      double a[4] = {0.0, 0.0, 0.0, 0.0};  // (thousands of them in a long batch)
#pragma unroll 8
      for (int k = 0; k < n; ++k) {
        const f32x4 x = *(const f32x4_u4*)(src + k * step + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] += (double)x[i];
      }
      s = f32x4{(float)a[0], (float)a[1], (float)a[2], (float)a[3]};
    } else {
      s = em_sum4(src, D, list, n, c);
    }
    s *= scale;
    if (ACC) s += *(const f32x4_u4*)(o + c);
    *(f32x4_u4*)(o + c) = s;
  }
  for (int64_t c = D4 + threadIdx.x; c < D; c += 256) {
    float s = 0.f;
    if (pieces) {
      double a = 0.0;
      for (int k = 0; k < n; ++k) a += (double)src[k * step + c];
      s = (float)a;
    } else {
      for (int k = 0; k < n; ++k) s += src[(int64_t)list[k] * D + c];
    }
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

static hipError_t embed_rows(const float* de, int64_t V, int64_t D, float scale, float* dW,
                             bool accumulate, const EmbedWs& w, hipStream_t stream) {
  if (accumulate)
    hipLaunchKernelGGL(embed_row_kernel<true>, dim3((unsigned)V), dim3(256), 0, stream, de, D,
                       scale, dW, w);
  else
    hipLaunchKernelGGL(embed_row_kernel<false>, dim3((unsigned)V), dim3(256), 0, stream, de, D,
                       scale, dW, w);
  return hipGetLastError();
}

// the positions by id (w.sorted), the rows' counts and places, and their pieces
template <typename I>
static void embed_digits(const I* ids, int64_t T, int64_t V, EmbedWs& w, hipStream_t stream) {
  const int64_t pieces = em_pieces(T), most = V > pieces ? V : pieces;
  const unsigned blocks = (unsigned)em_blocks(T), tb = (unsigned)((T + 255) / 256);
  hipLaunchKernelGGL(embed_digit_clear_kernel, dim3((unsigned)((most + 255) / 256)), dim3(256), 0,
                     stream, w, V, pieces);
  int* pos[2] = {w.sorted, w.other};
  int in = 1;
  for (int shift = 0; V >> shift != 0; shift += kEmDigit, in ^= 1) {
    const int *k = w.key[in], *p = pos[in];
    int *ko = w.key[in ^ 1], *po = pos[in ^ 1], *total = w.total + (shift / kEmDigit << kEmDigit);
    if (shift == 0) {
      hipLaunchKernelGGL((embed_digit_count_kernel<I, true>), dim3(blocks), dim3(1024), 0, stream,
                         ids, k, T, V, shift, w.digits, total);
    } else {
      hipLaunchKernelGGL((embed_digit_count_kernel<I, false>), dim3(blocks), dim3(1024), 0, stream,
                         ids, k, T, V, shift, w.digits, total);
    }
    hipLaunchKernelGGL(embed_digit_scan_kernel, dim3(1 << kEmDigit), dim3(256), 0, stream,
                       w.digits, total, (int)blocks);
    if (shift == 0) {
      hipLaunchKernelGGL((embed_digit_place_kernel<I, true>), dim3(blocks), dim3(1024), 0, stream,
                         ids, k, p, T, V, shift, w.digits, ko, po);
    } else {
      hipLaunchKernelGGL((embed_digit_place_kernel<I, false>), dim3(blocks), dim3(1024), 0, stream,
                         ids, k, p, T, V, shift, w.digits, ko, po);
    }
  }
  w.sorted = pos[in];
  const int* key = w.key[in];
  hipLaunchKernelGGL(embed_digit_ends_kernel, dim3(tb), dim3(256), 0, stream, key, T, V, w);
  hipLaunchKernelGGL(embed_digit_rows_kernel, dim3((unsigned)((V + 255) / 256)), dim3(256), 0,
                     stream, V, w);
  hipLaunchKernelGGL(embed_digit_pieces_kernel, dim3(tb), dim3(256), 0, stream, key, T, V, w);
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
  EmbedWs w = em_ws(workspace, T, V);
  const unsigned vb = (unsigned)((V + 255) / 256), tb = (unsigned)((T + 255) / 256);
  const unsigned pieces = (unsigned)em_pieces(T);
  if (T > kEmSearch) {
    embed_digits(ids, T, V, w, stream);
    hipLaunchKernelGGL(embed_digit_sum_kernel, dim3(pieces), dim3(256), 0, stream, de, D, w);
    hipLaunchKernelGGL(embed_fold_kernel, dim3(pieces), dim3(256), 0, stream, D, w);
    return embed_rows(de, V, D, scale, dW, accumulate, w, stream);
  }
  hipLaunchKernelGGL(embed_clear_kernel, dim3(vb), dim3(256), 0, stream, w, V);
  if (V <= kEmCountV)
    hipLaunchKernelGGL(embed_count_lds_kernel<I>, dim3((unsigned)((T + 1023) / 1024)), dim3(1024),
                       0, stream, ids, T, (int)V, w);
  else
    hipLaunchKernelGGL(embed_count_kernel<I>, dim3(tb), dim3(256), 0, stream, ids, T, V, w);
  hipLaunchKernelGGL(embed_place_kernel, dim3(vb), dim3(256), 0, stream, V, w);
  hipLaunchKernelGGL(embed_sort_kernel<I>, dim3(tb), dim3(256), 0, stream, ids, T, V, w);
  hipLaunchKernelGGL(embed_piece_kernel<I>, dim3(pieces), dim3(1024), 0, stream, ids, T, de, D, w);
  return embed_rows(de, V, D, scale, dW, accumulate, w, stream);
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
