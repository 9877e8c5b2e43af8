// The products of the head's loss (tmamba_head.h) on the gfx950 matrix cores,
// 16-bit operands (bfloat16 or float16), float32 sums:
//   logits   z[v, t]  = W[v, :] . h[t, :]        -> running softmax sums, or dlogits G
//   dh       dh[t, :] = sum_v G[t, v] W[v, :]
//   dW       dW[v, :] = sum_t G[t, v] h[t, :]
// Logits are made in the registers of a tile and never stored: forward, a
// lane keeps the maximum and the sum of exponentials of its tokens over all the
// words that its workgroup walks; backward the tile becomes 16-bit dlogits of one
// piece of the vocabulary, which dh and dW contract.
//
// One main loop for the three.  The first operand lies along the contraction (W
// for the logits, G for dh) or across it (G for dW), the second across it (h^T for
// the logits, W for dh, h for dW).  Tiles are staged in LDS in their natural order
// by direct-to-LDS loads, 32 steps of the contraction a stage.  Across: rows of 512
// bytes, in 32-byte units that are XOR-permuted against bank conflicts, read with
// the transpose read ds_read_b64_tr_b16, two an operand; a ring of four stages, loaded
// three ahead.  Along: 128-byte rows, the lines of the caches, hold two stages (with
// 64-byte rows, one stage, the requests to the L2 double: 16384 tokens of 50000 x 2048
// in 13.6 ms, 12.3 so); their 16-byte pieces are XOR-permuted, one ds_read_b128 is an
// operand; three pairs of stages, loaded two pairs ahead.
//
// Tile 256 x 256 of 4 waves, 128 x 128 each (4 x 4 blocks of 32 x 32,
// accumulators in AGPRs, one wave a SIMD), every MFMA a slot of its own with the
// reads of the next step and the loads of stage + 3 dealt over the slots.  Nothing
// spills: accumulators leave their registers a block at a time.
//
// Bound: the matrix cores under the power cap (a stage of a full tile takes 0.77 us, 1.36
// PFLOP/s, at 1.7 to 1.85 GHz).  16384 tokens of 50000 x 2048: softmax sums 2.50 to 2.60 ms (1.29
// to 1.34 PFLOP/s), dlogits 2.85 to 2.94, dh 2.53 to 2.60, dW 2.45 to 2.53; a tile's epilogue adds 3 us to the sums (its first
// loads are then already under way) and 7 to the dlogits.  (Up to 64
// tokens: head_dw_few_kernel below, and the softmax sums in head_loss.hip.)
#include <type_traits>

#include "common.hpp"
#include "head.hpp"
#include "launchers.hpp"

namespace tmk {

namespace {

constexpr int kBK = 32, kRing = 4;
constexpr int kTM = 256, kTN = 256;
constexpr int kOp = kTM * kBK * 2;  // an operand's bytes of a stage
// LDS: the ring of the second operand, then the first's: a ring, or three pairs
constexpr int kLdsB = kRing * kOp;
template <bool ALONG>
constexpr int kLds = kLdsB + (ALONG ? 6 : kRing) * kOp;
constexpr int kLoads = 8;  // direct-to-LDS loads of a wave and stage
constexpr float kLog2e = 1.4426950408889634f;

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

typedef uint16_t __attribute__((may_alias)) any16;

enum Mode { kStats, kDlogits, kDh, kDw };

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// lane i: 16 bytes at base + voff -> LDS lds_base + 16 i (lds_base wave-uniform)
__device__ __forceinline__ void dma16(const void* base, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff),
               "s"(base), "s"(lds_base)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// A stage's end.  No wait for LDS reads: those of the slot that the next stage's loads
// write have fed an MFMA of the stage, and those of the next slot are waited for where they
// are used (16384 tokens of 50000 x 2048: 12.29 ms with lgkmcnt(0) here, 12.19 without).
template <int kVm>
__device__ __forceinline__ void stage_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kVm) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

template <bool F16>
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return mfma32(as_bf16x8(a), as_bf16x8(b), c);
}

// two values rounded to nearest even
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (F16) {
    typedef __attribute__((ext_vector_type(2))) _Float16 h2;
    return __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
  } else {
    typedef __attribute__((ext_vector_type(2))) __bf16 b2;
    return __builtin_bit_cast(uint32_t, b2{(__bf16)a, (__bf16)b});
  }
}

// An accumulator block as values of their own: without the opaque copy the compiler wants
// all of the accumulators in vector registers at once, and spills them there.  (Not one
// by one: a wave is alone on its SIMD, and sixteen independent values hide the latencies of
// what is done to them.)
__device__ __forceinline__ f32x16 acc_block(f32x16 v) {
  asm("" : "+v"(v));
  return v;
}

// across: XOR applied to the 32-byte unit index of row r (the four rows of a
// transpose read land in distinct bank groups)
__device__ __forceinline__ int swz(int r) { return (r & 3) ^ ((r & 3) << 1); }
// across: byte offset of (row r, column c) of a 256-column operand, c % 4 == 0
__device__ __forceinline__ uint32_t off_across(int r, int c) {
  return (uint32_t)(r * 512 + 32 * ((c >> 4) ^ swz(r)) + 2 * (c & 15));
}
// along: byte offset of 16-byte piece p of row r
__device__ __forceinline__ uint32_t off_along(int r, int p) {
  return (uint32_t)(r * 128 + 16 * (p ^ ((r >> 1) & 7)));
}

// An operand's loads and the addresses they need: four of a wave and stage.  Along,
// the two stages of a pair load half of the rows each.  Rows (columns) past the
// array re-read its last one, and what they bring is not stored; steps past the
// contraction's end re-read its last ones, against zeros in the other operand.
template <bool ALONG>
struct Loader {
  const uint8_t* base;  // the array, at the tile's first row (along) or column (across)
  // along: byte offsets of the lane's rows in the array, of its piece in a row (the same
  // for all); across: of its rows in a stage, of its columns
  uint32_t row[ALONG ? 8 : 4];
  uint32_t col[ALONG ? 1 : 4];
  int64_t pitch;  // bytes of a row
  int end, rest;  // the contraction's last stage (along: pair), and its steps

  // left: rows (along) or columns (across; a multiple of 8) of the array from the tile on
  __device__ __forceinline__ void begin(const uint16_t* b, int left, int64_t pitch_, int K,
                                        int wave, int lane) {
    base = reinterpret_cast<const uint8_t*>(b);
    pitch = 2 * pitch_;
    constexpr int kSteps = ALONG ? 2 * kBK : kBK;
    end = __builtin_amdgcn_readfirstlane((K - 1) / kSteps);
    rest = __builtin_amdgcn_readfirstlane(K - end * kSteps);
    const int most = left < 256 ? left : 256;
    if constexpr (ALONG) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // 8 rows a load; wave w's are 64 w ..
        const int r = 64 * wave + 8 * i + (lane >> 3);
        row[i] = (uint32_t)(r < most ? r : most - 1) * (uint32_t)pitch;
      }
      // (r >> 1) & 7 = (4 i + (lane >> 4)) & 7: the upper bit is i's parity
      col[0] = 16u * (uint32_t)((lane & 7) ^ (lane >> 4));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 2 * (wave * 4 + i) + (lane >> 5), p = lane & 31;
        const int c = 8 * (2 * ((p >> 1) ^ swz(r)) + (p & 1));
        row[i] = (uint32_t)r * (uint32_t)pitch;
        col[i] = 2u * (uint32_t)(c < most ? c : most - 8);
      }
    }
  }
  struct At {
    const uint8_t* b;
    uint32_t last;
  };
  // st: a stage (across), or a pair (along)
  __device__ __forceinline__ At stage(int st) const {
    constexpr int kSteps = ALONG ? 2 * kBK : kBK;
    st = st < end ? st : end;
    const int64_t k0 = (int64_t)st * kSteps;
    const int left = st < end ? kSteps : rest;
    if constexpr (ALONG)  // (whole pieces: the rows go on to a multiple of 8)
      return At{base + 2 * k0, 16u * (uint32_t)((left - 1) >> 3)};
    else
      return At{base + k0 * pitch, (uint32_t)(left - 1) * (uint32_t)pitch};
  }
  template <int I>
  __device__ __forceinline__ void load(const At& a, uint32_t dst) const {
    if constexpr (ALONG) {
      const uint32_t c = I & 1 ? col[0] ^ 64u : col[0];
      dma16(a.b, row[I] + (c < a.last ? c : a.last), dst + 1024 * I);
    } else {
      dma16(a.b, (row[I] < a.last ? row[I] : a.last) + col[I], dst + 1024 * I);
    }
  }
};

// What a stage's loads need, and the loads
template <bool ALONG>
struct Loads {
  const Loader<ALONG>& la;
  const Loader<false>& lb;
  uint32_t lds0;  // the wave's part of the ring
  int s_beg, s_end;

  // Stages and slots are counted from s_beg.  Past the range the last stage is loaded again.
  struct Stage {
    typename Loader<ALONG>::At a;
    typename Loader<false>::At b;
    uint32_t adst, bdst;
  };
  // the loads that go with stage i: the second operand's stage i + 3 and the first's, or
  // half of its pair i / 2 + 2, to slot aslot
  __device__ __forceinline__ Stage begin(int i, uint32_t aslot, int wave) const {
    const int st = s_beg + i + 3 < s_end ? s_beg + i + 3 : s_end - 1;
    Stage d;
    d.b = lb.stage(st);
    d.bdst = lds0 + (uint32_t)((i + 3) & 3) * kOp + 4096u * wave;
    if constexpr (ALONG) {
      const int pair = s_beg / 2 + (i >> 1) + 2, end = (s_end - 1) / 2;
      d.a = la.stage(pair < end ? pair : end);
      d.adst = lds0 + kLdsB + aslot * (2 * kOp) + 8192u * wave;
    } else {
      d.a = la.stage(st);
      d.adst = lds0 + kLdsB + (uint32_t)((i + 3) & 3) * kOp + 4096u * wave;
    }
    return d;
  }
  // load J of the eight of stage i (PAR = i % 2)
  template <int J, int PAR>
  __device__ __forceinline__ void piece(const Stage& d) const {
    if constexpr (J < 4)
      la.template load<ALONG ? 4 * PAR + J : J>(d.a, d.adst);
    else
      lb.template load<J - 4>(d.b, d.bdst);
  }
  // before the main loop: three stages of the second operand, three stages or two pairs of the
  // first (along, the third pair's slot is not written)
  __device__ __forceinline__ void first(int wave) const {
    static_for<0, 4>([&](auto p_tag) {
      constexpr int p = decltype(p_tag)::value;
      if constexpr (!ALONG && p == 0) return;
      const Stage d = begin(p - 4, ALONG ? (uint32_t)(p / 2) : 0u, wave);
      // (stage p - 4: the second operand's p - 1, the first's p - 1 or pair p / 2)
      static_for<0, kLoads>([&](auto j_tag) {
        if constexpr (p > 0 || decltype(j_tag)::value < 4)
          piece<decltype(j_tag)::value, p % 2>(d);
      });
    });
  }
};

template <bool ALONG>
__device__ __forceinline__ Loads<ALONG> loads_of(uint8_t* lds, const Loader<ALONG>& la,
                                                 const Loader<false>& lb, int s_beg, int s_end) {
  return Loads<ALONG>{la, lb, (uint32_t)(uintptr_t)lds, s_beg, s_end};
}

// The main loop: acc = the tile's sums over stages s_beg .. s_end - 1, both
// multiples of the ring (4 stages, 128 steps), s_end > s_beg.  One of the operands holds
// zeros up to a multiple of 128 steps, so that there is no other end.  A tile has 64 BB
// columns, the first of those that are loaded.  Loads::first has been called.
template <bool F16, bool ALONG, int BB>
__device__ __forceinline__ void product(uint8_t* lds, const Loads<ALONG>& ld,
                                        f32x16 (&acc)[4][BB]) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wy = wave >> 1, wx = wave & 1;
  const int l32 = lane & 31, half = lane >> 5;

#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int b = 0; b < BB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;

  stage_barrier<kLoads>();

  // per-lane byte offsets of the operand reads: across, of the four blocks in a stage;
  // along, of the four steps of a pair
  const int trow = 8 * half + ((lane & 15) >> 2);
  const int tcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  uint32_t aoff[4], boff[BB];
#pragma unroll
  for (int x = 0; x < 4; ++x)
    aoff[x] = kLdsB + (ALONG ? off_along(wy * 128 + l32, 2 * x + half)
                             : off_across(trow, wy * 128 + 32 * x + tcol));
#pragma unroll
  for (int x = 0; x < BB; ++x) boff[x] = off_across(trow, wx * (32 * BB) + 32 * x + tcol);
  auto across = [&](uint32_t off, int t) {
    const s16x4 lo =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + off + 16 * t * 512));
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + off + (16 * t + 4) * 512));
    const u32x2 l = __builtin_bit_cast(u32x2, lo), u = __builtin_bit_cast(u32x2, hi);
    return u32x4{l.x, l.y, u.x, u.y};
  };
  // operands of block x, step t of the stage in slot S (along: of the pair whose slot's
  // offset is apair)
  auto frag_a = [&](uint32_t apair, auto s_tag, int x, int t) {
    constexpr int S = decltype(s_tag)::value;
    if constexpr (ALONG)
      return *reinterpret_cast<const u32x4*>(lds + (aoff[2 * (S & 1) + t] + apair) + 4096 * x);
    else
      return across(aoff[x] + S * kOp, t);
  };
  auto frag_b = [&](auto s_tag, int x, int t) {
    return across(boff[x] + decltype(s_tag)::value * kOp, t);
  };
  u32x4 af[2][4], bf[2][BB];
  auto read_op = [&](uint32_t apair, auto s_tag, auto t_tag, auto x_tag) {
    constexpr int T = decltype(t_tag)::value, X = decltype(x_tag)::value;
    if constexpr (X == 0)
      af[T][0] = frag_a(apair, s_tag, 0, T);
    else if constexpr (X <= BB)
      bf[T][X - 1] = frag_b(s_tag, X - 1, T);
    else
      af[T][X - BB] = frag_a(apair, s_tag, X - BB, T);
  };

  // One full stage, i % 4 = S.  The MFMAs of its first step cover the reads of its
  // second one and the loads, those of the second the first reads of the next stage, dealt
  // evenly.  a0, a1: slots (0 .. 2) of the pairs of this stage and the next one, a2 of the pair
  // that is loaded.
  auto stage = [&](auto s_tag, int i, uint32_t a0, uint32_t a1, uint32_t a2) {
    constexpr int S = decltype(s_tag)::value;
    constexpr int kMf = 4 * BB, kReads = 4 + BB;
    typedef std::integral_constant<int, (S + 1) & 3> Next;
    const typename Loads<ALONG>::Stage d = ld.begin(i, a2, wave);
    const uint32_t p0 = a0 * (2 * kOp), p1 = (S & 1 ? a1 : a0) * (2 * kOp);
    static_for<0, 2 * kMf>([&](auto k_tag) {
      constexpr int k = decltype(k_tag)::value;
      constexpr int t = k / kMf, m = k % kMf, a = m / BB, b = m % BB;
      acc[a][b] = mfma<F16>(af[t][a], bf[t][b], acc[a][b]);
      // reads ceil(m kReads / kMf) .. of the step and, an MFMA later, the loads
      static_for<(m * kReads + kMf - 1) / kMf, ((m + 1) * kReads + kMf - 1) / kMf>([&](auto x_tag) {
        if constexpr (t == 0)
          read_op(p0, s_tag, std::integral_constant<int, 1>{}, x_tag);
        else
          read_op(p1, Next{}, std::integral_constant<int, 0>{}, x_tag);
      });
      if constexpr (t == 0)
        static_for<m * kLoads / kMf, (m + 1) * kLoads / kMf>([&](auto j_tag) {
          ld.template piece<decltype(j_tag)::value, S & 1>(d);
        });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  uint32_t a0 = 0, a1 = 1, a2 = 2;  // slots of this pair, the next one and the one to load
  auto turn = [&]() {
    const uint32_t t = a0;
    a0 = a1;
    a1 = a2;
    a2 = t;
  };
  static_for<0, 4 + BB>([&](auto x_tag) {
    read_op(0, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, x_tag);
  });
  for (int i0 = 0; i0 < ld.s_end - ld.s_beg; i0 += kRing) {
    static_for<0, kRing>([&](auto s_tag) {
      constexpr int S = decltype(s_tag)::value;
      stage(s_tag, i0 + S, a0, a1, a2);
      if constexpr (S & 1) turn();
      stage_barrier<kLoads>();
    });
  }
  // every load has landed before the ring is used again
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  // (they stay in the accumulator registers until the epilogue takes them block by block)
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int b = 0; b < BB; ++b) asm volatile("" : "+a"(acc[a][b]));
}

// stages of a contraction of k steps
__device__ __forceinline__ int stages(int k) {
  return (k + kRing * kBK - 1) / (kRing * kBK) * kRing;
}

// The items (token tile, word tile), words fastest, that workgroup w of P has:
// a run floor(w N / P) .. floor((w + 1) N / P) - 1 of all N
__device__ __forceinline__ int64_t run_begin(int64_t w, int64_t N, int64_t P) { return w * N / P; }

// Sizes and what is left of them are int where they are compared: this compiler takes the
// condition of a select from the wrong register when a branch goes by the same signed
// 64-bit comparison (the words past the last were not masked).

}  // namespace

// A wave's 32 rows of 128 16-bit values from LDS to memory, whole lines: rows of 256 bytes
// from `mine` on, piece p of row r at p ^ (r & 15), to rows `pitch` elements apart; what lies
// past rows_left and cols_left (a multiple of 8) is not written.
__device__ __forceinline__ void store_rows(const uint8_t* mine, uint16_t* to, int64_t pitch,
                                           int rows_left, int cols_left) {
  const int lane = threadIdx.x & 63, r0 = lane >> 4, p = lane & 15;
  __builtin_amdgcn_wave_barrier();  // (a wave reads only what it wrote)
  to += r0 * pitch + 8 * p;
  mine += r0 * 256;
  const int left = 8 * p < cols_left ? rows_left - r0 : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (4 * i < left)
      st16(to + 4 * i * pitch,
           *reinterpret_cast<const u32x4*>(mine + 1024 * i + 16 * (p ^ ((r0 + 4 * i) & 15))));
  __builtin_amdgcn_wave_barrier();
}

// Logits: A = W (words), B = h^T (64 BB tokens), so that a lane has one
// token a block and 64 of its logits.  Lane: token 32 b + l32, words 32 a +
// 8 (i / 4) + 4 half + i % 4.
//
// kStats: part[(workgroup + token tile)][wave row][256][2 or 3] = maximum and sum
// of 2^(log2e (z - maximum)) over the run's words, and the same at the temperature
// where TEMP.  A workgroup walks many word tiles of one token tile, so
// a step of the softmax costs no memory.
// kDlogits: G[row][word - w0] in 16 bits; w and words are those from w0 on.
template <bool F16, Mode MODE, bool TEMP, int BB>
__global__ __launch_bounds__(256) void head_logits_kernel(
    const uint16_t* __restrict__ ht, int64_t tp, const uint16_t* __restrict__ w, int D,
    const int* __restrict__ count, int words, float inv_tau,
    float* __restrict__ part, const HeadRow* __restrict__ rows, uint16_t* __restrict__ G,
    int64_t ld, int w0, const int* __restrict__ mantissa) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds<true>];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wy = wave >> 1, wx = wave & 1, l32 = lane & 31, half = lane >> 5;
  constexpr int kT = 64 * BB;  // tokens of a tile
  const int n = __builtin_amdgcn_readfirstlane(*count);
  const int nt = (MODE == kStats ? n + kT - 1 : (n + 127) / 128 * 128 + kT - 1) / kT, nv = (words + kTM - 1) / kTM;
  const int64_t N = (int64_t)nt * nv, P = N < gridDim.x ? N : gridDim.x;  // (no empty runs)
  const int64_t wg = xcd_remap(blockIdx.x, gridDim.x);
  if (wg >= P) return;
  const int64_t i0 = run_begin(wg, N, P);
  const int items = (int)(run_begin(wg + 1, N, P) - i0);
  const int nst = stages(D);
  const float k1 = kLog2e, k2 = kLog2e * inv_tau;
  const float unit = MODE == kDlogits ? 1.0f / __int_as_float(*mantissa) : 0.f;

  float mx[BB], sm[BB], st[BB];  // the running maximum, its sum, the sum at the temperature
  auto reset = [&]() {
#pragma unroll
    for (int b = 0; b < BB; ++b) {
      mx[b] = -__builtin_inff();
      sm[b] = st[b] = 0.f;
    }
  };
  auto flush = [&](int tile) {  // the two halves of a token's words, then one entry a wave
    constexpr int E = TEMP ? 3 : 2;
#pragma unroll
    for (int b = 0; b < BB; ++b) {
      const float om = __shfl_xor(mx[b], 32, 64), os = __shfl_xor(sm[b], 32, 64);
      const float m = fmaxf(mx[b], om);
      const float ref = m == -__builtin_inff() ? 0.f : m;
      const float s = sm[b] * __builtin_amdgcn_exp2f((mx[b] - ref) * k1) +
                      os * __builtin_amdgcn_exp2f((om - ref) * k1);
      float* p = part + ((((wg + tile) * 2 + wy) * 256) + wx * (32 * BB) + 32 * b + l32) * E;
      float sT = 0.f;
      if constexpr (TEMP) {
        const float ot = __shfl_xor(st[b], 32, 64);
        sT = st[b] * __builtin_amdgcn_exp2f((mx[b] - ref) * k2) +
             ot * __builtin_amdgcn_exp2f((om - ref) * k2);
      }
      if (half == 0) {
        p[0] = m;
        p[1] = s;
        if constexpr (TEMP) p[2] = sT;
      }
    }
  };

  int tile = -1;
  Loader<true> la;
  Loader<false> lb;
  const Loads<true> loads = loads_of(lds, la, lb, 0, nst);
  // an item's first loads are under way while the one before it is finished
  auto first = [&](int nt_i, int nv_i) {
    la.begin(w + (int64_t)nv_i * kTM * D, words - nv_i * kTM, D, D, wave, lane);
    lb.begin(ht + nt_i * kT, (int)(tp - nt_i * kT), tp, nst * kBK, wave, lane);
    loads.first(wave);
  };
  int nt_i = (int)(i0 / nv), nv_i = (int)(i0 % nv);
  first(nt_i, nv_i);
  for (int item = 0; item < items; ++item) {
    if (nt_i != tile) {
      if constexpr (MODE == kStats) {
        if (tile >= 0) flush(tile);
        reset();
      }
      tile = nt_i;
    }
    const int v0 = nv_i * kTM + wy * 128, t0 = nt_i * kT + wx * (32 * BB);  // the wave's first ones
    const int v_left = words - v0 < 128 ? words - v0 : 128;
    f32x16 acc[4][BB];
    product<F16, true, BB>(lds, loads, acc);
    if (++nv_i == nv) {
      nv_i = 0;
      ++nt_i;
    }
    if (item + 1 < items) first(nt_i, nv_i);
    if constexpr (MODE == kStats) {
      const int left = v_left - 4 * half;
      auto softmax = [&](auto full_tag) {
        constexpr bool FULL = decltype(full_tag)::value;
        auto block = [&](int a, int b) {
          f32x16 z = acc_block(acc[a][b]);
          if constexpr (!FULL) {  // past the last word: no logit
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (32 * a + 8 * (i / 4) + i % 4 >= left) z[i] = -__builtin_inff();
          }
          return z;
        };
#pragma unroll
        for (int b = 0; b < BB; ++b) {
          float m4[4] = {mx[b], mx[b], mx[b], mx[b]};
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const f32x16 z = block(a, b);
#pragma unroll
            for (int i = 0; i < 16; ++i) m4[i % 4] = fmaxf(m4[i % 4], z[i]);
            __builtin_amdgcn_sched_barrier(0);
          }
          const float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          const float ref = m == -__builtin_inff() ? 0.f : m;
          const float c1 = -ref * k1, c2 = -ref * k2;
          float s4[4] = {0.f, 0.f, 0.f, 0.f}, t4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            const f32x16 z = block(a, b);
            float e[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
              e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], k1, c1));
#pragma unroll
            for (int i = 0; i < 16; ++i) s4[i % 4] += e[i];
            if constexpr (TEMP) {
#pragma unroll
              for (int i = 0; i < 16; ++i)
                e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], k2, c2));
#pragma unroll
              for (int i = 0; i < 16; ++i) t4[i % 4] += e[i];
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          sm[b] = sm[b] * __builtin_amdgcn_exp2f((mx[b] - ref) * k1) +
                  ((s4[0] + s4[1]) + (s4[2] + s4[3]));
          if constexpr (TEMP)
            st[b] = st[b] * __builtin_amdgcn_exp2f((mx[b] - ref) * k2) +
                    ((t4[0] + t4[1]) + (t4[2] + t4[3]));
          mx[b] = m;
        }
      };
      if (v_left == 128)
        softmax(std::true_type{});
      else
        softmax(std::false_type{});
    } else {
      // a token's words pass through LDS, so that whole lines are stored (from the
      // registers, 32 bytes of 32 rows a store, a tile took 11 us more): 32 tokens of a wave at a
      // time, in the third pair's slot, which the next item's first loads leave alone
      uint8_t* mine = lds + kLdsB + 4 * kOp + wave * (32 * 256);
#pragma unroll
      for (int b = 0; b < BB; ++b) {
        const int r = t0 + 32 * b + l32;
        // rows and words past the last are zeros, for dW's and dh's contractions
        HeadRow hr = r < n ? rows[r] : HeadRow{0.f, 0.f, 0.f, 0.f};
        hr.c1 *= unit;
        hr.c2 *= unit;
        const int left = v_left - 4 * half;
        uint8_t* row = mine + l32 * 256 + 8 * half;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const f32x16 z = acc_block(acc[a][b]);
          float p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i)
            p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], k1, -hr.lse));
#pragma unroll
          for (int i = 0; i < 16; ++i) p[i] *= hr.c1;
          if constexpr (TEMP) {
            float q[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
              q[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i], k2, -hr.lse_t));
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = __builtin_fmaf(hr.c2, q[i], p[i]);
          }
          if (v_left < 128) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (32 * a + 8 * (i / 4) + i % 4 >= left) p[i] = 0.f;
          }
#pragma unroll
          for (int q = 0; q < 4; ++q)  // words 32 a + 8 q + 4 half ..
            *reinterpret_cast<u32x2*>(row + 16 * ((4 * a + q) ^ (l32 & 15))) =
                u32x2{pack2<F16>(p[4 * q], p[4 * q + 1]), pack2<F16>(p[4 * q + 2], p[4 * q + 3])};
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!TEMP) {  // the label's word
          asm volatile("" ::: "memory");
          const int c = __float_as_int(hr.lse_t) - w0 - v0;
          if (half == 0 && c >= 0 && c < 128)
            *reinterpret_cast<any16*>(mine + l32 * 256 + 16 * ((c >> 3) ^ (l32 & 15)) +
                                      2 * (c & 7)) = (uint16_t)pack2<F16>(hr.c2, 0.f);
          asm volatile("" ::: "memory");
        }
        store_rows(mine, G + (int64_t)(t0 + 32 * b) * ld + v0, ld, 32, 128);
      }
    }
  }
  if constexpr (MODE == kStats)
    if (tile >= 0) flush(tile);
}

// The wave's 128 x 128 to an output, what lies inside: put(value, old) for every element,
// old read from there if ADD.  Row by row through a pitch that the compiler cannot take
// apart (precomputed offsets would need the accumulators' registers); a block's sixteen old
// values are read before the first is written (one by one, each waiting for its read, the
// sums of a tile of dh took 120 us).
template <bool ADD, bool FULL, typename T, typename Put>
__device__ __forceinline__ void write_as(T* base, int64_t pitch, int rows_left, int cols_left,
                                         const f32x16 (&acc)[4][4], Put put) {
  const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
  int64_t pv = pitch;
  asm volatile("" : "+v"(pv));
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    if (!FULL && 32 * a >= rows_left) break;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (FULL || 32 * b + l32 < cols_left) {
        T* const p0 = base + (int64_t)(32 * a) * pitch + 32 * b + (4 * half * pv + l32);
        const int left = rows_left - 32 * a - 4 * half;
        T old[16];
        if constexpr (ADD) {
          T* p = p0;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (FULL || 8 * (i / 4) + i % 4 < left) old[i] = *p;
            if (i < 15) p += i % 4 == 3 ? 5 * pv : pv;
          }
        }
        const f32x16 v = acc_block(acc[a][b]);
        T* p = p0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (FULL || 8 * (i / 4) + i % 4 < left) *p = put(v[i], ADD ? old[i] : T(0.f));
          if (i < 15) p += i % 4 == 3 ? 5 * pv : pv;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}
template <bool ADD, typename T, typename Put>
__device__ __forceinline__ void write_tile(T* base, int64_t pitch, int rows_left, int cols_left,
                                           const f32x16 (&acc)[4][4], Put put) {
  if (rows_left >= 128 && cols_left >= 128)
    write_as<ADD, true>(base, pitch, rows_left, cols_left, acc, put);
  else if (rows_left > 0 && cols_left > 0)
    write_as<ADD, false>(base, pitch, rows_left, cols_left, acc, put);
}

// dh: A = G (tokens; along the words), B = W (across).  The parts of the
// contraction and the pieces of the vocabulary meet in part[s][row][D].
template <bool F16, bool ADD>
__global__ __launch_bounds__(256) void head_dh_kernel(
    const uint16_t* __restrict__ G, int64_t ld, const uint16_t* __restrict__ w, int D,
    const int* __restrict__ count, int64_t T, int words, HeadCut plan, int all,
    float* __restrict__ part, int* __restrict__ used) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds<true>];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wy = wave >> 1, wx = wave & 1;
  const int n = __builtin_amdgcn_readfirstlane(*count);
  const int nt = (n + kTM - 1) / kTM, nd = (D + kTN - 1) / kTN;
  const int64_t tiles = (int64_t)nt * nd, P = gridDim.x;
  const int64_t wg = xcd_remap(blockIdx.x, gridDim.x);
  const HeadCut cut = head_cut(plan, all, T, n, D, (int)P);
  const int parts = cut.parts, per = cut.per;
  if (blockIdx.x == 0 && threadIdx.x == 0) *used = parts;
  const int nst = stages(words);
  for (int64_t item = wg; item < tiles * parts; item += P) {
    const int s = (int)(item / tiles), tile = (int)(item % tiles);
    const int m0 = tile / nd * kTM, d0 = tile % nd * kTN;
    const int s_end = s * per + per < nst ? s * per + per : nst;
    if (s * per >= s_end) continue;  // a last piece of fewer words: its part adds nothing
    f32x16 acc[4][4];
    {
      Loader<true> la;
      la.begin(G + (int64_t)m0 * ld, n - m0, ld, nst * kBK, wave, lane);
      Loader<false> lb;
      lb.begin(w + d0, D - d0, D, words, wave, lane);
      const Loads<true> l = loads_of(lds, la, lb, s * per, s_end);
      l.first(wave);
      product<F16, true, 4>(lds, l, acc);
    }
    const int r0 = m0 + wy * 128, c0 = d0 + wx * 128;
    float* out = part + ((int64_t)s * n + r0) * D + c0;
    write_tile<ADD>(out, D, n - r0, D - c0, acc, [](float v, float old) { return v + old; });
  }
}

// dW: G (words) and hs (columns), both across the tokens.  PARTS: to part[s][word][D],
// unscaled; else to dW's rows, times 2^exp[0] (float at exp[2]).  Float32: A = G, a lane has a column and
// stores 128 bytes of a row with its neighbours.  16 bits: A = hs, a lane has a word and four
// columns in a row, which pass through LDS as the dlogits do (with A = G, 2 bytes a lane and
// LDS write: 64 tokens, 50000 words 82 us, 65 so).
template <bool F16, bool PARTS, typename O, bool ACC>
__global__ __launch_bounds__(256) void head_dw_kernel(
    const uint16_t* __restrict__ G, int64_t ld, const uint16_t* __restrict__ hs, int D,
    const int* __restrict__ count, int words, int parts, int per, const int* __restrict__ exp,
    O* __restrict__ dw) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLds<false> + (sizeof(O) == 2 ? 4 * 32 * 256 : 0)];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wy = wave >> 1, wx = wave & 1, l32 = lane & 31, half = lane >> 5;
  const int n = __builtin_amdgcn_readfirstlane(*count);
  const int nv = (words + kTM - 1) / kTM, nd = (D + kTN - 1) / kTN;
  const int64_t tiles = (int64_t)nv * nd, P = gridDim.x;
  const int64_t wg = xcd_remap(blockIdx.x, gridDim.x);
  const int nst = stages(n);
  constexpr bool SWAP = sizeof(O) == 2;
  const int e = PARTS ? 0 : __builtin_amdgcn_readfirstlane(exp[0]);
  const float mant = PARTS ? 1.0f : __int_as_float(__builtin_amdgcn_readfirstlane(exp[2]));
  for (int64_t item = wg; item < tiles * parts; item += P) {
    const int s = (int)(item / tiles), tile = (int)(item % tiles);
    const int m0 = tile / nd * kTM, d0 = tile % nd * kTN;
    const int s_end = s * per + per < nst ? s * per + per : nst;
    const int r0 = m0 + (SWAP ? wx : wy) * 128, c0 = d0 + (SWAP ? wy : wx) * 128;
    O* out = dw + ((int64_t)s * words + r0) * D + c0;
    if (s * per >= s_end) {  // fewer rows than the parts were made for
      if constexpr (!ACC)
        for (int r = 0; r < 128 && r0 + r < words; ++r)
          for (int c = lane; c < 128 && c0 + c < D; c += 64) out[(int64_t)r * D + c] = O(0.f);
      continue;
    }
    f32x16 acc[4][4];
    {
      Loader<false> g, h;
      g.begin(G + m0, (int)ld - m0, ld, nst * kBK, wave, lane);
      h.begin(hs + d0, D - d0, D, n, wave, lane);
      const Loads<false> l = loads_of(lds, SWAP ? h : g, SWAP ? g : h, s * per, s_end);
      l.first(wave);
      product<F16, false, 4>(lds, l, acc);
    }
    if constexpr (SWAP) {
      uint8_t* mine = lds + kLds<false> + wave * (32 * 256);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        uint8_t* row = mine + l32 * 256 + 8 * half;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          f32x16 v = acc_block(acc[a][b]);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = ldexpf(mant * v[i], e);
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<u32x2*>(row + 16 * ((4 * a + q) ^ (l32 & 15))) =
                u32x2{pack2<F16>(v[4 * q], v[4 * q + 1]), pack2<F16>(v[4 * q + 2], v[4 * q + 3])};
          __builtin_amdgcn_sched_barrier(0);
        }
        store_rows(mine, reinterpret_cast<uint16_t*>(out) + (int64_t)(32 * b) * D, D,
                   words - r0 - 32 * b, D - c0);
      }
    } else {
      write_tile<ACC>(out, D, words - r0, D - c0, acc, [&](float v, O old) {
        if constexpr (PARTS)
          return v;
        else if constexpr (ACC)
          return old + ldexpf(mant * v, e);
        else
          return ldexpf(mant * v, e);
      });
    }
  }
}

// dW (+)= 2^exp[0] (float at exp[2]) times the sum of the parts, in their order; n elements, a multiple of 8
template <typename O, bool ACC>
__global__ __launch_bounds__(256) void head_dw_sum_kernel(const float* __restrict__ part,
                                                          int64_t n, int parts,
                                                          const int* __restrict__ exp,
                                                          O* __restrict__ dw) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  f32x4 v = *reinterpret_cast<const f32x4*>(part + i);
  for (int s = 1; s < parts; ++s) v += *reinterpret_cast<const f32x4*>(part + s * n + i);
  const int e = exp[0];
  const float mant = __int_as_float(exp[2]);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float x = ldexpf(mant * v[j], e);
    if constexpr (ACC)
      dw[i + j] += x;
    else
      dw[i + j] = (O)x;
  }
}

// dW of up to 64 tokens: it is written, and little else.  A workgroup has 256 columns d, whose h it
// keeps in registers as matrix operands, and a run of words, 128 of G at a time through LDS; a wave
// has 64 of the columns.  Rows of the product are columns d, in an order in which a lane's sixteen
// and its other block's are neighbours, columns are words; 32 words x 64 columns at a time
// pass through LDS, so that whole lines are stored.  Two workgroups a CU.
// Bound: HBM's writes.
template <bool F16, typename O, bool ACC>
__global__ __launch_bounds__(256, 2) void head_dw_few_kernel(
    const uint16_t* __restrict__ G, int64_t ld, const uint16_t* __restrict__ hs, int D,
    const int* __restrict__ count, int words, int runs, const int* __restrict__ exp,
    O* __restrict__ dw) {
  constexpr int kWords = 128, kPitch = 2 * kWords;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[64 * 512 + 64 * kPitch];
  uint8_t* const gt = lds + 64 * 512;  // G's tile; before it h's, then the waves' results
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nd = (D + 255) / 256, id = (int)xcd_remap(blockIdx.x, gridDim.x);
  const int d0 = id % nd * 256, run = id / nd;
  const int eights = (words + 7) / 8;
  const int v_beg = 8 * (int)((int64_t)run * eights / runs);
  int v_end = 8 * (int)((int64_t)(run + 1) * eights / runs);
  v_end = v_end < words ? v_end : words;
  const int n = __builtin_amdgcn_readfirstlane(*count), steps = (n + 15) / 16;
  const int e = exp[0];
  const float mant = __int_as_float(exp[2]);

  u32x4 next[4];
  auto load = [&](int v0) {  // 64 rows of 128 words
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 256 * j + tid, r = i >> 4, c = v0 + 8 * (i & 15);
      next[j] = ld16(G + r * ld + (c < ld ? c : ld - 8));
    }
  };
  load(v_beg);
  // h's 64 x 256: column 64 k + 32 half + 16 x + 4 a + b lies at 64 k + 32 x + 8 a + 4 half + b
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int i = 256 * j + tid, r = i >> 5, c = 8 * (i & 31);
    u32x4 v = {0, 0, 0, 0};
    if (r < n && d0 + c < D) v = ld16(hs + (int64_t)r * D + d0 + c);
    const int at = (c & ~63) + 32 * ((c >> 4) & 1) + 2 * (c & 8) + 4 * ((c >> 5) & 1);
    *reinterpret_cast<u32x2*>(lds + off_across(r, at)) = u32x2{v.x, v.y};
    *reinterpret_cast<u32x2*>(lds + off_across(r, at + 8)) = u32x2{v.z, v.w};
  }
  __syncthreads();
  const int trow = 8 * half + ((lane & 15) >> 2);
  const int tcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto across = [&](const uint8_t* at, int pitch) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * pitch));
    const u32x2 l = __builtin_bit_cast(u32x2, lo), u = __builtin_bit_cast(u32x2, hi);
    return u32x4{l.x, l.y, u.x, u.y};
  };
  auto off_g = [&](int r, int c) { return r * kPitch + 32 * ((c >> 4) ^ swz(r)) + 2 * (c & 15); };
  u32x4 hf[4][2];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int x = 0; x < 2; ++x)
      hf[t][x] = across(lds + off_across(trow, 64 * wave + 32 * x + tcol) + 16 * t * 512, 512);

  constexpr int kEl = 16 / sizeof(O), kPieces = 64 / kEl, kRows = 64 / kPieces;  // of a store
  uint8_t* const mine = lds + wave * 8192;
  const int sr = lane / kPieces, sp = lane % kPieces, sc = d0 + 64 * wave + kEl * sp;
  for (int v0 = v_beg; v0 < v_end; v0 += kWords) {
    __syncthreads();  // h's operands, or the tile before, have been read
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 256 * j + tid;
      st16(gt + off_g(i >> 4, 8 * (i & 15)), next[j]);
    }
    __syncthreads();
    if (v0 + kWords < v_end) load(v0 + kWords);
#pragma unroll 1
    for (int b = 0; b < kWords / 32; ++b) {
      const int left = v_end - v0 - 32 * b;
      if (left <= 0) break;
      f32x16 acc[2] = {};
      const uint8_t* gp = gt + off_g(trow, 32 * b + tcol);
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (t < steps) {
          const u32x4 gf = across(gp + 16 * t * kPitch, kPitch);
#pragma unroll
          for (int x = 0; x < 2; ++x) acc[x] = mfma<F16>(hf[t][x], gf, acc[x]);
        }
      // a lane: word l32, columns 32 half + 16 x + i of the wave's 64
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int i = 0; i < 16; i += kEl) {
          u32x4 o;
          if constexpr (sizeof(O) == 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = __float_as_uint(ldexpf(mant * acc[x][i + k], e));
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              o[k] = pack2<F16>(ldexpf(mant * acc[x][i + 2 * k], e),
                                ldexpf(mant * acc[x][i + 2 * k + 1], e));
          }
          const int piece = (32 * half + 16 * x + i) / kEl;
          st16(mine + l32 * (64 * sizeof(O)) + 16 * (piece ^ (l32 & (kPieces - 1))), o);
        }
      }
      __builtin_amdgcn_wave_barrier();
      O* to = dw + (int64_t)(v0 + 32 * b + sr) * D + sc;
      const int rows = sc < D ? left - sr : 0;
      u32x4 old[32 / kRows];
      if constexpr (ACC) {
#pragma unroll
        for (int k = 0; k < 32 / kRows; ++k)
          if (kRows * k < rows) old[k] = ld16(to + (int64_t)kRows * k * D);
      }
#pragma unroll
      for (int k = 0; k < 32 / kRows; ++k) {
        const int r = kRows * k + sr;
        u32x4 o = *reinterpret_cast<const u32x4*>(mine + r * (64 * sizeof(O)) +
                                                  16 * (sp ^ (r & (kPieces - 1))));
        if constexpr (ACC) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            o[q] = __float_as_uint(__uint_as_float(o[q]) + __uint_as_float(old[k][q]));
        }
        if (kRows * k < rows) st16(to + (int64_t)kRows * k * D, o);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

#define TM_HEAD_GRID(GRID) dim3((unsigned)(GRID)), dim3(256), 0, stream

static int64_t grid_of(int64_t items) {
  const int64_t cus = current_cu_count();
  return items < cus ? items : cus;
}

// Tokens of a tile of logits: 64 and 192 (the softmax sums only), 128 or 256.  A stage takes
// 0.52 us a workgroup of 64, 0.58 of 128 (both by their loads), 0.68 of 192, 0.80 of 256.  So
// narrow tiles are for few words, where 256 would leave workgroups idle (300 tokens of 5000 x
// 2048: 36 us, 51 with 256), and where they waste less of the last tile (300 of 50000: 93 us,
// 113 with 256; 800 of 50000: 178, 208).  Dlogits are kept, in rows to the next multiple of 256, and
// their products contract them 128 at a time: tiles of 192 would run past the last row.
int head_tile_tokens(int64_t T, int64_t words, bool stats) {
  const int64_t P = current_cu_count(), nv = (words + kTM - 1) / kTM;
  const double us[4] = {0.52, 0.58, 0.68, 0.80};
  int best = 256;
  double least = 0;
  for (int tile = 256; tile >= 64; tile -= 64) {
    if (!stats && tile != 256 && tile != 128) continue;
    const int64_t items = (T + tile - 1) / tile * nv;
    const double cost = (double)((items + P - 1) / P) * us[tile / 64 - 1];
    if (tile == 256 || cost < least) {
      least = cost;
      best = tile;
    }
  }
  return best;
}

int head_logits_grid(int64_t T, int64_t words, int tile) {
  return (int)grid_of((T + tile - 1) / tile * ((words + kTM - 1) / kTM));
}

int64_t head_part_floats(int64_t T, int64_t words) {
  const int tile = head_tile_tokens(T, words, true);
  return (current_cu_count() + (T + tile - 1) / tile + 1) * 2 * 256 * 3;
}

template <bool F16, Mode MODE, int BB>
static hipError_t run_logits(const HeadIn& in, const uint16_t* ht, const int* count, int64_t w0,
                             int64_t n, float* part, const HeadRow* rows, const int* mantissa,
                             uint16_t* G, int64_t ld, hipStream_t stream) {
  const int64_t T = MODE == kStats ? in.T : (in.T + 127) / 128 * 128;
  const int grid = head_logits_grid(T, n, 64 * BB);
  const uint16_t* w = in.w + w0 * in.D;
  if (in.K > 0 && in.tau != 1.0f)
    hipLaunchKernelGGL((head_logits_kernel<F16, MODE, true, BB>), TM_HEAD_GRID(grid), ht,
                       head_padded(in.T), w, in.D, count, (int)n, 1.0f / in.tau, part, rows, G, ld,
                       (int)w0, mantissa);
  else
    hipLaunchKernelGGL((head_logits_kernel<F16, MODE, false, BB>), TM_HEAD_GRID(grid), ht,
                       head_padded(in.T), w, in.D, count, (int)n, 1.0f, part, rows, G, ld, (int)w0,
                       mantissa);
  return hipGetLastError();
}

hipError_t launch_head_logits(const HeadIn& in, const uint16_t* ht, const int* count, float* part,
                              hipStream_t stream) {
  const int tile = head_tile_tokens(in.T, in.V, true);
#define TM_HEAD_LOGITS(F16, BB) \
  run_logits<F16, kStats, BB>(in, ht, count, 0, in.V, part, nullptr, nullptr, nullptr, 0, stream)
  if (tile == 64) return in.f16 ? TM_HEAD_LOGITS(true, 1) : TM_HEAD_LOGITS(false, 1);
  if (tile == 128) return in.f16 ? TM_HEAD_LOGITS(true, 2) : TM_HEAD_LOGITS(false, 2);
  if (tile == 192) return in.f16 ? TM_HEAD_LOGITS(true, 3) : TM_HEAD_LOGITS(false, 3);
  return in.f16 ? TM_HEAD_LOGITS(true, 4) : TM_HEAD_LOGITS(false, 4);
#undef TM_HEAD_LOGITS
}

hipError_t launch_head_dlogits(const HeadIn& in, const uint16_t* ht, const int* count,
                               const HeadRow* rows, const int* mantissa, int64_t w0, int64_t n,
                               uint16_t* G, int64_t ld, hipStream_t stream) {
#define TM_HEAD_DLOGITS(F16, BB) \
  run_logits<F16, kDlogits, BB>(in, ht, count, w0, n, nullptr, rows, mantissa, G, ld, stream)
  if (head_tile_tokens(in.T, n, false) == 128)
    return in.f16 ? TM_HEAD_DLOGITS(true, 2) : TM_HEAD_DLOGITS(false, 2);
  return in.f16 ? TM_HEAD_DLOGITS(true, 4) : TM_HEAD_DLOGITS(false, 4);
#undef TM_HEAD_DLOGITS
}

hipError_t launch_head_dh(const HeadIn& in, const int* count, const uint16_t* G, int64_t ld,
                          int64_t w0, int64_t n, HeadCut plan, int nst, bool add, float* part_h,
                          int* used, hipStream_t stream) {
  const uint16_t* w = in.w + w0 * in.D;
#define TM_HEAD_DH(F16, ADD)                                                                    \
  hipLaunchKernelGGL((head_dh_kernel<F16, ADD>), TM_HEAD_GRID(current_cu_count()), G, ld, w, in.D, \
                     count, in.T, (int)n, plan, nst, part_h, used)
  if (in.f16) {
    if (add)
      TM_HEAD_DH(true, true);
    else
      TM_HEAD_DH(true, false);
  } else {
    if (add)
      TM_HEAD_DH(false, true);
    else
      TM_HEAD_DH(false, false);
  }
#undef TM_HEAD_DH
  return hipGetLastError();
}

template <bool F16, typename O, bool ACC>
static hipError_t run_dw(const HeadIn& in, const int* count, const uint16_t* G, int64_t ld,
                         const uint16_t* hs, int64_t n, int parts, int per, const int* exp, O* dw,
                         float* part_w, hipStream_t stream) {
  const int64_t nd = (in.D + kTN - 1) / kTN, items = ((n + kTM - 1) / kTM) * nd * parts;
  // few tokens: 64 of 50000 x 2048 in 45 us, 66 by the tiles of products
  if (in.T <= 64) {
    const int64_t most = (n + 63) / 64, all = 2 * current_cu_count() / nd;
    const int64_t runs = all < 1 ? 1 : all < most ? all : most;
    hipLaunchKernelGGL((head_dw_few_kernel<F16, O, ACC>), TM_HEAD_GRID(runs * nd), G, ld, hs, in.D,
                       count, (int)n, (int)runs, exp, dw);
    return hipGetLastError();
  }
  if (parts == 1) {
    hipLaunchKernelGGL((head_dw_kernel<F16, false, O, ACC>), TM_HEAD_GRID(grid_of(items)), G, ld,
                       hs, in.D, count, (int)n, 1, per, exp, dw);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((head_dw_kernel<F16, true, float, false>), TM_HEAD_GRID(grid_of(items)), G, ld,
                     hs, in.D, count, (int)n, parts, per, exp, part_w);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t all = n * in.D;
  hipLaunchKernelGGL((head_dw_sum_kernel<O, ACC>), TM_HEAD_GRID((all / 4 + 255) / 256), part_w, all,
                     parts, exp, dw);
  return hipGetLastError();
}

hipError_t launch_head_dw(const HeadIn& in, const int* count, const uint16_t* G, int64_t ld,
                          const uint16_t* hs, int64_t w0, int64_t n, int parts, int per,
                          const int* exp, void* dw, int dw_type, bool accumulate, float* part_w,
                          hipStream_t stream) {
#define TM_HEAD_DW(F16, O, ACC)                                                                 \
  run_dw<F16, O, ACC>(in, count, G, ld, hs, n, parts, per, exp, static_cast<O*>(dw) + w0 * in.D, \
                      part_w, stream)
  if (dw_type == 0) {
    if (accumulate) return in.f16 ? TM_HEAD_DW(true, float, true) : TM_HEAD_DW(false, float, true);
    return in.f16 ? TM_HEAD_DW(true, float, false) : TM_HEAD_DW(false, float, false);
  }
  return in.f16 ? TM_HEAD_DW(true, _Float16, false) : TM_HEAD_DW(false, __bf16, false);
#undef TM_HEAD_DW
}

}  // namespace tmk
