// The selective scan over packed sequences (formulas: seq_scan_dev.hpp).
//
// scan_y_kernel: a workgroup of four waves walks the tiles of 64 tokens of one
// sequence (or of a segment of it) and one head, the state in registers
// (32 float32 a lane: wave w holds states 32 w .. + 31 of the 64 channels) and,
// as two bfloat16 terms, in LDS for the products that read it.  Of y^T (64
// channels x 64 tokens) wave w makes tokens 16 w .. + 15:
//   g = B C^T (rows s, columns t: its lanes then hold exactly what the next
//       product wants of it), times e^{c_t - c_s} dt'_s, in two terms;
//   y^T = x^T g + e^{c_t} S C^T + D x^T.
// The state takes the tile's e^{c_Q - c_s} dt'_s x_s B_s^T.
//
// Where there are too few sequences and heads to fill the chip, a sequence is
// cut into segments: scan_state_kernel makes each segment's own state,
// scan_pass_kernel (or the segments' workgroups themselves, where those are few)
// the states between the segments, then scan_y_kernel walks all segments at once.
//
// Why tiles of 64 and four waves: two workgroups fit a CU (69 KiB of LDS, mostly
// the state's terms, which every wave reads), so that one computes while the
// other waits; 128 tokens and eight waves would leave one, and more of g that is
// thrown away.  No single thing bounds it: of 180 us for 16384 tokens of 64 heads
// in eight sequences (3.3 times the 53 us of reading u and writing y) the matrix
// products busy the SIMDs 30 us, the vector instructions 80, LDS 85, and what
// they wait for each other in a tile's chain is the rest.
#include "seq_scan_dev.hpp"

namespace tmk {

// ---- tiles of 64 tokens: B or C rows (128 wide) and x or dy rows (64 wide) ----
// staged through registers by 256 threads: 4 and 2 vectors of 16 bytes each
struct TileRegs {
  u32x4 m[4], v[2];
};
// rows t0 .. t0 + 63 of mat (128 columns) and vec (64 columns); from t1 on, row
// t1 - 1 again: a load under a condition would make the compiler wait for every
// one before it, so none is, and tile_store puts zeros in their place
__device__ __forceinline__ void tile_load(TileRegs& r, const uint16_t* mat, int64_t ldm,
                                          const uint16_t* vec, int64_t ldv, int t0, int t1) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    r.m[q] = ld16(mat + min(t0 + q * 16 + (tid >> 4), t1 - 1) * ldm + (tid & 15) * 8);
#pragma unroll
  for (int q = 0; q < 2; ++q)
    r.v[q] = ld16(vec + min(t0 + q * 32 + (tid >> 3), t1 - 1) * ldv + (tid & 7) * 8);
}
// n: rows that are there
__device__ __forceinline__ void tile_store(const TileRegs& r, uint8_t* m, uint8_t* v, int n) {
  const int tid = threadIdx.x;
  const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int row = q * 16 + (tid >> 4);
    st16(m + row * kScRowN + (tid & 15) * 16, row < n ? r.m[q] : zero);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int row = q * 32 + (tid >> 3);
    st16(v + row * kScRowP + (tid & 7) * 16, row < n ? r.v[q] : zero);
  }
}

// Values of x in a tile that are not finite.  A token's x stands in the products of
// all the tile's tokens, with zeros for those before it, and zero times infinity is
// not zero: such a value goes into LDS as zero, its token is noted, and what depends
// on it is made NaN after the products (one prompt of 16384 tokens: 241 us, 237
// without).  Values of B, C and dt need none of it: the products of a token before
// them are other rows, columns or masked ones.
struct Spoilt {
  int first[kSqP];  // a channel's first such token, kScQ: none
  int any;
};
__device__ __forceinline__ void spoilt_clear(Spoilt& p, int i) {
  if (i < kSqP) p.first[i] = kScQ;
  if (i == 0) p.any = 0;
}
// zeros in their place in this thread's part of x (TileRegs::v)
__device__ __forceinline__ void spoilt_take(TileRegs& r, Spoilt& p, int n) {
  typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
  u16x2 m = {0, 0};
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, r.v[q][k] & 0x7FFF7FFFu));
  if (m.x < 0x7F80 && m.y < 0x7F80) return;
  const int tid = threadIdx.x;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int row = q * 32 + (tid >> 3);
    if (row >= n) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t half = 0xFFFFu << (16 * i), most = 0x7F80u << (16 * i);
        if ((r.v[q][k] & most) != most) continue;
        r.v[q][k] &= ~half;
        atomicMin(&p.first[(tid & 7) * 8 + 2 * k + i], row);
        p.any = 1;
      }
  }
}

// The wave's state slice += sum_s coef_s vec_s mat_s^T over the tile: rows
// (states) 32 w + 16 nb + 4 (lane / 16) + i, columns (channels) 16 pb + lane % 16.
template <int NT>
__device__ __forceinline__ void state_add(f32x4 (&S)[2][4], const uint8_t* m, const uint8_t* v,
                                          const float* coef) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int r = 32 * kb + 8 * g;
    float w[8];
    const f32x4 w0 = *(const f32x4*)(coef + r), w1 = *(const f32x4*)(coef + r + 4);
    w[0] = w0.x, w[1] = w0.y, w[2] = w0.z, w[3] = w0.w;
    w[4] = w1.x, w[5] = w1.y, w[6] = w1.z, w[7] = w1.w;
    bf16x8 a[2][NT];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      const u32x4 raw = __builtin_bit_cast(u32x4, tr_op(m, kScRowN, r, r + 4, 32 * wave + 16 * nb));
      float f[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf_lo(raw[i]) * w[2 * i];
        f[2 * i + 1] = bf_hi(raw[i]) * w[2 * i + 1];
      }
      split8<NT>(f, a[nb]);
    }
#pragma unroll
    for (int pb = 0; pb < 4; ++pb) {
      const bf16x8 b = tr_op(v, kScRowP, r, r + 4, 16 * pb);
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int q = 0; q < NT; ++q) S[nb][pb] = mfma16(a[nb][q], b, S[nb][pb]);
    }
  }
}

// ---- a segment's own state -------------------------------------------------
// REV false: vec = x, mat = B, coefficient e^{c_Q - c_s} dt'_s, tiles forward:
// the state at the segment's end from the segment alone, at its place; its
// sequence's last segment has no use for it.  REV true: vec = dy, mat = C,
// coefficient e^{c_t}, tiles backward: the gradient with respect to the state before
// the segment, at the place of the one before; not for the first segment.  grid:
// scan_grid, 256 threads.
template <bool F32, bool REV, int NT>
__global__ __launch_bounds__(256, 4) void scan_state_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u,
    const uint16_t* __restrict__ dy, int T, int nheads, const int* __restrict__ off, int nseq,
    int segT, const float* __restrict__ dt_bias, const float* __restrict__ A_log,
    float* __restrict__ state, float* __restrict__ decay) {
  __shared__ __attribute__((aligned(16))) uint8_t m[kScQ * kScRowN], v[kScQ * kScRowP];
  __shared__ Toks<kScQ> tks[2];
  __shared__ __attribute__((aligned(16))) float coefs[2][kScQ];
  const int h = blockIdx.x, sl = blockIdx.y + blockIdx.z * gridDim.y;
  const Slot s = slot_find(off, nseq, T, segT, sl);
  if (s.t0 >= s.t1 || (REV ? s.k == 0 : s.t1 == s.en)) return;
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const uint16_t* mat = u + d + (REV ? kSqN : 0);
  const uint16_t* vec = REV ? dy + h * kSqP : u + h * kSqP;
  const int64_t ldv = REV ? d : cd;
  const float bias = dt_bias[h], rate = sc_rate(A_log[h]);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  f32x4 S[2][4];
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int pb = 0; pb < 4; ++pb) S[nb][pb] = f32x4{0.f, 0.f, 0.f, 0.f};
  float dec = 1.f;
  const int nt = (s.t1 - s.t0 + kScQ - 1) / kScQ;
  TileRegs r;
  float raw = 0.f;
  auto tile_at = [&](int q) { return s.t0 + (REV ? nt - 1 - q : q) * kScQ; };
  auto load = [&](int q) {
    const int t0 = tile_at(q);
    tile_load(r, mat, cd, vec, ldv, t0, min(s.t1, t0 + kScQ));
  };
  auto raw_load = [&](int q) {
    if (q < nt) raw = tok_raw<F32>(zx, Z, nheads, h, min(tile_at(q) + lane, T - 1)) + bias;
  };
  auto toks = [&](int q) {  // by one wave, a tile ahead
    const float rr[1] = {raw};
    Toks<kScQ>& tk = tks[q & 1];
    toks_make<kScQ>(tk, rr, min(s.t1, tile_at(q) + kScQ) - tile_at(q), rate);
    coefs[q & 1][lane] = REV ? tk.ec[lane] : tk.eq[lane] * tk.dt[lane];
  };
  load(0);
  if (wave == 0) {
    raw_load(0);
    toks(0);
    raw_load(1);
  }
  for (int q = 0; q < nt; ++q) {
    tile_store(r, m, v, s.t1 - tile_at(q));
    __syncthreads();
    if (q + 1 < nt) {
      load(q + 1);
      if (wave == 0) {
        toks(q + 1);
        raw_load(q + 2);
      }
    }
    const float last = tks[q & 1].last;
    const float* coef = coefs[q & 1];
    dec *= last;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) S[nb][pb] *= last;
    state_add<NT>(S, m, v, coef);
    __syncthreads();
  }
  const int64_t at = (int64_t)(sl - s.i - (REV ? 1 : 0)) * nheads + h;
  float* o = state + at * kScState + (lane & 15) * kSqN + 32 * wave + 4 * (lane >> 4);
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int pb = 0; pb < 4; ++pb) *(f32x4*)(o + 16 * pb * kSqN + 16 * nb) = S[nb][pb];
  if (threadIdx.x == 0) decay[at] = dec;
}

// ---- the states between the segments, in place of the segments' own ---------
// grid (kScState / 1024, nheads, nseq), 256 threads, 4 values each.  REV false: at a
// segment's place, the state behind it, from init on; true: the gradient of that
// state, from zero behind the last segment.  first: receives init of sequences of
// more than one segment, at the first one's place (float16), or NULL.
template <bool REV>
__global__ __launch_bounds__(256) void scan_pass_kernel(float* __restrict__ state,
                                                        const float* __restrict__ decay, int T,
                                                        int nheads, const int* __restrict__ off,
                                                        int segT,
                                                        const uint16_t* __restrict__ init,
                                                        uint16_t* __restrict__ first) {
  const int h = blockIdx.y, i = blockIdx.z;
  const int st = off ? slot_off(off, T, i) : 0, en = off ? slot_off(off, T, i + 1) : T;
  const int nk = en > st ? (en - st + segT - 1) / segT : 0;
  if (nk <= 1) return;
  const int64_t base = st / segT;
  const int e = (int)(blockIdx.x * 256 + threadIdx.x) * 4;
  f32x4 E = {0.f, 0.f, 0.f, 0.f};
  if (!REV && init) {
    const u32x2 w = *(const u32x2*)(init + ((int64_t)i * nheads + h) * kScState + e);
    if (first) *(u32x2*)(first + (base * nheads + h) * kScState + e) = w;
    E = f32x4{h2f((uint16_t)w.x), h2f((uint16_t)(w.x >> 16)), h2f((uint16_t)w.y),
              h2f((uint16_t)(w.y >> 16))};
  }
  auto at = [&](int k) { return state + ((base + k) * nheads + h) * kScState + e; };
  // two segments' loads are issued together, and before the two before them are
  // stored, as a wait for loads is one for older stores too (one prompt of 16384
  // tokens backward, two passes: 1140 us in all, four at a time 1163; its scan with 8
  // heads: 61, 58, and 67 one at a time)
  constexpr int kAhead = 2;
  f32x4 own[2][kAhead];
  float dec[2][kAhead];
  auto load = [&](int b, int kb) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int k = min(kb + q, nk - 2), kk = REV ? nk - 2 - k : k;
      own[b][q] = *(const f32x4*)at(kk);
      dec[b][q] = decay[(base + kk) * nheads + h];
    }
  };
  auto walk = [&](int b, int kb) {
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      const int k = kb + q;
      if (k >= nk - 1) break;
      E = E * dec[b][q] + own[b][q];
      *(f32x4*)at(REV ? nk - 2 - k : k) = E;
    }
  };
  load(0, 0);
  for (int kb = 0; kb < nk - 1; kb += 2 * kAhead) {
    load(1, kb + kAhead);
    walk(0, kb);
    load(0, kb + 2 * kAhead);
    walk(1, kb + kAhead);
  }
}

// Tokens that a segment's last tile may have for it to be taken token by token:
// 16 sequences of one token: 21 us as tiles, 16 so (most of a tile's time is
// its chain of products and barriers, whatever it holds)
constexpr int kScShort = 4;

// ---- y ---------------------------------------------------------------------
// grid: scan_grid, 256 threads.  state: the states behind the segments, or, with
// decay, the segments' own ones; NULL where every sequence is one segment (one
// workgroup a head and sequence then, which may write over init).  first: init of the
// sequences of more segments, where it is written over, or NULL.
template <bool F32>
__global__ __launch_bounds__(256, 2) void scan_y_kernel(
    const typename Zx<F32>::T* __restrict__ zx, const uint16_t* __restrict__ u, int T, int nheads,
    const int* __restrict__ off, int nseq, int segT, const float* __restrict__ dt_bias,
    const float* __restrict__ A_log, const float* __restrict__ Dp, const uint16_t* init,
    const uint16_t* __restrict__ first, const float* __restrict__ state,
    const float* __restrict__ decay, uint16_t* final_, uint16_t* __restrict__ y) {
  __shared__ __attribute__((aligned(16))) uint8_t Bt[kScQ * kScRowN], xt[kScQ * kScRowP];
  __shared__ __attribute__((aligned(16))) uint8_t Sl[2][kSqP * kScRowS];  // the state's terms
  __shared__ Toks<kScQ> tks[2];
  __shared__ __attribute__((aligned(16))) float coefs[2][kScQ];
  __shared__ __attribute__((aligned(16))) Spoilt spoilt[2];
  const int h = blockIdx.x, sl = blockIdx.y + blockIdx.z * gridDim.y;
  const Slot s = slot_find(off, nseq, T, segT, sl);
  const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t sat = ((int64_t)s.i * nheads + h) * kScState;
  if (s.t0 >= s.t1) {
    // an empty sequence's state stays what it was
    if (s.k == 0 && s.en <= s.st && final_ && final_ != init)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = (q * 256 + (int)threadIdx.x) * 8;
        st16(final_ + sat + e, init ? ld16(init + sat + e) : u32x4{0, 0, 0, 0});
      }
    return;
  }
  const int d = nheads * kSqP, cd = d + 2 * kSqN;
  const int64_t Z = (int64_t)2 * d + 2 * kSqN + nheads;
  const float bias = dt_bias[h], rate = sc_rate(A_log[h]), skip = Dp[h];
  const uint16_t *Bg = u + d, *Cg = Bg + kSqN, *xg = u + h * kSqP;
  TileRegs r;
  bf16x8 cn[4];
  float raw;
  // this wave's 16 rows of C as operands (their columns contiguous)
  auto load = [&](int t0) {
    const int t1 = min(s.t1, t0 + kScQ);
    tile_load(r, Bg, cd, xg, cd, t0, t1);
    // (behind the last token: its C again, for a y that is not stored)
    const int64_t t = min(t0 + 16 * wave + col, t1 - 1);
#pragma unroll
    for (int k = 0; k < 4; ++k) cn[k] = as_bf16x8(ld16(Cg + t * cd + 32 * k + 8 * g));
  };
  // wave 0 (whose tokens have the fewest tokens before them) makes the token
  // values a tile ahead, of dt loaded yet a tile earlier
  auto raw_load = [&](int t0) {
    raw = tok_raw<F32>(zx, Z, nheads, h, min(t0 + lane, T - 1)) + bias;
  };
  auto toks = [&](int t0, int buf) {
    const float rr[1] = {raw};
    toks_make<kScQ>(tks[buf], rr, min(s.t1, t0 + kScQ) - t0, rate);
    coefs[buf][lane] = tks[buf].eq[lane] * tks[buf].dt[lane];
  };
  if (wave == 0) raw_load(s.t0);
  load(s.t0);
  if (s.t1 - s.t0 > kScShort) {  // (there are tiles)
    spoilt_clear(spoilt[0], threadIdx.x);
    __syncthreads();
  }
  // C of this lane's states and the last tile's first tokens, in case it is short
  u32x2 cv[kScShort][2];
  const int tail = s.t0 + (s.t1 - s.t0 - 1) / kScQ * kScQ;
#pragma unroll
  for (int q = 0; q < kScShort; ++q)
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
      cv[q][nb] = *(const u32x2*)(Cg + (int64_t)min(tail + q, s.t1 - 1) * cd + 32 * wave +
                                  16 * nb + 4 * g);
  // (all of the above on their way before the state's own loads are waited for)
  f32x4 S[2][4];
  const int sof = col * kSqN + 32 * wave + 4 * g;  // of S[0][0] in a state
  const int place = sl - s.i;  // of this segment's state
  if (state && !decay && s.k > 0) {
    const float* p = state + ((int64_t)(place - 1) * nheads + h) * kScState + sof;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) S[nb][pb] = *(const f32x4*)(p + 16 * pb * kSqN + 16 * nb);
  } else if (init) {
    const uint16_t* p = first && s.t1 < s.en
                            ? first + ((int64_t)place * nheads + h) * kScState + sof
                            : init + sat + sof;
    u32x2 w[2][4];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) w[nb][pb] = *(const u32x2*)(p + 16 * pb * kSqN + 16 * nb);
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb)
        S[nb][pb] = f32x4{h2f((uint16_t)w[nb][pb].x), h2f((uint16_t)(w[nb][pb].x >> 16)),
                          h2f((uint16_t)w[nb][pb].y), h2f((uint16_t)(w[nb][pb].y >> 16))};
  } else {
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) S[nb][pb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (decay)  // the segments' own states: take those of the segments before this one
    for (int k = s.k; k > 0; --k) {
      const int64_t at = (int64_t)(place - k) * nheads + h;
      const float dec = decay[at];
      const float* p = state + at * kScState + sof;
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int pb = 0; pb < 4; ++pb)
          S[nb][pb] = S[nb][pb] * dec + *(const f32x4*)(p + 16 * pb * kSqN + 16 * nb);
    }
  if (wave == 0) {
    toks(s.t0, 0);
    raw_load(s.t0 + kScQ);
  }
  int buf = 0;
  int t0 = s.t0;
  for (; s.t1 - t0 > kScShort; t0 += kScQ, buf ^= 1) {
    const int t1 = min(s.t1, t0 + kScQ);
    spoilt_take(r, spoilt[buf], t1 - t0);
    tile_store(r, Bt, xt, t1 - t0);
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        const float f[4] = {S[nb][pb].x, S[nb][pb].y, S[nb][pb].z, S[nb][pb].w};
        uint32_t a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          a[i] = bf_pack(f[2 * i], f[2 * i + 1]);
          b[i] = bf_pack(f[2 * i] - bf_lo(a[i]), f[2 * i + 1] - bf_hi(a[i]));
        }
        const int at = (16 * pb + col) * kScRowS + 2 * (32 * wave + 16 * nb + 4 * g);
        *(u32x2*)(Sl[0] + at) = u32x2{a[0], a[1]};
        *(u32x2*)(Sl[1] + at) = u32x2{b[0], b[1]};
      }
    bf16x8 C[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) C[k] = cn[k];
    __syncthreads();
    const Toks<kScQ>& tk = tks[buf];
    const float* coef = coefs[buf];
    const Spoilt& sp = spoilt[buf];
    const int any = sp.any;
    spoilt_clear(spoilt[buf ^ 1], threadIdx.x);
    if (t0 + kScQ < s.t1) {
      load(t0 + kScQ);
      if (wave == 0) {
        toks(t0 + kScQ, buf ^ 1);
        raw_load(t0 + 2 * kScQ);
      }
    }

    // e^{c_t} S C^T first: scaled, it is what the tile's own product adds to
    const int tt = 16 * wave + col;  // this lane's token in the tile
    f32x4 acc[4];
    {
      // operands a step (32 states) ahead of the products that take them: left
      // to itself the compiler waits for LDS before every other product
      bf16x8 sf[2][4][2];
      auto fetch = [&](int k) {
#pragma unroll
        for (int pb = 0; pb < 4; ++pb)
#pragma unroll
          for (int q = 0; q < 2; ++q) sf[k & 1][pb][q] = row_op(Sl[q], kScRowS, 16 * pb, 32 * k);
      };
      fetch(0);
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) acc[pb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k < 3) fetch(k + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 1; q >= 0; --q)
#pragma unroll
          for (int pb = 0; pb < 4; ++pb) acc[pb] = mfma16(sf[k & 1][pb][q], C[k], acc[pb]);
        __builtin_amdgcn_sched_barrier(0);
      }
      const float et = tk.ec[tt];
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) acc[pb] *= et;
    }
    // g of this wave's tokens with the s up to them, 32 at a time
    const float thi = tk.hi[tt], tlo = tk.lo[tt];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      if (2 * kb > wave) break;
      float gv[8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int sb = 2 * kb + half;
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
        if (sb <= wave)
#pragma unroll
          for (int k = 0; k < 4; ++k) a = mfma16(row_op(Bt, kScRowN, 16 * sb, 32 * k), C[k], a);
        const int s0 = 16 * sb + 4 * g;
        const f32x4 shi = *(const f32x4*)(tk.hi + s0), slo = *(const f32x4*)(tk.lo + s0),
                    sdt = *(const f32x4*)(tk.dt + s0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f((thi - shi[i]) + (tlo - slo[i]));
          gv[4 * half + i] = s0 + i <= tt ? a[i] * e * sdt[i] : 0.f;
        }
      }
      bf16x8 gt[2];
      split8<2>(gv, gt);
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        const bf16x8 xo = tr_op(xt, kScRowP, 32 * kb + 4 * g, 32 * kb + 16 + 4 * g, 16 * pb);
        acc[pb] = mfma16(xo, gt[1], acc[pb]);
        acc[pb] = mfma16(xo, gt[0], acc[pb]);
      }
    }
    const bool spoils = __builtin_amdgcn_readfirstlane(any) != 0;
    if (spoils)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (tt >= sp.first[16 * pb + 4 * g + i]) acc[pb][i] = __builtin_nanf("");
    if (t0 + tt < t1) {
      uint16_t* o = y + (int64_t)(t0 + tt) * d + h * kSqP + 4 * g;
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        const u32x2 xw = *(const u32x2*)(xt + tt * kScRowP + 2 * (16 * pb + 4 * g));
        const f32x4 a = acc[pb];
        *(u32x2*)(o + 16 * pb) =
            u32x2{bf_pack(__builtin_fmaf(skip, bf_lo(xw.x), a.x), __builtin_fmaf(skip, bf_hi(xw.x), a.y)),
                  bf_pack(__builtin_fmaf(skip, bf_lo(xw.y), a.z), __builtin_fmaf(skip, bf_hi(xw.y), a.w))};
      }
    }
    // the state at the tile's end
    const float last = tk.last;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) S[nb][pb] *= last;
    state_add<2>(S, Bt, xt, coef);
    if (spoils)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb)
        if (sp.first[16 * pb + col] < kScQ)
#pragma unroll
          for (int nb = 0; nb < 2; ++nb) S[nb][pb] = f32x4{1.f, 1.f, 1.f, 1.f} * __builtin_nanf("");
    __syncthreads();
  }
  if (t0 < s.t1) {
    // at most kScShort tokens are left: the recurrence itself, a token at a time
    tile_store(r, Bt, xt, s.t1 - t0);
    __syncthreads();
    const Toks<kScQ>& tk = tks[buf];
    float(*red)[4][kSqP] = (float(*)[4][kSqP])Sl;  // y of a token by waves
#pragma unroll
    for (int q = 0; q < kScShort; ++q) {
      if (t0 + q >= s.t1) break;
      const float dt = tk.dt[q];
      const float dec = q == 0 ? tk.ec[0]
                               : __builtin_amdgcn_exp2f((tk.hi[q] - tk.hi[q - 1]) +
                                                        (tk.lo[q] - tk.lo[q - 1]));
      u32x2 bw[2];
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
        bw[nb] = *(const u32x2*)(Bt + q * kScRowN + 2 * (32 * wave + 16 * nb + 4 * g));
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        const float dx =
            dt * __uint_as_float((uint32_t)*(const uint16_t*)(xt + q * kScRowP + 2 * (16 * pb + col)) << 16);
        float v = 0.f;
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
          const float bf[4] = {bf_lo(bw[nb].x), bf_hi(bw[nb].x), bf_lo(bw[nb].y), bf_hi(bw[nb].y)};
          const float cf[4] = {bf_lo(cv[q][nb].x), bf_hi(cv[q][nb].x), bf_lo(cv[q][nb].y),
                               bf_hi(cv[q][nb].y)};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float sn = __builtin_fmaf(S[nb][pb][i], dec, dx * bf[i]);
            S[nb][pb][i] = sn;
            v = __builtin_fmaf(sn, cf[i], v);
          }
        }
        v += __uint_as_float(lane_xchg<16>(__float_as_uint(v)));
        v += __uint_as_float(lane_xchg<32>(__float_as_uint(v)));
        if (g == 0) red[q][wave][16 * pb + col] = v;
      }
    }
    __syncthreads();
    const int q = wave, p = lane;  // a wave a token
    if (t0 + q < s.t1) {
      const float x = __uint_as_float((uint32_t)*(const uint16_t*)(xt + q * kScRowP + 2 * p) << 16);
      const float v = (red[q][0][p] + red[q][1][p]) + (red[q][2][p] + red[q][3][p]);
      y[(int64_t)(t0 + q) * d + h * kSqP + p] = bf_rne(__builtin_fmaf(skip, x, v));
    }
  }
  if (final_ && s.t1 == s.en) {
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int pb = 0; pb < 4; ++pb) {
        const f32x4 v = S[nb][pb];
        *(u32x2*)(final_ + sat + (16 * pb + col) * kSqN + 32 * wave + 16 * nb + 4 * g) =
            u32x2{(uint32_t)f2h(v.x) | ((uint32_t)f2h(v.y) << 16),
                  (uint32_t)f2h(v.z) | ((uint32_t)f2h(v.w) << 16)};
      }
  }
}

// Tokens of a segment: as many segments of all heads as the chip takes
// workgroups at once (512), whatever the sequences' lengths, which the host does
// not know.  Two sequences of 8192 tokens and 64 heads: 247 us, 437 in one
// segment each; one of 4096: 79 and 215; eight of 2048, where one segment each
// would do: 168 and 163.  Above 256 heads two segments of all of them do not fit
// (16384 tokens of 400 heads 1181 us, 1541 in 1.3; 1000 of 520 121, 160 in 960 + 40).
// Up to 512 tokens in one segment, whatever the heads: 300 tokens in three sequences
// 13 us, 16 in segments of 128, in one 21 and 19; 512 in one 30 and 22; 150 15 and 18.
static int64_t scan_seg(int64_t T, int64_t nheads) {
  if (T <= 512 || nheads > 256) return T;
  const int64_t seg = T * nheads / 512 / kScQ * kScQ;
  return seg < 128 ? 128 : seg;
}
// A workgroup adds the own states of this many segments before its own up by
// itself; with more, a launch makes the states between the segments.
constexpr int kScOwn = 16;

int64_t seq_scan_bytes(int64_t T, int64_t nheads) {
  const int64_t seg = scan_seg(T, nheads);
  if (seg >= T) return 0;
  // the states and decays in float32, the first segments' initial states in float16
  return state_count(T, seg) * nheads * (kScState * 6 + 4) + 16;
}

// Heads vary fastest: workgroups go to the eight XCDs in turn, and slots without
// tokens (every second one where sequences are one segment long) would leave
// XCDs idle.  y and z: the slots (65535 at most in one dimension).
static dim3 scan_grid(int64_t slots, int64_t nheads) {
  const int64_t y = slots < 32768 ? slots : 32768;
  return dim3((unsigned)nheads, (unsigned)y, (unsigned)((slots + y - 1) / y));
}

template <bool F32, bool REV, int NT>
static hipError_t scan_state_go(const SeqIn& in, const uint16_t* u, const uint16_t* dy, int segT,
                                const float* dt_bias, const float* A_log, float* state,
                                float* decay, hipStream_t stream) {
  hipLaunchKernelGGL((scan_state_kernel<F32, REV, NT>),
                     scan_grid(slot_count(in.T, in.nseq, segT), in.nheads), dim3(256), 0, stream,
                     (const typename Zx<F32>::T*)in.zx, u, dy, in.T, in.nheads, in.offsets,
                     in.nseq, segT, dt_bias, A_log, state, decay);
  return hipGetLastError();
}

template <bool REV>
static hipError_t scan_pass_go(const SeqIn& in, int segT, float* state, const float* decay,
                               const uint16_t* init, uint16_t* first, hipStream_t stream) {
  hipLaunchKernelGGL(scan_pass_kernel<REV>,
                     dim3(kScState / 1024, (unsigned)in.nheads, (unsigned)in.nseq), dim3(256), 0,
                     stream, state, decay, in.T, in.nheads, in.offsets, segT, init, first);
  return hipGetLastError();
}

// Every chunk by itself, then one launch that adds them up (102 + 77 us at 16384
// tokens of 64 heads, by the memory's rate; workgroups that walk through the
// sequences and write each state once took 190, too few loads in flight).
template <bool F32, bool REV>
static hipError_t chunk_states_go(const SeqIn& in, const uint16_t* u, const uint16_t* dy,
                                  const float* dt_bias, const float* A_log, float* state,
                                  float* decay, hipStream_t stream) {
  const hipError_t e =
      scan_state_go<F32, REV, 3>(in, u, dy, kScChunk, dt_bias, A_log, state, decay, stream);
  return e != hipSuccess ? e : scan_pass_go<REV>(in, kScChunk, state, decay, nullptr, nullptr, stream);
}

hipError_t launch_chunk_states(const SeqIn& in, const uint16_t* u, const uint16_t* dy, bool rev,
                               const float* dt_bias, const float* A_log, float* state,
                               float* decay, hipStream_t stream) {
  if (in.f32)
    return rev ? chunk_states_go<true, true>(in, u, dy, dt_bias, A_log, state, decay, stream)
               : chunk_states_go<true, false>(in, u, dy, dt_bias, A_log, state, decay, stream);
  return rev ? chunk_states_go<false, true>(in, u, dy, dt_bias, A_log, state, decay, stream)
             : chunk_states_go<false, false>(in, u, dy, dt_bias, A_log, state, decay, stream);
}

hipError_t launch_seq_scan(const SeqIn& in, const uint16_t* u, const float* dt_bias,
                           const float* A_log, const float* D, const uint16_t* ssm_in,
                           uint16_t* ssm_out, uint16_t* y, void* workspace, hipStream_t stream) {
  const int64_t seg = scan_seg(in.T, in.nheads);
  float *state = nullptr, *decay = nullptr;
  uint16_t* first = nullptr;
  const int64_t slots = slot_count(in.T, in.nseq, seg);
  if (seg < in.T) {
    // in place, a workgroup that has ended may have written what another would
    // still begin with: then the launch in between keeps the initial states
    const bool over = ssm_in && ssm_in == ssm_out, own = in.T / seg <= kScOwn && !over;
    const int64_t n = state_count(in.T, seg) * in.nheads;
    state = (float*)workspace;
    decay = state + n * kScState;
    hipError_t e = in.f32 ? scan_state_go<true, false, 2>(in, u, nullptr, (int)seg, dt_bias, A_log,
                                                          state, decay, stream)
                          : scan_state_go<false, false, 2>(in, u, nullptr, (int)seg, dt_bias, A_log,
                                                           state, decay, stream);
    if (e == hipSuccess && !own) {
      if (over) first = (uint16_t*)(decay + (n + 3) / 4 * 4);
      e = scan_pass_go<false>(in, (int)seg, state, decay, ssm_in, first, stream);
      decay = nullptr;
    }
    if (e != hipSuccess) return e;
  }
  const dim3 grid = scan_grid(slots, in.nheads);
  if (in.f32)
    hipLaunchKernelGGL(scan_y_kernel<true>, grid, dim3(256), 0, stream, (const float*)in.zx, u,
                       in.T, in.nheads, in.offsets, in.nseq, (int)seg, dt_bias, A_log, D, ssm_in,
                       first, state, decay, ssm_out, y);
  else
    hipLaunchKernelGGL(scan_y_kernel<false>, grid, dim3(256), 0, stream, (const uint16_t*)in.zx,
                       u, in.T, in.nheads, in.offsets, in.nseq, (int)seg, dt_bias, A_log, D,
                       ssm_in, first, state, decay, ssm_out, y);
  return hipGetLastError();
}

}  // namespace tmk
