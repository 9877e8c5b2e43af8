// C ABI of tmamba_seq.h: argument checks, then one launcher.
#include "../../include/tmamba_seq.h"

#include <initializer_list>

#include "abi_checks.hpp"
#include "seq_launch.hpp"

using namespace tmk_abi;

namespace {

// tokens and rows of an embedding: a workgroup of 256 threads each stays within
// a launch's 2^32 threads
constexpr int64_t kMaxTokens = int64_t(1) << 23;

struct Sizes {
  int64_t T, H, d, cd, Z, es;  // es: bytes of an element of zxbcdt
};

bool seq_sizes(int64_t T, int64_t nseq, int64_t H, int32_t z_f32, Sizes* s) {
  if (T < 1 || T > kMaxTokens || nseq < 1 || nseq > 65535 || H < 1 || H > 4096) return false;
  *s = Sizes{T, H, 64 * H, 64 * H + 256, 128 * H + 256 + H, z_f32 ? 4 : 2};
  int64_t b;  // the largest arrays: float32 zxbcdt, float16 states
  return bytes_of(T, s->Z, 4, &b) && bytes_of(nseq, H, 64 * 128 * 2, &b);
}

// outs: no overlap with an input or with each other; [0] .. are (pointer, bytes)
bool apart(std::initializer_list<Span> ins, std::initializer_list<Span> outs) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Span& i : ins)
      if (overlap(*o, i)) return false;
    for (auto p = o + 1; p != outs.end(); ++p)
      if (overlap(*o, *p)) return false;
  }
  return true;
}

Span opt(const void* p, int64_t bytes) { return span(p, p ? bytes : 0); }

bool all_aligned(std::initializer_list<const void*> ps, uintptr_t a) {
  for (const void* p : ps)
    if (!aligned(p, a)) return false;
  return true;
}

tm_status ws_checked(const void* ws, int64_t have, int64_t need) {
  if (need > 0 && !ws) return TM_EINVAL;
  if (have < need) return TM_ESHAPE;
  if (!aligned(ws, 256)) return TM_EALIGN;
  return TM_OK;
}

// zxbcdt's flag and pointer, the offsets
tm_status in_checked(const void* zx, int32_t z_f32, int64_t T, int32_t nseq, int32_t nheads,
                     const int32_t* offsets, Sizes* s) {
  if (!zx || (z_f32 & ~1)) return TM_EINVAL;
  if (!seq_sizes(T, nseq, nheads, z_f32, s)) return TM_ESHAPE;
  if (!offsets && nseq != 1) return TM_EINVAL;
  if (!aligned(zx, (uintptr_t)s->es) || !aligned(offsets, 4)) return TM_EALIGN;
  return TM_OK;
}

tmk::SeqIn seq_in(const void* zx, int32_t z_f32, int64_t T, int32_t nseq, int32_t nheads,
                  const int32_t* offsets) {
  return tmk::SeqIn{zx, z_f32 != 0, (int)T, nseq, nheads, offsets};
}

bool embed_sizes(int64_t T, int64_t V, int64_t D) {
  int64_t b;
  return T >= 1 && T <= kMaxTokens && V >= 1 && V <= kMaxTokens && D >= 1 &&
         D <= (int64_t(1) << 30) &&
         bytes_of(T, D, 4, &b) && bytes_of(V, D, 4, &b);
}

}  // namespace

extern "C" {

tm_status tm_mixer_conv(const void* zxbcdt, int32_t z_f32, int64_t T, int32_t nseq, int32_t nheads,
                        const int32_t* offsets, const float* conv_w, const float* conv_b,
                        const uint16_t* ring_in, const int32_t* ring_pos, uint16_t* ring_out,
                        uint16_t* u, tm_stream stream) {
  Sizes s;
  if (!conv_w || !conv_b || !u) return TM_EINVAL;
  if (tm_status st = in_checked(zxbcdt, z_f32, T, nseq, nheads, offsets, &s)) return st;
  if ((ring_in || ring_out) && !ring_pos) return TM_EINVAL;
  if (!all_aligned({conv_w, conv_b, ring_pos}, 4) || !all_aligned({ring_in, ring_out}, 8) ||
      !aligned(u, 16))
    return TM_EALIGN;
  const int64_t rb = nseq * s.cd * 8;
  const Span ri = opt(ring_in, rb), zx = span(zxbcdt, T * s.Z * s.es),
             of = opt(offsets, (nseq + 1) * 4), w = span(conv_w, s.cd * 16),
             b = span(conv_b, s.cd * 4), p = opt(ring_pos, 4);
  if (!apart({ri, zx, of, w, b, p}, {span(u, T * s.cd * 2)}) ||
      !apart({zx, of, w, b, p, span(u, T * s.cd * 2)}, {opt(ring_out, rb)}) ||
      (ring_out != ring_in && overlap(opt(ring_out, rb), ri)))
    return TM_EINVAL;
  return hip_status(tmk::launch_seq_conv(seq_in(zxbcdt, z_f32, T, nseq, nheads, offsets), conv_w,
                                         conv_b, ring_in, ring_pos, ring_out, u, to_hip(stream)));
}

int64_t tm_mixer_conv_bwd_workspace(int64_t T, int32_t nheads) {
  Sizes s;
  return seq_sizes(T, 1, nheads, 1, &s) ? tmk::seq_conv_bwd_bytes(T, nheads) : -1;
}

tm_status tm_mixer_conv_bwd(const void* zxbcdt, int32_t z_f32, int64_t T, int32_t nseq,
                            int32_t nheads, const int32_t* offsets, const float* conv_w,
                            const float* conv_b, const uint16_t* du, void* dzxbcdt, float* dconv_w,
                            float* dconv_b, void* workspace, int64_t workspace_bytes,
                            tm_stream stream) {
  Sizes s;
  if (!conv_w || !conv_b || !du || !dzxbcdt || !dconv_w || !dconv_b) return TM_EINVAL;
  if (tm_status st = in_checked(zxbcdt, z_f32, T, nseq, nheads, offsets, &s)) return st;
  const int64_t need = tmk::seq_conv_bwd_bytes(T, nheads);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!all_aligned({conv_w, conv_b, dconv_w, dconv_b}, 4) || !aligned(du, 16) ||
      !aligned(dzxbcdt, (uintptr_t)s.es))
    return TM_EALIGN;
  const int64_t zb = T * s.Z * s.es;
  if (!apart({span(zxbcdt, zb), opt(offsets, (nseq + 1) * 4), span(conv_w, s.cd * 16),
              span(conv_b, s.cd * 4), span(du, T * s.cd * 2)},
             {span(dzxbcdt, zb), span(dconv_w, s.cd * 16), span(dconv_b, s.cd * 4),
              span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_seq_conv_bwd(seq_in(zxbcdt, z_f32, T, nseq, nheads, offsets),
                                             conv_w, conv_b, du, dzxbcdt, dconv_w, dconv_b,
                                             workspace, to_hip(stream)));
}

int64_t tm_mixer_scan_workspace(int64_t T, int32_t nseq, int32_t nheads) {
  Sizes s;
  return seq_sizes(T, nseq, nheads, 1, &s) ? tmk::seq_scan_bytes(T, nheads) : -1;
}

tm_status tm_mixer_scan(const uint16_t* u, const void* zxbcdt, int32_t z_f32, int64_t T,
                        int32_t nseq, int32_t nheads, const int32_t* offsets, const float* dt_bias,
                        const float* A_log, const float* D, const uint16_t* ssm_in,
                        uint16_t* ssm_out, uint16_t* y, void* workspace, int64_t workspace_bytes,
                        tm_stream stream) {
  Sizes s;
  if (!u || !dt_bias || !A_log || !D || !y) return TM_EINVAL;
  if (tm_status st = in_checked(zxbcdt, z_f32, T, nseq, nheads, offsets, &s)) return st;
  const int64_t need = tmk::seq_scan_bytes(T, nheads);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!all_aligned({dt_bias, A_log, D}, 4) || !all_aligned({u, y, ssm_in, ssm_out}, 16))
    return TM_EALIGN;
  const int64_t sb = (int64_t)nseq * s.H * 64 * 128 * 2;
  const Span ui = span(u, T * s.cd * 2), zx = span(zxbcdt, T * s.Z * s.es),
             of = opt(offsets, (nseq + 1) * 4), a = span(dt_bias, s.H * 4),
             b = span(A_log, s.H * 4), c = span(D, s.H * 4), si = opt(ssm_in, sb),
             so = opt(ssm_out, sb), yo = span(y, T * s.d * 2), w = opt(workspace, need);
  if (!apart({ui, zx, of, a, b, c, si}, {yo, w}) || !apart({ui, zx, of, a, b, c, yo, w}, {so}) ||
      (ssm_out != ssm_in && overlap(so, si)))
    return TM_EINVAL;
  return hip_status(tmk::launch_seq_scan(seq_in(zxbcdt, z_f32, T, nseq, nheads, offsets), u,
                                         dt_bias, A_log, D, ssm_in, ssm_out, y, workspace,
                                         to_hip(stream)));
}

int64_t tm_mixer_scan_bwd_workspace(int64_t T, int32_t nseq, int32_t nheads) {
  Sizes s;
  return seq_sizes(T, nseq, nheads, 1, &s) ? tmk::seq_scan_bwd_bytes(T, nseq, nheads) : -1;
}

tm_status tm_mixer_scan_bwd(const uint16_t* u, const void* zxbcdt, int32_t z_f32, int64_t T,
                            int32_t nseq, int32_t nheads, const int32_t* offsets,
                            const float* dt_bias, const float* A_log, const float* D,
                            const uint16_t* dy, void* dzxbcdt, uint16_t* du, float* ddt_bias,
                            float* dA_log, float* dD, void* workspace, int64_t workspace_bytes,
                            tm_stream stream) {
  Sizes s;
  if (!u || !dt_bias || !A_log || !D || !dy || !dzxbcdt || !du || !ddt_bias || !dA_log || !dD)
    return TM_EINVAL;
  if (tm_status st = in_checked(zxbcdt, z_f32, T, nseq, nheads, offsets, &s)) return st;
  const int64_t need = tmk::seq_scan_bwd_bytes(T, nseq, nheads);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!all_aligned({dt_bias, A_log, D, ddt_bias, dA_log, dD}, 4) ||
      !all_aligned({u, dy, du}, 16) || !aligned(dzxbcdt, (uintptr_t)s.es))
    return TM_EALIGN;
  const int64_t zb = T * s.Z * s.es, ub = T * s.cd * 2, hb = s.H * 4;
  if (!apart({span(u, ub), span(zxbcdt, zb), opt(offsets, (nseq + 1) * 4), span(dt_bias, hb),
              span(A_log, hb), span(D, hb), span(dy, T * s.d * 2)},
             {span(dzxbcdt, zb), span(du, ub), span(ddt_bias, hb), span(dA_log, hb), span(dD, hb),
              span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_seq_scan_bwd(seq_in(zxbcdt, z_f32, T, nseq, nheads, offsets), u,
                                             dt_bias, A_log, D, dy, dzxbcdt, du, ddt_bias, dA_log,
                                             dD, workspace, to_hip(stream)));
}

tm_status tm_mixer_norm(const uint16_t* y, const void* zxbcdt, int32_t z_f32, int64_t T,
                        int32_t nseq, int32_t nheads, const int32_t* offsets, const float* norm_w,
                        float eps, uint16_t* out, tm_stream stream) {
  Sizes s;
  if (!y || !norm_w || !out) return TM_EINVAL;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return TM_EINVAL;
  if (tm_status st = in_checked(zxbcdt, z_f32, T, nseq, nheads, offsets, &s)) return st;
  if (!aligned(norm_w, 4) || !all_aligned({y, out}, 16)) return TM_EALIGN;
  if (!apart({span(y, T * s.d * 2), span(zxbcdt, T * s.Z * s.es), span(norm_w, s.d * 4),
              opt(offsets, (nseq + 1) * 4)},
             {span(out, T * s.d * 2)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_seq_norm(seq_in(zxbcdt, z_f32, T, nseq, nheads, offsets), y, norm_w,
                                         eps, out, to_hip(stream)));
}

int64_t tm_mixer_norm_bwd_workspace(int64_t T, int32_t nheads) {
  Sizes s;
  return seq_sizes(T, 1, nheads, 1, &s) ? tmk::seq_norm_bwd_bytes(T, nheads) : -1;
}

tm_status tm_mixer_norm_bwd(const uint16_t* y, const void* zxbcdt, int32_t z_f32, int64_t T,
                            int32_t nseq, int32_t nheads, const int32_t* offsets,
                            const float* norm_w, float eps, const uint16_t* dout, void* dzxbcdt,
                            uint16_t* dy, float* dnorm_w, void* workspace,
                            int64_t workspace_bytes, tm_stream stream) {
  Sizes s;
  if (!y || !norm_w || !dout || !dzxbcdt || !dy || !dnorm_w) return TM_EINVAL;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return TM_EINVAL;
  if (tm_status st = in_checked(zxbcdt, z_f32, T, nseq, nheads, offsets, &s)) return st;
  const int64_t need = tmk::seq_norm_bwd_bytes(T, nheads);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!all_aligned({norm_w, dnorm_w}, 4) || !all_aligned({y, dout, dy}, 16) ||
      !aligned(dzxbcdt, (uintptr_t)s.es))
    return TM_EALIGN;
  const int64_t zb = T * s.Z * s.es, yb = T * s.d * 2;
  if (!apart({span(y, yb), span(zxbcdt, zb), span(norm_w, s.d * 4), span(dout, yb),
              opt(offsets, (nseq + 1) * 4)},
             {span(dzxbcdt, zb), span(dy, yb), span(dnorm_w, s.d * 4), span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_seq_norm_bwd(seq_in(zxbcdt, z_f32, T, nseq, nheads, offsets), y,
                                             norm_w, eps, dout, dzxbcdt, dy, dnorm_w, workspace,
                                             to_hip(stream)));
}

tm_status tm_embed(const void* ids, int32_t ids_i64, int64_t T, const void* weight, int32_t w_type,
                   int64_t V, int64_t D, float scale, float* out, tm_stream stream) {
  if (!ids || !weight || !out || (ids_i64 & ~1) || w_type < 0 || w_type > 2) return TM_EINVAL;
  if (!std::isfinite(scale)) return TM_EINVAL;
  if (!embed_sizes(T, V, D)) return TM_ESHAPE;
  const int64_t ib = ids_i64 ? 8 : 4, wb = w_type == 0 ? 4 : 2;
  if (!aligned(ids, (uintptr_t)ib) || !aligned(weight, (uintptr_t)wb) || !aligned(out, 4))
    return TM_EALIGN;
  if (!apart({span(ids, T * ib), span(weight, V * D * wb)}, {span(out, T * D * 4)}))
    return TM_EINVAL;
  return hip_status(
      tmk::launch_embed(ids, ids_i64 != 0, T, weight, w_type, V, D, scale, out, to_hip(stream)));
}

int64_t tm_embed_bwd_workspace(int64_t T, int64_t V, int64_t D) {
  return embed_sizes(T, V, D) ? tmk::embed_bwd_bytes(T, V, D) : -1;
}

tm_status tm_embed_bwd(const void* ids, int32_t ids_i64, int64_t T, const float* dout, int64_t V,
                       int64_t D, float scale, float* dW, int32_t accumulate, void* workspace,
                       int64_t workspace_bytes, tm_stream stream) {
  if (!ids || !dout || !dW || (ids_i64 & ~1) || (accumulate & ~1)) return TM_EINVAL;
  if (!std::isfinite(scale)) return TM_EINVAL;
  if (!embed_sizes(T, V, D)) return TM_ESHAPE;
  const int64_t need = tmk::embed_bwd_bytes(T, V, D);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  const int64_t ib = ids_i64 ? 8 : 4;
  if (!aligned(ids, (uintptr_t)ib) || !aligned(dout, 4) || !aligned(dW, 4)) return TM_EALIGN;
  if (!apart({span(ids, T * ib), span(dout, T * D * 4)},
             {span(dW, V * D * 4), span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_embed_bwd(ids, ids_i64 != 0, T, dout, V, D, scale, dW,
                                          accumulate != 0, workspace, to_hip(stream)));
}

}  // extern "C"
