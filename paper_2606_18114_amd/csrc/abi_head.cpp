// C ABI of tmamba_head.h: argument checks, then one launcher.
#include "../../include/tmamba_head.h"

#include <initializer_list>

#include "abi_checks.hpp"
#include "head.hpp"

using namespace tmk_abi;

namespace {

// a workgroup of 256 threads a token stays under a launch's 2^32 threads (the block norm's, of up to
// 512, are dealt over two dimensions)
constexpr int64_t kMaxTokens = int64_t(1) << 23;

// outs: no overlap with an input or with each other
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

tm_status ws_checked(const void* ws, int64_t have, int64_t need) {
  if (need > 0 && !ws) return TM_EINVAL;
  if (have < need) return TM_ESHAPE;
  if (!aligned(ws, 256)) return TM_EALIGN;
  return TM_OK;
}

bool head_sizes(int64_t T, int64_t V, int64_t D) {
  return T >= 1 && T <= kMaxTokens && V >= 1 && V <= kMaxTokens && D >= 8 && D <= 65536 &&
         D % 8 == 0;
}

bool norm_sizes(int64_t T, int64_t D) {
  return T >= 1 && T <= kMaxTokens && D >= 1 && D <= (int64_t(1) << 20);
}

// what the two calls of the loss share; with a teacher alpha and tau count
tm_status head_checked(const void* h, const void* W, int32_t type, int64_t T, int64_t V, int64_t D,
                       const void* labels, int32_t labels_i64, const void* top_ids,
                       int32_t ids_i64, int32_t K, float alpha, float tau, tmk::HeadIn* in) {
  if (!h || !W || !labels || (type != 1 && type != 2) || (labels_i64 & ~1) || (ids_i64 & ~1))
    return TM_EINVAL;
  if (K < 0 || K > 1024 || !head_sizes(T, V, D) || T * (K + 1) >= (int64_t(1) << 31))
    return TM_ESHAPE;
  if ((K > 0) != (top_ids != nullptr)) return TM_EINVAL;
  if (K > 0 && (!(alpha >= 0.0f && alpha <= 1.0f) || !(tau >= 0x1p-10f && tau <= 0x1p10f)))
    return TM_EINVAL;
  if (!aligned(h, 16) || !aligned(W, 16) || !aligned(labels, labels_i64 ? 8 : 4) ||
      !aligned(top_ids, ids_i64 ? 8 : 4))
    return TM_EALIGN;
  *in = tmk::HeadIn{static_cast<const uint16_t*>(h), static_cast<const uint16_t*>(W), type == 2,
                    T, V, (int)D, labels, top_ids, labels_i64 != 0, ids_i64 != 0, K,
                    K > 0 ? alpha : 0.0f, K > 0 ? tau : 1.0f};
  return TM_OK;
}

}  // namespace

extern "C" {

int64_t tm_head_loss_workspace(int64_t T, int64_t V, int64_t D) {
  return head_sizes(T, V, D) ? tmk::head_loss_bytes(T, V, D) : -1;
}

tm_status tm_head_loss(const void* h, const void* W, int32_t type, int64_t T, int64_t V, int64_t D,
                       const void* labels, int32_t labels_i64, const void* top_ids,
                       int32_t ids_i64, const void* top, int32_t top_type, int32_t K, float alpha,
                       float tau, float* loss, float* stats, void* workspace,
                       int64_t workspace_bytes, tm_stream stream) {
  tmk::HeadIn in;
  if (!loss || !stats || top_type < 0 || top_type > 2) return TM_EINVAL;
  if (tm_status st = head_checked(h, W, type, T, V, D, labels, labels_i64, top_ids, ids_i64, K,
                                  alpha, tau, &in))
    return st;
  if ((K > 0) != (top != nullptr)) return TM_EINVAL;
  const int64_t need = tmk::head_loss_bytes(T, V, D), te = top_type == 0 ? 4 : 2;
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!aligned(top, (uintptr_t)te) || !aligned(loss, 4) || !aligned(stats, 4)) return TM_EALIGN;
  if (!apart({span(h, T * D * 2), span(W, V * D * 2), span(labels, T * (labels_i64 ? 8 : 4)),
              opt(top_ids, T * K * (ids_i64 ? 8 : 4)), opt(top, T * K * te)},
             {span(loss, T * 4), span(stats, tmk::head_stats_floats(T, K) * 4),
              span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_head_loss(in, top, top_type, loss, stats, workspace,
                                          to_hip(stream)));
}

int64_t tm_head_loss_bwd_workspace(int64_t T, int64_t V, int64_t D) {
  return head_sizes(T, V, D) ? tmk::head_loss_bwd_bytes(T, V, D) : -1;
}

tm_status tm_head_loss_bwd(const void* h, const void* W, int32_t type, int64_t T, int64_t V,
                           int64_t D, const void* labels, int32_t labels_i64, const void* top_ids,
                           int32_t ids_i64, int32_t K, float alpha, float tau, const float* stats,
                           const float* dloss, void* dh, void* dW, int32_t dW_type,
                           int32_t accumulate, void* workspace, int64_t workspace_bytes,
                           tm_stream stream) {
  tmk::HeadIn in;
  if (!stats || !dloss || (!dh && !dW) || (accumulate & ~1)) return TM_EINVAL;
  if (tm_status st = head_checked(h, W, type, T, V, D, labels, labels_i64, top_ids, ids_i64, K,
                                  alpha, tau, &in))
    return st;
  if ((dW_type != 0 && dW_type != type) || (accumulate && dW_type != 0)) return TM_EINVAL;
  const int64_t need = tmk::head_loss_bwd_bytes(T, V, D);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!aligned(stats, 4) || !aligned(dloss, 4) || !aligned(dh, 16) || !aligned(dW, 16))
    return TM_EALIGN;
  if (!apart({span(h, T * D * 2), span(W, V * D * 2), span(labels, T * (labels_i64 ? 8 : 4)),
              opt(top_ids, T * K * (ids_i64 ? 8 : 4)),
              span(stats, tmk::head_stats_floats(T, K) * 4), span(dloss, T * 4)},
             {opt(dh, T * D * 2), opt(dW, V * D * (dW_type == 0 ? 4 : 2)),
              span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_head_loss_bwd(in, stats, dloss, static_cast<uint16_t*>(dh), dW,
                                              dW_type == 0 ? 0 : 1, accumulate != 0, workspace,
                                              to_hip(stream)));
}

tm_status tm_block_norm(const float* residual, const float* y, int64_t T, int64_t D, const float* w,
                        float eps, float* residual_out, uint16_t* x, tm_stream stream) {
  if (!residual || !w || !x || (y && !residual_out)) return TM_EINVAL;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return TM_EINVAL;
  if (!norm_sizes(T, D)) return TM_ESHAPE;
  if (!aligned(residual, 4) || !aligned(y, 4) || !aligned(w, 4) || !aligned(residual_out, 4) ||
      !aligned(x, 2))
    return TM_EALIGN;
  const int64_t b = T * D * 4;
  const Span r = span(residual, b), out = opt(residual_out, b);
  if (residual_out != residual && overlap(out, r)) return TM_EINVAL;
  if (!apart({r}, {span(x, b / 2)}) || !apart({opt(y, b), span(w, D * 4)}, {out, span(x, b / 2)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_block_norm(residual, y, T, (int)D, w, eps, residual_out, x,
                                           to_hip(stream)));
}

int64_t tm_block_norm_bwd_workspace(int64_t T, int64_t D) {
  return norm_sizes(T, D) ? tmk::block_norm_bwd_bytes(T, D) : -1;
}

tm_status tm_block_norm_bwd(const float* r, int64_t T, int64_t D, const float* w, float eps,
                            const uint16_t* dx, const float* dresidual, float* dr, float* dw,
                            void* workspace, int64_t workspace_bytes, tm_stream stream) {
  if (!r || !w || !dx || !dr || !dw) return TM_EINVAL;
  if (!(eps >= 0.0f) || !std::isfinite(eps)) return TM_EINVAL;
  if (!norm_sizes(T, D)) return TM_ESHAPE;
  const int64_t need = tmk::block_norm_bwd_bytes(T, D);
  if (tm_status st = ws_checked(workspace, workspace_bytes, need)) return st;
  if (!aligned(r, 4) || !aligned(w, 4) || !aligned(dx, 2) || !aligned(dresidual, 4) ||
      !aligned(dr, 4) || !aligned(dw, 4))
    return TM_EALIGN;
  const int64_t b = T * D * 4;
  const Span g = opt(dresidual, b);
  if (dr != dresidual && overlap(span(dr, b), g)) return TM_EINVAL;
  if (!apart({span(r, b), span(w, D * 4), span(dx, b / 2)},
             {span(dr, b), span(dw, D * 4), span(workspace, need)}) ||
      !apart({g}, {span(dw, D * 4), span(workspace, need)}))
    return TM_EINVAL;
  return hip_status(tmk::launch_block_norm_bwd(r, T, (int)D, w, eps, dx, dresidual, dr, dw,
                                               workspace, to_hip(stream)));
}

}  // extern "C"
