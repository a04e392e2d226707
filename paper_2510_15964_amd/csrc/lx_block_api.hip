// Host side of the calls between and behind a layer's halves: dropout, the norm of a sum with its residual, the loss over a
// vocabulary.  Argument checks and dispatch, as in lx_api.hip.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/lx.h"
#include "lx_host.h"
#include "lx_launch.h"
#include "vocab.h"

namespace lx {

static inline lx_status done(hipError_t e) { return e == hipSuccess ? LX_OK : LX_ERR_RUNTIME; }

static lx_status rows_size(lx_dtype dt, int32_t T, int32_t d) {
  if (dt != LX_F32 && !is16(dt)) return LX_ERR_UNSUPPORTED;
  if (T <= 0 || d <= 0) return LX_ERR_INVALID_ARG;
  return LX_OK;
}
// A tensor [T, d]; one that is written must not meet itself.  `vec` stays true if its runs of eight lie at multiples of 16 bytes.
static bool rows_of(lx_dtype dt, const void* p, int64_t stride, int32_t T, int32_t d, bool written, long long& to, bool& vec) {
  const uintptr_t size = esize(dt);
  to = T > 1 ? stride : 0;       // (one row has any stride)
  if ((uintptr_t)p % size != 0 || to < 0 || (written && T > 1 && to < d)) return false;
  vec &= (uintptr_t)p % 16 == 0 && to * (long long)size % 16 == 0 && d % 8 == 0;
  return true;
}
static lx_status drop_of(float p, const int64_t* rng, int32_t site, DropArgs& drop) {
  if (!(p >= 0) || !(p < 1)) return LX_ERR_INVALID_ARG;
  const long below = std::lrint((double)p * 65536);
  if (below >= 65536 || (below > 0 && (!rng || (uintptr_t)rng % 8 != 0))) return LX_ERR_INVALID_ARG;
  drop = {(const long long*)rng, site, (unsigned)below, (float)(65536.0 / (double)(65536 - below))};
  return LX_OK;
}

static lx_status dropout_impl(lx_dtype dt, int32_t T, int32_t d, const void* X, const void* R, void* out, const int64_t* st, float p,
                              const int64_t* rng, int32_t site, void* stream) {
  lx_status s = rows_size(dt, T, d);
  if (s != LX_OK) return s;
  RowsArgs a = {};
  DropArgs drop = {};
  bool vec = true;
  if (!X || !out || !st || !rows_of(dt, X, st[0], T, d, false, a.is[0], vec) || (R && !rows_of(dt, R, st[1], T, d, false, a.is[1], vec)) ||
      !rows_of(dt, out, st[2], T, d, true, a.os[0], vec))
    return LX_ERR_INVALID_ARG;
  s = drop_of(p, rng, site, drop);
  if (s != LX_OK) return s;
  if (T == 1) a.is[0] = a.is[1] = a.os[0] = d;
  a.in[0] = X, a.in[1] = R, a.out[0] = out, a.T = T, a.d = d;
  return done(launch_dropout(dt, a, drop, vec, (hipStream_t)stream));
}

static lx_status norm_common(lx_dtype dt, int32_t T, int32_t d, float eps, const void* weight, bool& vec) {
  const lx_status s = rows_size(dt, T, d);
  if (s != LX_OK) return s;
  if (d > kNormWidest) return LX_ERR_UNSUPPORTED;
  if (!(eps >= 0) || !std::isfinite(eps) || (uintptr_t)weight % esize(dt) != 0) return LX_ERR_INVALID_ARG;
  vec = (uintptr_t)weight % 16 == 0;
  return LX_OK;
}

static lx_status norm_fwd_impl(lx_dtype dt, int32_t T, int32_t d, float eps, const void* weight, const void* X, const void* R, void* H, void* Y,
                               const int64_t* st, uint8_t* Y8, float* scales, int32_t group, float p, const int64_t* rng, int32_t site,
                               void* stream) {
  bool vec = true;
  lx_status s = norm_common(dt, T, d, eps, weight, vec);
  if (s != LX_OK) return s;
  RowsArgs a = {};
  DropArgs drop = {};
  if (!X || !st || (!Y && !Y8) || !Y8 != !scales || !rows_of(dt, X, st[0], T, d, false, a.is[0], vec) ||
      (R && !rows_of(dt, R, st[1], T, d, false, a.is[1], vec)) || (H && !rows_of(dt, H, st[2], T, d, true, a.os[0], vec)) ||
      (Y && !rows_of(dt, Y, st[3], T, d, true, a.os[1], vec)) || (uintptr_t)scales % 4 != 0)
    return LX_ERR_INVALID_ARG;
  if (Y8) {
    if (group <= 0 || d % group != 0) return LX_ERR_INVALID_ARG;
    if (group != d && group != 32 && group != 64 && group != 128 && group != 256 && group != 512) return LX_ERR_UNSUPPORTED;
    vec &= (uintptr_t)Y8 % 8 == 0;
  }
  s = drop_of(p, rng, site, drop);
  if (s != LX_OK) return s;
  a.in[0] = X, a.in[1] = R, a.out[0] = H, a.out[1] = Y, a.T = T, a.d = d;
  const NormArgs n = {weight, eps, Y8, scales, group, nullptr};
  return done(launch_norm_fwd(dt, a, drop, n, vec, (hipStream_t)stream));
}

static lx_status norm_bwd_impl(lx_dtype dt, int32_t T, int32_t d, float eps, const void* weight, const void* dY, const void* H, const void* dH,
                               void* dX, void* dR, const int64_t* st, float* dW, float p, const int64_t* rng, int32_t site, void* ws,
                               size_t ws_bytes, void* stream) {
  bool vec = true;
  lx_status s = norm_common(dt, T, d, eps, weight, vec);
  if (s != LX_OK) return s;
  RowsArgs a = {};
  DropArgs drop = {};
  if (!dY || !H || !st || (!dX && !dR && !dW) || !rows_of(dt, dY, st[0], T, d, false, a.is[0], vec) ||
      !rows_of(dt, H, st[1], T, d, false, a.is[1], vec) || (dH && !rows_of(dt, dH, st[2], T, d, false, a.is[2], vec)) ||
      (dX && !rows_of(dt, dX, st[3], T, d, true, a.os[0], vec)) || (dR && !rows_of(dt, dR, st[4], T, d, true, a.os[1], vec)) ||
      (uintptr_t)dW % 4 != 0)
    return LX_ERR_INVALID_ARG;
  s = drop_of(p, rng, site, drop);
  if (s != LX_OK) return s;
  if (dW) {
    if (!aligned16(ws)) return LX_ERR_INVALID_ARG;
    if (!ws || ws_bytes < lx_rms_norm_bwd_workspace_bytes(T, d)) return LX_ERR_WORKSPACE;
  }
  a.in[0] = dY, a.in[1] = H, a.in[2] = dH, a.out[0] = dX, a.out[1] = dR, a.T = T, a.d = d;
  const NormArgs n = {weight, eps, nullptr, nullptr, 0, dW ? (float*)ws : nullptr};
  return done(launch_norm_bwd(dt, a, drop, n, dW, vec, (hipStream_t)stream));
}

static lx_status vocab_size(lx_dtype dt, int32_t T, int32_t d, int32_t V) {
  if (!is16(dt) && dt != LX_F32) return LX_ERR_UNSUPPORTED;
  if (T <= 0 || d <= 0 || V <= 0) return LX_ERR_INVALID_ARG;
  if (d % 64 != 0 || d > 32768 || V > 1 << 20 || T > INT32_MAX - kVocabPieceMost) return LX_ERR_UNSUPPORTED;
  return LX_OK;
}
static lx_status vocab_loss_impl(lx_dtype dt, int32_t T, int32_t d, int32_t V, const void* X, int64_t xs, const void* W, const int32_t* targets,
                                 const float* weights, float* loss, float* lse, void* dX, int64_t dxs, void* dW, lx_dtype dw_dt, void* ws,
                                 size_t ws_bytes, void* stream) {
  const lx_status s = vocab_size(dt, T, d, V);
  if (s != LX_OK) return s;
  if (!X || !W || !targets || !loss || ((uintptr_t)X | (uintptr_t)dX) % esize(dt) != 0 || !aligned16(W) || !aligned16(dW) || !aligned16(ws) ||
      ((uintptr_t)targets | (uintptr_t)weights | (uintptr_t)loss | (uintptr_t)lse) % 4 != 0)
    return LX_ERR_INVALID_ARG;
  if (T > 1 && (xs < 0 || (dX && dxs < d))) return LX_ERR_INVALID_ARG;
  if (dW && dw_dt != dt && dw_dt != LX_F32) return LX_ERR_UNSUPPORTED;
  const bool grads = dX || dW, f32 = dw_dt == LX_F32;
  // the longest pieces that the workspace has room for
  int rows = vocab_rows(T, V, grads, dt == LX_F32);
  auto room_of = [&] { return dt == LX_F32 ? vocab_room_plain(rows, V) : vocab_room(rows, T, d, V, grads, dW != nullptr, f32); };
  VocabRoom room = room_of();
  while (room.bytes > ws_bytes && rows > kVocabTile) rows -= kVocabTile, room = room_of();
  if (!ws || room.bytes > ws_bytes) return LX_ERR_WORKSPACE;
  if (dt == LX_F32) {
    const PlainVocabArgs p = {T, d, V, (const float*)X, T > 1 ? xs : 0, (const float*)W, targets, weights, loss, lse, (float*)dX, T > 1 ? dxs : 0, (float*)dW};
    return done(launch_vocab_loss_plain(p, room, ws, (hipStream_t)stream));
  }
  VocabArgs a = {};
  a.T = T, a.d = d, a.V = V, a.dt = dt16(dt), a.X = (const uint16_t*)X, a.xs = T > 1 ? xs : 0, a.W = (const uint16_t*)W, a.targets = targets;
  a.weights = weights, a.loss = loss, a.lse = lse, a.dX = (uint16_t*)dX, a.dxs = T > 1 ? dxs : 0, a.dW = dW, a.dw_f32 = f32;
  return done(launch_vocab_loss(a, room, ws, (hipStream_t)stream));
}

}  // namespace lx

using namespace lx;

extern "C" {

lx_status lx_dropout(lx_dtype dt, int32_t T, int32_t d, const void* X, const void* residual, void* out, const int64_t strides[3], float p,
                     const int64_t* rng, int32_t site, void* stream) {
  const lx_status s = dropout_impl(dt, T, d, X, residual, out, strides, p, rng, site, stream);
  LX_LOGF("lx_dropout dt=%d T=%d d=%d p=%g site=%d -> %s", (int)dt, T, d, (double)p, site, lx_status_string(s));
  return s;
}

lx_status lx_rms_norm_fwd(lx_dtype dt, int32_t T, int32_t d, float eps, const void* weight, const void* X, const void* residual, void* H, void* Y,
                          const int64_t strides[4], uint8_t* Y8, float* scales, int32_t group, float p, const int64_t* rng, int32_t site,
                          void* stream) {
  const lx_status s = norm_fwd_impl(dt, T, d, eps, weight, X, residual, H, Y, strides, Y8, scales, group, p, rng, site, stream);
  LX_LOGF("lx_rms_norm_fwd dt=%d T=%d d=%d group=%d p=%g -> %s", (int)dt, T, d, Y8 ? group : 0, (double)p, lx_status_string(s));
  return s;
}

size_t lx_rms_norm_bwd_workspace_bytes(int32_t T, int32_t d) {
  return T <= 0 || d <= 0 || d > kNormWidest ? 0 : round256((size_t)norm_bwd_parts(T, d) * d * sizeof(float));
}
lx_status lx_rms_norm_bwd(lx_dtype dt, int32_t T, int32_t d, float eps, const void* weight, const void* dY, const void* H, const void* dH, void* dX,
                          void* dR, const int64_t strides[5], float* dW, float p, const int64_t* rng, int32_t site, void* workspace,
                          size_t workspace_bytes, void* stream) {
  const lx_status s = norm_bwd_impl(dt, T, d, eps, weight, dY, H, dH, dX, dR, strides, dW, p, rng, site, workspace, workspace_bytes, stream);
  LX_LOGF("lx_rms_norm_bwd dt=%d T=%d d=%d dW=%d p=%g -> %s", (int)dt, T, d, dW != nullptr, (double)p, lx_status_string(s));
  return s;
}

size_t lx_vocab_loss_workspace_bytes(lx_dtype dt, int32_t T, int32_t d, int32_t V, int32_t gradients, lx_dtype dW_dt, int32_t tokens) {
  if (vocab_size(dt, T, d, V) != LX_OK || tokens < 0) return 0;
  const bool grads = gradients != 0, dW = gradients & LX_GRAD_W;
  int rows = vocab_rows(T, V, grads, dt == LX_F32);
  if (tokens > 0 && tokens < rows) rows = (tokens + kVocabTile - 1) / kVocabTile * kVocabTile;
  return dt == LX_F32 ? vocab_room_plain(rows, V).bytes : vocab_room(rows, T, d, V, grads, dW, dW_dt == LX_F32).bytes;
}
lx_status lx_vocab_loss(lx_dtype dt, int32_t T, int32_t d, int32_t V, const void* X, int64_t x_stride, const void* W, const int32_t* targets,
                        const float* weights, float* loss, float* lse, void* dX, int64_t dx_stride, void* dW, lx_dtype dW_dt, void* workspace,
                        size_t workspace_bytes, void* stream) {
  const lx_status s = vocab_loss_impl(dt, T, d, V, X, x_stride, W, targets, weights, loss, lse, dX, dx_stride, dW, dW_dt, workspace, workspace_bytes,
                                      stream);
  LX_LOGF("lx_vocab_loss dt=%d T=%d d=%d V=%d dX=%d dW=%d ws=%zu -> %s", (int)dt, T, d, V, dX != nullptr, dW != nullptr, workspace_bytes,
          lx_status_string(s));
  return s;
}

}  // extern "C"
