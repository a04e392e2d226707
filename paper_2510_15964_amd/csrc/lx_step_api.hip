// Host side of the calls around attention and the gradients: rotary positions, key ranges of packed documents, attention with
// rules on its scores, clipping by the global norm.  Argument checks and dispatch, as in lx_api.hip.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "../../include/lx.h"
#include "lx_host.h"
#include "lx_launch.h"

namespace lx {

static inline lx_status done(hipError_t e) { return e == hipSuccess ? LX_OK : LX_ERR_RUNTIME; }

static lx_status rope_table_impl(int32_t rot, int32_t n_pos, double base, const lx_rope_scaling* s, float* table, void* stream) {
  if (!table || rot <= 0 || rot % 2 != 0 || n_pos <= 0 || !(base > 0) || !std::isfinite(base)) return LX_ERR_INVALID_ARG;
  lx_rope_scaling p = {LX_ROPE_PLAIN, 1.f, 0.f, 0.f, 0.f, 1.f};
  if (s) p = *s;
  if (p.kind < LX_ROPE_PLAIN || p.kind > LX_ROPE_PARTS) return LX_ERR_UNSUPPORTED;
  if (!std::isfinite(p.gain)) return LX_ERR_INVALID_ARG;
  if (p.kind != LX_ROPE_PLAIN && (!(p.factor > 0) || !std::isfinite(p.factor))) return LX_ERR_INVALID_ARG;
  if (p.kind == LX_ROPE_BASE && rot == 2) return LX_ERR_INVALID_ARG;
  if (p.kind == LX_ROPE_PARTS && (!(p.trained_length > 0) || !std::isfinite(p.trained_length) || !std::isfinite(p.low_turns) ||
                                  !std::isfinite(p.high_turns) || !(p.high_turns > p.low_turns)))
    return LX_ERR_INVALID_ARG;
  if ((int64_t)n_pos * (rot / 2) > INT32_MAX) return LX_ERR_UNSUPPORTED;      // (threads of a launch: a 32-bit number)
  return done(launch_rope_table(rot, n_pos, base, p.kind, p.factor, p.trained_length, p.low_turns, p.high_turns, p.gain, table,
                                (hipStream_t)stream));
}

static lx_status rope_impl(lx_dtype dt, int32_t B, int32_t S, int32_t D, int32_t rot, int32_t layout, int32_t inverse, const float* table,
                           int32_t n_pos, const int32_t* positions, const lx_rope_tensor* tensors, int32_t n, void* stream) {
  if (dt != LX_F32 && !is16(dt)) return LX_ERR_UNSUPPORTED;
  if (layout != LX_ROPE_HALF && layout != LX_ROPE_INTERLEAVED) return LX_ERR_UNSUPPORTED;
  if (B <= 0 || S <= 0 || D <= 0 || rot <= 0 || rot % 2 != 0 || rot > D || n_pos <= 0 || !table || !tensors || n < 1 || n > 2)
    return LX_ERR_INVALID_ARG;
  if ((int64_t)B * S > INT32_MAX || (int64_t)B * S > (int64_t)UINT32_MAX / D - 256) return LX_ERR_UNSUPPORTED;      // (threads of a launch)
  if (!positions && S > n_pos) return LX_ERR_INVALID_ARG;
  if ((uintptr_t)table % 4 != 0 || (uintptr_t)positions % 4 != 0) return LX_ERR_INVALID_ARG;
  RopeArgs a = {};
  a.n = n, a.B = B, a.S = S, a.D = D, a.rot = rot, a.inverse = inverse != 0, a.n_pos = n_pos, a.table = table, a.positions = positions;
  int64_t heads = 0;
  for (int i = 0; i < n; ++i) {
    const lx_rope_tensor& t = tensors[i];
    const int64_t sizes[3] = {B, t.heads, S};
    if (!t.in || !t.out || t.heads <= 0) return LX_ERR_INVALID_ARG;
    if ((uintptr_t)t.in % esize(dt) != 0 || (uintptr_t)t.out % esize(dt) != 0) return LX_ERR_INVALID_ARG;
    for (int k = 0; k < 3; ++k) {
      if (t.in_strides[k] < 0 || t.out_strides[k] < 0 || (sizes[k] > 1 && t.out_strides[k] < D)) return LX_ERR_INVALID_ARG;
      if (t.in == t.out && sizes[k] > 1 && t.in_strides[k] != t.out_strides[k]) return LX_ERR_INVALID_ARG;
      a.t[i].is[k] = sizes[k] > 1 ? t.in_strides[k] : 0;      // (a dimension of one has any stride)
      a.t[i].os[k] = sizes[k] > 1 ? t.out_strides[k] : 0;
    }
    a.t[i].in = t.in, a.t[i].out = t.out, a.t[i].heads = t.heads;
    heads += t.heads;
  }
  if (heads > 65535) return LX_ERR_UNSUPPORTED;
  return done(launch_rope(dt, layout, a, (hipStream_t)stream));
}

static lx_status key_ranges_impl(int32_t B, int32_t S, const int32_t* begin, const int32_t* end, const int32_t* prefix, int32_t n,
                                 int32_t causal, int32_t* lo, int32_t* hi, void* stream) {
  if (B <= 0 || S <= 0 || n < 0 || !lo || !hi || (n > 0 && (!begin || !end))) return LX_ERR_INVALID_ARG;
  if (((uintptr_t)begin | (uintptr_t)end | (uintptr_t)prefix | (uintptr_t)lo | (uintptr_t)hi) % 4 != 0) return LX_ERR_INVALID_ARG;
  if ((int64_t)B * S > INT32_MAX - 1) return LX_ERR_UNSUPPORTED;
  return done(launch_key_ranges(B, S, begin, end, prefix, n, causal != 0, lo, hi, (hipStream_t)stream));
}

// A tensor of the two attention calls; one that is written must not meet itself.
static bool score_tensor(ScoreTensor& t, const void* p, const int64_t* st, const int64_t (&sizes)[3], int32_t D, bool written) {
  if (!p || !st || !aligned16(p)) return false;
  long long s[3];
  for (int k = 0; k < 3; ++k) {
    s[k] = sizes[k] > 1 ? st[k] : 0;       // (a dimension of one has any stride)
    if (s[k] < 0 || s[k] % 8 != 0 || (written && sizes[k] > 1 && s[k] < D)) return false;
  }
  t.p = p, t.sb = s[0], t.sh = s[1], t.ss = s[2];
  return true;
}
static lx_status score_sizes(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D) {
  if (dt != LX_F32 && !is16(dt)) return LX_ERR_UNSUPPORTED;
  if (B <= 0 || Hq <= 0 || Hkv <= 0 || Sq <= 0 || Sk <= 0 || D <= 0 || Hq % Hkv != 0) return LX_ERR_INVALID_ARG;
  if ((D != 64 && D != 128) || B > 65535 || Hq > 65535) return LX_ERR_UNSUPPORTED;
  // Rows of statistics are counted in 32 bits, and the threads of a launch: 256 for 128 rows, or 64 for one in 32-bit precision.
  if (((int64_t)Sq + 64) * Hq * B > INT32_MAX || Sk > INT32_MAX - 256) return LX_ERR_UNSUPPORTED;
  constexpr int64_t kWorkgroups = ((int64_t)1 << 24) - 64;
  if (((int64_t)Sq + 127) / 128 * Hq * B > kWorkgroups || ((int64_t)Sk + 127) / 128 * Hkv * B > kWorkgroups) return LX_ERR_UNSUPPORTED;
  if (dt == LX_F32 && (Sq > 1 << 25 || Sk > 1 << 25)) return LX_ERR_UNSUPPORTED;
  return LX_OK;
}
static lx_status score_rules(const lx_score_rules* r, ScoreArgs& a) {
  if (!r || !std::isfinite(r->scale) || !(r->cap >= 0) || !std::isfinite(r->cap) || !r->key_lo != !r->key_hi) return LX_ERR_INVALID_ARG;
  if (((uintptr_t)r->slopes | (uintptr_t)r->q_start | (uintptr_t)r->key_lo | (uintptr_t)r->key_hi) % 4 != 0) return LX_ERR_INVALID_ARG;
  a.scale = r->scale, a.cap = r->cap, a.causal = r->causal != 0;
  a.slopes = r->slopes, a.q_start = r->q_start, a.key_lo = r->key_lo, a.key_hi = r->key_hi;
  return LX_OK;
}

static lx_status score_fwd_impl(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D, const lx_score_rules* rules,
                                const void* Q, const int64_t* qs, const void* K, const int64_t* ks, const void* V, const int64_t* vs, void* O,
                                const int64_t* os, float* LSE, void* ws, size_t ws_bytes, void* stream) {
  lx_status s = score_sizes(dt, B, Hq, Hkv, Sq, Sk, D);
  if (s != LX_OK) return s;
  ScoreArgs a = {};
  s = score_rules(rules, a);
  if (s != LX_OK) return s;
  const int64_t q[3] = {B, Hq, Sq}, k[3] = {B, Hkv, Sk};
  if (!score_tensor(a.Q, Q, qs, q, D, false) || !score_tensor(a.K, K, ks, k, D, false) || !score_tensor(a.V, V, vs, k, D, false) ||
      !score_tensor(a.O, O, os, q, D, true) || (uintptr_t)LSE % 4 != 0)
    return LX_ERR_INVALID_ARG;
  a.LSE = LSE, a.B = B, a.Hq = Hq, a.Hkv = Hkv, a.Sq = Sq, a.Sk = Sk, a.D = D;
  const size_t need = lx_score_attn_fwd_workspace_bytes(dt, B, Hq, Hkv, Sq, Sk, D);
  if (need && !aligned16(ws)) return LX_ERR_INVALID_ARG;
  if (need && (!ws || ws_bytes < need)) return LX_ERR_WORKSPACE;
  return done(dt == LX_F32 ? launch_score_fwd_plain(a, (hipStream_t)stream) : launch_score_fwd_bf16(dt16(dt), a, ws, (hipStream_t)stream));
}

static lx_status score_bwd_impl(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D, const lx_score_rules* rules,
                                const void* Q, const void* K, const void* V, const void* O, const float* LSE, const void* dO, void* dQ, void* dK,
                                void* dV, const int64_t* st, void* ws, size_t ws_bytes, void* stream) {
  lx_status s = score_sizes(dt, B, Hq, Hkv, Sq, Sk, D);
  if (s != LX_OK) return s;
  ScoreArgs a = {};
  s = score_rules(rules, a);
  if (s != LX_OK) return s;
  const int64_t q[3] = {B, Hq, Sq}, k[3] = {B, Hkv, Sk};
  if (!st || !LSE || (uintptr_t)LSE % 4 != 0 || !score_tensor(a.Q, Q, st, q, D, false) || !score_tensor(a.K, K, st + 3, k, D, false) ||
      !score_tensor(a.V, V, st + 6, k, D, false) || !score_tensor(a.O, O, st + 9, q, D, false) ||
      !score_tensor(a.dO, dO, st + 12, q, D, false) || !score_tensor(a.dQ, dQ, st + 15, q, D, true) ||
      !score_tensor(a.dK, dK, st + 18, k, D, true) || !score_tensor(a.dV, dV, st + 21, k, D, true))
    return LX_ERR_INVALID_ARG;
  a.LSE = const_cast<float*>(LSE), a.B = B, a.Hq = Hq, a.Hkv = Hkv, a.Sq = Sq, a.Sk = Sk, a.D = D;
  if (!aligned16(ws)) return LX_ERR_INVALID_ARG;
  if (!ws || ws_bytes < lx_score_attn_bwd_workspace_bytes(dt, B, Hq, Hkv, Sq, Sk, D)) return LX_ERR_WORKSPACE;
  const int64_t rows = (int64_t)B * Hq * Sq;
  a.center = (double*)ws, a.Delta = a.center + rows, a.lse64 = a.Delta + rows;
  return done(dt == LX_F32 ? launch_score_bwd_plain(a, (hipStream_t)stream) : launch_score_bwd_bf16(dt16(dt), a, ws, (hipStream_t)stream));
}

// Pieces of a set, or -1 (an argument) or -2 (too many).
static int64_t grad_pieces(const lx_grad_tensor* t, int32_t n) {
  if (n < 0 || (n > 0 && !t)) return -1;
  int64_t pieces = 0;
  const lx_grad_tensor* some = nullptr;       // a tensor that is not empty
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].dt != LX_F32 && t[i].dt != LX_BF16 && t[i].dt != LX_F16) return -2;
    if (t[i].n < 0 || (t[i].n > 0 && !t[i].in)) return -1;
    const uintptr_t size = esize((lx_dtype)t[i].dt);
    if ((uintptr_t)t[i].in % size != 0 || (uintptr_t)t[i].out % size != 0) return -1;
    if (t[i].n > 0 && !some) some = t + i;
    if (t[i].n > 0 && !t[i].out != !some->out) return -1;
    const int64_t p = t[i].n / kGradPiece + (t[i].n % kGradPiece != 0);
    if (p > INT32_MAX - pieces) return -2;
    pieces += p;
  }
  return pieces;
}

}  // namespace lx

using namespace lx;

extern "C" {

lx_status lx_rope_table(int32_t rot, int32_t n_pos, double base, const lx_rope_scaling* scaling, float* table, void* stream) {
  const lx_status s = rope_table_impl(rot, n_pos, base, scaling, table, stream);
  LX_LOGF("lx_rope_table rot=%d n_pos=%d base=%g kind=%d -> %s", rot, n_pos, base, scaling ? scaling->kind : 0, lx_status_string(s));
  return s;
}

lx_status lx_rope(lx_dtype dt, int32_t B, int32_t S, int32_t D, int32_t rot, int32_t layout, int32_t inverse, const float* table, int32_t n_pos,
                  const int32_t* positions, const lx_rope_tensor* tensors, int32_t n_tensors, void* stream) {
  const lx_status s = rope_impl(dt, B, S, D, rot, layout, inverse, table, n_pos, positions, tensors, n_tensors, stream);
  LX_LOGF("lx_rope dt=%d B=%d S=%d D=%d rot=%d layout=%d inverse=%d tensors=%d -> %s", (int)dt, B, S, D, rot, layout, inverse, n_tensors,
          lx_status_string(s));
  return s;
}

lx_status lx_attn_key_ranges(int32_t B, int32_t S, const int32_t* doc_begin, const int32_t* doc_end, const int32_t* doc_prefix, int32_t n_docs,
                             int32_t causal, int32_t* key_lo, int32_t* key_hi, void* stream) {
  const lx_status s = key_ranges_impl(B, S, doc_begin, doc_end, doc_prefix, n_docs, causal, key_lo, key_hi, stream);
  LX_LOGF("lx_attn_key_ranges B=%d S=%d docs=%d causal=%d -> %s", B, S, n_docs, causal, lx_status_string(s));
  return s;
}

size_t lx_score_attn_fwd_workspace_bytes(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D) {
  if (score_sizes(dt, B, Hq, Hkv, Sq, Sk, D) != LX_OK || dt == LX_F32) return 0;
  return score_fwd_bytes(B, Hq, Hkv, Sq, Sk, D);
}
size_t lx_score_attn_bwd_workspace_bytes(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D) {
  if (score_sizes(dt, B, Hq, Hkv, Sq, Sk, D) != LX_OK) return 0;
  return dt == LX_F32 ? round256(3 * (size_t)B * Hq * Sq * sizeof(double)) : score_bwd_bytes(B, Hq, Hkv, Sq, Sk, D);
}

lx_status lx_score_attn_fwd(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D, const lx_score_rules* rules,
                            const void* Q, const int64_t q_strides[3], const void* K, const int64_t k_strides[3], const void* V,
                            const int64_t v_strides[3], void* O, const int64_t o_strides[3], float* LSE, void* workspace, size_t workspace_bytes,
                            void* stream) {
  const lx_status s = score_fwd_impl(dt, B, Hq, Hkv, Sq, Sk, D, rules, Q, q_strides, K, k_strides, V, v_strides, O, o_strides, LSE, workspace,
                                     workspace_bytes, stream);
  LX_LOGF("lx_score_attn_fwd dt=%d B=%d Hq=%d Hkv=%d Sq=%d Sk=%d D=%d ws=%zu -> %s", (int)dt, B, Hq, Hkv, Sq, Sk, D, workspace_bytes,
          lx_status_string(s));
  return s;
}

lx_status lx_score_attn_bwd(lx_dtype dt, int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq, int32_t Sk, int32_t D, const lx_score_rules* rules,
                            const void* Q, const void* K, const void* V, const void* O, const float* LSE, const void* dO, void* dQ, void* dK,
                            void* dV, const int64_t strides[24], void* workspace, size_t workspace_bytes, void* stream) {
  const lx_status s = score_bwd_impl(dt, B, Hq, Hkv, Sq, Sk, D, rules, Q, K, V, O, LSE, dO, dQ, dK, dV, strides, workspace, workspace_bytes, stream);
  LX_LOGF("lx_score_attn_bwd dt=%d B=%d Hq=%d Hkv=%d Sq=%d Sk=%d D=%d ws=%zu -> %s", (int)dt, B, Hq, Hkv, Sq, Sk, D, workspace_bytes,
          lx_status_string(s));
  return s;
}

size_t lx_grad_table_bytes(const lx_grad_tensor* tensors, int32_t n_tensors) {
  const int64_t pieces = grad_pieces(tensors, n_tensors);
  return pieces < 0 ? 0 : (size_t)n_tensors * sizeof(GradEntry) + (size_t)pieces * sizeof(int) + 8;
}
lx_status lx_grad_table_build(const lx_grad_tensor* tensors, int32_t n_tensors, void* table, size_t table_bytes, int32_t* pieces) {
  const int64_t n = grad_pieces(tensors, n_tensors);
  if (n == -2) return LX_ERR_UNSUPPORTED;
  if (n < 0 || !table || !pieces || (uintptr_t)table % 8 != 0 || table_bytes < lx_grad_table_bytes(tensors, n_tensors)) return LX_ERR_INVALID_ARG;
  GradEntry* e = (GradEntry*)table;
  int* of = (int*)(e + n_tensors);
  int32_t at = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    e[i] = {tensors[i].in, tensors[i].out, (long long)tensors[i].n, tensors[i].dt, at};
    for (int64_t k = 0; k < tensors[i].n; k += kGradPiece) of[at++] = i;
  }
  *pieces = at;
  return LX_OK;
}
size_t lx_grad_norm_clip_workspace_bytes(int32_t pieces) {
  return round256((size_t)(pieces < 1 ? 1 : pieces < kGradSums ? pieces : kGradSums) * sizeof(double));
}
lx_status lx_grad_norm_clip(const void* table, int32_t n_tensors, int32_t pieces, float max_norm, float* norm, void* workspace,
                            size_t workspace_bytes, void* stream) {
  lx_status s = LX_OK;
  if (!table || n_tensors < 0 || pieces < 0 || !norm || !(max_norm >= 0) || (uintptr_t)table % 8 != 0 || (uintptr_t)workspace % 8 != 0 || (uintptr_t)norm % 4 != 0)
    s = LX_ERR_INVALID_ARG;
  else if (!workspace || workspace_bytes < lx_grad_norm_clip_workspace_bytes(pieces))
    s = LX_ERR_WORKSPACE;
  else
    s = done(launch_grad_norm_clip((const GradEntry*)table, n_tensors, pieces, max_norm, norm, (double*)workspace, (hipStream_t)stream));
  LX_LOGF("lx_grad_norm_clip tensors=%d pieces=%d max_norm=%g -> %s", n_tensors, pieces, (double)max_norm, lx_status_string(s));
  return s;
}

}  // extern "C"
