// The loss over a vocabulary: pieces of the tokens, workspace, tiles and how launches deal their work.  Plain C++ for host and device.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "ffn_plan.h"

namespace lx {

constexpr int kVocabTile = 256;                 // the widest tile's tokens and rows of the vocabulary: what buffers are padded to
constexpr int kVocabPieceMost = 65536;          // tokens of a piece, each of whose workgroups counts the targets before its own
constexpr size_t kVocabPieceBytes = (size_t)1 << 30;   // of a piece's probabilities, where the library chooses

// ---- tiles, by ffn_plan.h's times of a launch -------------------------------------------------------

// The 64 x 64 tile here, whose weight side comes from memory and not from a list's few blocks, and lies as columns for dX: a step takes 0.22 us
// and 0.27 (35 tokens, d = 2368, 4370 rows: logits 11.9, by the 64 x 128 tile 15.2; dX of 2 tokens, 889 rows 7.5, by 64 x 256 10.6;
// of 77, d = 2816, 3846 rows uncut 19.6, by 64 x 256 cut 12.1 and 5).
LX_HD TileInfo vocab_tile(int id, float step) {
  TileInfo t = kTileInfo[id];
  if (id == kT11) t.step[0] = step, t.step[1] = 2.f * step;
  return t;
}
// Logits: `n` tokens, V columns, d / 64 steps.  Exponentials and statistics add to a round what they take for the elements of a CU's tiles.
constexpr int kLogitTiles[] = {kT44, kT24, kT14Deep, kT12, kT11};
LX_HD float logit_cost(int id, int n, int d, int V) {
  TileInfo t = vocab_tile(id, 0.22f);
  t.round += 4.f / 16 * (float)(t.tm * t.tn * t.resident);
  return tile_cost(t, t.resident, ceil_div(n, 64 * t.tm) * ceil_div(V, 64 * t.tn), (float)(d / 64));
}
inline int plan_logits(int n, int d, int V) {
  int best = kT44;
  for (int id : kLogitTiles)
    if (logit_cost(id, n, d, V) < logit_cost(best, n, d, V)) best = id;
  return best;
}

// dX and dW: units (tiles of rows x columns), whole rounds of workgroups as they are, the rest with the contraction, `steps` of 64, cut into
// pieces, whose results are added in order: as many pieces as cost least, if there is room for their results (`room`: elements).  Host
// and kernels each make the plan, so its arithmetic is not fused: the same sizes give the same plan everywhere.
constexpr int kDxTiles[] = {kT44, kT24, kT14Deep, kT11}, kDwTiles[] = {kT44, kT24};
struct CutPlan {
  int GM, GN, full, rest, pieces, steps;
  float cost;
};
LX_HD CutPlan cut_plan(int id, int rows, int columns, int steps, long long room) {
#ifdef __clang__
#pragma clang fp contract(off)
#endif
  const TileInfo t = vocab_tile(id, 0.27f);
  CutPlan p = {ceil_div(rows, 64 * t.tm), ceil_div(columns, 64 * t.tn), 0, 0, 1, steps, 0.f};
  const int units = p.GM * p.GN;
  p.full = units / kCUs * kCUs;
  p.rest = units - p.full;
  float least = 0.f;
  if (p.rest > 0)
    for (int wgs = 0; wgs <= 2 * kCUs; wgs = wgs ? 2 * wgs : kCUs / 4) {      // (as they are; a quarter of a round, half of one, one, two)
      const int k = wgs ? wgs / p.rest : 1;
      if (k < 1 || (k > 1 && (k > steps || (long long)k * p.rest * (t.tm * t.tn * 4096) > room))) continue;
      // (a piece's way through memory: written and read in fp32; the launch that adds them)
      const float c = (float)ceil_div(p.rest * k, kCUs) * (t.round + (float)ceil_div(steps, k) * t.step[0]) +
                      (k > 1 ? (float)(p.rest * k * t.tm * t.tn) * (4096 * 8 / 4.5e6f) + 6.f : 0.f);
      if (!wgs || c < least) least = c, p.pieces = k;
    }
  p.cost = least + (float)(p.full / kCUs) * (t.round + (float)steps * t.step[0]);
  if (p.pieces == 1) p.full = units, p.rest = 0;
  return p;
}
LX_HD CutPlan dx_plan(int id, int n, int d, int V, long long room) { return cut_plan(id, n, d, ceil_div(V, 64), room); }
LX_HD CutPlan dw_plan(int id, int n, int d, int V, long long room) { return cut_plan(id, V, d, ceil_div(n, 64), room); }
template <size_t N, class Plan>
inline int cheapest(const int (&ids)[N], Plan plan) {
  int best = ids[0];
  for (int id : ids)
    if (plan(id).cost < plan(best).cost) best = id;
  return best;
}
inline int plan_dx(int n, int d, int V, long long room) {
  return cheapest(kDxTiles, [&](int id) { return dx_plan(id, n, d, V, room); });
}
inline int plan_dw(int n, int d, int V, long long room) {
  return cheapest(kDwTiles, [&](int id) { return dw_plan(id, n, d, V, room); });
}
// What workgroup w does: a unit, steps lo .. hi - 1 of it, and where its results go if it is not whole (-1).  Workgroup w runs on XCD w % 8.
struct CutItem {
  int unit, lo, hi, slot;
};
LX_HD bool cut_item(const CutPlan& p, int w, CutItem& it) {
  const int Lf = ceil_div(p.full, 8), cut = p.rest * p.pieces, Lr = ceil_div(cut, 8), s = w / 8, x = w % 8;
  it = {x * Lf + s, 0, p.steps, -1};
  if (s < Lf) return it.unit < p.full;
  const int y = x * Lr + s - Lf;
  if (s - Lf >= Lr || y >= cut) return false;
  const int piece = y / p.rest;            // an XCD works on few pieces
  it.unit = p.full + y % p.rest;
  it.slot = (y % p.rest) * p.pieces + piece;
  it.lo = (int)((long long)p.steps * piece / p.pieces);
  it.hi = (int)((long long)p.steps * (piece + 1) / p.pieces);
  return true;
}
// Whole tiles, in bands of four tiles of tokens: XCD w % 8 takes an eighth of them.
LX_HD bool xcd_item(int w, int GM, int GN, GridItem& it) {
  const int total = GM * GN, L = ceil_div(total, 8), slot = w / 8, idx = w % 8 * L + slot;
  if (slot >= L || idx >= total) return false;
  it = grid_item(idx, GM, GN, 4);
  return true;
}
inline int eights(int x) { return ceil_div(x, 8) * 8; }      // workgroups, an equal number to each XCD
// Pieces that a launch has room for, two rounds of workgroups at most.
inline int cut_slots(int id, long long room) {
  const long long slots = room / (kTileInfo[id].tm * kTileInfo[id].tn * 4096);
  return (int)(slots < 2 * kCUs ? slots : 2 * kCUs);
}
// Workgroups of dX's launch, whose kernel alone knows how many of the n tokens have a target: enough for any number of them.
inline int dx_grid(int id, int n, int d, long long room) {
  return eights(ceil_div(n, 64 * kTileInfo[id].tm) * ceil_div(d, 64 * kTileInfo[id].tn)) + eights(cut_slots(id, room));
}

// A piece's part of the workspace, for up to `rows` tokens (a multiple of kVocabTile).
struct VocabRoom {
  size_t head, list, target, weight, z, factor, lacks, stats, x, tail, p, part, dw, spans, order, lo, bytes;
  int rows, units;       // units: columns of statistics per token
  long long slots;       // elements of the pieces of dX and dW that there is room for
  long long ldp;         // elements between rows of the probabilities
};
inline size_t vocab_align(size_t x) { return (x + 255) & ~(size_t)255; }
inline VocabRoom vocab_room(int rows, int T, int d, int V, bool grads, bool dw, bool dw_f32) {
  VocabRoom r = {};
  const size_t tiles = ((size_t)V + kVocabTile - 1) / kVocabTile, n = (size_t)rows;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += vocab_align(bytes);
    return here;
  };
  r.rows = rows;
  r.units = (int)tiles * 8;      // (of 32 columns at least)
  r.ldp = (long long)tiles * kVocabTile;
  r.head = take(256);
  r.list = take(n * 4);
  r.target = take(n * 4);
  r.weight = take(n * 4);
  r.z = take(n * 8);
  r.factor = take(n * 4);
  r.lacks = take(n * 4);
  r.stats = take(n * r.units * 8);
  r.x = take(n * d * 2);
  r.tail = take((size_t)64 * d * 2);
  if (grads) {
    r.p = take(n * r.ldp * 2);
    // (two rounds of the widest tile; of a small call as many pieces of each product as it has, of 8 steps)
    const long long width = (d + kVocabTile - 1) / kVocabTile * kVocabTile, two = 2ll * kCUs * kVocabTile * kVocabTile;
    const long long dx = (long long)n * width * ((V + 511) / 512), dw_ = dw ? (long long)tiles * kVocabTile * width * ((n + 511) / 512) : 0;
    r.slots = dx < dw_ ? dw_ : dx;
    if (r.slots > two) r.slots = two;
    r.part = take((size_t)r.slots * 4);
  }
  if (dw) {       // (tiles of the vocabulary of 128 rows at least, 64 tokens more for each, and 64 that are read and not used)
    r.spans = take(2 * tiles * 8);
    r.order = take((n + 128 * tiles + 64) * 4);
    r.lo = take((n + 64 * tiles) * kVocabTile * 2);
  }
  if (dw && !dw_f32 && T > rows) r.dw = take((size_t)V * d * 4);
  r.bytes = at;
  return r;
}
// Tokens of a piece: the whole call, or as many as fit kVocabPieceBytes, in pieces of equal length.
inline int vocab_rows(int T, int V, bool grads, bool f32) {
  const long long row = ((long long)V + kVocabTile - 1) / kVocabTile * (f32 ? kVocabTile * 4 : grads ? kVocabTile * 2 : 64);
  long long most = (long long)(kVocabPieceBytes / (size_t)row) / kVocabTile * kVocabTile;
  most = most < kVocabTile ? kVocabTile : most > kVocabPieceMost ? kVocabPieceMost : most;
  const long long pieces = (T + most - 1) / most, even = (T + pieces - 1) / pieces;
  return (int)((even + kVocabTile - 1) / kVocabTile * kVocabTile);
}

// Single precision: the logits themselves.
inline VocabRoom vocab_room_plain(int rows, int V) {
  VocabRoom r = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += vocab_align(bytes);
    return here;
  };
  r.rows = rows;
  r.ldp = ((long long)V + 63) / 64 * 64;
  r.head = take(256);
  r.list = take((size_t)rows * 4);
  r.target = take((size_t)rows * 4);
  r.p = take((size_t)rows * r.ldp * 4);
  r.bytes = at;
  return r;
}

}  // namespace lx
