// How the loss over a vocabulary cuts its work (csrc/vocab_plan.h), as C functions.
#include <string.h>

#include "../paper_2510_15964_amd/csrc/log_steps.h"
#include "../paper_2510_15964_amd/csrc/vocab_plan.h"

using namespace lx;

static void write(const CutPlan& p, int* out) {
  const int v[] = {p.GM, p.GN, p.full, p.rest, p.pieces, p.steps};
  for (int i = 0; i < 6; ++i) out[i] = v[i];
}

extern "C" {
int logits_tile(int n, int d, int V) { return plan_logits(n, d, V); }
int dx_tile(int n, int d, int V, long long room) { return plan_dx(n, d, V, room); }
int dw_tile(int n, int d, int V, long long room) { return plan_dw(n, d, V, room); }
void tile_size(int id, int* out) { out[0] = 64 * kTileInfo[id].tm, out[1] = 64 * kTileInfo[id].tn; }
void dx(int id, int n, int d, int V, long long room, int* out) { write(dx_plan(id, n, d, V, room), out); }
void dw(int id, int n, int d, int V, long long room, int* out) { write(dw_plan(id, n, d, V, room), out); }
int grid_dx(int id, int n, int d, long long room) { return dx_grid(id, n, d, room); }
int slots(int id, long long room) { return cut_slots(id, room); }
// Of every workgroup: unit, lo, hi, slot; how many have something to do.
int items(const int* plan, int grid, int* out) {
  const CutPlan p = {plan[0], plan[1], plan[2], plan[3], plan[4], plan[5], 0.f};
  int n = 0;
  for (int w = 0; w < grid; ++w) {
    CutItem it;
    if (!cut_item(p, w, it)) continue;
    int* o = out + 4 * n++;
    o[0] = it.unit, o[1] = it.lo, o[2] = it.hi, o[3] = it.slot;
  }
  return n;
}
int tiles(int GM, int GN, int* out) {
  int n = 0;
  for (int w = 0; w < eights(GM * GN); ++w) {
    GridItem it;
    if (xcd_item(w, GM, GN, it)) out[2 * n] = it.m, out[2 * n + 1] = it.n, ++n;
  }
  return n;
}
int rows(int T, int V, int grads, int f32) { return vocab_rows(T, V, grads, f32); }
long long room(int rows, int T, int d, int V, int grads, int dw, int dw_f32, long long* slots) {
  const VocabRoom r = vocab_room(rows, T, d, V, grads, dw, dw_f32);
  *slots = r.slots;
  return (long long)r.bytes;
}
// Bytes for the order of the tokens by their target's tile, and for what G lacks.
void lacks_room(int rows, int T, int d, int V, int dw_f32, long long* out) {
  const VocabRoom r = vocab_room(rows, T, d, V, true, true, dw_f32);
  out[0] = (long long)(r.lo - r.order), out[1] = (long long)((r.dw ? r.dw : r.bytes) - r.lo);
}
// The step of exp(y), as the kernels keep it, and the power of two that it stands for.
int step(float y) {
  const float f = log_step(y);
  unsigned u;
  memcpy(&u, &f, 4);
  return (int)(u & 0xffff);
}
float power(int step) { return step_log2((unsigned)step); }
// What a plan is taken to cost.
float dx_cost(int id, int n, int d, int V, long long room) { return dx_plan(id, n, d, V, room).cost; }
float dw_cost(int id, int n, int d, int V, long long room) { return dw_plan(id, n, d, V, room).cost; }
}
