// Loss over a vocabulary with its gradients, 16-bit operands:  z = X W^T,  loss = log sum exp z - z_target,
// G = weight (softmax(z) - [target]),  dX = G W,  dW = G^T X.
//
// Three products of 2 n V d operations, n the number of tokens that have a target, which bound the call; nothing of the size of
// z outlives a piece of the tokens, whose exponentials lie in the workspace in 16 bits:
//   gather  the tokens that have a target, one after the other: the others are not multiplied, and what they hold has no effect
//   logits  z, tile by tile in registers; of each token and unit of columns, the target's column left out, the largest z and the sum of
//           exp(z - largest), in fp32; exp(z - largest) 2^15 in half precision
//   rows    the loss, and the exponentials in place times exp(largest - lse) weight, rounded to the element type: G
//   dX, dW  products of G
// The exponentials' first rounding, 2^-11 at most, is lost beside the second where that is one to bfloat16; the target's column is made from
// the other columns' sum, so that a token whose target is all but certain has an exact gradient, and an exact loss by log1p.
#include <type_traits>

#include "ffn_plan.h"
#include "ffn_tile.h"
#include "vocab.h"

namespace lx {

constexpr float kLog2e = 1.4426950408889634f;
// Half precision: gradients are scaled by a power of two, so that the largest weight's are at most 2^14.
constexpr float kHalfTop = 16384.f;

struct VocabHead {       // of a piece
  int n;                 // tokens that have a target
  float scale, unscale;  // of G
};

// Pointers into the workspace.
struct VocabPiece {
  VocabHead* head;
  int *list, *target;
  float *weight, *at;    // per token: its weight, its target's z
  float2* stats;         // [rows][units]: largest z, sum
  uint16_t *x, *tail, *p;
  f32x4* part;
  float* dw;
  int rows, units, first, count;      // rows that there is room for; the piece's tokens: first .. first + count - 1 of the call's
  long long ldp;
};

// ---- gather ----------------------------------------------------------------------------------------

// 64 tokens to a workgroup, which counts the targets before its own; the workgroups behind those copy the last V % 64 rows of W
// and zeros into a block of 64 rows of their own, which the products read in their place.
template <bool VEC>
__global__ __launch_bounds__(256) void vocab_gather(VocabArgs a, VocabPiece q) {
  __shared__ int counts[2][4];
  __shared__ float tops[4];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, chunks = (q.count + 63) / 64;
  const int first = blockIdx.x * 64;
  if ((int)blockIdx.x >= chunks) {
    const int r0 = a.V / 64 * 64;
    for (int r = ((int)blockIdx.x - chunks) * 4 + wave; r < 64; r += 64)
      for (int c = lane * 8; c < a.d; c += 8 * kWave)
        *reinterpret_cast<uint4*>(q.tail + (long long)r * a.d + c) =
            r0 + r < a.V ? *reinterpret_cast<const uint4*>(a.W + (long long)(r0 + r) * a.d + c) : make_uint4(0, 0, 0, 0);
    return;
  }
  const int* targets = a.targets + q.first;
  const float* weights = a.weights ? a.weights + q.first : nullptr;
  int before = 0, all = 0;
  float top = 0;
  for (int t = threadIdx.x; t < q.count; t += 256) {
    const bool held = (unsigned)targets[t] < (unsigned)a.V;
    all += held;
    before += held && t < first;
    if (held) top = fmaxf(top, weights ? fabsf(weights[t]) : 1.f);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    before += __shfl_xor(before, o);
    all += __shfl_xor(all, o);
    top = fmaxf(top, __shfl_xor(top, o));
  }
  if (lane == 0) counts[0][wave] = before, counts[1][wave] = all, tops[wave] = top;
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) before += counts[0][w], all += counts[1][w], top = fmaxf(top, tops[w]);
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) {
      // a power of two: bfloat16 has the range of fp32
      float s = 1.f;
      if (a.dt == kF16 && top > 0 && top < 3e38f) s = exp2f(floorf(log2f(kHalfTop / top)));
      s = fminf(fmaxf(s, 0x1p-100f), 0x1p100f);
      *q.head = {all, s, 1.f / s};
    }
    // the rows up to the next 64, which dW's product reads
    for (int r = all + wave; r < (all + 63) / 64 * 64; r += 4)
      for (int c = lane * 8; c < a.d; c += 8 * kWave) *reinterpret_cast<uint4*>(q.x + (long long)r * a.d + c) = make_uint4(0, 0, 0, 0);
  }
  const int mine = first + lane < q.count ? targets[first + lane] : -1;
  const unsigned long long held = __ballot((unsigned)mine < (unsigned)a.V);
  if (wave == 0 && first + lane < q.count) {
    const long long t = q.first + first + lane;
    if (held >> lane & 1) {
      const int to = before + __popcll(held & ((1ull << lane) - 1));
      q.list[to] = (int)t;
      q.target[to] = mine;
      q.weight[to] = weights ? weights[first + lane] : 1.f;
    } else {
      a.loss[t] = 0.f;
      if (a.lse) a.lse[t] = 0.f;
    }
  }
  for (int i = wave; i < 64 && first + i < q.count; i += 4) {
    const long long t = q.first + first + i;
    if (held >> i & 1) {
      const int to = before + __popcll(held & ((1ull << i) - 1));
      const uint16_t* x = a.X + t * a.xs;
      for (int c = lane * 8; c < a.d; c += 8 * kWave) {
        uint4 v;
        if constexpr (VEC) {
          v = *reinterpret_cast<const uint4*>(x + c);
        } else {
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = (uint32_t)x[c + 2 * k] | (uint32_t)x[c + 2 * k + 1] << 16;
          v = make_uint4(w[0], w[1], w[2], w[3]);
        }
        *reinterpret_cast<uint4*>(q.x + (long long)to * a.d + c) = v;
      }
    } else if (a.dX) {
      uint16_t* dx = a.dX + t * a.dxs;
      if constexpr (VEC) {
        for (int c = lane * 8; c < a.d; c += 8 * kWave) *reinterpret_cast<uint4*>(dx + c) = make_uint4(0, 0, 0, 0);
      } else {
        for (int c = lane; c < a.d; c += kWave) dx[c] = 0;
      }
    }
  }
}

// ---- the products ----------------------------------------------------------------------------------

// Transfers of a product's two operands: instruction u of wavefront w brings eight rows of a stage, rows 8 g .. of its
// operand with g = w + 8 u (the token side's first), 64 elements of each.  An operand that lies as columns (TRA, TRB): eight
// contraction indices, 64 columns.  The weight side may change to other rows at step `turn`.
template <class Tl>
struct VocabSrc {
  const uint16_t* base[Tl::kIss];
  const uint16_t* other[Tl::kIss - Tl::kIssA];
  uint32_t voff_b, voff_a;
  long long step_b, step_a, off_b, off_a;
  int turn;
  __device__ __forceinline__ int live() const { return Tl::kIss; }
  __device__ __forceinline__ bool busy(int) const { return true; }
  // ld: elements between memory's rows
  __device__ __forceinline__ void places(int wave, long long ld_b, long long ld_a) {
    const int lane = threadIdx.x % kWave, lr = lane / 8;
    auto place = [&](long long ld, bool columns) {
      const int swz = columns ? column_swz(8 * wave + lr) : tile_swz<Tl>(8 * wave + lr);
      return (uint32_t)(lr * ld * 2 + (((lane % 8) ^ swz) << 4));
    };
    voff_b = place(ld_b, Tl::TRB);
    voff_a = place(ld_a, Tl::TRA);
    turn = -1;
  }
  __device__ __forceinline__ void begin(int s) {
    off_b = s * step_b;
    off_a = s * step_a;
    if (Tl::TRA && s == turn) {
      off_a = 0;
#pragma unroll
      for (int u = Tl::kIssA; u < Tl::kIss; ++u) base[u] = other[u - Tl::kIssA];
    }
  }
  __device__ __forceinline__ void dma(int u, uint32_t lds) const {
    if (u < Tl::kIssA)
      dma16_s(base[u] + off_b, voff_b, lds + u * (Tl::kWaves * 1024));
    else
      dma16_s(base[u] + off_a, voff_a, lds + u * (Tl::kWaves * 1024));
  }
};
// Step numbers are those of the whole contraction; a part of it starts at `lo`.
template <class Src>
struct FromStep {
  Src& src;
  int lo;
  __device__ __forceinline__ int live() const { return src.live(); }
  __device__ __forceinline__ bool busy(int w) const { return src.busy(w); }
  __device__ __forceinline__ void begin(int s) { src.begin(lo + s); }
  __device__ __forceinline__ void dma(int u, uint32_t lds) const { src.dma(u, lds); }
};

template <class Tl>
__device__ __forceinline__ void clear(typename Tl::Acc (&acc)[Tl::NI][Tl::TI]) {
#pragma unroll
  for (int x = 0; x < Tl::NI; ++x)
#pragma unroll
    for (int y = 0; y < Tl::TI; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// A wavefront's 16 TI x 16 NI results -> its own part of LDS as 16-bit elements, four consecutive columns of a row at a time
// (pack(ni, ti)), and from there in runs of 16 bytes, whole rows of 32 NI bytes next to one another: put(row, slot, run).
template <class Tl, class Pack, class Put>
__device__ __forceinline__ void rows_out(uint32_t lds, Pack pack, Put put) {
  constexpr int kSlots = 2 * Tl::NI, kRows = 16 * Tl::TI;
  const int lane = threadIdx.x % kWave, r = lane % 16, q = lane / 16;
  const uint32_t mine = lds + (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (kRows * kSlots * 16);
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti)
#pragma unroll
    for (int ni = 0; ni < Tl::NI; ++ni) {
      const int row = 16 * ti + r, slot = (2 * ni + q / 2) ^ (row & (kSlots - 1));
      lds_write8(mine + (uint32_t)(row * kSlots + slot) * 16 + q % 2 * 8, pack(ni, ti));
    }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (no other wavefront writes or reads there)
#pragma unroll
  for (int x = 0; x < kRows * kSlots / kWave; ++x) {
    const int at = x * kWave + lane, row = at / kSlots, slot = at % kSlots;
    put(row, slot, lds_read16(mine + (uint32_t)(row * kSlots + (slot ^ (row & (kSlots - 1)))) * 16));
  }
}

// The item of a workgroup: XCD w % 8 takes an eighth of the items, in bands of four token tiles.
__device__ __forceinline__ bool xcd_item(int w, int GM, int GN, GridItem& it) {
  const int total = GM * GN, L = (total + 7) / 8, slot = w / 8, idx = w % 8 * L + slot;
  if (slot >= L || idx >= total) return false;
  it = grid_item(idx, GM, GN, 4);
  return true;
}

//     TM TN WM WN NST PH
using LogitTile = Tile<4, 4, 4, 2, 2, 2>;
using DxTile = Tile<4, 4, 4, 2, 2, 2, 2, 16, true, false>;     // W as columns
using DwTile = Tile<4, 4, 4, 2, 2, 2, 2, 16, true, true>;      // both

// z of a tile, its statistics, its exponentials if GRAD.
template <class Tl, int DT, bool GRAD>
__global__ __launch_bounds__(Tl::kTileThreads, Tl::kMinWaves) void vocab_logits(VocabArgs a, VocabPiece q) {
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  const int n = q.head->n, GM = (n + 64 * Tl::TM - 1) / (64 * Tl::TM), GN = (a.V + 64 * Tl::TN - 1) / (64 * Tl::TN);
  GridItem it;
  if (!xcd_item(blockIdx.x, GM, GN, it)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.m * 64 * Tl::TM, n0 = it.n * 64 * Tl::TN;
  VocabSrc<Tl> src;
  src.places(wave, a.d, a.d);
  src.step_b = src.step_a = kBK;
#pragma unroll
  for (int u = 0; u < Tl::kIss; ++u) {
    const int g = wave + Tl::kWaves * u;
    if (u < Tl::kIssA) {
      src.base[u] = q.x + (long long)(i0 + 8 * g) * a.d;      // (rows behind the last one: whatever lies there, for results that are not stored)
    } else {
      const int r = n0 + 8 * (g - 8 * Tl::TM), over = a.V / 64 * 64;
      src.base[u] = r + 8 <= over ? a.W + (long long)r * a.d : q.tail + (long long)(r - over < 64 ? r - over : 0) * a.d;
    }
  }
  const int wm = wave / Tl::WN, wn = wave % Tl::WN, lane = threadIdx.x % kWave;
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  run_tile<Tl, DT>(a.d / kBK, lds_addr(ring), wm, wn, src, acc);
  // a lane: columns c0 + 16 ni + v of its tokens t0 + 16 ti
  const int t0 = i0 + 16 * Tl::TI * wm + lane % 16, u0 = n0 + 16 * Tl::NI * wn, c0 = u0 + lane / 16 * 4;
  if (u0 + 16 * Tl::NI > a.V) {
#pragma unroll
    for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (c0 + 16 * ni + v >= a.V)
#pragma unroll
          for (int ti = 0; ti < Tl::TI; ++ti) acc[ni][ti][v] = -INFINITY;
  }
  const int unit = u0 / (16 * Tl::NI);
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti) {
    const int t = t0 + 16 * ti, rel = (t < n ? q.target[t] : -1) - c0;
    // the target, if it is here, is taken out: beside one that is all but certain the others would vanish in half precision
    const bool here = rel >= 0 && rel < 16 * Tl::NI && rel % 16 < 4;
    if (__ballot(here)) {
      float z = 0;
#pragma unroll
      for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (rel == 16 * ni + v) z = acc[ni][ti][v], acc[ni][ti][v] = -INFINITY;
      if (here) q.at[t] = z;
    }
    float top = acc[0][ti][0];
#pragma unroll
    for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
      for (int v = 0; v < 4; ++v) top = fmaxf(top, acc[ni][ti][v]);
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    float sum = 0;
    const float from = top == -INFINITY ? 0.f : top;      // (nothing but the target, or columns behind the vocabulary)
#pragma unroll
    for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float e = __builtin_amdgcn_exp2f(fmaf(acc[ni][ti][v] - from, kLog2e, 15.f));
        sum += e;
        if (GRAD) acc[ni][ti][v] = e;
      }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (lane < 16 && t < n) q.stats[(long long)t * q.units + unit] = make_float2(top, sum * 0x1p-15f);
  }
  if constexpr (GRAD) {
    lds_barrier();       // nobody reads the ring any more
    uint16_t* p = q.p + (long long)(i0 + 16 * Tl::TI * wm) * q.ldp + u0;
    rows_out<Tl>(lds_addr(ring),
                 [&](int ni, int ti) {
                   const f32x4 v = acc[ni][ti];
                   return make_uint2(pack2<kF16>(v[0], v[1]), pack2<kF16>(v[2], v[3]));
                 },
                 [&](int row, int slot, uint4 v) { *reinterpret_cast<uint4*>(p + row * q.ldp + slot * 8) = v; });
  }
}

// A token's statistics joined, its loss, and its row of G.  units: of `width` columns each.
template <int DT, bool GRAD>
__global__ __launch_bounds__(256) void vocab_rows_kernel(VocabArgs a, VocabPiece q, int units, int width) {
  extern __shared__ float factor[];
  __shared__ float part[2][4];
  const int n = q.head->n, t = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  if (t >= n) {      // rows up to the next 64, which dW's product reads
    if (GRAD && t < (n + 63) / 64 * 64)
      for (long long c = threadIdx.x * 8; c < q.ldp; c += 2048) *reinterpret_cast<uint4*>(q.p + t * q.ldp + c) = make_uint4(0, 0, 0, 0);
    return;
  }
  const float2* stats = q.stats + (long long)t * q.units;
  const float z = q.at[t];
  float top = z, sum = 0;
  for (int u = threadIdx.x; u < units; u += 256) top = fmaxf(top, stats[u].x);
#pragma unroll
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (lane == 0) part[0][wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
  for (int u = threadIdx.x; u < units; u += 256) {
    const float2 s = stats[u];
    const float f = __builtin_amdgcn_exp2f((s.x - top) * kLog2e);
    sum = fmaf(s.y, f, sum);
    if (GRAD) factor[u] = f;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) part[1][wave] = sum;
  __syncthreads();
  sum = (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);      // of all but the target
  const float mine = __builtin_amdgcn_exp2f((z - top) * kLog2e), total = sum + mine;
  if (threadIdx.x == 0) {
    const float lse = top + logf(total);
    a.loss[q.list[t]] = mine > 0.5f * total ? log1pf(sum / mine) : (top - z) + logf(total);
    if (a.lse) a.lse[q.list[t]] = lse;
  }
  if constexpr (GRAD) {
    const float w = q.weight[t] * q.head->scale, f = w / total * 0x1p-15f;
    const int target = q.target[t];
    const float g = -w * (sum / total);
    uint16_t* p = q.p + t * q.ldp;
    for (int c = threadIdx.x * 8; c < (int)q.ldp; c += 2048) {
      const float k = factor[c / width] * f;
      const uint4 v = *reinterpret_cast<const uint4*>(p + c);
      const uint32_t in[4] = {v.x, v.y, v.z, v.w};
      float e[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) e[2 * i] = to_f32<kF16>(in[i] & 0xffff) * k, e[2 * i + 1] = to_f32<kF16>(in[i] >> 16) * k;
      if (target - c >= 0 && target - c < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (target - c == i) e[i] = g;
      *reinterpret_cast<uint4*>(p + c) = make_uint4(pack2<DT>(e[0], e[1]), pack2<DT>(e[2], e[3]), pack2<DT>(e[4], e[5]), pack2<DT>(e[6], e[7]));
    }
  }
}

// How dX's units (tiles of 256 tokens x 256 columns), whose number the device knows, are shared: whole rounds of workgroups as they are,
// the rest with the vocabulary cut into pieces of at least kLeastSteps steps, whose results are added in order.
constexpr int kLeastSteps = 8;
struct DxPlan {
  int GM, GN, full, rest, pieces, steps;
};
__device__ __forceinline__ DxPlan dx_plan(int n, int d, int V) {
  DxPlan p;
  p.GM = (n + kVocabTile - 1) / kVocabTile, p.GN = (d + kVocabTile - 1) / kVocabTile;
  p.steps = (V + 63) / 64;
  const int units = p.GM * p.GN;
  p.full = units / kCUs * kCUs;
  p.rest = units - p.full;
  p.pieces = p.rest ? min(kCUs / p.rest, max(p.steps / kLeastSteps, 1)) : 1;
  if (p.pieces == 1) p.full = units, p.rest = 0;
  return p;
}

template <int DT>
__global__ __launch_bounds__(DxTile::kTileThreads, DxTile::kMinWaves) void vocab_dx(VocabArgs a, VocabPiece q) {
  using Tl = DxTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  const DxPlan p = dx_plan(q.head->n, a.d, a.V);
  const int Lf = (p.full + 7) / 8, cut = p.rest * p.pieces, Lr = (cut + 7) / 8, s = blockIdx.x / 8, x = blockIdx.x % 8;
  int unit, lo = 0, hi = p.steps, slot = -1;
  if (s < Lf) {
    unit = x * Lf + s;
    if (unit >= p.full) return;
  } else {
    const int y = x * Lr + s - Lf;
    if (s - Lf >= Lr || y >= cut) return;
    const int piece = y / p.rest;            // an XCD works on few pieces
    unit = p.full + y % p.rest;
    slot = (y % p.rest) * p.pieces + piece;
    lo = (int)((long long)p.steps * piece / p.pieces);
    hi = (int)((long long)p.steps * (piece + 1) / p.pieces);
  }
  const GridItem it = grid_item(unit, p.GM, p.GN, 4);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.m * kVocabTile, n0 = it.n * kVocabTile;
  VocabSrc<Tl> src;
  src.places(wave, q.ldp, a.d);
  src.step_b = kBK;
  src.step_a = 64ll * a.d;
  if (a.V % 64) src.turn = a.V / 64;
#pragma unroll
  for (int u = 0; u < Tl::kIss; ++u) {
    const int g = wave + Tl::kWaves * u;
    if (u < Tl::kIssA) {
      src.base[u] = q.p + (long long)(i0 + 8 * g) * q.ldp;
    } else {                 // columns past the edge: the last 64 again, not stored
      const int c = min(n0 + (g / 8 - Tl::TM) * 64, a.d - 64);
      src.base[u] = a.W + (long long)(8 * (g % 8)) * a.d + c;
      src.other[u - Tl::kIssA] = q.tail + (long long)(8 * (g % 8)) * a.d + c;
    }
  }
  const int wm = wave / Tl::WN, wn = wave % Tl::WN, lane = threadIdx.x % kWave;
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  FromStep<VocabSrc<Tl>> part = {src, lo};
  run_tile<Tl, DT>(hi - lo, lds_addr(ring), wm, wn, part, acc);
  if (slot >= 0) {       // [wavefront][accumulator][lane][4 registers]
    f32x4* to = q.part + ((size_t)slot * Tl::kWaves + wave) * (Tl::NI * Tl::TI) * kWave + lane;
#pragma unroll
    for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
      for (int ti = 0; ti < Tl::TI; ++ti) to[(ni * Tl::TI + ti) * kWave] = acc[ni][ti];
    return;
  }
  lds_barrier();       // nobody reads the ring any more
  const float k = q.head->unscale;
  const int n = q.head->n, r0 = i0 + 16 * Tl::TI * wm, c0 = n0 + 16 * Tl::NI * wn;
  const bool whole = ((uintptr_t)a.dX | (uintptr_t)(a.dxs * 2)) % 16 == 0;
  rows_out<Tl>(lds_addr(ring),
               [&](int ni, int ti) {
                 const f32x4 v = acc[ni][ti];
                 return make_uint2(pack2<DT>(v[0] * k, v[1] * k), pack2<DT>(v[2] * k, v[3] * k));
               },
               [&](int row, int at, uint4 v) {
                 if (r0 + row >= n || c0 + at * 8 >= a.d) return;
                 uint16_t* to = a.dX + q.list[r0 + row] * a.dxs + c0 + at * 8;
                 if (whole) {
                   *reinterpret_cast<uint4*>(to) = v;
                 } else {
                   const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                   for (int i = 0; i < 8; ++i) to[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
                 }
               });
}

// The pieces of dX's cut units added in order: one workgroup to 16 accumulators' columns of a wavefront of the product.
template <int DT>
__global__ __launch_bounds__(256) void vocab_dx_sum(VocabArgs a, VocabPiece q) {
  using Tl = DxTile;
  const DxPlan p = dx_plan(q.head->n, a.d, a.V);
  if ((int)blockIdx.x >= p.rest) return;
  const GridItem it = grid_item(p.full + blockIdx.x, p.GM, p.GN, 4);
  const int lane = threadIdx.x % kWave, wave = blockIdx.y, ni = blockIdx.z, ti = threadIdx.x / kWave;
  const f32x4* from = q.part + (((size_t)blockIdx.x * p.pieces * Tl::kWaves + wave) * (Tl::NI * Tl::TI) + ni * Tl::TI + ti) * kWave + lane;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < p.pieces; ++i) v += from[(size_t)i * (Tl::kWaves * Tl::NI * Tl::TI * kWave)];
  const int row = it.m * kVocabTile + 16 * (Tl::TI * (wave / Tl::WN) + ti) + lane % 16;
  const int c = it.n * kVocabTile + 16 * (Tl::NI * (wave % Tl::WN) + ni) + lane / 16 * 4;
  if (row >= q.head->n || c >= a.d) return;
  const float k = q.head->unscale;
  uint16_t* to = a.dX + q.list[row] * a.dxs + c;
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = (uint16_t)pack2<DT>(v[i] * k, 0.f);
}

// dW of a tile of the vocabulary over a piece's tokens.  first / last: of the call's pieces.  With several pieces the sums lie in fp32 in
// `sums` (dW itself if it is fp32) in between.
template <int DT>
__global__ __launch_bounds__(DwTile::kTileThreads, DwTile::kMinWaves) void vocab_dw(VocabArgs a, VocabPiece q, float* sums, bool first, bool last) {
  using Tl = DwTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  GridItem it;
  if (!xcd_item(blockIdx.x, (a.V + kVocabTile - 1) / kVocabTile, (a.d + kVocabTile - 1) / kVocabTile, it)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.m * kVocabTile, n0 = it.n * kVocabTile;
  VocabSrc<Tl> src;
  src.places(wave, q.ldp, a.d);
  src.step_b = 64 * q.ldp;
  src.step_a = 64ll * a.d;
#pragma unroll
  for (int u = 0; u < Tl::kIss; ++u) {
    const int g = wave + Tl::kWaves * u;
    if (u < Tl::kIssA)
      src.base[u] = q.p + (8 * (g % 8)) * q.ldp + i0 + g / 8 * 64;
    else                     // columns past the edge: the last 64 again, not stored
      src.base[u] = q.x + (long long)(8 * (g % 8)) * a.d + min(n0 + (g / 8 - Tl::TM) * 64, a.d - 64);
  }
  const int wm = wave / Tl::WN, wn = wave % Tl::WN, lane = threadIdx.x % kWave;
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  run_tile<Tl, DT>((q.head->n + 63) / 64, lds_addr(ring), wm, wn, src, acc);
  const float k = q.head->unscale;
  const int r0 = i0 + 16 * Tl::TI * wm, c0 = n0 + 16 * Tl::NI * wn;
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti)
#pragma unroll
    for (int ni = 0; ni < Tl::NI; ++ni) {
      const int r = r0 + 16 * ti + lane % 16, c = c0 + 16 * ni + lane / 16 * 4;
      acc[ni][ti] *= k;
      if (!sums || r >= a.V || c >= a.d) continue;
      f32x4* to = reinterpret_cast<f32x4*>(sums + (long long)r * a.d + c);
      if (!first) acc[ni][ti] += *to;
      if (a.dw_f32 || !last) *to = acc[ni][ti];
    }
  if (a.dw_f32 || !last) return;
  lds_barrier();       // nobody reads the ring any more
  uint16_t* out = (uint16_t*)a.dW;
  rows_out<Tl>(lds_addr(ring),
               [&](int ni, int ti) {
                 const f32x4 v = acc[ni][ti];
                 return make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
               },
               [&](int row, int at, uint4 v) {
                 if (r0 + row < a.V && c0 + at * 8 < a.d) *reinterpret_cast<uint4*>(out + (long long)(r0 + row) * a.d + c0 + at * 8) = v;
               });
}

// ---- launches --------------------------------------------------------------------------------------

template <int DT>
static hipError_t vocab_piece(const VocabArgs& a, const VocabPiece& q, bool first, bool last, hipStream_t st) {
  const int GN = (a.V + kVocabTile - 1) / kVocabTile, GD = (a.d + kVocabTile - 1) / kVocabTile, GM = (q.count + kVocabTile - 1) / kVocabTile;
  const bool grads = a.dX || a.dW, vec = ((uintptr_t)a.X | (uintptr_t)(a.xs * 2) | (uintptr_t)a.dX | (uintptr_t)(a.dxs * 2)) % 16 == 0;
  const int gather = (q.count + 63) / 64 + (a.V % 64 ? 16 : 0);
  if (vec)
    hipLaunchKernelGGL(vocab_gather<true>, dim3(gather), dim3(256), 0, st, a, q);
  else
    hipLaunchKernelGGL(vocab_gather<false>, dim3(gather), dim3(256), 0, st, a, q);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int tiles = (GM * GN + 7) / 8 * 8, width = 16 * LogitTile::NI, units = GN * (kVocabTile / width), rows = (q.count + 63) / 64 * 64;
  if (grads) {
    hipLaunchKernelGGL((vocab_logits<LogitTile, DT, true>), dim3(tiles), dim3(LogitTile::kTileThreads), 0, st, a, q);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((vocab_rows_kernel<DT, true>), dim3(rows), dim3(256), units * sizeof(float), st, a, q, units, width);
  } else {
    hipLaunchKernelGGL((vocab_logits<LogitTile, DT, false>), dim3(tiles), dim3(LogitTile::kTileThreads), 0, st, a, q);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((vocab_rows_kernel<DT, false>), dim3(rows), dim3(256), 0, st, a, q, units, width);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.dX) {
    const int whole = (GM * GD + 7) / 8 * 8;
    hipLaunchKernelGGL(vocab_dx<DT>, dim3(whole + kCUs), dim3(DxTile::kTileThreads), 0, st, a, q);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int most = GM * GD < kCUs / 2 ? GM * GD : kCUs / 2;      // (more are not cut)
    hipLaunchKernelGGL(vocab_dx_sum<DT>, dim3(most, DxTile::kWaves, DxTile::NI), dim3(256), 0, st, a, q);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.dW) {
    float* sums = a.dw_f32 ? (float*)a.dW : first && last ? nullptr : q.dw;
    hipLaunchKernelGGL(vocab_dw<DT>, dim3((GN * GD + 7) / 8 * 8), dim3(DwTile::kTileThreads), 0, st, a, q, sums, first, last);
    e = hipGetLastError();
  }
  return e;
}

hipError_t launch_vocab_loss(const VocabArgs& a, const VocabRoom& room, void* ws, hipStream_t st) {
  ProfScope prof(kKVocab, st);
  char* at = (char*)ws;
  VocabPiece q = {};
  q.head = (VocabHead*)(at + room.head), q.list = (int*)(at + room.list), q.target = (int*)(at + room.target);
  q.weight = (float*)(at + room.weight), q.at = (float*)(at + room.at), q.stats = (float2*)(at + room.stats);
  q.x = (uint16_t*)(at + room.x), q.tail = (uint16_t*)(at + room.tail), q.p = (uint16_t*)(at + room.p), q.part = (f32x4*)(at + room.part);
  q.dw = (float*)(at + room.dw);
  q.rows = room.rows, q.units = room.units, q.ldp = room.ldp;
  for (int t = 0; t < a.T; t += room.rows) {
    q.first = t;
    q.count = a.T - t < room.rows ? a.T - t : room.rows;
    const bool last = t + q.count == a.T;
    const hipError_t e = a.dt == kF16 ? vocab_piece<kF16>(a, q, t == 0, last, st) : vocab_piece<kBf16>(a, q, t == 0, last, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace lx
