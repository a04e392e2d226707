// Loss over a vocabulary with its gradients, 16-bit operands:  z = X W^T,  loss = log sum exp z - z_target,
// G = weight (softmax(z) - [target]),  dX = G W,  dW = G^T X.
//
// Three products of 2 n V d operations, n the number of tokens that have a target, which bound the call; nothing of the size of
// z outlives a piece of the tokens, whose exponentials lie in the workspace in 16 bits:
//   gather  the tokens that have a target, one after the other: the others are not multiplied, and what they hold has no effect; the
//           target's z by itself, in 64 bits, for all of a small loss hangs on it
//   logits  z, tile by tile in registers; of each token and unit of columns, the target's column left out, a reference and the sum of
//           exp(z - reference), in fp32; the exponentials in 16 bits.  References, see Kept below, are a unit's own or the token's.
//   rows    the loss; the exponentials, where they are not relative to one reference, in place times what they lack: G
//   dX, dW  products of G
// The target's column is made from the other columns' sum, so that a token whose target is all but certain has an exact gradient, and
// an exact loss by log1p.  It is most of a token's G, as a rule, and what its rounding to 16 bits takes away is made up: in dX, a single row
// of W's, at the end; in dW, rows of X, by further steps of the product (lacks below).
#include <type_traits>

#include "ffn_tile.h"
#include "log_steps.h"
#include "vocab.h"

namespace lx {

constexpr float kLog2e = 1.4426950408889634f;
// Half precision: gradients are scaled by a power of two, so that the largest weight's are at most 2^14.
constexpr float kHalfTop = 16384.f;

// How the exponentials are kept.
//   kNot     not at all: no gradients
//   kApart   relative to the unit's largest z, times 2^15, in half precision, which has the range of the G that it is for; rows makes G of
//            them in place, which moves a piece's exponentials twice
//   kSteps   bfloat16: the same, as steps of their logarithm (log_steps.h), which has bfloat16's range and half precision's error: a rounding that
//            is lost beside that of G to bfloat16
//   kOne     bfloat16, which has the range of fp32: relative to one number per token, about the target's z, so that they are G but for a
//            factor of the row, which dX takes at its end.  A unit whose exponentials add up to 2^60 or more takes them as many powers of
//            two lower as bring its largest to 1, and rows brings that token's others to the lowest ones, by a power of two again: no bit of
//            them is rounded twice.  (2^60: the row's factor stays a normal number for weights down to 2^-51, and the sums of dX stay in
//            range with W up to 2^50.)  For dW the factor would be one of the contraction's index.
// 8192 tokens, 60 % with a target, d = 2048, 50272 rows, bfloat16: rows 181 us with kSteps (175 in half precision with kApart), 10 with kOne.
enum Kept { kNot, kApart, kSteps, kOne };
constexpr bool in_place(Kept k) { return k == kApart || k == kSteps; }

struct VocabHead {       // of a piece
  int n;                 // tokens that have a target
  float scale, unscale;  // of G
};

// Pointers into the workspace.
struct VocabPiece {
  VocabHead* head;
  int *list, *target;
  double* z;             // per token: its target's z
  float* weight;
  float *factor, *lacks; // what dX's rows are multiplied with, and how much of W's row of the target they lack
  float2* stats;         // [rows][units]: reference (with kOne: powers of two above the token's), sum
  uint16_t *x, *tail, *p;
  int2* spans;           // dW: of each tile of the vocabulary where its tokens start in order and lo, and their number
  int* order;            // tokens by the tile of their target
  uint16_t* lo;          // [tokens in that order][columns of a tile]: what G lacks
  f32x4* part;
  float* dw;
  int units, first, count;      // the piece's tokens: first .. first + count - 1 of the call's
  long long ldp;
  long long slots;       // elements of the pieces of dX and dW
};

// ---- gather ----------------------------------------------------------------------------------------

// `per` tokens to a workgroup, which counts the targets before its own, a wavefront takes one row after the other; the workgroups behind those
// copy the last V % 64 rows of W and zeros into a block of 64 rows of their own, which the products read in their place.
// At most kGatherWorkgroups, a row to a wavefront while they suffice: small calls are a chain of loads, and in large ones the counting is
// what costs.  777 tokens of 768 elements 7.2 us (four rows at a time to a wavefront: 11.3), 8192 of 2048 24 (40; with 2048 workgroups 28), 65536 of
// 768 76 (378; 101).
constexpr int kGatherWorkgroups = 1024;
template <bool VEC>
__device__ __forceinline__ uint4 load8(const uint16_t* p) {
  if constexpr (VEC) return *reinterpret_cast<const uint4*>(p);
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = (uint32_t)p[2 * k] | (uint32_t)p[2 * k + 1] << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool VEC>
__device__ __forceinline__ void store8(uint16_t* p, uint4 v) {
  if constexpr (VEC) {
    *reinterpret_cast<uint4*>(p) = v;
  } else {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = (uint16_t)(w[k / 2] >> 16 * (k % 2));
  }
}
// Eight products of 16-bit elements added in 64 bits.
template <int DT>
__device__ __forceinline__ double dot8(const uint4& u, const uint4& v, double sum) {
  const uint32_t x[4] = {u.x, u.y, u.z, u.w}, y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum = fma((double)to_f32<DT>(x[i] & 0xffff), (double)to_f32<DT>(y[i] & 0xffff), sum);
    sum = fma((double)to_f32<DT>(x[i] >> 16), (double)to_f32<DT>(y[i] >> 16), sum);
  }
  return sum;
}
// f(t, targets[t]) of all t < n, a workgroup's threads in turn, eight loads of each on their way at once (the last turns of an unrolled loop come one by one: 8192 tokens of
// 2048 elements gathered in 34 us instead of 24).
template <int THREADS, class F>
__device__ __forceinline__ void each_target(const int* targets, int n, F f) {
  for (int first = threadIdx.x; first < n; first += 8 * THREADS) {
    int v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = first + i * THREADS < n ? targets[first + i * THREADS] : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (first + i * THREADS < n) f(first + i * THREADS, v[i]);
  }
}
// top: of the weights.  G's scale is a power of two; bfloat16 has the range of fp32.
template <int DT>
__device__ __forceinline__ VocabHead head(int n, float top) {
  float s = 1.f;
  if (DT == kF16 && top > 0 && top < 3e38f) s = exp2f(floorf(log2f(kHalfTop / top)));
  s = fminf(fmaxf(s, 0x1p-100f), 0x1p100f);
  return {n, s, 1.f / s};
}
// A row by a wavefront, zeros where `from` is null.
template <bool FROM, bool TO>
__device__ __forceinline__ void copy_row(uint16_t* to, const uint16_t* from, int d) {
  const int lane = threadIdx.x % kWave;
  if (from) {
#pragma unroll 4
    for (int c = lane * 8; c < d; c += 8 * kWave) store8<TO>(to + c, load8<FROM>(from + c));
  } else {
#pragma unroll 4
    for (int c = lane * 8; c < d; c += 8 * kWave) store8<TO>(to + c, make_uint4(0, 0, 0, 0));
  }
}
template <bool VEC, int DT>
__global__ __launch_bounds__(256) void vocab_gather(VocabArgs a, VocabPiece q, int per) {
  __shared__ int counts[2][4];
  __shared__ float tops[4];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, chunks = (q.count + per - 1) / per;
  const int first = blockIdx.x * per;
  if ((int)blockIdx.x >= chunks) {
    const int r0 = a.V / 64 * 64, r = ((int)blockIdx.x - chunks) * 4 + wave;
    return copy_row<true, true>(q.tail + (long long)r * a.d, r0 + r < a.V ? a.W + (long long)(r0 + r) * a.d : nullptr, a.d);
  }
  const int* targets = a.targets + q.first;
  const float* weights = a.weights ? a.weights + q.first : nullptr;
  int before = 0, all = 0;
  float top = 0;
  each_target<256>(targets, q.count, [&](int t, int target) {
    const bool held = (unsigned)target < (unsigned)a.V;
    all += held;
    before += held && t < first;
    if (DT == kF16 && blockIdx.x == 0 && held) top = fmaxf(top, weights ? fabsf(weights[t]) : 1.f);
  });
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
    if (threadIdx.x == 0) *q.head = head<DT>(all, top);
    // the rows up to the next 64, which dW's product reads
    if (a.dW)
      for (int r = all + wave; r < (all + 63) / 64 * 64; r += 4) copy_row<true, true>(q.x + (long long)r * a.d, nullptr, a.d);
  }
  const int mine = lane < per && first + lane < q.count ? targets[first + lane] : -1;
  const unsigned long long held = __ballot((unsigned)mine < (unsigned)a.V);
  if (wave == 0 && lane < per && first + lane < q.count) {
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
  for (int i = wave; i < per && first + i < q.count; i += 4) {
    const long long t = q.first + first + i;
    if (held >> i & 1) {
      const int place = before + __popcll(held & ((1ull << i) - 1));
      const uint16_t *x = a.X + t * a.xs, *w = a.W + (long long)__shfl(mine, i) * a.d;
      uint16_t* to = q.x + (long long)place * a.d;
      double dot = 0;
#pragma unroll 4
      for (int c = lane * 8; c < a.d; c += 8 * kWave) {
        const uint4 v = load8<VEC>(x + c);
        dot = dot8<DT>(v, load8<true>(w + c), dot);
        store8<true>(to + c, v);
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) dot += __shfl_xor(dot, o);
      if (lane == 0) q.z[place] = dot;
    } else if (a.dX) {
      copy_row<true, VEC>(a.dX + t * a.dxs, nullptr, a.d);
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
  int first, steps;        // the contraction starts at step `first` and goes round: see first_step
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
    first = 0;
    steps = 0x7fffffff;
  }
  __device__ __forceinline__ void begin(int s) {
    s += first;
    if (s >= steps) s -= steps;
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
// dW's, of `main` steps and then those of what G lacks: another buffer for the first operand, rows of X in the order of `order` for the second one.
template <class Tl>
struct DwSrc : VocabSrc<Tl> {
  const int* order;
  int main, width, ld, token;      // width, ld: elements between memory's rows, of what lacks and of X; the lane's token of the next such step
  long long far, back;             // from base to there
  __device__ __forceinline__ void begin(int s) {
    if (s < main) {
      this->off_b = s * this->step_b;
      this->off_a = s * this->step_a;
      return;
    }
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, lr = lane / 8, swz = ((lane % 8) ^ column_swz(8 * wave + lr)) << 4;
    this->off_b = far + (long long)(s - main) * (64 * width);
    this->off_a = back;
    this->voff_b = (uint32_t)(lr * width * 2 + swz);
    this->voff_a = (uint32_t)token * (uint32_t)(ld * 2) + (uint32_t)swz;      // (65536 rows of 65536 bytes at most)
    token = order[64 * (s - main + 1)];
  }
};
// Step numbers are those of the whole contraction; a part of it starts at `lo`.
template <class Src>
struct FromStep {
  Src& src;
  int lo;
  __device__ __forceinline__ void begin(int s) { src.begin(lo + s); }
  __device__ __forceinline__ void dma(int u, uint32_t lds) const { src.dma(u, lds); }
};

// The same of up to 64 tokens where they lie in X, an address per lane, and of W's rows alone: rows behind the last one are the last
// one again.
template <class Tl>
struct DirectSrc {
  const uint16_t* x[Tl::kIssA];
  const uint16_t* w;
  uint32_t voff[Tl::kIss - Tl::kIssA];
  long long off;
  int first, steps;      // as above
  __device__ __forceinline__ void begin(int s) {
    s += first;
    off = (long long)(s < steps ? s : s - steps) * kBK;
  }
  __device__ __forceinline__ void dma(int u, uint32_t lds) const {
    if (u < Tl::kIssA)
      dma16_v(x[u < Tl::kIssA ? u : 0] + off, lds + u * (Tl::kWaves * 1024));
    else
      dma16_s(w + off, voff[u < Tl::kIssA ? 0 : u - Tl::kIssA], lds + u * (Tl::kWaves * 1024));
  }
};

// Where the contraction of z's tiles starts.  Rows of W lie a power of two apart, as a rule, so that the same 128 bytes of all rows are in few
// of the memory's channels: workgroups that all start with them ask these alone.  With one tile of tokens every tile of the
// vocabulary starts a step further on (16 tokens, d = 2048, 50272 rows: 53.7 -> 41.4 us); with more, workgroups share the bytes
// that they read, and do not wait for the memory (an eighth further on per XCD: no difference).
__device__ __forceinline__ int first_step(int GM, int tile, int steps) { return GM == 1 ? tile % steps : 0; }

template <class Tl>
__device__ __forceinline__ void clear(typename Tl::Acc (&acc)[Tl::NI][Tl::TI]) {
#pragma unroll
  for (int x = 0; x < Tl::NI; ++x)
#pragma unroll
    for (int y = 0; y < Tl::TI; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// 16 of a wavefront's rows, 16 NI results each -> its own part of LDS as 16-bit elements, four consecutive columns of a row at a time
// (pack(ni)), and from there in runs of 16 bytes, whole rows of 32 NI bytes next to one another: put(row, slot, run).
template <class Tl, class Pack, class Put>
__device__ __forceinline__ void rows_out(uint32_t lds, int ti, Pack pack, Put put) {
  constexpr int kSlots = 2 * Tl::NI;
  const int lane = threadIdx.x % kWave, r = lane % 16, q = lane / 16;
  const uint32_t mine = lds + (uint32_t)(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * Tl::TI + ti) * (16 * kSlots * 16);
#pragma unroll
  for (int ni = 0; ni < Tl::NI; ++ni)
    lds_write8(mine + (uint32_t)(r * kSlots + ((2 * ni + q / 2) ^ (r & (kSlots - 1)))) * 16 + q % 2 * 8, pack(ni));
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (no other wavefront writes or reads there)
#pragma unroll
  for (int x = 0; x < (16 * kSlots + kWave - 1) / kWave; ++x) {
    const int at = x * kWave + lane, row = at / kSlots, slot = at % kSlots;
    if (16 * kSlots % kWave == 0 || row < 16) put(16 * ti + row, slot, lds_read16(mine + (uint32_t)(row * kSlots + (slot ^ (row & (kSlots - 1)))) * 16));
  }
}

// The tiles of vocab_plan.h, as in the FFN's products.   TM TN WM WN NST PH; COLUMNS_A, COLUMNS_B: the operands that lie as columns
template <int ID, bool COLUMNS_A, bool COLUMNS_B>
struct TileOf;
template <bool A, bool B>
struct TileOf<kT44, A, B> { using T = Tile<4, 4, 4, 2, 2, 2, 2, 16, A, B>; };
template <bool A, bool B>
struct TileOf<kT24, A, B> { using T = Tile<2, 4, 2, 4, 3, 2, 2, 16, A, B>; };
template <bool A, bool B>
struct TileOf<kT14Deep, A, B> { using T = Tile<1, 4, 2, 4, 4, 2, 2, 16, A, B>; };
template <>
struct TileOf<kT12, false, false> { using T = Tile<1, 2, 1, 4, 3, 2>; };
template <>
struct TileOf<kT11, false, false> { using T = Tile<1, 1, 2, 2, 4, 2>; };
template <>
struct TileOf<kT11, true, false> { using T = Tile<1, 1, 4, 1, 4, 2, 2, 16, true, false>; };      // (whole groups of 64 columns)

// A piece's results: [wavefront][accumulator][lane][4 registers]
template <class Tl>
__device__ __forceinline__ void store_piece(f32x4* part, int slot, const typename Tl::Acc (&acc)[Tl::NI][Tl::TI]) {
  f32x4* to = part + ((size_t)slot * Tl::kWaves + threadIdx.x / kWave) * (Tl::NI * Tl::TI) * kWave + threadIdx.x % kWave;
#pragma unroll
  for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
    for (int ti = 0; ti < Tl::TI; ++ti) to[(ni * Tl::TI + ti) * kWave] = acc[ni][ti];
}
// Four results of a cut unit, its pieces added in order, with their row and column: accumulator blockIdx.z, threadIdx / 64 of wavefront
// blockIdx.y.  (A workgroup to all 16-column groups of a wavefront takes 46 us for 125 MB, one to each 34; in a whole call 41.)
template <class Tl>
__device__ __forceinline__ f32x4 add_pieces(const CutPlan& p, const f32x4* part, int& row, int& column) {
  const GridItem it = grid_item(p.full + blockIdx.x, p.GM, p.GN, 4);
  const int lane = threadIdx.x % kWave, wave = blockIdx.y, ni = blockIdx.z, ti = threadIdx.x / kWave;
  const f32x4* from = part + (((size_t)blockIdx.x * p.pieces * Tl::kWaves + wave) * (Tl::NI * Tl::TI) + ni * Tl::TI + ti) * kWave + lane;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = 0; i < p.pieces; ++i) v += from[(size_t)i * (Tl::kWaves * Tl::NI * Tl::TI * kWave)];
  row = it.m * 64 * Tl::TM + 16 * (Tl::TI * (wave / Tl::WN) + ti) + lane % 16;
  column = it.n * 64 * Tl::TN + 16 * (Tl::NI * (wave % Tl::WN) + ni) + lane / 16 * 4;
  return v;
}

// kOne: what a token's exponentials are relative to.
__device__ __forceinline__ float one_reference(double z) { return (float)z == -INFINITY ? 0.f : (float)z; }

// The statistics of a tile's z, and its exponentials.  target(t, ti): of token t, -1 behind the last one.
template <class Tl, Kept KEPT, class Target>
__device__ __forceinline__ void logits_out(const VocabArgs& a, const VocabPiece& q, int n, int i0, int n0, int wm, int wn, uint32_t ring,
                                           Target target, typename Tl::Acc (&acc)[Tl::NI][Tl::TI]) {
  // a lane: columns c0 + 16 ni + v of its tokens t0 + 16 ti
  const int lane = threadIdx.x % kWave, t0 = i0 + 16 * Tl::TI * wm + lane % 16, u0 = n0 + 16 * Tl::NI * wn, c0 = u0 + lane / 16 * 4;
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
  uint16_t* p = q.p + (long long)(i0 + 16 * Tl::TI * wm) * q.ldp + u0;
  if (KEPT != kNot) lds_barrier();       // nobody reads the ring any more
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti) {
    const int t = t0 + 16 * ti, rel = target(t, ti) - c0;
    // the target, if it is here, is taken out: beside one that is all but certain the others would vanish in half precision
    const bool here = rel >= 0 && rel < 16 * Tl::NI && rel % 16 < 4;
    if (__ballot(here)) {
#pragma unroll
      for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          acc[ni][ti][v] = rel == 16 * ni + v ? -INFINITY : acc[ni][ti][v];      // (a select: as a branch the accumulators go through scratch memory)
    }
    float ref = KEPT == kOne && t < n ? one_reference(q.z[t]) : 0.f, up = KEPT == kOne ? 0.f : 15.f, sum = 0;
    auto largest = [&] {
      float top = acc[0][ti][0];
#pragma unroll
      for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
        for (int v = 0; v < 4; ++v) top = fmaxf(top, acc[ni][ti][v]);
      top = fmaxf(top, __shfl_xor(top, 16));
      return fmaxf(top, __shfl_xor(top, 32));
    };
    f32x4 e[Tl::NI];       // with kSteps their steps
    auto exponentials = [&](float from) {
      sum = 0;
#pragma unroll
      for (int ni = 0; ni < Tl::NI; ++ni)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float y = acc[ni][ti][v] - from, x = __builtin_amdgcn_exp2f(fmaf(y, kLog2e, up));
          sum += x;
          e[ni][v] = KEPT == kSteps ? log_step(y) : x;
        }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
    };
    auto own = [&] {
      ref = largest();
      exponentials(ref == -INFINITY ? 0.f : ref);      // (nothing but the target, or columns behind the vocabulary)
    };
    if constexpr (KEPT == kOne) {
      exponentials(ref);
      const bool far = !(sum < 0x1p60f);      // (NaN too)
      if (__ballot(far)) {
        const float top = largest();
        if (far) up = -ceilf((top - ref) * kLog2e);
        exponentials(ref);
      }
      ref = -up;
    } else {
      own();
      sum *= 0x1p-15f;
    }
    if (lane < 16 && t < n) q.stats[(long long)t * q.units + unit] = make_float2(ref, sum);
    // (each 16 tokens on their way while the next ones' exponentials are made)
    auto pair = [&](float lo, float hi) {
      if constexpr (KEPT == kSteps)
        return (__builtin_bit_cast(uint32_t, lo) & 0xffffu) | __builtin_bit_cast(uint32_t, hi) << 16;
      else
        return pack2<(KEPT == kOne ? kBf16 : kF16)>(lo, hi);
    };
    if constexpr (KEPT != kNot)
      rows_out<Tl>(ring, ti, [&](int ni) { return make_uint2(pair(e[ni][0], e[ni][1]), pair(e[ni][2], e[ni][3])); },
                   [&](int row, int slot, uint4 v) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)(p + row * q.ldp + slot * 8)); });
  }
}

// z of a tile.  Bound by the matrix instructions, and after them by the exponentials, which nothing overlaps: a CU holds one tile of
// 256 x 256, and smaller ones read more.  4096 tokens, d = 4096, 50272 rows, half precision, no gradients: 1273 us, 1.33 PFLOP/s (the
// library's product alone, 8192 tokens, d = 2048: 1.19).  The stores 16 tokens at a time between the exponentials, and past the caches,
// took 979 to 898 at 4900 tokens, d = 2048, bfloat16.
template <class Tl, int DT, Kept KEPT>
__global__ __launch_bounds__(Tl::kTileThreads, Tl::kMinWaves) void vocab_logits(VocabArgs a, VocabPiece q) {
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  const int n = q.head->n, GM = ceil_div(n, 64 * Tl::TM), GN = ceil_div(a.V, 64 * Tl::TN);
  GridItem it;
  if (!xcd_item(blockIdx.x, GM, GN, it)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.m * 64 * Tl::TM, n0 = it.n * 64 * Tl::TN;
  VocabSrc<Tl> src;
  src.places(wave, a.d, a.d);
  src.step_b = src.step_a = kBK;
  src.steps = a.d / kBK;
  src.first = first_step(GM, it.n, src.steps);
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
  const int wm = wave / Tl::WN, wn = wave % Tl::WN;
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  run_tile<Tl, DT>(a.d / kBK, lds_addr(ring), wm, wn, src, acc);
  logits_out<Tl, KEPT>(a, q, n, i0, n0, wm, wn, lds_addr(ring), [&](int t, int) { return t < n ? q.target[t] : -1; }, acc);
}

// z of up to 64 tokens with nothing gathered before: every workgroup finds the tokens that have a target, the first one writes down
// which they are, and those behind the tiles, kFewRows wavefronts, bring what the gradients read.  16 tokens, d = 2048, 50272 rows, no
// gradients: the gathering launch was 9.4 of 62 us.
constexpr int kFewRows = 3 * 64;
template <class Tl, int DT, Kept KEPT>
__global__ __launch_bounds__(Tl::kTileThreads, Tl::kMinWaves) void vocab_logits_few(VocabArgs a, VocabPiece q, int tiles) {
  static_assert(Tl::TM == 1, "one tile of tokens");
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, n0 = blockIdx.x * 64 * Tl::TN;
  const int mine = lane < q.count ? a.targets[q.first + lane] : -1;
  const unsigned long long all = __ballot((unsigned)mine < (unsigned)a.V);
  const int n = __popcll(all);
  const bool held = all >> lane & 1;
  int* list = reinterpret_cast<int*>(ring);
  const int rank = __popcll(all & ((1ull << lane) - 1));
  if (wave == 0 && held) list[rank] = lane, list[64 + rank] = mine;
  if (blockIdx.x == 0 && wave == 0) {
    const long long t = q.first + lane;
    const float weight = held && a.weights ? a.weights[t] : held ? 1.f : 0.f;
    float top = fabsf(weight);
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    if (lane == 0) *q.head = head<DT>(n, top);
    if (held) {
      q.list[rank] = (int)t;
      q.target[rank] = mine;
      q.weight[rank] = weight;
    } else if (lane < q.count) {
      a.loss[t] = 0.f;
      if (a.lse) a.lse[t] = 0.f;
    }
  }
  __syncthreads();
  if constexpr (KEPT != kNot)
    if ((int)blockIdx.x >= tiles) {      // W's last rows; X for dW; dX of tokens without a target
      const int job = ((int)blockIdx.x - tiles) * Tl::kWaves + wave, r = job % 64, last = a.V / 64 * 64;
      if (job < 64) {
        if (last < a.V) copy_row<true, true>(q.tail + (long long)r * a.d, last + r < a.V ? a.W + (long long)(last + r) * a.d : nullptr, a.d);
      } else if (job < 128) {
        if (a.dW && n) copy_row<true, true>(q.x + (long long)r * a.d, r < n ? a.X + (q.first + list[r]) * a.xs : nullptr, a.d);
      } else if (job < kFewRows) {
        if (a.dX && r < q.count && !(all >> r & 1)) copy_row<true, true>(a.dX + (long long)(q.first + r) * a.dxs, nullptr, a.d);
      }
      return;
    }
  if (n == 0) return;
  DirectSrc<Tl> src;
  const int lr = lane / 8;
#pragma unroll
  for (int u = 0; u < Tl::kIss; ++u) {
    const int g = wave + Tl::kWaves * u;
    const int seg = ((lane % 8) ^ tile_swz<Tl>(lr)) * 8;
    if (u < Tl::kIssA)
      src.x[u < Tl::kIssA ? u : 0] = a.X + (q.first + list[min(8 * g + lr, n - 1)]) * a.xs + seg;
    else
      src.voff[u < Tl::kIssA ? 0 : u - Tl::kIssA] = (uint32_t)(((long long)(min(n0 + 8 * (g - 8) + lr, a.V - 1) - n0) * a.d + seg) * 2);
  }
  src.w = a.W + (long long)n0 * a.d;
  src.steps = a.d / kBK;
  src.first = first_step(1, blockIdx.x, src.steps);
  const int wm = wave / Tl::WN, wn = wave % Tl::WN;
  int targets[Tl::TI];
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti) {
    const int t = 16 * (Tl::TI * wm + ti) + lane % 16;
    targets[ti] = t < n ? list[64 + t] : -1;
  }
  __syncthreads();       // the ring is filled over the list
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  run_tile<Tl, DT>(a.d / kBK, lds_addr(ring), wm, wn, src, acc);
  logits_out<Tl, KEPT>(a, q, n, 0, n0, wm, wn, lds_addr(ring), [&](int, int ti) { return targets[ti]; }, acc);
}

// A token's statistics joined, its loss, and what its row of G lacks.  units: of `width` columns each; direct: nothing was gathered,
// and z is made here.  summing: threads that add statistics.  Few rows: gridDim.y workgroups make G, a part of the row each (17 rows of 39596 elements 13.6 -> 8.8 us).
constexpr int kRowThreads = 512;      // at most: as many as have something to do
constexpr int kFactors = 2048;        // units at a time
template <int DT, Kept KEPT>
__global__ __launch_bounds__(kRowThreads) void vocab_rows_kernel(VocabArgs a, VocabPiece q, int units, int width, int summing, bool direct) {
  __shared__ float factors[kFactors], tops[kRowThreads / kWave], sums[kRowThreads / kWave];
  __shared__ double dots[kRowThreads / kWave];
  __shared__ int apart;      // kOne: whether references differ
  const int threads = blockDim.x;
  const int n = q.head->n, t = blockIdx.x, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  if (t >= n) {      // rows up to the next 64, which dW's product reads
    if (in_place(KEPT) && blockIdx.y == 0 && t < (n + 63) / 64 * 64)
      for (long long c = threadIdx.x * 8; c < q.ldp; c += 8 * threads) *reinterpret_cast<uint4*>(q.p + t * q.ldp + c) = make_uint4(0, 0, 0, 0);
    return;
  }
  const float2* stats = q.stats + (long long)t * q.units;
  const int target = q.target[t];
  const long long token = q.list[t];
  // the thread's units, eight at a time, which are all of them but in the largest vocabularies
  const int own = (int)threadIdx.x < summing ? threadIdx.x : units;
  float2 s[8];
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = first + i * summing < units ? stats[first + i * summing] : make_float2(-INFINITY, 0.f);
  };
  double z = 0;
  float top = -INFINITY, sum = 0;
  if (KEPT == kOne && threadIdx.x == 0) apart = 0;
  if (direct)
    for (int c = threadIdx.x * 8; c < a.d; c += 8 * threads)
      z = dot8<DT>(load8<true>(a.X + token * a.xs + c), load8<true>(a.W + (long long)target * a.d + c), z);
  for (int first = own; first < units; first += 8 * summing) {
    load(first);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, s[i].x);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    top = fmaxf(top, __shfl_xor(top, o));
    if (direct) z += __shfl_xor(z, o);
  }
  if (lane == 0) tops[wave] = top, dots[wave] = z;
  __syncthreads();
  z = direct ? 0 : q.z[t];
  for (int k = 0; k < threads / kWave; ++k) top = fmaxf(top, tops[k]), z += direct ? dots[k] : 0;
  // All is relative to the largest reference, or to the target's z where that is larger; with kOne that is not above the reference.
  if (KEPT != kOne) top = fmaxf(top, (float)z);
  auto above = [&](float ref) {
    if (ref == top) return 1.f;
    return KEPT == kOne ? ldexpf(1.f, (int)fmaxf(ref - top, -1000.f)) : expf(ref - top);
  };
  bool differ = false;
  for (int first = own; first < units; first += 8 * summing) {
    if (units > 8 * summing) load(first);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum = fmaf(s[i].y, above(s[i].x), sum);
      differ |= s[i].x != top && first + i * summing < units;
    }
  }
  if (KEPT == kOne && differ) apart = 1;
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = 0;
  for (int k = 0; k < threads / kWave; ++k) sum += sums[k];      // of all but the target
  const double at = KEPT == kOne ? (double)one_reference(z) + (double)top * 0.69314718055994530942 : (double)top;
  const float behind = (float)(at - z), mine = expf(-behind), total = sum + mine;
  const float weight = KEPT == kNot ? 0.f : q.weight[t], g = -weight * (sum / total);      // G in the target's place
  if (threadIdx.x == 0 && blockIdx.y == 0) {
    a.loss[token] = mine > 0.5f * total ? log1pf(sum / mine) : behind + logf(total);
    if (a.lse) a.lse[token] = (float)at + logf(total);
  }
  if constexpr (KEPT == kNot) return;
  uint16_t* p = q.p + t * q.ldp;
  if constexpr (KEPT == kOne) {
    if (threadIdx.x == 0) q.factor[t] = weight / total, q.lacks[t] = g;
    if (!apart) return;      // (0 in the target's place)
  }
  const float scale = KEPT == kOne ? 1.f : q.head->scale, f = KEPT == kOne ? 1.f : weight * scale / total * (KEPT == kApart ? 0x1p-15f : 1.f);
  if (in_place(KEPT) && threadIdx.x == 0 && blockIdx.y == 0) {
    q.factor[t] = q.head->unscale;
    q.lacks[t] = g - to_f32<DT>(pack2<DT>(g * scale, 0.f) & 0xffff) * q.head->unscale;
  }
  auto kept = [](uint32_t x) {
    if constexpr (KEPT == kSteps)
      return __builtin_amdgcn_exp2f(step_log2(x));
    else
      return to_f32<KEPT == kOne ? kBf16 : kF16>(x);
  };
  // kOne: the difference of two references may be more powers of two than a factor holds, where exponentials of 2^59 are still numbers after it.
  auto times = [](float x, float k) { return KEPT == kOne ? ldexpf(x, (int)fmaxf(k, -1000.f)) : x * k; };
  const int part = ceil_div(units, (int)gridDim.y), last = min((int)(blockIdx.y + 1) * part, units);
  for (int u0 = blockIdx.y * part; u0 < last; u0 += kFactors) {
    const int u1 = min(u0 + kFactors, last);
    for (int u = u0 + (int)threadIdx.x; u < u1; u += threads) {
      factors[u - u0] = KEPT == kOne ? stats[u].x - top : above(stats[u].x) * f;
    }
    __syncthreads();
#pragma unroll 4
    for (int c = u0 * width + (int)threadIdx.x * 8; c < u1 * width; c += 8 * threads) {
      const float k = factors[c / width - u0];
      const uint4 v = *reinterpret_cast<const uint4*>(p + c);
      const uint32_t in[4] = {v.x, v.y, v.z, v.w};
      float e[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) e[2 * i] = times(kept(in[i] & 0xffff), k), e[2 * i + 1] = times(kept(in[i] >> 16), k);
      if (in_place(KEPT) && target - c >= 0 && target - c < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (target - c == i) e[i] = g * scale;
      *reinterpret_cast<uint4*>(p + c) = make_uint4(pack2<DT>(e[0], e[1]), pack2<DT>(e[2], e[3]), pack2<DT>(e[4], e[5]), pack2<DT>(e[6], e[7]));
    }
    __syncthreads();
  }
}

// What G's rounding in the targets' columns takes from dW, as further indices of its contraction: of each tile of `width` rows of the
// vocabulary the tokens whose target is one of them, in their order and filled up to the next 64 with zeros, the token itself and a row with what G
// lacks.  A tile's tokens start behind those of smaller targets, 64 for each tile before, so that nobody waits for another one's
// number.  gridDim.y shares of the tokens.  dW in bfloat16 is 2.4e-3 of its norm off without them, 1.7e-3 with them, which is its own rounding.
constexpr int kLackThreads = 512;
template <int DT>
__global__ __launch_bounds__(kLackThreads) void vocab_lacks(VocabArgs a, VocabPiece q, int width) {
  constexpr int kWaves = kLackThreads / kWave;
  __shared__ int counts[3][kWaves], found[kWaves], columns[kLackThreads];
  __shared__ uint32_t values[kLackThreads];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, v0 = blockIdx.x * width, n = q.head->n;
  const int t0 = (int)((long long)n * blockIdx.y / gridDim.y), t1 = (int)((long long)n * (blockIdx.y + 1) / gridDim.y);
  int below = 0, all = 0, before = 0;
  each_target<kLackThreads>(q.target, n, [&](int t, int target) {
    const bool in = (unsigned)(target - v0) < (unsigned)width;
    below += target < v0, all += in, before += in && t < t0;
  });
#pragma unroll
  for (int o = 32; o; o >>= 1) below += __shfl_xor(below, o), all += __shfl_xor(all, o), before += __shfl_xor(before, o);
  if (lane == 0) counts[0][wave] = below, counts[1][wave] = all, counts[2][wave] = before;
  __syncthreads();
  below = all = before = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) below += counts[0][w], all += counts[1][w], before += counts[2][w];
  const int start = below + 64 * blockIdx.x;
  if (blockIdx.y == 0 && threadIdx.x == 0) q.spans[blockIdx.x] = make_int2(start, all);
  if (all == 0) return;
  // a row of zeros but for one element
  auto row = [&](int at, int column, uint32_t value) {
    for (int c = lane * 8; c < width; c += 8 * kWave) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (column == c + 2 * i ? value : 0) | (column == c + 2 * i + 1 ? value << 16 : 0);
      *reinterpret_cast<uint4*>(q.lo + (long long)at * width + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  };
  const float scale = q.head->scale;
  int at = start + before;
  for (int t = t0; t < t1; t += kLackThreads) {
    const int mine = t + (int)threadIdx.x, column = mine < t1 ? q.target[mine] - v0 : -1;
    const bool in = (unsigned)column < (unsigned)width;
    const unsigned long long held = __ballot(in);
    if (lane == 0) found[wave] = __popcll(held);
    __syncthreads();
    int rank = __popcll(held & ((1ull << lane) - 1)), sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) rank += w < wave ? found[w] : 0, sum += found[w];
    if (in) {
      q.order[at + rank] = mine;
      columns[rank] = column;
      values[rank] = pack2<DT>(q.lacks[mine] * scale, 0.f) & 0xffff;
    }
    __syncthreads();
    for (int k = wave; k < sum; k += kWaves) row(at + k, columns[k], values[k]);
    at += sum;
    __syncthreads();
  }
  if (blockIdx.y == gridDim.y - 1)
    for (int k = all + wave; k < (all + 63) / 64 * 64; k += kWaves) {
      row(start + k, -1, 0);
      if (lane == 0) q.order[start + k] = 0;
    }
}

// Four columns of a row of dX from the product's: times the row's factor, and what the target's column lacked.
template <int DT>
__device__ __forceinline__ uint2 dx_columns(const VocabArgs& a, const VocabPiece& q, int row, int column, const f32x4& v) {
  const float k = q.factor[row], lacks = q.lacks[row];
  const uint2 w = *reinterpret_cast<const uint2*>(a.W + (long long)q.target[row] * a.d + column);
  return make_uint2(pack2<DT>(fmaf(lacks, to_f32<DT>(w.x & 0xffff), v[0] * k), fmaf(lacks, to_f32<DT>(w.x >> 16), v[1] * k)),
                    pack2<DT>(fmaf(lacks, to_f32<DT>(w.y & 0xffff), v[2] * k), fmaf(lacks, to_f32<DT>(w.y >> 16), v[3] * k)));
}

// dX of a tile of tokens x columns: G's rows, W as columns by LDS's transposing reads.  Bound by the matrix instructions: 1213 us, 1.32 PFLOP/s,
// at 3900 tokens, d = 4096, 50272 rows, bfloat16, whose tiles are one round of workgroups; 1.16 at 4900 tokens, d = 2048, whose 160 tiles
// are cut into 480 pieces, two rounds (the library, 8192 tokens, d = 2048: 1.24).
template <int ID, int DT>
__global__ __launch_bounds__(512, 2) void vocab_dx(VocabArgs a, VocabPiece q) {
  using Tl = typename TileOf<ID, true, false>::T;      // W as columns
  static_assert(Tl::kTileThreads <= 512, "threads");
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  const CutPlan p = dx_plan(ID, q.head->n, a.d, a.V, q.slots);
  CutItem cut;
  if (!cut_item(p, blockIdx.x, cut)) return;
  const GridItem it = grid_item(cut.unit, p.GM, p.GN, 4);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.m * 64 * Tl::TM, n0 = it.n * 64 * Tl::TN;
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
  const int wm = wave / Tl::WN, wn = wave % Tl::WN;
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  FromStep<VocabSrc<Tl>> part = {src, cut.lo};
  run_tile<Tl, DT>(cut.hi - cut.lo, lds_addr(ring), wm, wn, part, acc);
  if (cut.slot >= 0) return store_piece<Tl>(q.part, cut.slot, acc);
  lds_barrier();       // nobody reads the ring any more
  const int n = q.head->n, r0 = i0 + 16 * Tl::TI * wm, c0 = n0 + 16 * Tl::NI * wn;
  const bool whole = ((uintptr_t)a.dX | (uintptr_t)(a.dxs * 2)) % 16 == 0;
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti) {
    const int mine = min(r0 + 16 * ti + (int)threadIdx.x % 16, n - 1), column = c0 + (int)threadIdx.x % kWave / 16 * 4;
    rows_out<Tl>(lds_addr(ring), ti, [&](int ni) { return dx_columns<DT>(a, q, mine, min(column + 16 * ni, a.d - 4), acc[ni][ti]); },
                 [&](int row, int at, uint4 v) {
                   if (r0 + row >= n || c0 + at * 8 >= a.d) return;
                   uint16_t* to = a.dX + q.list[r0 + row] * a.dxs + c0 + at * 8;
                   if (whole)
                     store8<true>(to, v);
                   else
                     store8<false>(to, v);
                 });
  }
}

// The pieces of dX's cut units added.
template <class Tl, int ID, int DT>
__global__ __launch_bounds__(64 * Tl::TI) void vocab_dx_sum(VocabArgs a, VocabPiece q) {
  const CutPlan p = dx_plan(ID, q.head->n, a.d, a.V, q.slots);
  if ((int)blockIdx.x >= p.rest) return;
  int row, c;
  const f32x4 v = add_pieces<Tl>(p, q.part, row, c);
  if (row >= q.head->n || c >= a.d) return;
  uint16_t* to = a.dX + q.list[row] * a.dxs + c;
  const uint2 w = dx_columns<DT>(a, q, row, c, v);
  if (((uintptr_t)a.dX | (uintptr_t)(a.dxs * 2)) % 8 == 0)
    *reinterpret_cast<uint2*>(to) = w;
  else
    to[0] = (uint16_t)w.x, to[1] = (uint16_t)(w.x >> 16), to[2] = (uint16_t)w.y, to[3] = (uint16_t)(w.y >> 16);
}

// dW of a tile of the vocabulary over a piece's tokens.  first / last: of the call's pieces.  With several pieces the sums lie in fp32 in
// `sums` (dW itself if it is fp32) in between.  Both operands lie as columns.  Bound as dX is: 1240 us, 1.29 PFLOP/s, as there
// (the library, 8192 tokens, d = 2048: 1.03).
template <int ID, int DT>
__global__ __launch_bounds__(512, 2) void vocab_dw(VocabArgs a, VocabPiece q, float* sums, bool first, bool last) {
  using Tl = typename TileOf<ID, true, true>::T;
  static_assert(Tl::kWaves == 8, "DwSrc: a wavefront brings the same eight indices by every instruction");
  __shared__ __attribute__((aligned(1024))) uint16_t ring[Tl::NST * Tl::kElems];
  const CutPlan p = dw_plan(ID, q.head->n, a.d, a.V, q.slots);
  CutItem cut;
  if (!cut_item(p, blockIdx.x, cut)) return;
  const GridItem it = grid_item(cut.unit, p.GM, p.GN, 4);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i0 = it.m * 64 * Tl::TM, n0 = it.n * 64 * Tl::TN;
  const int2 span = q.spans[it.m];
  DwSrc<Tl> src;
  src.places(wave, q.ldp, a.d);
  src.step_b = 64 * q.ldp;
  src.step_a = 64ll * a.d;
  src.main = cut.hi - cut.lo;
  src.width = 64 * Tl::TM;
  src.ld = a.d;
  src.order = q.order + span.x + threadIdx.x / 8;      // (a wavefront brings eight indices of each step)
  src.token = span.y ? src.order[0] : 0;
  src.back = -(64ll * cut.lo + 8 * wave) * a.d;
#pragma unroll
  for (int u = 0; u < Tl::kIss; ++u) {
    const int g = wave + Tl::kWaves * u;
    if (u < Tl::kIssA)
      src.base[u] = q.p + (64ll * cut.lo + 8 * (g % 8)) * q.ldp + i0 + g / 8 * 64;
    else                     // columns past the edge: the last 64 again, not stored
      src.base[u] = q.x + (64ll * cut.lo + 8 * (g % 8)) * a.d + min(n0 + (g / 8 - Tl::TM) * 64, a.d - 64);
  }
  src.far = q.lo + (long long)(span.x + 8 * wave) * src.width - src.base[0];      // (the same columns)
  const int wm = wave / Tl::WN, wn = wave % Tl::WN, lane = threadIdx.x % kWave;
  typename Tl::Acc acc[Tl::NI][Tl::TI];
  clear<Tl>(acc);
  run_tile<Tl, DT>(src.main + (cut.hi == p.steps ? ceil_div(span.y, 64) : 0), lds_addr(ring), wm, wn, src, acc);
  if (cut.slot >= 0) return store_piece<Tl>(q.part, cut.slot, acc);
  const float k = q.head->unscale;
  const int r0 = i0 + 16 * Tl::TI * wm, c0 = n0 + 16 * Tl::NI * wn, r = r0 + lane % 16, c = c0 + lane / 16 * 4;
  // the sum so far of the lane's four elements
  auto place = [&](int ni, int ti) { return reinterpret_cast<f32x4*>(sums + (long long)(r + 16 * ti) * a.d + c + 16 * ni); };
  auto held = [&](int ni, int ti) { return r + 16 * ti < a.V && c + 16 * ni < a.d; };
  if (a.dw_f32 || !last) {
#pragma unroll
    for (int ti = 0; ti < Tl::TI; ++ti)
#pragma unroll
      for (int ni = 0; ni < Tl::NI; ++ni) {
        if (!held(ni, ti)) continue;
        const f32x4 v = acc[ni][ti] * k;
        *place(ni, ti) = first ? v : v + *place(ni, ti);
      }
    return;
  }
  lds_barrier();       // nobody reads the ring any more
  uint16_t* out = (uint16_t*)a.dW;
#pragma unroll
  for (int ti = 0; ti < Tl::TI; ++ti)
    rows_out<Tl>(lds_addr(ring), ti,
                 [&](int ni) {
                   f32x4 v = acc[ni][ti] * k;
                   if (!first && held(ni, ti)) v += *place(ni, ti);
                   return make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
                 },
                 [&](int row, int at, uint4 v) {
                   if (r0 + row < a.V && c0 + at * 8 < a.d)
                     __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4*)(out + (long long)(r0 + row) * a.d + c0 + at * 8));
                 });
}

// The pieces of dW's cut units added.
template <class Tl, int ID, int DT>
__global__ __launch_bounds__(64 * Tl::TI) void vocab_dw_sum(VocabArgs a, VocabPiece q, float* sums, bool first, bool last) {
  const CutPlan p = dw_plan(ID, q.head->n, a.d, a.V, q.slots);
  if ((int)blockIdx.x >= p.rest) return;
  int row, c;
  f32x4 v = add_pieces<Tl>(p, q.part, row, c);
  if (row >= a.V || c >= a.d) return;
  v *= q.head->unscale;
  const long long at = (long long)row * a.d + c;
  if (sums) {
    f32x4* to = reinterpret_cast<f32x4*>(sums + at);
    if (!first) v += *to;
    if (a.dw_f32 || !last) {
      *to = v;
      return;
    }
  }
  *reinterpret_cast<uint2*>((uint16_t*)a.dW + at) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
}

// ---- launches --------------------------------------------------------------------------------------

template <class Tl, int DT, Kept KEPT>
static hipError_t launch_rows(const VocabArgs& a, const VocabPiece& q, hipStream_t st, bool direct = false) {
  constexpr int kWidth = 16 * Tl::NI;
  const int units = ceil_div(a.V, 64 * Tl::TN) * (64 * Tl::TN / kWidth), rows = in_place(KEPT) ? (q.count + 63) / 64 * 64 : q.count;
  // Eight units' statistics per thread, with and without gradients, so that the sums are the same; a run of 8 elements per thread and turn.
  // (4900 tokens of 393 units by a wavefront each 10.5 us, by seven 22.)
  auto waves = [](int work) { return work >= kRowThreads ? kRowThreads : ceil_div(work, kWave) * kWave; };
  const int summing = waves(ceil_div(units, 8)), threads = max(summing, waves(in_place(KEPT) ? (int)(q.ldp / 8) : direct ? a.d / 8 : 1));
  const int parts = in_place(KEPT) && rows < 2 * kCUs ? min(2 * kCUs / rows, ceil_div(units * kWidth, 8 * kRowThreads)) : 1;
  hipLaunchKernelGGL((vocab_rows_kernel<DT, KEPT>), dim3(rows, parts), dim3(threads), 0, st, a, q, units, kWidth, summing, direct);
  return hipGetLastError();
}
template <int ID, int DT, Kept KEPT>
static hipError_t launch_logits(const VocabArgs& a, const VocabPiece& q, hipStream_t st) {
  using Tl = typename TileOf<ID, false, false>::T;
  const int grid = eights(ceil_div(q.count, 64 * Tl::TM) * ceil_div(a.V, 64 * Tl::TN));
  hipLaunchKernelGGL((vocab_logits<Tl, DT, KEPT>), dim3(grid), dim3(Tl::kTileThreads), 0, st, a, q);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_rows<Tl, DT, KEPT>(a, q, st);
}
template <int DT, Kept KEPT>
static hipError_t launch_logits(int tile, const VocabArgs& a, const VocabPiece& q, hipStream_t st) {
  switch (tile) {
    case kT44: return launch_logits<kT44, DT, KEPT>(a, q, st);
    case kT24: return launch_logits<kT24, DT, KEPT>(a, q, st);
    case kT14Deep: return launch_logits<kT14Deep, DT, KEPT>(a, q, st);
    case kT12: return launch_logits<kT12, DT, KEPT>(a, q, st);
    default: return launch_logits<kT11, DT, KEPT>(a, q, st);
  }
}
template <int ID, int DT, Kept KEPT>
static hipError_t launch_logits_few(const VocabArgs& a, const VocabPiece& q, hipStream_t st) {
  using Tl = typename TileOf<ID, false, false>::T;
  const int tiles = ceil_div(a.V, 64 * Tl::TN);
  hipLaunchKernelGGL((vocab_logits_few<Tl, DT, KEPT>), dim3(tiles + (KEPT == kNot ? 0 : kFewRows / Tl::kWaves)), dim3(Tl::kTileThreads), 0, st, a, q, tiles);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_rows<Tl, DT, KEPT>(a, q, st, true);
}
template <int DT, Kept KEPT>
static hipError_t launch_logits_few(int tile, const VocabArgs& a, const VocabPiece& q, hipStream_t st) {
  switch (tile) {
    case kT11: return launch_logits_few<kT11, DT, KEPT>(a, q, st);
    case kT12: return launch_logits_few<kT12, DT, KEPT>(a, q, st);
    default: return launch_logits_few<kT14Deep, DT, KEPT>(a, q, st);
  }
}
template <int DT>
static hipError_t launch_gather(const VocabArgs& a, const VocabPiece& q, bool vec, hipStream_t st) {
  const int per = 4 * ceil_div(q.count, 4 * kGatherWorkgroups), grid = ceil_div(q.count, per) + (a.V % 64 ? 16 : 0);
  static_assert(kVocabPieceMost / kGatherWorkgroups <= kWave, "a lane per token");
  if (vec)
    hipLaunchKernelGGL((vocab_gather<true, DT>), dim3(grid), dim3(256), 0, st, a, q, per);
  else
    hipLaunchKernelGGL((vocab_gather<false, DT>), dim3(grid), dim3(256), 0, st, a, q, per);
  return hipGetLastError();
}
template <int ID, int DT>
static hipError_t launch_dx(const VocabArgs& a, const VocabPiece& q, hipStream_t st) {
  using Tl = typename TileOf<ID, true, false>::T;
  // (the device's number of tokens decides: as many workgroups as any number of them may have)
  const int GM = ceil_div(q.count, 64 * Tl::TM), units = GM * ceil_div(a.d, 64 * Tl::TN), slots = cut_slots(ID, q.slots);
  // One tile of tokens is one for any number of them, and so is its plan: where that cuts nothing the kernel gets no room to.
  const bool whole = GM == 1 && dx_plan(ID, q.count, a.d, a.V, q.slots).pieces == 1;
  VocabPiece o = q;
  if (whole) o.slots = 0;
  hipLaunchKernelGGL((vocab_dx<ID, DT>), dim3(dx_grid(ID, q.count, a.d, o.slots)), dim3(Tl::kTileThreads), 0, st, a, o);
  const hipError_t e = hipGetLastError();
  const int cut = units < slots / 2 ? units : slots / 2;
  if (e != hipSuccess || cut == 0 || whole) return e;
  hipLaunchKernelGGL((vocab_dx_sum<Tl, ID, DT>), dim3(cut, Tl::kWaves, Tl::NI), dim3(64 * Tl::TI), 0, st, a, q);
  return hipGetLastError();
}
template <int ID, int DT>
static hipError_t launch_dw(const VocabArgs& a, const VocabPiece& q, bool first, bool last, hipStream_t st) {
  using Tl = typename TileOf<ID, true, true>::T;
  // (what is looked at is the targets, once per workgroup: as many shares as there are CUs for, of 1024 tokens at least)
  const int tiles = ceil_div(a.V, 64 * Tl::TM), shares = tiles < 2 * kCUs ? 2 * kCUs / tiles : 1, most = ceil_div(q.count, 1024);
  hipLaunchKernelGGL((vocab_lacks<DT>), dim3(tiles, shares < most ? shares : most), dim3(kLackThreads), 0, st, a, q, 64 * Tl::TM);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  float* sums = a.dw_f32 ? (float*)a.dW : first && last ? nullptr : q.dw;
  // (cut if it would be for all of the piece's tokens: the units' number is not the tokens')
  VocabPiece whole = q;
  const CutPlan p = dw_plan(ID, q.count, a.d, a.V, q.slots);
  if (p.pieces == 1) whole.slots = 0;
  hipLaunchKernelGGL((vocab_dw<ID, DT>), dim3(eights(p.GM * p.GN) + eights(cut_slots(ID, whole.slots))), dim3(512), 0, st, a, whole, sums, first, last);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.pieces == 1) return e;
  hipLaunchKernelGGL((vocab_dw_sum<Tl, ID, DT>), dim3(p.rest, Tl::kWaves, Tl::NI), dim3(64 * Tl::TI), 0, st, a, q, sums, first, last);
  return hipGetLastError();
}

template <int DT>
static hipError_t vocab_piece(const VocabArgs& a, const VocabPiece& q, bool first, bool last, hipStream_t st) {
  const bool grads = a.dX || a.dW, vec = ((uintptr_t)a.X | (uintptr_t)(a.xs * 2) | (uintptr_t)a.dX | (uintptr_t)(a.dxs * 2)) % 16 == 0;
  const int tile = plan_logits(q.count, a.d, a.V);
  const bool one = DT == kBf16 && a.dX && !a.dW;
  constexpr Kept kept = DT == kBf16 ? kSteps : kApart;
  hipError_t e = hipSuccess;
  if (q.count <= 64 && vec) {
    e = grads ? launch_logits_few<DT, kept>(tile, a, q, st) : launch_logits_few<DT, kNot>(tile, a, q, st);
  } else {
    e = launch_gather<DT>(a, q, vec, st);
    if (e != hipSuccess) return e;
    if constexpr (DT == kBf16) e = one ? launch_logits<DT, kOne>(tile, a, q, st) : e;
    if (!one) e = grads ? launch_logits<DT, kept>(tile, a, q, st) : launch_logits<DT, kNot>(tile, a, q, st);
  }
  if (e == hipSuccess && a.dX) switch (plan_dx(q.count, a.d, a.V, q.slots)) {
      case kT44: e = launch_dx<kT44, DT>(a, q, st); break;
      case kT24: e = launch_dx<kT24, DT>(a, q, st); break;
      case kT14Deep: e = launch_dx<kT14Deep, DT>(a, q, st); break;
      default: e = launch_dx<kT11, DT>(a, q, st); break;
    }
  if (e == hipSuccess && a.dW) e = plan_dw(q.count, a.d, a.V, q.slots) == kT24 ? launch_dw<kT24, DT>(a, q, first, last, st) : launch_dw<kT44, DT>(a, q, first, last, st);
  return e;
}

hipError_t launch_vocab_loss(const VocabArgs& a, const VocabRoom& room, void* ws, hipStream_t st) {
  ProfScope prof(kKVocab, st);
  char* at = (char*)ws;
  VocabPiece q = {};
  q.head = (VocabHead*)(at + room.head), q.list = (int*)(at + room.list), q.target = (int*)(at + room.target);
  q.weight = (float*)(at + room.weight), q.z = (double*)(at + room.z), q.factor = (float*)(at + room.factor), q.lacks = (float*)(at + room.lacks), q.stats = (float2*)(at + room.stats);
  q.x = (uint16_t*)(at + room.x), q.tail = (uint16_t*)(at + room.tail), q.p = (uint16_t*)(at + room.p), q.part = (f32x4*)(at + room.part);
  q.dw = (float*)(at + room.dw);
  q.spans = (int2*)(at + room.spans), q.order = (int*)(at + room.order), q.lo = (uint16_t*)(at + room.lo);
  q.units = room.units, q.ldp = room.ldp, q.slots = room.slots;
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
