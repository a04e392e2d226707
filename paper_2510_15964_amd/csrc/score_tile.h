// What the 16-bit kernels of attention with rules on its scores share (score_bf16.hip, score_token.hip): LDS tiles and their reads,
// the rules, intervals of keys, and the online softmax of a tile.
#pragma once
#include <type_traits>

#include "lx_dev.h"
#include "lx_launch.h"
#include "score_plan.h"

namespace lx {

constexpr int kSThreads = 256, kSWaves = kSThreads / kWave;      // of a team: a workgroup has one or two, with the same own rows
constexpr int kOwn = 32 * kSWaves;       // own rows of a workgroup
constexpr float kSLog2e = 1.4426950408889634f, kSLn2 = 0.6931471805599453f;
constexpr float kSSlack = 8.f;           // log2 units by which a score may exceed the reference point of its row
constexpr int kIntMax = 0x7fffffff;
constexpr float kFloatMax = 3.402823466e38f;

// Waits here for loads whose results a loop uses: otherwise the compiler waits inside it, for everything in flight.
__device__ __forceinline__ void settle(float& x) { asm volatile("" : "+v"(x)); }
template <int N>
__device__ __forceinline__ void settle(uint4 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i].x), "+v"(f[i].y), "+v"(f[i].z), "+v"(f[i].w));
}
// What the 16-byte slots of a tile's row are XORed with.  Rows of 2D bytes put the same slot of 16 rows (D = 128) or of eight
// pairs (D = 64) into the same banks; lanes 0..3, 12..15, 20..27 of a half wavefront (and the others) are served together by a
// 16-byte read, all 32 by a transposing one, whose lanes cover four rows by 64 bytes.  For both no two of them meet in a bank.
// Rows 16 apart have the same.
template <int D>
__device__ __forceinline__ constexpr int score_swz(int row) {
  return D == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row & 2) << 1 | (row >> 2 & 3);
}

// dma16 with a wave-uniform base and a 32-bit offset per lane (dma16_s names no memory clobber)
__device__ __forceinline__ void score_dma16(const char* base, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
// Transfers of one [64 x D] tile: an instruction moves 1 KiB, D / 32 of them per wavefront.  A lane's rows are 64 / (D / 32) apart, so
// they have the same slot, and all of them the same offset from a base of their own: one register per tensor and scalar
// additions.  (With an address per lane and instruction the transfers were a sixth of a tile's vector instructions.)  Tiles that
// end beyond the tensor, and strides whose offsets leave 32 bits, take an address per lane.  Without KEEP the offset is made for
// every tile: the key side at D = 128 has no register for it.
template <int D, bool KEEP = true>
struct ScoreDma {
  static constexpr int kSlots = D / 8, kRowsPer = 64 / kSlots, kStep = kRowsPer * kSWaves, kPerWave = kTileRows / kStep;
  static_assert(kStep % 16 == 0, "rows 16 apart have the same swizzle");
  uint32_t off, wave_lds;
  long long row_bytes;
  static __device__ __forceinline__ int row_of(int thread) { return kRowsPer * (thread / kWave % kSWaves) + thread % kWave / kSlots; }
  static __device__ __forceinline__ int slot_of(int thread) { return ((thread % kWave % kSlots) ^ score_swz<D>(row_of(thread))) * 16; }
  __device__ __forceinline__ void init(const ScoreTensor& t) {
    wave_lds = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave % kSWaves) * 1024;
    row_bytes = 2 * t.ss;
    if constexpr (KEEP) off = (uint32_t)(row_of(threadIdx.x) * row_bytes) + slot_of(threadIdx.x);
  }
  // rows past `last` repeat it
  __device__ __forceinline__ void issue(uint32_t tile, const char* base, int last) const {
    const uint32_t to = tile + wave_lds;
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));      // (what is made of it is made here, not kept)
    if (last >= kTileRows - 1 && row_bytes < (1ll << 32) / kTileRows) {
      const uint32_t v = KEEP ? off : (uint32_t)row_of(thread) * (uint32_t)row_bytes + slot_of(thread);
#pragma unroll
      for (int u = 0; u < kPerWave; ++u) score_dma16(base + u * kStep * row_bytes, v, to + u * (kSWaves * 1024));
    } else {
      const int row = row_of(thread), slot = slot_of(thread);
#pragma unroll
      for (int u = 0; u < kPerWave; ++u)
        dma16(base + (long long)min(row + kStep * u, last) * row_bytes + slot, to + u * (kSWaves * 1024));
    }
  }
};

// LDS offsets of a lane in a [64 x D] tile: of its 16-byte operand pieces (row lane%32, columns 16kk + 8(lane/32)..) and of the
// transposing reads (rows 4(lane/32) + (lane%16)/4, columns 16((lane/16)%2) + 4(lane%4)).  A k slice, column tile or half slice
// is an XOR of the slot's bits, which the addresses of tiles leave clear; rows, and a second tile, are immediates.
template <int D>
struct ScoreOff {
  uint32_t rows, tr;
  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x % kWave, h = lane / 32, r = lane % 32, i = lane % 16 / 4;
    rows = r * 2 * D + ((h ^ score_swz<D>(r)) << 4);
    const int tr_row = 4 * h + i, col = 16 * (lane / 16 % 2) + 4 * (lane % 4);
    tr = tr_row * 2 * D + (((col >> 3) ^ score_swz<D>(tr_row)) << 4) + (col & 7) * 2;
  }
};
// v ^ C, made where it is used: left to itself the compiler keeps a register for every C, up to 25 of them
template <int C>
__device__ __forceinline__ uint32_t flip(uint32_t v) {
  if constexpr (C == 0) return v;
  uint32_t r;
  asm volatile("v_xor_b32 %0, %2, %1" : "=v"(r) : "v"(v), "n"(C));
  return r;
}
// operand of k slice kk, rows 32t .. of the tile `at` bytes behind the one that `rows` (address + ScoreOff::rows) is of
template <int D>
__device__ __forceinline__ uint4 read_piece(uint32_t rows, int at, int t, int kk) {
  auto from = [&](uint32_t v) { return lds_read16(v + at + 32 * t * 2 * D); };
  switch (kk) {
    case 0: return from(flip<0>(rows));
    case 1: return from(flip<1 << 5>(rows));
    case 2: return from(flip<2 << 5>(rows));
    case 3: return from(flip<3 << 5>(rows));
    case 4: return from(flip<4 << 5>(rows));
    case 5: return from(flip<5 << 5>(rows));
    case 6: return from(flip<6 << 5>(rows));
    default: return from(flip<7 << 5>(rows));
  }
}
// transposed operand: columns 32ct + lane%32, and the 16 rows 32t + 16j .. in the order of the accumulators' registers 8j .. 8j + 7;
// tr: address + ScoreOff::tr
template <int D>
__device__ __forceinline__ uint4 read_piece_tr(uint32_t tr, int at, int t, int j, int ct) {
  auto from = [&](uint32_t a, uint32_t b) {
    const uint2 lo = lds_read8_tr(a + at + (32 * t + 16 * j) * 2 * D), hi = lds_read8_tr(b + at + (32 * t + 16 * j + 8) * 2 * D);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  switch (ct) {
    case 0: return from(flip<0>(tr), flip<32>(tr));
    case 1: return from(flip<1 << 6>(tr), flip<(1 << 6) + 32>(tr));
    case 2: return from(flip<2 << 6>(tr), flip<(2 << 6) + 32>(tr));
    default: return from(flip<3 << 6>(tr), flip<(3 << 6) + 32>(tr));
  }
}
// accumulator registers 8j .. 8j + 7, rounded
template <int DT>
__device__ __forceinline__ uint4 pack_piece(const f32x16& p, int j) {
  return make_uint4(pack2<DT>(p[8 * j], p[8 * j + 1]), pack2<DT>(p[8 * j + 2], p[8 * j + 3]), pack2<DT>(p[8 * j + 4], p[8 * j + 5]),
                    pack2<DT>(p[8 * j + 6], p[8 * j + 7]));
}
// what the rounding to `p` left of them, rounded
template <int DT>
__device__ __forceinline__ uint4 rest_piece(const f32x16& p, int j, uint4 rounded) {
  const uint32_t w[4] = {rounded.x, rounded.y, rounded.z, rounded.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = pack2<DT>(p[8 * j + 2 * i] - to_f32<DT>(w[i] & 0xffff), p[8 * j + 2 * i + 1] - to_f32<DT>(w[i] >> 16));
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// sum + the product of two pairs of elements
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ float dot2(uint32_t x, uint32_t y, float sum) {
  if constexpr (DT == kF16)
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x), __builtin_bit_cast(f16x2, y), sum, false);
  else
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v, x), __builtin_bit_cast(bf16x2v, y), sum, false);
}
template <int DT>
constexpr uint32_t kOnes = DT == kF16 ? 0x3c003c00u : 0x3f803f80u;
// sum + the eight elements of a packed piece
template <int DT>
__device__ __forceinline__ float add_piece(uint4 p, float sum) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) sum = dot2<DT>(w[i], kOnes<DT>, sum);
  return sum;
}

template <class T>
__device__ __forceinline__ const char* score_row(const ScoreTensor& t, int b, int h, T s) {
  return (const char*)t.p + 2 * (b * t.sb + h * t.sh + (long long)s * t.ss);
}
// D elements of an own row as k slices of an operand
template <int D>
__device__ __forceinline__ void load_own(const ScoreTensor& t, int b, int h, int s, uint4 (&f)[D / 16]) {
  const uint4* p = (const uint4*)score_row(t, b, h, s) + threadIdx.x % kWave / 32;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) f[kk] = p[2 * kk];
}
// the sum of an own row's squares
template <int DT, int N>
__device__ __forceinline__ float own_squares(const uint4 (&f)[N]) {
  float sum = 0.f;
#pragma unroll
  for (int kk = 0; kk < N; ++kk) {
    const uint32_t x[4] = {f[kk].x, f[kk].y, f[kk].z, f[kk].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = to_f32<DT>(x[i / 2] >> (i % 2 * 16) & 0xffff);
      sum = fmaf(v, v, sum);
    }
  }
  return sum + __shfl_xor(sum, 32);
}
// the own rows' columns of a product, times c
template <int D, int DT>
__device__ __forceinline__ void store_own(const ScoreTensor& t, int b, int h, int s, const f32x16 (&acc)[D / 32], float c) {
  uint2* p = (uint2*)const_cast<char*>(score_row(t, b, h, s)) + threadIdx.x % kWave / 32;
#pragma unroll
  for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      p[8 * ct + 2 * i] = make_uint2(pack2<DT>(acc[ct][4 * i] * c, acc[ct][4 * i + 1] * c), pack2<DT>(acc[ct][4 * i + 2] * c, acc[ct][4 * i + 3] * c));
}

// e of a number that is not negative, 2^(e - 1) <= x < 2^e; 0 of zero and of what is not finite
__device__ __forceinline__ int exponent_of(float x) { return __builtin_amdgcn_frexp_expf(x); }
__device__ __forceinline__ float times_pow2(float x, int e) { return __builtin_amdgcn_ldexpf(x, e); }
__device__ __forceinline__ float finite_or_zero(float x) { return x < INFINITY ? x : 0.f; }

// row, relative to 4(lane/32), of accumulator register v
__device__ __forceinline__ constexpr int acc_row(int v) { return 8 * (v / 4) + v % 4; }

// How scores are capped.  kInExponent: s = cap (1 - 2 r), r = 1 / (1 + e^(2 s / cap)), without the constant part.  r is half a unit in the last
// place off and more, so that s is off by up to 2^-22 of the cap: 3e-5 of natural units at kExponentCap, below what the products of
// 16-bit numbers themselves leave.  kAnyCap: beyond, where that would be seen (1.5e-3 at 1e4, 0.16 at 1e6), small arguments by the
// series of tanh, which does not cancel; about ten vector instructions more per score (4 x 2048, 32 heads on 8, D = 128, forward 203
// us with a cap of 15, 230 with one of 200, backward 555 and 789).
enum CapKind { kNoCap, kInExponent, kAnyCap };
constexpr float kExponentCap = 128.f;
// The constant part, in log2 units.
__host__ __device__ __forceinline__ float cap_base(float cap) { return cap > 0.f && cap <= kExponentCap ? cap * kSLog2e : 0.f; }

// The rules: of a product of Q and K the score in log2 units less `base`, the cap, and with CAP the factor of its derivative.
template <int CAP, bool BIAS>
struct FastRules {
  float c, slope;         // CAP: 2 scale log2(e) / cap; otherwise scale log2(e)
  float minus2, plain;    // kInExponent: -2 cap log2(e); kAnyCap: cap log2(e), scale log2(e)
  // UNIFORM: h is the wavefront's
  template <bool UNIFORM>
  __device__ __forceinline__ void init(const ScoreArgs& a, int h) {
    auto uniform = [](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); };
    auto finite = [](float x) { return fminf(fmaxf(x, -kFloatMax), kFloatMax); };      // (times a product of zero: zero)
    c = uniform(CAP ? finite(2.f * kSLog2e * a.scale / a.cap) : a.scale * kSLog2e);
    minus2 = uniform(CAP == kAnyCap ? finite(a.cap * kSLog2e) : -2.f * base(a));
    plain = CAP == kAnyCap ? uniform(a.scale * kSLog2e) : 0.f;
    slope = 0.f;
    if constexpr (BIAS) {
      slope = a.slopes ? a.slopes[h] * kSLog2e : 0.f;
      settle(slope);
      if constexpr (UNIFORM) slope = uniform(slope);
    }
  }
  static __device__ __forceinline__ float base(const ScoreArgs& a) { return CAP == kInExponent ? cap_base(a.cap) : 0.f; }
  // with kInExponent, of a product: -r; the score is its product with -minus2
  __device__ __forceinline__ float negative_rate(float x) const { return __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(x * c)); }
  // r: 1 / (1 + e^(2 s / cap)), tanh = 1 - 2 r; with kAnyCap 1 - tanh^2
  __device__ __forceinline__ float score(float x, float dist, float& r) const {
    float s;
    if constexpr (CAP) {
      const float z = x * c;
      r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z));
      s = minus2 * r;
      if constexpr (CAP == kAnyCap) {
        // tanh y = y f(y^2) up to y = 1/4, where the first term left out is 8e-9 of the whole
        const float y = z * (0.5f * kSLn2), yy = y * y;
        const float f = fmaf(yy, fmaf(yy, fmaf(yy, fmaf(yy, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f), t = y * f;
        const bool small = fabsf(y) < 0.25f;
        s = small ? x * plain * f : fmaf(-2.f, s, minus2);
        r = small ? fmaf(-t, t, 1.f) : 4.f * fmaf(-r, r, r);
      }
    } else {
      s = x * c;
    }
    if constexpr (BIAS) s = fmaf(-slope, fabsf(dist), s);
    return s;
  }
  // The bias of a tile all of whose queries attend no key behind them is linear in the key: -slope (pos - k).  What depends on the
  // accumulator's register is where the sums of the first product begin (lift), the rest is one number per own row and 32
  // keys: no vector instructions for the bias, which otherwise takes three per score.
  static constexpr bool kMayBeLinear = BIAS && !CAP;
  // (c: so that a slope divided by it stays far from infinite)
  __device__ __forceinline__ bool linear(int after) const { return kMayBeLinear && !after && c > 0x1p-64f; }
  __device__ __forceinline__ void lift(f32x16& l) const {
    if constexpr (kMayBeLinear) {
      const float each = c > 0.f ? slope / c : 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) l[v] = each * (float)acc_row(v);
    }
  }
  // 1 - tanh^2, over kDerivative
  static __device__ __forceinline__ float derivative(float r) { return CAP == kInExponent ? fmaf(-r, r, r) : CAP ? r : 1.f; }
  static constexpr float kDerivative = CAP == kInExponent ? 4.f : 1.f;
};

// f(std::true_type or false_type): whether the bias is linear, as one branch around a loop, not one in it.
template <int CAP, bool BIAS, class F>
__device__ __forceinline__ void by_linear(const FastRules<CAP, BIAS>& rules, int after, F f) {
  if constexpr (FastRules<CAP, BIAS>::kMayBeLinear)
    if (rules.linear(after)) return f(std::true_type());
  f(std::false_type());
}

// The interval of keys of query q, as its first key and its length, and the query's position.
__device__ __forceinline__ void key_interval(const ScoreArgs& a, int b, int q, int start, int& lo, int& len) {
  int hi = a.Sk;
  lo = 0;
  if (a.causal) hi = (int)max(min((long long)hi, (long long)start + q + 1), 0ll);
  if (a.key_lo) {
    lo = max(lo, a.key_lo[(long long)b * a.Sq + q]);
    hi = min(hi, a.key_hi[(long long)b * a.Sq + q]);
  }
  len = hi > lo ? hi - lo : 0;      // (hi may be any number: no difference before this)
}
// The largest of the first 32 lanes' v, which the other 32 repeat, as a scalar.
__device__ __forceinline__ int max_of_half(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xf, 0xf, false));     // from 1, 2, 4 and 8 lanes before in a row of 16
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xf, 0xf, false));
  return max(__builtin_amdgcn_readlane(v, 15), __builtin_amdgcn_readlane(v, 31));
}
// The sum of the first 32 lanes' v, as a scalar.
__device__ __forceinline__ float sum_of_half(float v) {
  auto from = [&](auto lanes) {
    const int moved = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(lanes)::value, 0xf, 0xf, false);
    v += __builtin_bit_cast(float, moved);
  };
  from(std::integral_constant<int, 0x111>());      // 1, 2, 4 and 8 lanes before in a row of 16
  from(std::integral_constant<int, 0x112>());
  from(std::integral_constant<int, 0x114>());
  from(std::integral_constant<int, 0x118>());
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 15)) +
         __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 31));
}
// of numbers that are not negative
__device__ __forceinline__ float max_of_half(float x) { return __builtin_bit_cast(float, max_of_half(__builtin_bit_cast(int, x))); }
// What a set of queries attends: every tile that some query attends lies in first .. end - 1, and keys from all_from up to
// all_to - 1 are attended by all of them; after: some query attends a key behind its own position.
struct KeySpan {
  int first, end, all_from, all_to, after;
  __device__ __forceinline__ void of(bool there, int lo, int len, int pos) {
    after = there && len > 0 && lo + len - 1 > pos;
    first = there && len > 0 ? lo : kIntMax;
    end = there && len > 0 ? lo + len : 0;
    all_from = !there ? 0 : len > 0 ? lo : kIntMax;
    all_to = !there ? kIntMax : len > 0 ? lo + len : 0;
  }
  __device__ __forceinline__ void join(const KeySpan& o) {
    first = min(first, o.first), end = max(end, o.end), all_from = max(all_from, o.all_from), all_to = min(all_to, o.all_to);
    after |= o.after;
  }
  // as if of no queries, otherwise
  __device__ __forceinline__ void only_if(bool there) {
    first = there ? first : kIntMax, end = there ? end : 0, all_from = there ? all_from : 0, all_to = there ? all_to : kIntMax;
    after = there ? after : 0;
  }
  __device__ __forceinline__ bool touches(int k, int n) const { return k < end && first < k + n; }
  __device__ __forceinline__ bool covers(int k, int n) const { return all_from <= k && k + n <= all_to; }
};
__device__ __forceinline__ KeySpan scalar_span(const KeySpan& s) {
  return {__builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.end), __builtin_amdgcn_readfirstlane(s.all_from),
          __builtin_amdgcn_readfirstlane(s.all_to), __builtin_amdgcn_readfirstlane(s.after)};
}
// of the queries of a wavefront, a lane's and that of the lane 32 further being the same
__device__ __forceinline__ KeySpan span_of_wave(const KeySpan& s) {
  return {-max_of_half(-s.first), max_of_half(s.end), max_of_half(s.all_from), -max_of_half(-s.all_to), __any(s.after) != 0};
}
// of queries q .. q + n - 1, of Sq, where there are no intervals given
__device__ __forceinline__ KeySpan span_of_rows(const ScoreArgs& a, int start, int q, int n) {
  const int last = min(q + n, a.Sq) - 1;
  KeySpan s = {kIntMax, 0, 0, kIntMax, 0};
  if (last < q) return s;
  auto upto = [&](int r) { return a.causal ? (int)max(min((long long)a.Sk, (long long)start + r + 1), 0ll) : a.Sk; };
  s.end = upto(last);
  s.first = s.end > 0 ? 0 : kIntMax;
  s.all_to = upto(q);
  s.after = !a.causal && (long long)start + q < a.Sk - 1;
  return s;
}

// which of the keys from k0 on, a bit each, are among len keys from lo on
__device__ __forceinline__ unsigned long long keys_seen(int k0, int lo, int len) {
  const int from = min(max(lo - k0, 0), 64), to = min(max(lo - k0 + len, 0), 64);
  const unsigned long long below_to = to == 64 ? ~0ull : (1ull << to) - 1, below_from = from == 64 ? ~0ull : (1ull << from) - 1;
  return below_to & ~below_from;
}
// all ones where bit b of a word is set
__device__ __forceinline__ uint32_t spread_bit(uint32_t word, int b) { return (uint32_t)__builtin_amdgcn_sbfe((int)word, b, 1); }
// x, or -inf / 0 where the mask is zero
__device__ __forceinline__ float or_minus_inf(uint32_t mask, float x) {
  return __builtin_bit_cast(float, (mask & __builtin_bit_cast(uint32_t, x)) | (~mask & 0xff800000u));
}
__device__ __forceinline__ float or_zero(uint32_t mask, float x) { return __builtin_bit_cast(float, mask & __builtin_bit_cast(uint32_t, x)); }
// The largest of x and v.  (fmaxf first makes its arguments canonical, and a statement per instruction gets a wait behind each.)
__device__ __forceinline__ float max17(float x, const f32x16& v) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3\n\tv_max3_f32 %0, %0, %4, %5\n\tv_max3_f32 %0, %0, %6, %7\n\tv_max3_f32 %0, %0, %8, %9\n\t"
      "v_max3_f32 %0, %0, %10, %11\n\tv_max3_f32 %0, %0, %12, %13\n\tv_max3_f32 %0, %0, %14, %15\n\tv_max3_f32 %0, %0, %16, %17"
      : "=&v"(r)
      : "v"(x), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]), "v"(v[8]), "v"(v[9]), "v"(v[10]),
        "v"(v[11]), "v"(v[12]), "v"(v[13]), "v"(v[14]), "v"(v[15]));
  return r;
}
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
template <uint32_t EXP>
__device__ __forceinline__ ushort2v top_exponent(uint4 v, ushort2v top) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort2v, w[i] & EXP));
  return top;
}
// Zeroes what is not finite in a [64 x D] tile, a quarter of a row per thread, and says in which of the wavefront's 16 rows
// it found any.
template <int D, int DT>
__device__ __forceinline__ unsigned clear_not_finite(uint32_t tile) {
  constexpr uint32_t kExp = DT == kF16 ? 0x7c007c00u : 0x7f807f80u, kOne = DT == kF16 ? 0x04000400u : 0x00800080u;
  const uint32_t at = tile + threadIdx.x % kSThreads * (D / 2);
  ushort2v top = {0, 0};       // the largest exponent of each half
#pragma unroll
  for (int i = 0; i < D / 32; ++i) top = top_exponent<kExp>(lds_read16(at + 16 * i), top);
  // an exponent of ones and nothing else carries into the sign's place
  const bool found = (__builtin_bit_cast(uint32_t, top) + kOne) & 0x80008000u;
  if (found)
#pragma unroll
    for (int i = 0; i < D / 16; ++i) lds_write8(at + 8 * i, make_uint2(0, 0));
  const unsigned long long lanes = __ballot(found);
  if (!lanes) return 0;
  unsigned rows = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) rows |= (unsigned)((lanes >> (4 * r) & 15) != 0) << r;
  return rows;
}
__device__ __forceinline__ unsigned long long join_rows(unsigned mine, unsigned* part) {
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave % kSWaves] = mine;
  lds_barrier();
  const unsigned a = part[0] | part[1] << 16, b = part[2] | part[3] << 16;
  return (unsigned long long)__builtin_amdgcn_readfirstlane(b) << 32 | (unsigned)__builtin_amdgcn_readfirstlane(a);
}

// Of one own row: the reference point of its exponentials (0 for -inf), the sum of its probabilities and that of the rounded ones.
// O is normalised by the latter, of which it is made: a row dominated by a few keys otherwise carries their rounding errors as
// a whole, and Delta hands them on to the gradients.  LSE is of the unrounded ones.
template <int D>
struct ScoreRow {
  float m, ref, sum, weight;
  f32x16 o[D / 32];
  __device__ __forceinline__ void clear() {
    m = -INFINITY, ref = sum = weight = 0.f;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[ct][v] = 0.f;
  }
};

// Products issue a slot at a time, a matrix instruction and what may run under it, with the compiler's scheduler held off between
// slots: left to itself it reads an operand from LDS right before its product and waits for it.
__device__ __forceinline__ void end_slot() { __builtin_amdgcn_sched_barrier(0); }
constexpr int kAhead = 3;       // slots by which operands are read ahead
// A wavefront that issues products goes before one of the same SIMD that does its softmax, which so runs under them (D = 128, one
// call after the other: 8192 tokens, 32 heads on 8, forward 600 -> 593 us; 4 x 2048, capped, backward 644 -> 631).
template <int P>
__device__ __forceinline__ void wave_priority() { __builtin_amdgcn_s_setprio(P); }

// A tile of 32 NT keys from k0 on: K at tk, V AT bytes behind.  pos: the own query's position; lo, len: its keys; masked: not all of the
// tile's are among those of every query.
//
// A matrix instruction of 32 clocks leaves the SIMD's vector instructions about 16 (a loop of 32 of them and 288 others, two to
// four wavefronts, takes 595 - 638 ns, 470 and 356 without the ones or the others); rules run under the next 32 keys' scores,
// exponentials under the second product of the keys before.
//
// middle() runs between the products, when K has been read and V is not yet.
struct Nothing {
  __device__ __forceinline__ void operator()() const {}
};
template <int NT, int AT, bool LINEAR, int D, int DT, int CAP, bool BIAS, class Middle = Nothing>
__device__ __forceinline__ void attend_tile(uint32_t tk, const ScoreOff<D>& off, const uint4 (&qf)[D / 16],
                                            const FastRules<CAP, BIAS>& rules, const f32x16& lift, int k0, int pos, int lo, int len,
                                            bool masked, ScoreRow<D>& w, Middle middle = Nothing()) {
  constexpr int KK = D / 16, CT = D / 32, kScores = NT * KK, kGroups = 2 * NT;
  // Scores are products, or with a cap what takes the place of a tanh, times a positive number: made in the exponent.
  constexpr bool kPlain = !CAP && (!BIAS || LINEAR), kTimes = kPlain || (CAP == kInExponent && !BIAS);
  const float times = CAP ? -rules.minus2 : rules.c;
  const int half = threadIdx.x % kWave / 32;
  const uint32_t rows = tk + off.rows, tr = tk + off.tr;
  const float far = (float)(pos - k0 - 4 * half);
  f32x16 s[NT];
  float base[NT];         // of the scores, with kTimes
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    base[t] = LINEAR ? rules.slope * ((float)(32 * t) - far) : 0.f;
    if constexpr (LINEAR) s[t] = lift;
    else s[t] = f32x16{};
  }
  auto rule = [&](int t, int v) {
    float r;
    if constexpr (kTimes) s[t][v] = rules.negative_rate(s[t][v]);
    else s[t][v] = rules.score(s[t][v], far - (float)(32 * t + acc_row(v)), r);
  };
  uint4 in[kAhead + 1];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) in[n] = read_piece<D>(rows, 0, n / KK, n % KK);
  end_slot();
  wave_priority<1>();
#pragma unroll
  for (int n = 0; n < kScores; ++n) {
    const int t = n / KK, kk = n % KK, next = n + kAhead;
    if (next < kScores) in[next % (kAhead + 1)] = read_piece<D>(rows, 0, next / KK, next % KK);
    s[t] = mfma32<DT>(in[n % (kAhead + 1)], qf[kk], s[t]);
    if constexpr (!kPlain)
      if (t > 0 && kk >= KK / 2) {
#pragma unroll
        for (int e = 0; e < 32 / KK; ++e) rule(t - 1, (kk - KK / 2) * (32 / KK) + e);
      }
    end_slot();
  }
  wave_priority<0>();
  middle();
  // the first operands of the second product are on their way during the softmax
#pragma unroll
  for (int n = 0; n < kAhead; ++n) in[n] = read_piece_tr<D>(tr, AT, n / (2 * CT), n / CT % 2, n % CT);
  end_slot();
  if constexpr (!kPlain)
#pragma unroll
    for (int v = 0; v < 16; ++v) rule(NT - 1, v);
  if (masked) {
    const unsigned long long seen = keys_seen(k0, lo, len);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t word = (uint32_t)(seen >> (32 * t)) >> (4 * half);
#pragma unroll
      for (int v = 0; v < 16; ++v) s[t][v] = or_minus_inf(spread_bit(word, acc_row(v)), s[t][v]);
    }
  }
  float top;
  if constexpr (LINEAR) {
    top = fmaf(max17(-INFINITY, s[0]), rules.c, base[0]);
    if constexpr (NT == 2) top = fmaxf(top, fmaf(max17(-INFINITY, s[1]), rules.c, base[1]));
  } else {
    top = max17(-INFINITY, s[0]);
    if constexpr (NT == 2) top = max17(top, s[1]);
    if constexpr (kTimes) top *= times;
  }
  // The reference point only has to bound the scores up to a factor that fp32 holds comfortably: it follows the maximum when
  // that has moved by more than kSSlack, which most tiles do for no query of the wavefront.
  if (__any(top > w.m + kSSlack)) {
    const float both = fmaxf(top, __shfl_xor(top, 32)), next = both > w.m + kSSlack ? both : w.m;
    w.ref = next == -INFINITY ? 0.f : next;
    const float shrink = __builtin_amdgcn_exp2f(w.m - w.ref);
    w.sum *= shrink;
    w.weight *= shrink;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) w.o[ct] *= shrink;
    w.m = next;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) base[t] -= w.ref;
  auto expo = [&](int g, int e) {
    const float x = s[g / 2][8 * (g % 2) + e], y = __builtin_amdgcn_exp2f(kTimes ? fmaf(x, times, base[g / 2]) : x - w.ref);
    s[g / 2][8 * (g % 2) + e] = y;
    w.sum += y;
  };
  end_slot();
#pragma unroll
  for (int e = 0; e < 8; ++e) expo(0, e);
  // Over a cache the matrix unit is idle: P goes into the product in two parts, so that O carries its own rounding alone (1.65e-3 of its norm
  // in bf16, with P rounded 2.2e-3; 8 x 32 heads over 1024 keys, D = 64, 14.3 us, so 14.8; 4 x 8 over 32768, D = 128, 103 both).
  constexpr bool kRest = NT == 1;
  uint4 p, rest;
  auto pack = [&](int g) {
    p = pack_piece<DT>(s[g / 2], g % 2);
    w.weight = add_piece<DT>(p, w.weight);
    if constexpr (kRest) {
      rest = rest_piece<DT>(s[g / 2], g % 2, p);
      w.weight = add_piece<DT>(rest, w.weight);
    }
  };
  pack(0);
  end_slot();
  wave_priority<1>();
#pragma unroll
  for (int n = 0; n < kGroups * CT; ++n) {
    const int g = n / CT, ct = n % CT, next = n + kAhead;
    if (next < kGroups * CT) in[next % (kAhead + 1)] = read_piece_tr<D>(tr, AT, next / (2 * CT), next / CT % 2, next % CT);
    w.o[ct] = mfma32<DT>(in[n % (kAhead + 1)], p, w.o[ct]);
    if constexpr (kRest) w.o[ct] = mfma32<DT>(in[n % (kAhead + 1)], rest, w.o[ct]);
    if (g + 1 < kGroups) {
#pragma unroll
      for (int e = 0; e < 8 / CT; ++e) expo(g + 1, ct * (8 / CT) + e);
      if (ct == CT - 1) pack(g + 1);
    }
    end_slot();
  }
  wave_priority<0>();
}
// f(type with the constants D, DT, CAP, BIAS)
template <int D_, int DT_, int CAP_, bool BIAS_>
struct ScoreVariant {
  static constexpr int D = D_, DT = DT_, CAP = CAP_;
  static constexpr bool BIAS = BIAS_;
};
template <int D, int DT, class F>
static hipError_t by_rules(const ScoreArgs& a, F f) {
  if (a.cap > kExponentCap) return f(ScoreVariant<D, DT, kAnyCap, true>());
  if (a.cap > 0.f) return a.slopes ? f(ScoreVariant<D, DT, kInExponent, true>()) : f(ScoreVariant<D, DT, kInExponent, false>());
  // (without rules the largest product is taken for the largest score)
  return a.slopes || !(a.scale > 0.f) ? f(ScoreVariant<D, DT, kNoCap, true>()) : f(ScoreVariant<D, DT, kNoCap, false>());
}
template <class F>
static hipError_t by_variant(int dt, const ScoreArgs& a, F f) {
  if (a.D == 64) return dt == kF16 ? by_rules<64, kF16>(a, f) : by_rules<64, kBf16>(a, f);
  return dt == kF16 ? by_rules<128, kF16>(a, f) : by_rules<128, kBf16>(a, f);
}
inline size_t round_up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace lx
