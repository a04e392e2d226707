// What the 16-bit kernels of attention with rules on its scores share (score_bf16.hip, score_token.hip): LDS tiles and their reads,
// the rules, intervals of keys, and the online softmax of a tile.
#pragma once
#include "lx_dev.h"
#include "lx_launch.h"

namespace lx {

constexpr int kSThreads = 256, kSWaves = kSThreads / kWave;
constexpr int kOwn = 32 * kSWaves;       // own rows of a workgroup
constexpr int kTileRows = 64;            // rows of a streamed tile
constexpr float kSLog2e = 1.4426950408889634f, kSLn2 = 0.6931471805599453f;
constexpr float kSSlack = 8.f;           // log2 units by which a score may exceed the reference point of its row
constexpr int kIntMax = 0x7fffffff;

// What the 16-byte slots of a tile's row are XORed with.  Rows of 2D bytes put the same slot of 16 rows (D = 128) or of eight
// pairs (D = 64) into the same banks; lanes 0..3, 12..15, 20..27 of a half wavefront (and the others) are served together by a
// 16-byte read, all 32 by a transposing one, whose lanes cover four rows by 64 bytes.  For both no two of them meet in a bank.
// Rows 16 apart have the same.
template <int D>
__device__ __forceinline__ constexpr int score_swz(int row) {
  return D == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row & 2) << 1 | (row >> 2 & 3);
}

// Transfers of one [64 x D] tile: an instruction moves 1 KiB, D / 32 of them per wavefront.
template <int D>
struct ScoreDma {
  static constexpr int kSlots = D / 8, kRowsPer = 64 / kSlots, kPerWave = kTileRows / kRowsPer / kSWaves;
  int row[kPerWave], slot[kPerWave];
  uint32_t wave_lds;
  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    wave_lds = wave * 1024;
#pragma unroll
    for (int u = 0; u < kPerWave; ++u) {
      row[u] = kRowsPer * (wave + kSWaves * u) + lane / kSlots;
      slot[u] = ((lane % kSlots) ^ score_swz<D>(row[u])) * 16;
    }
  }
  // rows past `last` repeat it
  __device__ __forceinline__ void issue(uint32_t tile, const char* base, long long row_bytes, int last) const {
#pragma unroll
    for (int u = 0; u < kPerWave; ++u)
      dma16(base + (long long)min(row[u], last) * row_bytes + slot[u], tile + wave_lds + u * (kSWaves * 1024));
  }
};

// LDS offsets of a lane in a [64 x D] tile: of its 16-byte operand pieces (row lane%32, columns 16kk + 8(lane/32)..) and of the
// transposing reads (rows 4(lane/32) + (lane%16)/4, columns 16((lane/16)%2) + 4(lane%4)).  A k slice, column tile or half slice
// is an XOR, rows are added.
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
// operand of k slice kk, rows 32t ..
template <int D>
__device__ __forceinline__ uint4 read_piece(uint32_t tile, const ScoreOff<D>& off, int t, int kk) {
  return lds_read16(tile + (off.rows ^ (kk << 5)) + 32 * t * 2 * D);
}
// transposed operand: columns 32ct + lane%32, and the 16 rows 32t + 16j .. in the order of the accumulators' registers 8j .. 8j + 7
template <int D>
__device__ __forceinline__ uint4 read_piece_tr(uint32_t tile, const ScoreOff<D>& off, int t, int j, int ct) {
  const uint2 lo = lds_read8_tr(tile + (off.tr ^ (ct << 6)) + (32 * t + 16 * j) * 2 * D);
  const uint2 hi = lds_read8_tr(tile + (off.tr ^ (ct << 6) ^ (2 << 4)) + (32 * t + 16 * j + 8) * 2 * D);
  return make_uint4(lo.x, lo.y, hi.x, hi.y);
}
// accumulator registers 8j .. 8j + 7, rounded
template <int DT>
__device__ __forceinline__ uint4 pack_piece(const f32x16& p, int j) {
  return make_uint4(pack2<DT>(p[8 * j], p[8 * j + 1]), pack2<DT>(p[8 * j + 2], p[8 * j + 3]), pack2<DT>(p[8 * j + 4], p[8 * j + 5]),
                    pack2<DT>(p[8 * j + 6], p[8 * j + 7]));
}
// sum + the eight elements of a packed piece
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ float add_piece(uint4 p, float sum) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == kF16)
      sum = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w[i]), __builtin_bit_cast(f16x2, 0x3c003c00u), sum, false);
    else
      sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2v, w[i]), __builtin_bit_cast(bf16x2v, 0x3f803f80u), sum, false);
  }
  return sum;
}
// row, relative to 4(lane/32), of accumulator register v
__device__ __forceinline__ constexpr int acc_row(int v) { return 8 * (v / 4) + v % 4; }

template <class T>
__device__ __forceinline__ const char* score_row(const ScoreTensor& t, int b, int h, T s) {
  return (const char*)t.p + 2 * (b * t.sb + h * t.sh + (long long)s * t.ss);
}
// Waits here for loads whose results a loop uses: otherwise the compiler waits inside it, for everything in flight.
__device__ __forceinline__ void settle(float& x) { asm volatile("" : "+v"(x)); }
template <int N>
__device__ __forceinline__ void settle(uint4 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i].x), "+v"(f[i].y), "+v"(f[i].z), "+v"(f[i].w));
}
// D elements of an own row as k slices of an operand
template <int D>
__device__ __forceinline__ void load_own(const ScoreTensor& t, int b, int h, int s, uint4 (&f)[D / 16]) {
  const uint4* p = (const uint4*)score_row(t, b, h, s) + threadIdx.x % kWave / 32;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) f[kk] = p[2 * kk];
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

// The rules: of a product of Q and K the score in log2 units, and with CAP the factor of its derivative.
template <bool CAP, bool BIAS>
struct FastRules {
  float c, top, slope;       // CAP: 2 scale log2(e) / cap, cap log2(e); otherwise scale log2(e)
  __device__ __forceinline__ void init(const ScoreArgs& a, int h) {
    c = CAP ? 2.f * kSLog2e * a.scale / a.cap : a.scale * kSLog2e;
    top = CAP ? a.cap * kSLog2e : 0.f;
    slope = 0.f;
    if constexpr (BIAS) {
      slope = a.slopes ? a.slopes[h] * kSLog2e : 0.f;
      settle(slope);
    }
  }
  // r: 1 / (1 + e^(2 s / cap)), tanh = 1 - 2 r
  __device__ __forceinline__ float score(float x, float dist, float& r) const {
    float s;
    if constexpr (CAP) {
      r = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * c));
      s = fmaf(-2.f * top, r, top);
    } else {
      s = x * c;
    }
    if constexpr (BIAS) s = fmaf(-slope, fabsf(dist), s);
    return s;
  }
  // 1 - tanh^2
  static __device__ __forceinline__ float derivative(float r) { return CAP ? 4.f * r * (1.f - r) : 1.f; }
};

// The interval of keys of query q, as its first key and its length, and the query's position.
__device__ __forceinline__ void key_interval(const ScoreArgs& a, int b, int q, int start, int& lo, int& len) {
  int hi = a.Sk;
  lo = 0;
  if (a.causal) hi = (int)max(min((long long)hi, (long long)start + q + 1), 0ll);
  if (a.key_lo) {
    lo = max(lo, a.key_lo[(long long)b * a.Sq + q]);
    hi = min(hi, a.key_hi[(long long)b * a.Sq + q]);
  }
  len = max(hi - lo, 0);
}
// What a set of queries attends: every tile that some query attends lies in first .. end - 1, and keys from all_from up to
// all_to - 1 are attended by all of them.
struct KeySpan {
  int first, end, all_from, all_to;
  __device__ __forceinline__ void of(bool there, int lo, int len) {
    first = there && len > 0 ? lo : kIntMax;
    end = there && len > 0 ? lo + len : 0;
    all_from = !there ? 0 : len > 0 ? lo : kIntMax;
    all_to = !there ? kIntMax : len > 0 ? lo + len : 0;
  }
  __device__ __forceinline__ void join(const KeySpan& o) {
    first = min(first, o.first), end = max(end, o.end), all_from = max(all_from, o.all_from), all_to = min(all_to, o.all_to);
  }
  // over the lanes whose numbers differ in the bits of `lanes`
  template <int FROM>
  __device__ __forceinline__ void join_lanes() {
#pragma unroll
    for (int o = FROM; o; o >>= 1) join(KeySpan{__shfl_xor(first, o), __shfl_xor(end, o), __shfl_xor(all_from, o), __shfl_xor(all_to, o)});
  }
  __device__ __forceinline__ bool touches(int k, int n) const { return k < end && first < k + n; }
  __device__ __forceinline__ bool covers(int k, int n) const { return all_from <= k && k + n <= all_to; }
};
__device__ __forceinline__ KeySpan scalar_span(const KeySpan& s) {
  return {__builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.end), __builtin_amdgcn_readfirstlane(s.all_from),
          __builtin_amdgcn_readfirstlane(s.all_to)};
}
// of the workgroup: `part` in LDS, one per wavefront; contains a barrier
__device__ __forceinline__ KeySpan span_of_workgroup(const KeySpan& wave_span, KeySpan* part) {
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = wave_span;
  __syncthreads();
  KeySpan s = part[0];
#pragma unroll
  for (int w = 1; w < kSWaves; ++w) s.join(part[w]);
  return scalar_span(s);
}

// whether some of the rows of a tile from k0 on, a bit each, are among len keys from lo on
__device__ __forceinline__ bool meets(unsigned long long rows, int k0, int lo, int len) {
  const int from = min(max(lo - k0, 0), 64), to = min(max(lo - k0 + len, 0), 64);
  const unsigned long long below_to = to == 64 ? ~0ull : (1ull << to) - 1, below_from = from == 64 ? ~0ull : (1ull << from) - 1;
  return (rows & below_to & ~below_from) != 0;
}
// Zeroes what is not finite in a [64 x D] tile, a quarter of a row per thread, and says in which of the wavefront's 16 rows
// it found any.
template <int D, int DT>
__device__ __forceinline__ unsigned clear_not_finite(uint32_t tile) {
  constexpr uint32_t kExp = DT == kF16 ? 0x7c007c00u : 0x7f807f80u, kOne = DT == kF16 ? 0x04000400u : 0x00800080u;
  const uint32_t at = tile + threadIdx.x * (D / 2);
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const uint4 v = lds_read16(at + 16 * i);
    // an exponent of ones and nothing else carries into the sign's place
    any |= ((v.x & kExp) + kOne) | ((v.y & kExp) + kOne) | ((v.z & kExp) + kOne) | ((v.w & kExp) + kOne);
  }
  const bool found = any & 0x80008000u;
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
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = mine;
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

// A tile of 32 NT keys from k0 on: K at tk, V at tv.  pos: the own query's position; lo, len: its keys; masked: not all of the
// tile's are among those of every query.
template <int NT, int D, int DT, bool CAP, bool BIAS>
__device__ __forceinline__ void attend_tile(uint32_t tk, uint32_t tv, const ScoreOff<D>& off, const uint4 (&qf)[D / 16],
                                            const FastRules<CAP, BIAS>& rules, int k0, int pos, int lo, int len, bool masked,
                                            ScoreRow<D>& w) {
  const int half = threadIdx.x % kWave / 32;
  f32x16 s[NT] = {};
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t] = mfma32<DT>(read_piece<D>(tk, off, t, kk), qf[kk], s[t]);
  const float far = (float)(pos - k0 - 4 * half);
  const int from = k0 + 4 * half - lo;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      float r;
      s[t][v] = rules.score(s[t][v], far - (float)(32 * t + acc_row(v)), r);
    }
  if (masked)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if ((unsigned)(from + 32 * t + acc_row(v)) >= (unsigned)len) s[t][v] = -INFINITY;
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) top = fmaxf(top, s[t][v]);
  // The reference point only has to bound the scores up to a factor that fp32 holds comfortably: it follows the maximum when
  // that has moved by more than kSSlack, which most tiles do for no query of the wavefront.
  if (__any(top > w.m + kSSlack)) {
    const float both = fmaxf(top, __shfl_xor(top, 32)), next = both > w.m + kSSlack ? both : w.m;
    w.ref = next == -INFINITY ? 0.f : next;
    const float shrink = __builtin_amdgcn_exp2f(w.m - w.ref);
    w.sum *= shrink;
    w.weight *= shrink;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) w.o[ct] *= shrink;
    w.m = next;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      s[t][v] = __builtin_amdgcn_exp2f(s[t][v] - w.ref);
      w.sum += s[t][v];
    }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint4 p = pack_piece<DT>(s[t], j);
      w.weight = add_piece<DT>(p, w.weight);
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct) w.o[ct] = mfma32<DT>(read_piece_tr<D>(tv, off, t, j, ct), p, w.o[ct]);
    }
}
// f(type with the constants D, DT, CAP, BIAS)
template <int D_, int DT_, bool CAP_, bool BIAS_>
struct ScoreVariant {
  static constexpr int D = D_, DT = DT_;
  static constexpr bool CAP = CAP_, BIAS = BIAS_;
};
template <int D, int DT, class F>
static hipError_t by_rules(const ScoreArgs& a, F f) {
  if (a.cap > 0.f) return a.slopes ? f(ScoreVariant<D, DT, true, true>()) : f(ScoreVariant<D, DT, true, false>());
  return a.slopes ? f(ScoreVariant<D, DT, false, true>()) : f(ScoreVariant<D, DT, false, false>());
}
template <class F>
static hipError_t by_variant(int dt, const ScoreArgs& a, F f) {
  if (a.D == 64) return dt == kF16 ? by_rules<64, kF16>(a, f) : by_rules<64, kBf16>(a, f);
  return dt == kF16 ? by_rules<128, kF16>(a, f) : by_rules<128, kBf16>(a, f);
}
inline size_t round_up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace lx
