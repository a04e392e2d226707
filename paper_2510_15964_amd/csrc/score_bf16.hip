// Attention over dense keys with rules on its scores, 16-bit types: forward, and backward in two passes.
//
// A workgroup of four wavefronts owns 128 rows (queries: forward, dQ; keys: dK/dV), 32 to a wavefront, and streams tiles of 64
// rows of the other side through LDS.  All products run on the 32x32x16 MFMA with the own rows as columns: S^T = K Q^T, so a
// lane holds scores of one query and the accumulators of the first product are, packed, the operand of the second one (the
// MFMA's k index may be permuted as long as both operands agree); the k-major operands (V^T, K^T, Q^T, dO^T) come from the same
// row-major tiles by the transposing LDS read.
//
// The keys of a query are one interval, so a tile lies outside, inside or across it, and only tiles across the end of some
// query's interval pay for masks.  In those a masked pair's factor is set to zero after the exponential, and rows of the tile
// that are not finite are zeroed before they are multiplied (0 * NaN); a factor that an attended pair has with such a row
// becomes NaN, so that nothing is hidden.
//
// Softmax in the log2 domain, statistics and accumulators in fp32; P and dS are rounded to the element type once, for the second
// product.
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

// Workgroup `w` of N: those of an XCD (w % 8) are consecutive ones, so that they share keys in its L2.
__device__ __forceinline__ int deal(int w, int N) {
  const int x = w % 8, whole = N / 8, rest = N % 8;
  return x * whole + min(x, rest) + w / 8;
}
// workgroup -> (batch entry, head, tile of own rows), the last tile, whose queries attend most, first
struct ScoreWork {
  int b, h, tile;
  __device__ __forceinline__ ScoreWork(int heads, int tiles) {
    const int i = deal(blockIdx.x, gridDim.x), pair = i / tiles;
    tile = tiles - 1 - (i - pair * tiles);
    b = pair / heads;
    h = pair - b * heads;
  }
};

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kSThreads, 2) void score_fwd(const ScoreArgs a) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[2][2 * kTileRows * D];   // K tile, V tile
  __shared__ KeySpan part[kSWaves];
  __shared__ unsigned bad_part[kSWaves];
  const ScoreWork wk(a.Hq, (a.Sq + kOwn - 1) / kOwn);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, half = lane / 32;
  const int hk = wk.h / (a.Hq / a.Hkv), q = wk.tile * kOwn + 32 * wave + lane % 32, qc = min(q, a.Sq - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  int lo, len;
  key_interval(a, wk.b, qc, start, lo, len);
  KeySpan span;
  span.of(q < a.Sq, lo, len);
  span.join_lanes<16>();
  span = scalar_span(span);
  const KeySpan all = span_of_workgroup(span, part);

  uint4 qf[D / 16];
  load_own<D>(a.Q, wk.b, wk.h, qc, qf);
  FastRules<CAP, BIAS> rules;
  rules.init(a, wk.h);
  ScoreDma<D> dma;
  dma.init();
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[0][0]);
  auto issue = [&](int stage, int k0) {
    const uint32_t to = ring0 + stage * kStage;
    dma.issue(to, score_row(a.K, wk.b, hk, k0), 2 * a.K.ss, a.Sk - 1 - k0);
    dma.issue(to + kTile, score_row(a.V, wk.b, hk, k0), 2 * a.V.ss, a.Sk - 1 - k0);
  };

  settle(qf);
  f32x16 o[D / 32] = {};
  // O is normalised by the sum of the rounded probabilities that it is made of: a row dominated by a few keys otherwise carries
  // their rounding errors as a whole, and Delta hands them on to the gradients.  LSE is of the unrounded ones.
  float m = -INFINITY, ref = 0.f, sum = 0.f, weight = 0.f;
  if (all.first < all.end) issue(0, all.first);
  int stage = 0;
  for (int k0 = all.first; k0 < all.end; k0 += kTileRows, stage ^= 1) {
    if (k0 + kTileRows < all.end) {
      issue(stage ^ 1, k0 + kTileRows);
      wait_vmcnt<2 * ScoreDma<D>::kPerWave>();
    } else {
      wait_vmcnt<0>();
    }
    lds_barrier();
    const uint32_t tk = ring0 + stage * kStage, tv = tk + kTile;
    unsigned long long bad = 0;
    if (!all.covers(k0, kTileRows)) bad = join_rows(clear_not_finite<D, DT>(tv), bad_part);
    if (span.touches(k0, kTileRows)) {
      f32x16 s[2] = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[t] = mfma32<DT>(read_piece<D>(tk, off, t, kk), qf[kk], s[t]);
      const float far = (float)(start + qc - k0 - 4 * half);
      float top = -INFINITY;
      const bool masked = !span.covers(k0, kTileRows);
      const int from = k0 + 4 * half - lo;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          float r;
          s[t][v] = rules.score(s[t][v], far - (float)(32 * t + acc_row(v)), r);
        }
      if (masked)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if ((unsigned)(from + 32 * t + acc_row(v)) >= (unsigned)len) s[t][v] = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(top, s[t][v]);
      // The reference point only has to bound the scores up to a factor that fp32 holds comfortably: it follows the maximum when
      // that has moved by more than kSSlack, which most tiles do for no query of the wavefront.
      if (__any(top > m + kSSlack)) {
        const float both = fmaxf(top, __shfl_xor(top, 32)), next = both > m + kSSlack ? both : m;
        ref = next == -INFINITY ? 0.f : next;
        const float shrink = __builtin_amdgcn_exp2f(m - ref);
        sum *= shrink;
        weight *= shrink;
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct) o[ct] *= shrink;
        m = next;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          s[t][v] = __builtin_amdgcn_exp2f(s[t][v] - ref);
          sum += s[t][v];
        }
      if (bad) {
        const unsigned long long mine = bad >> (4 * half);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if ((mine >> (32 * t + acc_row(v)) & 1) && (unsigned)(from + 32 * t + acc_row(v)) < (unsigned)len) s[t][v] = __builtin_nanf("");
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 p = pack_piece<DT>(s[t], j);
          weight = add_piece<DT>(p, weight);
#pragma unroll
          for (int ct = 0; ct < D / 32; ++ct) o[ct] = mfma32<DT>(read_piece_tr<D>(tv, off, t, j, ct), p, o[ct]);
        }
    }
    lds_barrier();      // the stage is free
  }
  sum += __shfl_xor(sum, 32);
  weight += __shfl_xor(weight, 32);
  if (q < a.Sq) {
    store_own<D, DT>(a.O, wk.b, wk.h, q, o, weight == 0.f ? 0.f : 1.f / weight);
    if (a.LSE && half == 0) a.LSE[((long long)wk.b * a.Hq + wk.h) * a.Sq + q] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * kSLn2;
  }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// Statistics of the queries that the query side leaves for the key side, padded to whole tiles (lse2: +inf, delta: 0, no
// keys), and the span of every tile.
struct ScoreStats {
  float *lse2, *delta;      // [B, Hq, rows]
  int *lo, *len;            // [B, rows]
  KeySpan* span;            // [B, rows / 64]
  int rows;
};
__host__ __device__ inline int stat_rows(int Sq) { return (Sq + kTileRows - 1) / kTileRows * kTileRows; }

template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kSThreads, 2) void score_dq(const ScoreArgs a, const ScoreStats st) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[2][2 * kTileRows * D];   // K tile, V tile
  __shared__ KeySpan part[kSWaves];
  __shared__ unsigned bad_part[kSWaves];
  const ScoreWork wk(a.Hq, (a.Sq + kOwn - 1) / kOwn);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, half = lane / 32;
  const int hk = wk.h / (a.Hq / a.Hkv), q = wk.tile * kOwn + 32 * wave + lane % 32, qc = min(q, a.Sq - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  int lo, len;
  key_interval(a, wk.b, qc, start, lo, len);
  KeySpan span;
  span.of(q < a.Sq, lo, len);
  span.join_lanes<16>();
  span = scalar_span(span);
  const KeySpan all = span_of_workgroup(span, part);
  if (wk.h == 0) {
    // of the two tiles of 64 queries
    const int tile = 2 * wk.tile + wave / 2;
    KeySpan both = part[wave & ~1];
    both.join(part[wave | 1]);
    if (wave % 2 == 0 && lane == 0 && tile * kTileRows < st.rows) st.span[(long long)wk.b * (st.rows / kTileRows) + tile] = both;
    if (half == 0 && q < st.rows) {
      st.lo[(long long)wk.b * st.rows + q] = lo;
      st.len[(long long)wk.b * st.rows + q] = q < a.Sq ? len : 0;
    }
  }

  uint4 qf[D / 16], gf[D / 16];
  load_own<D>(a.Q, wk.b, wk.h, qc, qf);
  load_own<D>(a.dO, wk.b, wk.h, qc, gf);
  float delta = 0.f;
  {
    uint4 of[D / 16];
    load_own<D>(a.O, wk.b, wk.h, qc, of);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const uint32_t x[4] = {gf[kk].x, gf[kk].y, gf[kk].z, gf[kk].w}, y[4] = {of[kk].x, of[kk].y, of[kk].z, of[kk].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        delta = fmaf(to_f32<DT>(x[i] & 0xffff), to_f32<DT>(y[i] & 0xffff), delta);
        delta = fmaf(to_f32<DT>(x[i] >> 16), to_f32<DT>(y[i] >> 16), delta);
      }
    }
    delta += __shfl_xor(delta, 32);
  }
  const long long head_row = (long long)wk.b * a.Hq + wk.h;
  const float lse = a.LSE[head_row * a.Sq + qc];
  const bool none = len <= 0 || lse == -INFINITY;
  const float lse2 = none ? INFINITY : lse * kSLog2e;
  if (none) delta = 0.f;
  if (half == 0 && q < st.rows) {
    st.lse2[head_row * st.rows + q] = q < a.Sq ? lse2 : INFINITY;
    st.delta[head_row * st.rows + q] = q < a.Sq ? delta : 0.f;
  }
  FastRules<CAP, BIAS> rules;
  rules.init(a, wk.h);
  ScoreDma<D> dma;
  dma.init();
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[0][0]);
  auto issue = [&](int stage, int k0) {
    const uint32_t to = ring0 + stage * kStage;
    dma.issue(to, score_row(a.K, wk.b, hk, k0), 2 * a.K.ss, a.Sk - 1 - k0);
    dma.issue(to + kTile, score_row(a.V, wk.b, hk, k0), 2 * a.V.ss, a.Sk - 1 - k0);
  };

  settle(qf);
  settle(gf);
  f32x16 g[D / 32] = {};
  if (all.first < all.end) issue(0, all.first);
  int stage = 0;
  for (int k0 = all.first; k0 < all.end; k0 += kTileRows, stage ^= 1) {
    if (k0 + kTileRows < all.end) {
      issue(stage ^ 1, k0 + kTileRows);
      wait_vmcnt<2 * ScoreDma<D>::kPerWave>();
    } else {
      wait_vmcnt<0>();
    }
    lds_barrier();
    const uint32_t tk = ring0 + stage * kStage, tv = tk + kTile;
    unsigned long long bad = 0;
    if (!all.covers(k0, kTileRows)) bad = join_rows(clear_not_finite<D, DT>(tk), bad_part);
    if (span.touches(k0, kTileRows)) {
      const float far = (float)(start + qc - k0 - 4 * half);
      const bool masked = !span.covers(k0, kTileRows);
      const int from = k0 + 4 * half - lo;
      const unsigned long long mine = bad >> (4 * half);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          s = mfma32<DT>(read_piece<D>(tk, off, t, kk), qf[kk], s);
          dp = mfma32<DT>(read_piece<D>(tv, off, t, kk), gf[kk], dp);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          float r;
          const float p = __builtin_amdgcn_exp2f(rules.score(s[v], far - (float)(32 * t + acc_row(v)), r) - lse2);
          dp[v] = p * (dp[v] - delta);
          if constexpr (CAP) dp[v] *= rules.derivative(r);
        }
        if (masked)
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const bool seen = (unsigned)(from + 32 * t + acc_row(v)) < (unsigned)len;
            if (!seen) dp[v] = 0.f;
            if (bad && seen && (mine >> (32 * t + acc_row(v)) & 1)) dp[v] = __builtin_nanf("");
          }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 p = pack_piece<DT>(dp, j);
#pragma unroll
          for (int ct = 0; ct < D / 32; ++ct) g[ct] = mfma32<DT>(read_piece_tr<D>(tk, off, t, j, ct), p, g[ct]);
        }
      }
    }
    lds_barrier();
  }
  if (q < a.Sq) store_own<D, DT>(a.dQ, wk.b, wk.h, q, g, a.scale);
}

// The tiles of queries that attend some key of a block, head after head of a group: 64 tiles' spans at a time, one a lane.
struct QueryWalk {
  const KeySpan* span;      // of the batch entry
  int tiles, k, n, h, h_end, base;
  unsigned long long left;
  KeySpan mine;             // of tile base + lane
  __device__ __forceinline__ void load() {
    const int t = base + threadIdx.x % kWave;
    mine = span[min(t, tiles - 1)];
    left = __ballot(t < tiles && mine.touches(k, n));
  }
  __device__ __forceinline__ KeySpan span_here() const {
    const int l = __ffsll((long long)left) - 1;
    return {__builtin_amdgcn_readlane(mine.first, l), __builtin_amdgcn_readlane(mine.end, l), __builtin_amdgcn_readlane(mine.all_from, l),
            __builtin_amdgcn_readlane(mine.all_to, l)};
  }
  __device__ __forceinline__ void init(const KeySpan* s, int nt, int key, int keys, int first_head, int heads) {
    span = s, tiles = nt, k = key, n = keys, h = first_head, h_end = first_head + heads, base = 0;
    load();
    settle();
  }
  __device__ __forceinline__ void settle() {      // to the next tile, if there is one
    while (!left && h < h_end) {
      base += kWave;
      if (base >= tiles) base = 0, ++h;
      if (h < h_end) load();
    }
  }
  __device__ __forceinline__ bool there() const { return h < h_end; }
  __device__ __forceinline__ int tile() const { return base + __ffsll((long long)left) - 1; }
  __device__ __forceinline__ void next() {
    left &= left - 1;
    settle();
  }
};

template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kSThreads, 2) void score_dkv(const ScoreArgs a, const ScoreStats st) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStat = kTileRows * 4, kStage = 2 * kTile + 4 * kStat;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[2][kStage];   // Q tile, dO tile, lse2, delta, lo, len
  __shared__ unsigned bad_part[2][kSWaves];
  const ScoreWork wk(a.Hkv, (a.Sk + kOwn - 1) / kOwn);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), half = lane / 32;
  const int group = a.Hq / a.Hkv, k_wg = wk.tile * kOwn, k_wave = k_wg + 32 * wave, k = k_wave + lane % 32, kc = min(k, a.Sk - 1);
  const int n_wg = min(kOwn, a.Sk - k_wg), n_wave = max(min(32, a.Sk - k_wave), 0);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  const KeySpan* spans = st.span + (long long)wk.b * (st.rows / kTileRows);

  uint4 kf[D / 16], vf[D / 16];
  load_own<D>(a.K, wk.b, wk.h, kc, kf);
  load_own<D>(a.V, wk.b, wk.h, kc, vf);
  ScoreDma<D> dma;
  dma.init();
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[0][0]);
  QueryWalk walk;
  walk.init(spans, st.rows / kTileRows, k_wg, n_wg, wk.h * group, group);
  auto issue = [&](int stage, int h, int tile) {
    const uint32_t to = ring0 + stage * kStage;
    const int q0 = tile * kTileRows;
    dma.issue(to, score_row(a.Q, wk.b, h, q0), 2 * a.Q.ss, a.Sq - 1 - q0);
    dma.issue(to + kTile, score_row(a.dO, wk.b, h, q0), 2 * a.dO.ss, a.Sq - 1 - q0);
    const long long of_head = ((long long)wk.b * a.Hq + h) * st.rows + q0, of_row = (long long)wk.b * st.rows + q0;
    const void* from = wave == 0 ? (const void*)(st.lse2 + of_head) : wave == 1 ? (const void*)(st.delta + of_head)
                       : wave == 2 ? (const void*)(st.lo + of_row) : (const void*)(st.len + of_row);
    dma4((const char*)from + 4 * lane, to + 2 * kTile + wave * kStat);
  };

  settle(kf);
  settle(vf);
  f32x16 gk[D / 32] = {}, gv[D / 32] = {};
  FastRules<CAP, BIAS> rules;
  if (walk.there()) issue(0, walk.h, walk.tile());
  int stage = 0, rules_of = -1;
  while (walk.there()) {
    const int h = walk.h, tile = walk.tile(), q0 = tile * kTileRows;
    const KeySpan span = walk.span_here();
    if (h != rules_of) rules.init(a, h), rules_of = h;
    walk.next();
    if (walk.there()) {
      issue(stage ^ 1, walk.h, walk.tile());
      wait_vmcnt<2 * ScoreDma<D>::kPerWave + 1>();
    } else {
      wait_vmcnt<0>();
    }
    lds_barrier();
    const uint32_t tq = ring0 + stage * kStage, tg = tq + kTile, ts = tg + kTile + 16 * half;
    unsigned long long bad = 0;
    if (!span.covers(k_wg, n_wg)) {
      bad = join_rows(clear_not_finite<D, DT>(tq), bad_part[0]);
      bad |= join_rows(clear_not_finite<D, DT>(tg), bad_part[1]);
    }
    if (n_wave > 0 && span.touches(k_wave, n_wave)) {
      const float far = (float)(start + q0 + 4 * half - kc);
      const bool masked = !span.covers(k_wave, n_wave);
      const unsigned long long mine = bad >> (4 * half);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          s = mfma32<DT>(read_piece<D>(tq, off, t, kk), kf[kk], s);
          dp = mfma32<DT>(read_piece<D>(tg, off, t, kk), vf[kk], dp);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 lse2 = __builtin_bit_cast(f32x4, lds_read16(ts + (32 * t + 8 * i) * 4));
          const f32x4 delta = __builtin_bit_cast(f32x4, lds_read16(ts + kStat + (32 * t + 8 * i) * 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = 4 * i + e;
            float r;
            const float p = __builtin_amdgcn_exp2f(rules.score(s[v], far + (float)(32 * t + acc_row(v)), r) - lse2[e]);
            dp[v] = p * (dp[v] - delta[e]);
            if constexpr (CAP) dp[v] *= rules.derivative(r);
            s[v] = p;
          }
        }
        if (masked)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 lo4 = lds_read16(ts + 2 * kStat + (32 * t + 8 * i) * 4), len4 = lds_read16(ts + 3 * kStat + (32 * t + 8 * i) * 4);
            const unsigned lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, len[4] = {len4.x, len4.y, len4.z, len4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int v = 4 * i + e;
              const bool seen = (unsigned)k - lo[e] < len[e];
              if (!seen) s[v] = dp[v] = 0.f;
              if (bad && seen && (mine >> (32 * t + acc_row(v)) & 1)) s[v] = dp[v] = __builtin_nanf("");
            }
          }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 p = pack_piece<DT>(s, j), ds = pack_piece<DT>(dp, j);
#pragma unroll
          for (int ct = 0; ct < D / 32; ++ct) {
            gv[ct] = mfma32<DT>(read_piece_tr<D>(tg, off, t, j, ct), p, gv[ct]);
            gk[ct] = mfma32<DT>(read_piece_tr<D>(tq, off, t, j, ct), ds, gk[ct]);
          }
        }
      }
    }
    lds_barrier();
    stage ^= 1;
  }
  if (k < a.Sk) {
    store_own<D, DT>(a.dK, wk.b, wk.h, k, gk, a.scale);
    store_own<D, DT>(a.dV, wk.b, wk.h, k, gv, 1.f);
  }
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
static size_t round_up256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t score_fwd_bytes(int, int, int, int, int, int) { return 0; }
size_t score_bwd_bytes(int B, int Hq, int, int Sq, int, int) {
  const size_t rows = stat_rows(Sq);
  return 2 * round_up256(B * (size_t)Hq * rows * 4) + 2 * round_up256(B * rows * 4) + round_up256(B * (rows / kTileRows) * sizeof(KeySpan));
}

template <int D, int DT, bool CAP, bool BIAS>
static hipError_t run_fwd(const ScoreArgs& a, hipStream_t st) {
  ProfScope p(kKScoreFwd, st);
  hipLaunchKernelGGL((score_fwd<D, DT, CAP, BIAS>), dim3((unsigned)((a.Sq + kOwn - 1) / kOwn * a.Hq * a.B)), dim3(kSThreads), 0, st, a);
  return hipGetLastError();
}
template <int D, int DT, bool CAP, bool BIAS>
static hipError_t run_bwd(const ScoreArgs& a, const ScoreStats& s, hipStream_t st) {
  {
    ProfScope p(kKScoreDq, st);
    hipLaunchKernelGGL((score_dq<D, DT, CAP, BIAS>), dim3((unsigned)((a.Sq + kOwn - 1) / kOwn * a.Hq * a.B)), dim3(kSThreads), 0, st, a, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfScope p(kKScoreDkv, st);
  hipLaunchKernelGGL((score_dkv<D, DT, CAP, BIAS>), dim3((unsigned)((a.Sk + kOwn - 1) / kOwn * a.Hkv * a.B)), dim3(kSThreads), 0, st, a, s);
  return hipGetLastError();
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
hipError_t launch_score_fwd_bf16(int dt, const ScoreArgs& a, hipStream_t st) {
  return by_variant(dt, a, [&](auto v) { return run_fwd<v.D, v.DT, v.CAP, v.BIAS>(a, st); });
}
hipError_t launch_score_bwd_bf16(int dt, const ScoreArgs& a, void* workspace, hipStream_t st) {
  ScoreStats s;
  s.rows = stat_rows(a.Sq);
  char* p = (char*)workspace;
  auto take = [&](size_t bytes) {
    char* r = p;
    p += round_up256(bytes);
    return r;
  };
  s.lse2 = (float*)take((size_t)a.B * a.Hq * s.rows * 4);
  s.delta = (float*)take((size_t)a.B * a.Hq * s.rows * 4);
  s.lo = (int*)take((size_t)a.B * s.rows * 4);
  s.len = (int*)take((size_t)a.B * s.rows * 4);
  s.span = (KeySpan*)take((size_t)a.B * (s.rows / kTileRows) * sizeof(KeySpan));
  return by_variant(dt, a, [&](auto v) { return run_bwd<v.D, v.DT, v.CAP, v.BIAS>(a, s, st); });
}

}  // namespace lx
