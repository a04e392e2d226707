// Attention over dense keys with rules on its scores, 16-bit types: forward, and backward in two passes.
//
// A workgroup of four wavefronts owns 128 rows (queries: forward, dQ; keys: dK/dV), 32 to a wavefront, and streams tiles of 64
// rows of the other side through LDS.  All products run on the 32x32x16 MFMA with the own rows as columns: S^T = K Q^T, so a
// lane holds scores of one query and the accumulators of the first product are, packed, the operand of the second one (the
// MFMA's k index may be permuted as long as both operands agree); the k-major operands (V^T, K^T, Q^T, dO^T) come from the same
// row-major tiles by the transposing LDS read.
//
// The keys of a query are one interval, so a tile lies outside, inside or across it, and only tiles across the end of some
// query's interval pay for masks.  In those a masked pair's factor is set to zero after the exponential.  Where a sum then still
// comes out not finite (0 * NaN), the workgroup starts again, and zeroes rows of masked tiles that are not finite before they are
// multiplied; the result of an own row that attends such a row becomes NaN as a whole, so that nothing is hidden.
//
// Two stages of LDS and one barrier per tile: behind it the tile has arrived, and the stage of the one before, with which everybody
// is done, takes the transfer of the next.
//
// Softmax in the log2 domain, statistics and accumulators in fp32; P and dS are rounded to the element type once, for the second
// product, which takes nothing wider (what that leaves as a product of its own, as over a cache, would be half the forward pass's
// products again).  Delta comes from O as it is stored where that is exact enough, otherwise from the products.  dQ and dK are 2.1e-3 to
// 3.1e-3 (bf16) and 2.6e-4 to 3.9e-4 (f16) of their norm off, where products in fp32 would leave the rounding of the result alone, 1.7e-3
// and 2.1e-4; where keys have a mean along which the errors of dS add up, dQ more: 3.7e-3 with a mean of one deviation, 4.8e-3 of two.
//
// Bound by issue at large sizes: a tile's vector instructions take as long as its matrix instructions, or twice as long with a cap, and
// half of either hides the other; sustained launches also meet the power limit.  8192 tokens, 32 heads on 8, D = 128, forward 528 - 575
// us, 0.96 - 1.04 PFLOP/s of the causal half; 4 x 2048 alike, forward 156 - 162, backward 488 - 505, capped 203 and 555 - 565: of the
// products as built 0.86, 0.97, 0.68 and 0.86 PFLOP/s.  At a few tiles per wavefront by latency and by workgroups of different lengths: 8 x 32 heads of 1024, D = 64,
// documents of 300 on average with slopes 61, 91 and 100 (by rocprofv3), of which 20, 31 and 34 are launch, own rows and results.
#include "score_tile.h"

namespace lx {

// Which workgroup of which (sequence, key head) pair this is: number z of `each`, its query heads' tiles one after the other (forward,
// dQ) or its tiles of keys.  Workgroup w runs on XCD w % 8.  Whole rounds of eight pairs are dealt to the XCDs in turn, all workgroups
// of a pair to one, whose L2 then holds the pair's keys; the key head is a pair's fast index, so that with eight of them or
// more every XCD has heads of every sequence, whose documents differ in length (8 x 32 heads of 1024 tokens in documents of 300 on
// average, forward, a sequence to an XCD 100 us, so 55).  The workgroups of the last pairs are spread over all XCDs in runs;
// `even`: all are dealt one by one, where a round would be heads of few sequences that may differ in length.
constexpr int kSet = 4;
struct ScoreWork {
  int b, hk, z;
  bool there;
  __device__ __forceinline__ ScoreWork(const ScoreArgs& a, int each, int even) {
    const int P = a.B * a.Hkv, w = blockIdx.x;
    int pair;
    there = true;
    if (even) {
      pair = w / each;
      z = w - pair * each;
    } else {
      const int x = w % 8, s = w / 8, whole = P / 8 * each;
      if (s < whole) {
        // kSet pairs of an XCD at a time, whose first z come first
        const int set = s / (kSet * each), in = s - set * kSet * each, pairs = min(kSet, P / 8 - set * kSet);
        z = in / pairs;
        pair = (set * kSet + in - z * pairs) * 8 + x;
      } else {
        const int rest = P % 8 * each, run = (rest + 7) / 8, r = x * run + s - whole;
        there = s - whole < run && r < rest;
        pair = P / 8 * 8 + r / each;
        z = r % each;
      }
    }
    b = pair / a.Hkv;
    hk = pair - b * a.Hkv;
  }
};
static int score_even(const ScoreArgs& a) { return a.Hkv % 8 != 0 && (a.key_lo || a.q_start); }
static unsigned score_grid(const ScoreArgs& a, int each) {
  const long long P = (long long)a.B * a.Hkv;
  return (unsigned)(score_even(a) ? P * each : 8 * (P / 8 * each + (P % 8 * each + 7) / 8));
}
// of a query side: the query head and the tile of queries, the last, which attend most, first
struct QueryWork : ScoreWork {
  int h, tile;
  __device__ __forceinline__ QueryWork(const ScoreArgs& a, int even) : ScoreWork(a, a.Hq / a.Hkv * ((a.Sq + kOwn - 1) / kOwn), even) {
    const int group = a.Hq / a.Hkv, t = z / group;
    h = hk * group + z - t * group;
    tile = (a.Sq + kOwn - 1) / kOwn - 1 - t;
  }
};

// Spans of the wavefront's 32 queries and of the workgroup's, from the rules alone or from the intervals that there are.  part: LDS,
// a span per wavefront of a team, written in either case.
__device__ __forceinline__ void spans_of_queries(const ScoreArgs& a, int start, int tile, bool there, int lo, int len, int pos, KeySpan* part,
                                                 KeySpan& span, KeySpan& all) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave % kSWaves);
  if (a.key_lo) {
    span.of(there, lo, len, pos);
    span = span_of_wave(span);
  } else {
    span = scalar_span(span_of_rows(a, start, tile * kOwn + 32 * wave, 32));
  }
  if (threadIdx.x % kWave == 0) part[wave] = span;
  lds_barrier();
  all = part[0];
#pragma unroll
  for (int w = 1; w < kSWaves; ++w) all.join(part[w]);
  all = scalar_span(all);
}

// Accumulators handed from one team to the other through LDS: a wavefront's to the one with the same own rows.
template <int N>
__device__ __forceinline__ void hand_over(uint32_t to, const f32x16 (&acc)[N]) {
  const uint32_t at = to + threadIdx.x % kSThreads * 16;
#pragma unroll
  for (int ct = 0; ct < N; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      lds_write16(at + (4 * ct + i) * (16 * kSThreads),
                  __builtin_bit_cast(uint4, f32x4{acc[ct][4 * i], acc[ct][4 * i + 1], acc[ct][4 * i + 2], acc[ct][4 * i + 3]}));
}
// acc * c + what was handed over * d
template <int N>
__device__ __forceinline__ void take_over(uint32_t from, f32x16 (&acc)[N], float c, float d) {
  const uint32_t at = from + threadIdx.x % kSThreads * 16;
#pragma unroll
  for (int ct = 0; ct < N; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = __builtin_bit_cast(f32x4, lds_read16(at + (4 * ct + i) * (16 * kSThreads)));
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[ct][4 * i + e] = fmaf(acc[ct][4 * i + e], c, v[e] * d);
    }
}
template <int N>
constexpr uint32_t kHanded = N * 64 * kSThreads;      // bytes of N accumulators

// NaN if some of the accumulators are not finite, otherwise zero.
template <int N>
__device__ __forceinline__ float not_finite(const f32x16 (&acc)[N]) {
  float sum[4] = {};
#pragma unroll
  for (int ct = 0; ct < N; ++ct)
#pragma unroll
    for (int v = 0; v < 16; ++v) sum[v % 4] = fmaf(acc[ct][v], 0.f, sum[v % 4]);
  return sum[0] + sum[1] + sum[2] + sum[3];
}
// The keys of the tiles that a workgroup streams: rows behind the last attended one are among them.
__device__ __forceinline__ int whole_tiles(const KeySpan& all, int teams) {
  const int step = teams * kTileRows, n = max(all.end - min(all.first, all.end), 0);
  return (n + step - 1) / step * step;
}
// pass(), whose result says whether its sums are finite, and where some wavefront's are not once more, carefully: with rows that are
// not finite cleared in masked tiles.  To look for them in every masked tile from the start took a pass over the tile and two barriers
// (8 x 32 heads of 1024 tokens, D = 64, documents of 300 on average: forward 69 us, dQ 80, dK/dV 110, so 64, 74 and 101); a workgroup
// that meets one now takes twice its time.  pass is told which of the two it is, as a type.  redo: LDS, a number per wavefront; contains
// a barrier.
__device__ __forceinline__ bool any_wave(bool mine, int* redo) {
  if (threadIdx.x % kWave == 0) redo[threadIdx.x / kWave] = mine;
  lds_barrier();
  int any = 0;
  for (int w = 0; w < (int)blockDim.x / kWave; ++w) any |= redo[w];
  return __builtin_amdgcn_readfirstlane(any);
}
template <class Pass>
__device__ __forceinline__ void do_carefully(bool& careful, int* redo, Pass pass) {
  if (!careful && !any_wave(__any(pass(std::false_type()) != 0.f), redo)) return;        // (NaN differs from zero)
  careful = true;
  pass(std::true_type());       // (a copy of its own: as one loop with the first both hold more registers, up to 52 bytes of them in memory)
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <int D, int DT, int CAP, bool BIAS, int TEAMS>
__global__ __launch_bounds__(kSThreads * TEAMS, D == 64 && TEAMS == 1 ? 3 : 2) void score_fwd(const ScoreArgs a, const int even) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[TEAMS][2][2 * kTileRows * D];   // K tile, V tile
  __shared__ KeySpan part[TEAMS][kSWaves];
  __shared__ unsigned bad_part[TEAMS][kSWaves];
  __shared__ int redo[TEAMS * kSWaves];
  const QueryWork wk(a, even);
  if (!wk.there) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave % kSWaves, half = lane / 32;
  const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kSThreads);
  const int hk = wk.hk, q = wk.tile * kOwn + 32 * wave + lane % 32, qc = min(q, a.Sq - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  uint4 qf[D / 16];
  load_own<D>(a.Q, wk.b, wk.h, qc, qf);
  int lo, len;
  key_interval(a, wk.b, qc, start, lo, len);
  KeySpan span, all;
  spans_of_queries(a, start, wk.tile, q < a.Sq, lo, len, start + qc, part[team], span, all);

  FastRules<CAP, BIAS> rules;
  rules.template init<true>(a, wk.h);
  ScoreDma<D> dma_k, dma_v;
  dma_k.init(a.K);
  dma_v.init(a.V);
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[team][0][0]);
  auto issue = [&](int stage, int k0) {
    const uint32_t to = ring0 + stage * kStage;
    dma_k.issue(to, score_row(a.K, wk.b, hk, k0), a.Sk - 1 - k0);
    dma_v.issue(to + kTile, score_row(a.V, wk.b, hk, k0), a.Sk - 1 - k0);
  };

  settle(qf);
  ScoreRow<D> row;
  bool careful = false;
  auto attend = [&](auto is_linear) {
    constexpr bool linear = decltype(is_linear)::value;
    f32x16 lift = {};
    if constexpr (linear) rules.lift(lift);
    constexpr int kStep = TEAMS * kTileRows;
    const int first = min(all.first, all.end);      // (of queries that attend nothing all.first is the largest number)
    int k0 = first + team * kTileRows, stage = 0;
    if (k0 < all.end) issue(0, k0);
    for (int base = first; base < all.end; base += kStep, k0 += kStep, stage ^= 1) {
      wait_vmcnt<0>();
      lds_barrier();        // the tile is there, and everybody is done with the one before, whose stage is free
      if (k0 + kStep < all.end) issue(stage ^ 1, k0 + kStep);
      const bool mine = k0 < all.end;
      const uint32_t tk = ring0 + stage * kStage;
      unsigned long long bad = 0;
      if (careful && !all.covers(base, kStep)) bad = join_rows(mine ? clear_not_finite<D, DT>(tk + kTile) : 0, bad_part[team]);
      if (mine && span.touches(k0, kTileRows)) {
        attend_tile<2, kTile, linear, D, DT, CAP, BIAS>(tk, off, qf, rules, lift, k0, start + qc, lo, len, !span.covers(k0, kTileRows), row);
        if (bad && (bad & keys_seen(k0, lo, len))) row.weight = __builtin_nanf("");
      }
    }
  };
  do_carefully(careful, redo, [&](auto) {
    row.clear();
    by_linear(rules, all.after, attend);
    return all.covers(all.first, whole_tiles(all, TEAMS)) ? 0.f : not_finite(row.o);
  });
  if constexpr (TEAMS == 2) {
    lds_barrier();
    const uint32_t here = lds_addr(&ring[0][0][0]), stats = here + kHanded<D / 32> + threadIdx.x % kSThreads * 16;
    if (team == 1) {
      hand_over(here, row.o);
      lds_write16(stats, __builtin_bit_cast(uint4, f32x4{row.m, row.sum, row.weight, 0.f}));
    }
    lds_barrier();
    if (team == 1) return;
    const f32x4 other = __builtin_bit_cast(f32x4, lds_read16(stats));
    const float m = fmaxf(row.m, other[0]), ref = m == -INFINITY ? 0.f : m;
    const float c = __builtin_amdgcn_exp2f(row.m - ref), d = __builtin_amdgcn_exp2f(other[0] - ref);
    take_over(here, row.o, c, d);
    row.sum = fmaf(row.sum, c, other[1] * d);
    row.weight = fmaf(row.weight, c, other[2] * d);
    row.m = m;
  }
  row.sum += __shfl_xor(row.sum, 32);
  row.weight += __shfl_xor(row.weight, 32);
  if (q < a.Sq) {
    store_own<D, DT>(a.O, wk.b, wk.h, q, row.o, row.weight == 0.f ? 0.f : 1.f / row.weight);
    if (a.LSE && half == 0)
      a.LSE[((long long)wk.b * a.Hq + wk.h) * a.Sq + q] = row.sum == 0.f ? -INFINITY : (row.m + rules.base(a) + __builtin_amdgcn_logf(row.sum)) * kSLn2;
  }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// Statistics of the queries that the query side leaves for the key side, padded to whole tiles (lse2: +inf, delta: 0, no
// keys), and the span of every tile.
struct ScoreStats {
  float *lse2, *delta;      // [B, Hq, rows]; delta: the negative of Delta
  float2* top;              // [B, Hq, rows / 32], f16: the largest |dO|^2, |Delta| of as many queries
  int *lo, *len;            // [B, rows]
  KeySpan* span;            // [B, rows / 64]
  int rows;
};
constexpr int kFewKeys = 32;
__host__ __device__ inline int stat_rows(int Sq) { return (Sq + kTileRows - 1) / kTileRows * kTileRows; }

template <int D, int DT, int CAP, bool BIAS, int TEAMS>
__global__ __launch_bounds__(kSThreads * TEAMS, D == 64 && TEAMS == 1 ? 3 : 2) void score_dq(const ScoreArgs a, const ScoreStats st, const int even) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[TEAMS][2][2 * kTileRows * D];   // K tile, V tile
  __shared__ KeySpan part[TEAMS][kSWaves], few_part[TEAMS][kSWaves];
  __shared__ int few_next[TEAMS][kSWaves];
  __shared__ float2 row_sums[TEAMS == 2 ? 2 : 1][kOwn];
  __shared__ float row_squares[kOwn];
  __shared__ unsigned bad_part[TEAMS][kSWaves];
  __shared__ int redo[TEAMS * kSWaves];
  const QueryWork wk(a, even);
  if (!wk.there) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave % kSWaves, half = lane / 32;
  const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kSThreads);
  const int hk = wk.hk, q = wk.tile * kOwn + 32 * wave + lane % 32, qc = min(q, a.Sq - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  uint4 qf[D / 16], gf[D / 16], of[D / 16];
  load_own<D>(a.Q, wk.b, wk.h, qc, qf);
  load_own<D>(a.dO, wk.b, wk.h, qc, gf);
  load_own<D>(a.O, wk.b, wk.h, qc, of);
  int lo, len;
  key_interval(a, wk.b, qc, start, lo, len);
  KeySpan span, all;
  spans_of_queries(a, start, wk.tile, q < a.Sq, lo, len, start + qc, part[team], span, all);
  if (wk.h == 0 && team == 0) {
    // of the two tiles of 64 queries
    const int tile = 2 * wk.tile + wave / 2;
    KeySpan both = span;
    both.join(part[0][wave ^ 1]);
    if (wave % 2 == 0 && lane == 0 && tile * kTileRows < st.rows) st.span[(long long)wk.b * (st.rows / kTileRows) + tile] = both;
    if (half == 0 && q < st.rows) {
      st.lo[(long long)wk.b * st.rows + q] = lo;
      st.len[(long long)wk.b * st.rows + q] = q < a.Sq ? len : 0;
    }
  }

  float delta = 0.f;       // of the stored O
  {
    float squares = 0.f;   // of its terms
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const uint32_t x[4] = {gf[kk].x, gf[kk].y, gf[kk].z, gf[kk].w}, y[4] = {of[kk].x, of[kk].y, of[kk].z, of[kk].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int shift = i % 2 * 16;
        const float dO = to_f32<DT>(x[i / 2] >> shift & 0xffff), O = to_f32<DT>(y[i / 2] >> shift & 0xffff);
        delta = fmaf(dO, O, delta);
        const float t = dO * (DT == kF16 ? fmaxf(fabsf(O), 0x1p-14f) : O);       // (half precision is no finer below)
        squares = fmaf(t, t, squares);
      }
    }
    delta += __shfl_xor(delta, 32);
    squares += __shfl_xor(squares, 32);
    if (half == 0 && team == 0) row_squares[32 * wave + lane] = squares;
  }
  const long long head_row = (long long)wk.b * a.Hq + wk.h;
  const float lse = a.LSE[head_row * a.Sq + qc];
  const bool none = len <= 0 || lse == -INFINITY;
  float lse2 = none ? INFINITY : lse * kSLog2e - FastRules<CAP, BIAS>::base(a);
  if (none) delta = 0.f;
  FastRules<CAP, BIAS> rules;
  rules.template init<true>(a, wk.h);
  ScoreDma<D> dma_k, dma_v;
  dma_k.init(a.K);
  dma_v.init(a.V);
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[team][0][0]);
  auto issue = [&](int stage, int k0) {
    const uint32_t to = ring0 + stage * kStage;
    dma_k.issue(to, score_row(a.K, wk.b, hk, k0), a.Sk - 1 - k0);
    dma_v.issue(to + kTile, score_row(a.V, wk.b, hk, k0), a.Sk - 1 - k0);
  };

  settle(qf);
  settle(gf);
  // Delta is the mean of dP under P.  From the stored O it is 2^-9 (bf16) of a row of V off, which is most of dS where few keys share a
  // query (dQ and dK of sequences of 5 tokens 3.8e-3 of their norm off, so 2.4e-3): there it is summed from the products, before the
  // pass.  The tiles that such queries attend, both teams alike.  (8 x 32 heads of 1024, documents of 300: dQ 71 us, so 75; three
  // sequences of 777 15.4 and 19; long sequences have them in one workgroup.)
  const bool few_keys = q < a.Sq && len > 0 && len <= kFewKeys;
  KeySpan few, few_all;
  few.of(few_keys, lo, len, start + qc);
  few = span_of_wave(few);
  if (lane == 0) few_part[team][wave] = few;
  lds_barrier();
  few_all = few_part[team][0];
#pragma unroll
  for (int w = 1; w < kSWaves; ++w) few_all.join(few_part[team][w]);
  few_all = scalar_span(few_all);
  if (few_all.end > 0) {
    const uint32_t rows = ring0 + off.rows;
    float sum = 0.f;
    for (int k0 = few_all.first; k0 < few_all.end;) {
      issue(0, k0);
      // the first key behind this tile that such a query attends: what lies between is not read
      const int next = -max_of_half(few_keys && lo + len - kTileRows > k0 ? -max(lo, k0 + kTileRows) : -kIntMax);
      if (lane == 0) few_next[team][wave] = next;
      wait_vmcnt<0>();
      lds_barrier();
      if (few.touches(k0, kTileRows)) {
        const float far = (float)(start + qc - k0 - 4 * half);
        const unsigned long long seen = keys_seen(k0, lo, len);
#pragma unroll 1
        for (int t = 0; t < 2; ++t) {
          f32x16 s = {}, dp = {};
          const uint32_t at = rows + t * (kTile / 2);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            s = mfma32<DT>(read_piece<D>(at, 0, 0, kk), qf[kk], s);
            dp = mfma32<DT>(read_piece<D>(at, kTile, 0, kk), gf[kk], dp);
          }
          const uint32_t word = (uint32_t)(seen >> (32 * t)) >> (4 * half);
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            float r;
            const float p = __builtin_amdgcn_exp2f(rules.score(s[v], far - (float)(32 * t + acc_row(v)), r) - lse2);
            sum += or_zero(spread_bit(word, acc_row(v)), p * dp[v]);
          }
        }
      }
      k0 = min(min(few_next[team][0], few_next[team][1]), min(few_next[team][2], few_next[team][3]));
      k0 = __builtin_amdgcn_readfirstlane(k0);
      lds_barrier();      // the stage is free
    }
    sum += __shfl_xor(sum, 32);
    if (few_keys && !none) delta = sum;
  }
  if (half == 0 && q < st.rows && team == 0) st.lse2[head_row * st.rows + q] = q < a.Sq ? lse2 : INFINITY;
  if (len == 1) lse2 = INFINITY;       // dS is zero, and so comes out as just that (what is not a number stays so)
  const bool stored = q < a.Sq && !none && len > kFewKeys;      // Delta is the stored O's
  // Half precision ends at 65504 and gets coarse below 2^-14, where gradients may well lie (dO of 1e-3, 4096 keys: dQ and dK 1.6e-3 off, so
  // 3.2e-4).  dS is made 2^up times as large, in the exponent, and dQ as much smaller.  A term of O is seldom much longer than O, so
  // that P |dP| is of the order of |dO| |O|: that comes near 2^2.  If some dS does not fit all the same, sums are not finite, and the
  // other pass brings |dO| near 2^-5, where rows of V of any size fit.
  constexpr int kNear = 2, kSafe = -5;
  auto half_exponent = [](float squared) { return (exponent_of(squared) + 1) >> 1; };
  int up = 0;
  const long long top_at = head_row * (st.rows / 32) + wk.tile * kSWaves + wave;
  const bool has_top = DT == kF16 && team == 0 && lane == 0 && (wk.tile * kSWaves + wave) * 32 < st.rows;
  if constexpr (DT == kF16) {
    const float norm = own_squares<DT>(gf), size = own_squares<DT>(of);
    up = norm > 0.f && norm < INFINITY && size < INFINITY ? (size > 0.f ? kNear : 0) - half_exponent(norm) - half_exponent(size) : 0;
    lse2 -= up;
    const float most = max_of_half(q < a.Sq && !none ? finite_or_zero(norm) : 0.f);
    if (has_top) st.top[top_at].x = most;
  }
  f32x16 g[D / 32];
  float gain = a.scale * FastRules<CAP, BIAS>::kDerivative;       // NaN where an attended key's row was cleared
  float sum = 0.f, square = 0.f;       // of P (dP - Delta), of dS
  bool careful = false;
  auto attend = [&](auto is_linear) __attribute__((always_inline)) {
    constexpr bool linear = decltype(is_linear)::value;
    f32x16 lift = {};
    if constexpr (linear) rules.lift(lift);
    // -Delta is where the sums of dP begin, unless there are no registers for it (168 with three wavefronts per SIMD)
    constexpr bool kFromDelta = D == 128 || TEAMS == 2;
    f32x16 from;
#pragma unroll
    for (int v = 0; v < 16; ++v) from[v] = kFromDelta ? -delta : 0.f;
    constexpr int kStep = TEAMS * kTileRows;
    const int first = min(all.first, all.end);      // (of queries that attend nothing all.first is the largest number)
    int k0 = first + team * kTileRows, stage = 0;
    if (k0 < all.end) issue(0, k0);
    for (int base = first; base < all.end; base += kStep, k0 += kStep, stage ^= 1) {
      wait_vmcnt<0>();
      lds_barrier();        // the tile is there, and everybody is done with the one before, whose stage is free
      if (k0 + kStep < all.end) issue(stage ^ 1, k0 + kStep);
      const bool mine = k0 < all.end;
      const uint32_t tk = ring0 + stage * kStage, rows = tk + off.rows, tr = tk + off.tr;
      unsigned long long bad = 0;
      if (careful && !all.covers(base, kStep)) bad = join_rows(mine ? clear_not_finite<D, DT>(tk) : 0, bad_part[team]);
      if (mine && span.touches(k0, kTileRows)) {
        const float far = (float)(start + qc - k0 - 4 * half);
        const bool masked = !span.covers(k0, kTileRows);
        const unsigned long long seen = keys_seen(k0, lo, len);
        if (bad & seen) gain = __builtin_nanf("");
        constexpr int KK = D / 16, CT = D / 32, kAheadQ = 2;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (!span.touches(k0 + 32 * t, 32)) continue;       // (half a tile; a copy of the forward loop for it costs more than it saves)
          f32x16 s = {}, dp = from;
          if constexpr (linear) s = lift;
          uint4 ka[kAheadQ + 1], va[kAheadQ + 1];
#pragma unroll
          for (int kk = 0; kk < kAheadQ; ++kk) ka[kk] = read_piece<D>(rows, 0, t, kk), va[kk] = read_piece<D>(rows, kTile, t, kk);
          end_slot();
          wave_priority<1>();
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            const int next = kk + kAheadQ;
            if (next < KK) {
              ka[next % (kAheadQ + 1)] = read_piece<D>(rows, 0, t, next);
              va[next % (kAheadQ + 1)] = read_piece<D>(rows, kTile, t, next);
            }
            s = mfma32<DT>(ka[kk % (kAheadQ + 1)], qf[kk], s);
            dp = mfma32<DT>(va[kk % (kAheadQ + 1)], gf[kk], dp);
            end_slot();
          }
          uint4 kt[kAheadQ + 2];
          wave_priority<0>();
#pragma unroll
          for (int n = 0; n <= kAheadQ; ++n) kt[n] = read_piece_tr<D>(tr, 0, t, n / CT, n % CT);
          end_slot();
          if constexpr (linear) {
            const float base = rules.slope * ((float)(32 * t) - far) - lse2;
#pragma unroll
            for (int v = 0; v < 16; ++v) dp[v] = __builtin_amdgcn_exp2f(fmaf(s[v], rules.c, base)) * (kFromDelta ? dp[v] : dp[v] - delta);
          } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              float r;
              const float p = __builtin_amdgcn_exp2f(rules.score(s[v], far - (float)(32 * t + acc_row(v)), r) - lse2);
              dp[v] = p * (kFromDelta ? dp[v] : dp[v] - delta);
              if constexpr (CAP) s[v] = rules.derivative(r);
            }
          }
          if (masked) {
            const uint32_t word = (uint32_t)(seen >> (32 * t)) >> (4 * half);
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const uint32_t bit = spread_bit(word, acc_row(v));
              dp[v] = or_zero(bit, dp[v]);
              if constexpr (CAP) s[v] = or_zero(bit, s[v]);
            }
          }
          if constexpr (CAP)
#pragma unroll
            for (int v = 0; v < 16; ++v) sum += dp[v], dp[v] *= s[v];
          const uint4 p = pack_piece<DT>(dp, 0), p1 = pack_piece<DT>(dp, 1);
          end_slot();
          wave_priority<1>();
#pragma unroll
          for (int n = 0; n < 2 * CT; ++n) {
            const int next = n + kAheadQ + 1;
            if (next < 2 * CT) kt[next % (kAheadQ + 2)] = read_piece_tr<D>(tr, 0, t, next / CT, next % CT);
            g[n % CT] = mfma32<DT>(kt[n % (kAheadQ + 2)], n < CT ? p : p1, g[n % CT]);
            if (n % (CT / 2) == 0) {       // a quarter of dS
              const uint4 ds = n < CT ? p : p1;
              const uint32_t lo2 = n % CT == 0 ? ds.x : ds.z, hi2 = n % CT == 0 ? ds.y : ds.w;
              if constexpr (!CAP) sum = dot2<DT>(hi2, kOnes<DT>, dot2<DT>(lo2, kOnes<DT>, sum));
              square = dot2<DT>(hi2, hi2, dot2<DT>(lo2, lo2, square));
            }
            end_slot();
          }
          wave_priority<0>();
        }
      }
    }
  };
  // One more pass for every workgroup where some wavefront's sums are not finite, and a shorter one for wavefronts whose Delta is not good
  // enough.  The stored O's is off by the rounding of O, u = 2^-9 / sqrt(3) of the root of `squares`, and puts that times sum P K into dQ;
  // next to it stands the rounding of dS, u of the root of sum dS^2 K^2.  Where the squares of the one are more than four times those of
  // the other, over the queries of a wavefront - scores that leave few keys their weight, values with a mean that their sum over the
  // keys keeps - sum P K is made, and taken off dQ as often as the sum of dS says, which ought to be zero (it carries dS's own rounding
  // too, whose part along the mean of the keys so goes as well).  The key side gets the exact Delta for all queries.
  // (Four: with the result's own and dS's the worst is sqrt(6) times 1.67e-3 for bf16, within the gate of 5e-3.  Normal data, 512 tokens, dQ
  // off by: bias of 2 and 4 per key 2.2e-3, without the correction 4.9e-3 and 1.3e-2; scores of deviation 16 2.1e-3 and 6e-3; values and
  // keys of mean 1 2.5e-3 and 1.6e-2.  The sums and the test: backward 4 x 2048, 32 heads on 8, D = 128, 488 us, so 500, with a cap 552
  // and 564; 8 x 32 heads of 1024, D = 64, 179 and 188.  All wavefronts corrected, scores of deviation 8: 669 and 238; a second whole
  // pass 696 and 255.  Documents of 300 with slopes from 0.84 down: dQ 84 without a correction, 90 with four, 106 with three.)
  constexpr float kWorthwhile = 4.f, kPart = FastRules<CAP, BIAS>::kDerivative;       // (dS is a part of itself)
  auto clear = [&] {
    sum = square = 0.f;
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) g[ct] = f32x16{};
  };
  clear();
  by_linear(rules, all.after, attend);
  int any;
  KeySpan wanted;
  for (;;) {
    sum += __shfl_xor(sum, 32);
    square += __shfl_xor(square, 32);
    if constexpr (TEAMS == 2) {
      if (half == 0) row_sums[team][32 * wave + lane] = make_float2(sum, square);
      lds_barrier();
      const float2 x = row_sums[0][32 * wave + lane % 32], y = row_sums[1][32 * wave + lane % 32];
      sum = x.x + y.x, square = x.y + y.y;
    }
    const float row_square = DT == kF16 ? times_pow2(square, -2 * up) : square, squares = row_squares[32 * wave + lane % 32];
    const bool counts = stored && row_square < INFINITY && squares < INFINITY;
    const bool repeat = sum_of_half(counts ? squares - kWorthwhile * kPart * kPart * row_square : 0.f) > 0.f;
    const bool again = !careful && (DT == kF16 || !all.covers(all.first, whole_tiles(all, TEAMS))) && __any(not_finite(g) != 0.f);      // (NaN differs from zero)
    wanted = span;
    wanted.only_if(repeat);
    if (lane == 0) redo[threadIdx.x / kWave] = again * 2 + repeat, part[team][wave] = wanted;
    lds_barrier();
    any = 0;
    for (int w = 0; w < TEAMS * kSWaves; ++w) any |= redo[w];
    any = __builtin_amdgcn_readfirstlane(any);
    if (any < 2) break;
    careful = true;
    if constexpr (DT == kF16) {
      const float norm = own_squares<DT>(gf);
      const int next = min(up, norm > 0.f && norm < INFINITY ? kSafe - half_exponent(norm) : 0);
      lse2 += up - next, up = next;
    }
    clear();
    attend(std::false_type());       // (a copy of its own: as one loop with the first both hold more registers, up to 52 bytes of them in memory)
  }
  if (stored) delta += DT == kF16 ? times_pow2(sum, -up) : sum;
  if (any) {
    all = part[team][0];
#pragma unroll
    for (int w = 1; w < kSWaves; ++w) all.join(part[team][w]);
    all = scalar_span(all);
    auto issue_k = [&](int stage, int k0) { dma_k.issue(ring0 + stage * kStage, score_row(a.K, wk.b, hk, k0), a.Sk - 1 - k0); };
    const float to_one = lse2 + up;
    f32x16 b[D / 32];
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) b[ct] = f32x16{};
    constexpr int kStep = TEAMS * kTileRows;
    int k0 = all.first + team * kTileRows, stage = 0;
    if (k0 < all.end) issue_k(0, k0);
    for (int base = all.first; base < all.end; base += kStep, k0 += kStep, stage ^= 1) {
      wait_vmcnt<0>();
      lds_barrier();
      if (k0 + kStep < all.end) issue_k(stage ^ 1, k0 + kStep);
      const bool mine = k0 < all.end;
      const uint32_t tk = ring0 + stage * kStage, rows = tk + off.rows, tr = tk + off.tr;
      if (careful && !all.covers(base, kStep)) join_rows(mine ? clear_not_finite<D, DT>(tk) : 0, bad_part[team]);
      if (!mine || !wanted.touches(k0, kTileRows)) continue;
      const float far = (float)(start + qc - k0 - 4 * half);
      const bool masked = !wanted.covers(k0, kTileRows);
      const unsigned long long seen = keys_seen(k0, lo, len);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (!wanted.touches(k0 + 32 * t, 32)) continue;
        f32x16 s = {};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) s = mfma32<DT>(read_piece<D>(rows, 0, t, kk), qf[kk], s);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          float r;
          s[v] = __builtin_amdgcn_exp2f(rules.score(s[v], far - (float)(32 * t + acc_row(v)), r) - to_one);
          if constexpr (CAP) s[v] *= rules.derivative(r);
        }
        if (masked) {
          const uint32_t word = (uint32_t)(seen >> (32 * t)) >> (4 * half);
#pragma unroll
          for (int v = 0; v < 16; ++v) s[v] = or_zero(spread_bit(word, acc_row(v)), s[v]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 p = pack_piece<DT>(s, j);
#pragma unroll
          for (int ct = 0; ct < D / 32; ++ct) b[ct] = mfma32<DT>(read_piece_tr<D>(tr, 0, t, j, ct), p, b[ct]);
        }
      }
    }
    if (wanted.end > 0)
#pragma unroll
      for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
        for (int v = 0; v < 16; ++v) g[ct][v] = fmaf(-sum, b[ct][v], g[ct][v]);
  }
  if (half == 0 && q < st.rows && team == 0) st.delta[head_row * st.rows + q] = q < a.Sq ? -delta : 0.f;
  if constexpr (DT == kF16) {
    const float most = max_of_half(q < a.Sq ? finite_or_zero(fabsf(delta)) : 0.f);
    if (has_top) st.top[top_at].y = most;
    gain = times_pow2(gain, -up);
  }
  if constexpr (TEAMS == 2) {
    lds_barrier();
    const uint32_t here = lds_addr(&ring[0][0][0]), gains = here + kHanded<D / 32> + threadIdx.x % kSThreads * 16;
    if (team == 1) {
      hand_over(here, g);
      lds_write16(gains, make_uint4(__builtin_bit_cast(uint32_t, gain), 0, 0, 0));
    }
    lds_barrier();
    if (team == 1) return;
    take_over(here, g, 1.f, 1.f);
    const float other = __builtin_bit_cast(float, lds_read4(gains));
    if (other != other) gain = other;
  }
  if (q < a.Sq) store_own<D, DT>(a.dQ, wk.b, wk.h, q, g, gain);
}

// The tiles of queries that attend some key of the workgroup's, head after head of a group.  What the keys of the workgroup and of
// the wavefront are to 64 tiles at a time is kept as a bit per tile.
struct QueryWalk {
  const KeySpan* span;      // of the batch entry
  int tiles, k_wg, n_wg, k_wave, n_wave, h, h_end, base;
  unsigned long long left, all_wg, some_wave, all_wave;
  __device__ __forceinline__ void load() {
    const int t = base + threadIdx.x % kWave;
    const KeySpan s = span[min(t, tiles - 1)];
    left = __ballot(t < tiles && s.touches(k_wg, n_wg));
    all_wg = __ballot(s.covers(k_wg, n_wg));
    some_wave = n_wave > 0 ? __ballot(s.touches(k_wave, n_wave)) : 0;
    all_wave = __ballot(s.covers(k_wave, n_wave));
  }
  __device__ __forceinline__ void init(const KeySpan* s, int nt, int keys, int Sk, int key, int first_head, int heads) {
    span = s, tiles = nt, h = first_head, h_end = first_head + heads, base = 0;
    k_wg = keys, n_wg = min(kOwn, Sk - k_wg), k_wave = key, n_wave = max(min(32, Sk - k_wave), 0);
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
  __device__ __forceinline__ int bit() const { return __ffsll((long long)left) - 1; }
  __device__ __forceinline__ int tile() const { return base + bit(); }
  __device__ __forceinline__ void next() {
    left &= left - 1;
    settle();
  }
};

// Where there are few tiles of keys the query heads of a group are shared out among n workgroups, which leave sums in fp32:
// [part][dK, dV][B, Hkv, Sk, D].
struct ScoreParts {
  int n;
  float* sums;
};
template <int D>
__device__ __forceinline__ void store_part(float* row, const f32x16 (&acc)[D / 32], float c) {
  f32x4* p = (f32x4*)row + threadIdx.x % kWave / 32;
#pragma unroll
  for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i) p[8 * ct + 2 * i] = f32x4{acc[ct][4 * i] * c, acc[ct][4 * i + 1] * c, acc[ct][4 * i + 2] * c, acc[ct][4 * i + 3] * c};
}

// What a team works on next: a tile of queries of a head.  `is`, as bits (truth values would be two scalar registers each): kThere,
// kTeams (some team has one), kTouches (the wavefront's keys), kMasked (not by all queries), kWhole (every query of the teams'
// tiles attends every key of the workgroup).
struct QueryItem {
  enum { kThere = 1, kTeams = 2, kTouches = 4, kMasked = 8, kWhole = 16 };
  int h, tile, is;
};
// Teams take the walk's tiles in turn.
template <int TEAMS>
__device__ __forceinline__ QueryItem next_item(QueryWalk& walk, int team) {
  QueryItem mine = {0, 0, QueryItem::kWhole};
#pragma unroll
  for (int t = 0; t < TEAMS; ++t) {
    if (!walk.there()) break;
    const int bit = walk.bit();
    mine.is |= QueryItem::kTeams;
    if (!(walk.all_wg >> bit & 1)) mine.is &= ~QueryItem::kWhole;
    if (t == team) {
      mine.h = walk.h, mine.tile = walk.tile();
      mine.is |= QueryItem::kThere | (int)(walk.some_wave >> bit & 1) * QueryItem::kTouches | (int)(~walk.all_wave >> bit & 1) * QueryItem::kMasked;
    }
    walk.next();
  }
  return mine;
}

// (dK, dV, the own rows and a tile of scores are 224 of 256 registers at D = 128: an operand's registers are filled again right behind
// its product, no further ahead; a register in scratch memory would cost the transfers ahead.)
template <int D, int DT, int CAP, bool BIAS, int TEAMS>
__global__ __launch_bounds__(kSThreads * TEAMS, D == 64 && TEAMS == 1 ? 3 : 2) void score_dkv(const ScoreArgs a, const ScoreStats st, const ScoreParts parts, const int even) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStat = kTileRows * 4, kStage = 2 * kTile + 4 * kStat;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[TEAMS][2][kStage];   // Q tile, dO tile, lse2, delta, lo, len
  __shared__ unsigned bad_part[TEAMS][2][kSWaves];
  __shared__ int redo[TEAMS * kSWaves];
  const ScoreWork wk(a, (a.Sk + kOwn - 1) / kOwn * parts.n, even);
  if (!wk.there) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave % kSWaves), half = lane / 32;
  const int team = TEAMS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kSThreads);
  const int group = a.Hq / a.Hkv, part = wk.z % parts.n, k_wg = wk.z / parts.n * kOwn, k_wave = k_wg + 32 * wave, k = k_wave + lane % 32, kc = min(k, a.Sk - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  const KeySpan* spans = st.span + (long long)wk.b * (st.rows / kTileRows);

  uint4 kf[D / 16], vf[D / 16];
  load_own<D>(a.K, wk.b, wk.hk, kc, kf);
  load_own<D>(a.V, wk.b, wk.hk, kc, vf);
  ScoreDma<D, D == 64> dma_q, dma_g;
  dma_q.init(a.Q);
  dma_g.init(a.dO);
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[team][0][0]);
  auto issue = [&](int stage, int h, int tile) {
    const uint32_t to = ring0 + stage * kStage;
    const int q0 = tile * kTileRows;
    dma_q.issue(to, score_row(a.Q, wk.b, h, q0), a.Sq - 1 - q0);
    dma_g.issue(to + kTile, score_row(a.dO, wk.b, h, q0), a.Sq - 1 - q0);
    const long long of_head = ((long long)wk.b * a.Hq + h) * st.rows + q0, of_row = (long long)wk.b * st.rows + q0;
    const void* from = wave == 0 ? (const void*)(st.lse2 + of_head) : wave == 1 ? (const void*)(st.delta + of_head)
                       : wave == 2 ? (const void*)(st.lo + of_row) : (const void*)(st.len + of_row);
    dma4((const char*)from + 4 * lane, to + 2 * kTile + wave * kStat);
  };

  // Half precision ends at 65504 and gets coarse below 2^-14.  Every dS is within `bound`, by |P (dP - Delta)| <= |dO| |V| + |Delta| with the
  // largest dO and Delta of the heads' queries and V of the wavefront's keys; most P are about 1 / Sk, and dP a sixteenth of the bound: at
  // a bound of 2^-6 Sk such a dS is 2^-10, and the four binades to 2^-14 are for large scores, where most are smaller (with 2^-8 Sk as the limit
  // dK of 21 queries was 6.6e-4 off for 2.9e-4; the times are the same).
  // Where that leaves the range, P is made `up` times as large and dS `up_ds` times, both powers of two, as far as 2^15 holds them, and
  // dV and dK as much smaller, by the second form of the pass, at once.  (4 x 2048, 32 heads on 8, D = 128, backward 525 us, with dO of 1e-3
  // 538; in the exponent, in every call, 561; a branch around it in the loop costs registers in memory.)
  float up = 1.f, up_ds = 1.f;
  bool careful = false;
  if constexpr (DT == kF16) {
    const int heads = group / parts.n, n = heads * (st.rows / 32);
    const float2* top = st.top + ((long long)wk.b * a.Hq + wk.hk * group + part * heads) * (st.rows / 32);
    float norm = 0.f, delta = 0.f;
    for (int i = lane; i < n; i += kWave) norm = fmaxf(norm, top[i].x), delta = fmaxf(delta, top[i].y);
    float v2 = finite_or_zero(own_squares<DT>(vf));
#pragma unroll
    for (int o = 32; o; o >>= 1) norm = fmaxf(norm, __shfl_xor(norm, o)), delta = fmaxf(delta, __shfl_xor(delta, o)), v2 = fmaxf(v2, __shfl_xor(v2, o));
    const int bound = exponent_of(1.001f * (__builtin_amdgcn_sqrtf(norm) * __builtin_amdgcn_sqrtf(v2) + delta)), keys = exponent_of((float)a.Sk);
    const int most = 15 - bound;
    if (most < 0 || keys > 13 || bound - keys < -6) {
      up = times_pow2(1.f, __builtin_amdgcn_readfirstlane(14));
      up_ds = times_pow2(1.f, __builtin_amdgcn_readfirstlane(min(most, 28)));
    }
    careful = any_wave(up != 1.f, redo);
  }
  settle(kf);
  settle(vf);
  f32x16 gk[D / 32], gv[D / 32];
  float gain = 1.f;       // NaN where an attending query's row was cleared
  FastRules<CAP, BIAS> rules;
  bool whole = true;       // all queries that were met attend all keys
  do_carefully(careful, redo, [&](auto second) {
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct) gk[ct] = gv[ct] = f32x16{};
    QueryWalk walk;
    walk.init(spans, st.rows / kTileRows, k_wg, a.Sk, k_wave, wk.hk * group + part * (group / parts.n), group / parts.n);
    int stage = 0, rules_of = -1;
    QueryItem now = next_item<TEAMS>(walk, team);
    if (now.is & QueryItem::kThere) issue(0, now.h, now.tile);
    while (now.is & QueryItem::kTeams) {
      const QueryItem next = next_item<TEAMS>(walk, team);
      if ((now.is & QueryItem::kThere) && now.h != rules_of) rules.template init<true>(a, now.h), rules_of = now.h;
      wait_vmcnt<0>();
      lds_barrier();
      if (next.is & QueryItem::kThere) issue(stage ^ 1, next.h, next.tile);
      const int q0 = now.tile * kTileRows;
      const uint32_t tq = ring0 + stage * kStage, tg = tq + kTile, ts = tg + kTile + 16 * half, rows = tq + off.rows, tr = tq + off.tr;
      unsigned long long bad = 0;
      whole = whole && (now.is & QueryItem::kWhole);
      if (careful && !(now.is & QueryItem::kWhole)) {
        bad = join_rows(now.is & QueryItem::kThere ? clear_not_finite<D, DT>(tq) : 0, bad_part[team][0]);
        bad |= join_rows(now.is & QueryItem::kThere ? clear_not_finite<D, DT>(tg) : 0, bad_part[team][1]);
      }
      if (now.is & QueryItem::kTouches) {
        const float far = (float)(start + q0 + 4 * half - kc);
        for (unsigned long long left = bad; left; left &= left - 1) {
          const int r = 4 * (__ffsll((long long)left) - 1);
          if ((unsigned)k - lds_read4(tg + kTile + 2 * kStat + r) < lds_read4(tg + kTile + 3 * kStat + r)) gain = __builtin_nanf("");
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // -Delta is where the sums of dP begin
          f32x16 s = {}, dp;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 delta = __builtin_bit_cast(f32x4, lds_read16(ts + kStat + (32 * t + 8 * i) * 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) dp[4 * i + e] = delta[e];
          }
          uint4 qa = read_piece<D>(rows, 0, t, 0), ga = read_piece<D>(rows, kTile, t, 0);
          end_slot();
          wave_priority<1>();
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            s = mfma32<DT>(qa, kf[kk], s);
            if (kk + 1 < D / 16) qa = read_piece<D>(rows, 0, t, kk + 1);
            end_slot();
            dp = mfma32<DT>(ga, vf[kk], dp);
            if (kk + 1 < D / 16) ga = read_piece<D>(rows, kTile, t, kk + 1);
            end_slot();
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i == 0) wave_priority<0>();
            const f32x4 lse2 = __builtin_bit_cast(f32x4, lds_read16(ts + (32 * t + 8 * i) * 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int v = 4 * i + e;
              float r;
              const float p = __builtin_amdgcn_exp2f(rules.score(s[v], far + (float)(32 * t + acc_row(v)), r) - lse2[e]);
              dp[v] *= p;
              if constexpr (CAP) dp[v] *= rules.derivative(r);
              s[v] = p;
            }
            end_slot();
          }
          if constexpr (DT == kF16 && decltype(second)::value)
#pragma unroll
            for (int v = 0; v < 16; ++v) s[v] *= up, dp[v] *= up_ds;
          if (now.is & QueryItem::kMasked)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint4 lo4 = lds_read16(ts + 2 * kStat + (32 * t + 8 * i) * 4), len4 = lds_read16(ts + 3 * kStat + (32 * t + 8 * i) * 4);
              const unsigned lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, len[4] = {len4.x, len4.y, len4.z, len4.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int v = 4 * i + e;
                if ((unsigned)k - lo[e] >= len[e]) s[v] = dp[v] = 0.f;
              }
              end_slot();
            }
          uint4 p[2], ds[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) p[j] = pack_piece<DT>(s, j), ds[j] = pack_piece<DT>(dp, j);
          ga = read_piece_tr<D>(tr, kTile, t, 0, 0);
          qa = read_piece_tr<D>(tr, 0, t, 0, 0);
          end_slot();
          constexpr int kCt = D / 32;
          wave_priority<1>();
#pragma unroll
          for (int i = 0; i < 2 * kCt; ++i) {
            gv[i % kCt] = mfma32<DT>(ga, p[i / kCt], gv[i % kCt]);
            if (i + 1 < 2 * kCt) ga = read_piece_tr<D>(tr, kTile, t, (i + 1) / kCt, (i + 1) % kCt);
            end_slot();
            gk[i % kCt] = mfma32<DT>(qa, ds[i / kCt], gk[i % kCt]);
            if (i + 1 < 2 * kCt) qa = read_piece_tr<D>(tr, 0, t, (i + 1) / kCt, (i + 1) % kCt);
            end_slot();
          }
          wave_priority<0>();
        }
      }
      stage ^= 1;
      now = next;
    }
    return whole ? 0.f : not_finite(gk) + not_finite(gv);
  });
  // one team finishes dK, the other dV
  if constexpr (TEAMS == 2) {
    lds_barrier();
    const uint32_t here = lds_addr(&ring[0][0][0]);
    uint32_t* gains = &bad_part[0][0][0];      // NaN of any wavefront's lane: whether, a bit per own row
    static_assert(sizeof(bad_part) >= 2 * kSWaves * sizeof(uint32_t), "a word per wavefront");
    const unsigned long long nan_rows = __ballot(gain != gain);
    if (lane == 0) gains[team * kSWaves + wave] = (uint32_t)nan_rows;
    if (team == 1) hand_over(here, gk);
    else hand_over(here + kHanded<D / 32>, gv);
    lds_barrier();
    if (gains[(team ^ 1) * kSWaves + wave] >> (lane % 32) & 1) gain = __builtin_nanf("");
    if (team == 0) take_over(here, gk, 1.f, 1.f);
    else take_over(here + kHanded<D / 32>, gv, 1.f, 1.f);
  }
  if (k < a.Sk) {
    const float gain_k = a.Sk == 1 ? gain * 0.f : a.scale * rules.kDerivative * gain / up_ds;       // (of one key: zero, and comes out as just that)
    gain /= up;
    if (parts.n > 1) {
      const long long row = ((long long)wk.b * a.Hkv + wk.hk) * a.Sk + k, of_part = (long long)a.B * a.Hkv * a.Sk * D;
      if (TEAMS == 1 || team == 0) store_part<D>(parts.sums + 2 * part * of_part + row * D, gk, gain_k);
      if (TEAMS == 1 || team == 1) store_part<D>(parts.sums + (2 * part + 1) * of_part + row * D, gv, gain);
    } else {
      if (TEAMS == 1 || team == 0) store_own<D, DT>(a.dK, wk.b, wk.hk, k, gk, gain_k);
      if (TEAMS == 1 || team == 1) store_own<D, DT>(a.dV, wk.b, wk.hk, k, gv, gain);
    }
  }
}

// Adds the parts of dK and dV in order: four elements of each per thread.
template <int D, int DT>
__global__ __launch_bounds__(256) void score_add_parts(const ScoreArgs a, const ScoreParts parts) {
  const long long of_part = (long long)a.B * a.Hkv * a.Sk * D, i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= of_part) return;
  f32x4 gk = {}, gv = {};
  for (int p = 0; p < parts.n; ++p) {
    gk += *(const f32x4*)(parts.sums + 2 * p * of_part + i);
    gv += *(const f32x4*)(parts.sums + (2 * p + 1) * of_part + i);
  }
  const long long row = i / D, pair = row / a.Sk;
  const int c = (int)(i % D), k = (int)(row - pair * a.Sk), b = (int)(pair / a.Hkv), hk = (int)(pair - (long long)b * a.Hkv);
  *(uint2*)(const_cast<char*>(score_row(a.dK, b, hk, k)) + 2 * c) = make_uint2(pack2<DT>(gk[0], gk[1]), pack2<DT>(gk[2], gk[3]));
  *(uint2*)(const_cast<char*>(score_row(a.dV, b, hk, k)) + 2 * c) = make_uint2(pack2<DT>(gv[0], gv[1]), pack2<DT>(gv[2], gv[3]));
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
// Parts that the heads of a group fall into on the key side: with at most half a workgroup per CU, the largest number that
// divides the group and leaves at most two of them per CU.  Sums in fp32 are written and read for it.  1 x 8 heads on one of 4096, D =
// 128, causal, 773 us in one part, 398 in two, 211 in four, 133 in eight; 4 x 32 on 4 of 512 115, 71, 51 and 51.
static int key_parts(int B, int Hq, int Hkv, int Sk) {
  const long long wgs = (long long)B * Hkv * ((Sk + kOwn - 1) / kOwn);
  const int group = Hq / Hkv;
  int n = 1;
  if (wgs <= kCUs / 2)
    for (int p = 2; p <= group && wgs * p <= 2 * kCUs; ++p)
      if (group % p == 0) n = p;
  return n;
}
// The workspace of a backward call, piece by piece.
struct ScoreRoom {
  char* at;
  size_t bytes = 0;
  explicit ScoreRoom(void* p) : at((char*)p) {}
  template <class T>
  T* take(size_t n) {
    T* r = at ? (T*)(at + bytes) : nullptr;
    bytes += round_up256(n * sizeof(T));
    return r;
  }
};
static size_t score_bwd_room(int B, int Hq, int Hkv, int Sq, int Sk, int D, void* workspace, ScoreStats& s, ScoreParts& parts) {
  ScoreRoom room(workspace);
  const size_t rows = s.rows = stat_rows(Sq);
  s.lse2 = room.take<float>(B * (size_t)Hq * rows);
  s.delta = room.take<float>(B * (size_t)Hq * rows);
  s.top = room.take<float2>(B * (size_t)Hq * (rows / 32));
  s.lo = room.take<int>(B * rows);
  s.len = room.take<int>(B * rows);
  s.span = room.take<KeySpan>(B * (rows / kTileRows));
  parts.n = key_parts(B, Hq, Hkv, Sk);
  parts.sums = parts.n > 1 ? room.take<float>(2 * (size_t)parts.n * B * Hkv * Sk * D) : nullptr;
  return room.bytes;
}
size_t score_bwd_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D) {
  ScoreStats s;
  ScoreParts parts;
  return score_bwd_room(B, Hq, Hkv, Sq, Sk, D, nullptr, s, parts);
}

// Teams per workgroup: two halve the tiles that a wavefront works on one after the other, and hold a CU together where half of
// the wavefronts would be left alone with the longest rows; they cost a merge and, where the workgroups fill the chip anyway, the
// freedom of two workgroups to be in different phases.  Over 84 launches of both head sizes, by number of workgroups, time with
// two teams over time with one: query sides up to 256 0.75 - 1.13, 0.93 on average; 512, causal and 2048 keys or more 0.84 - 0.96,
// otherwise 0.95 - 1.44; more 1.01 - 1.83.  Key side up to 256 0.70 - 0.97; 512 with masks and 2048 queries or more to a key 0.62 -
// 0.96, otherwise 0.94 - 1.30; more 1.04 - 1.21.
static int query_teams(const ScoreArgs& a) {
  const long long wgs = (long long)a.B * a.Hq * ((a.Sq + kOwn - 1) / kOwn);
  return wgs <= kCUs || (wgs <= 2 * kCUs && a.causal && !a.key_lo && a.Sk >= 2048) ? 2 : 1;
}
static int key_teams(const ScoreArgs& a, int parts) {
  const long long wgs = (long long)a.B * a.Hkv * ((a.Sk + kOwn - 1) / kOwn) * parts;
  return wgs <= kCUs || (wgs <= 2 * kCUs && (a.causal || a.key_lo) && (long long)a.Sq * (a.Hq / a.Hkv) / parts >= 2048) ? 2 : 1;
}
template <class V>
static hipError_t run_fwd(V, const ScoreArgs& a, hipStream_t st) {
  ProfScope p(kKScoreFwd, st);
  const dim3 grid(score_grid(a, a.Hq / a.Hkv * ((a.Sq + kOwn - 1) / kOwn)));
  if (query_teams(a) == 2)
    hipLaunchKernelGGL((score_fwd<V::D, V::DT, V::CAP, V::BIAS, 2>), grid, dim3(2 * kSThreads), 0, st, a, score_even(a));
  else
    hipLaunchKernelGGL((score_fwd<V::D, V::DT, V::CAP, V::BIAS, 1>), grid, dim3(kSThreads), 0, st, a, score_even(a));
  return hipGetLastError();
}
template <class V>
static hipError_t run_bwd(V, const ScoreArgs& a, const ScoreStats& s, const ScoreParts& parts, hipStream_t st) {
  {
    ProfScope p(kKScoreDq, st);
    const dim3 grid(score_grid(a, a.Hq / a.Hkv * ((a.Sq + kOwn - 1) / kOwn)));
    if (query_teams(a) == 2)
      hipLaunchKernelGGL((score_dq<V::D, V::DT, V::CAP, V::BIAS, 2>), grid, dim3(2 * kSThreads), 0, st, a, s, score_even(a));
    else
      hipLaunchKernelGGL((score_dq<V::D, V::DT, V::CAP, V::BIAS, 1>), grid, dim3(kSThreads), 0, st, a, s, score_even(a));
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfScope p(kKScoreDkv, st);
  const dim3 grid(score_grid(a, (a.Sk + kOwn - 1) / kOwn * parts.n));
  if (key_teams(a, parts.n) == 2)
    hipLaunchKernelGGL((score_dkv<V::D, V::DT, V::CAP, V::BIAS, 2>), grid, dim3(2 * kSThreads), 0, st, a, s, parts, score_even(a));
  else
    hipLaunchKernelGGL((score_dkv<V::D, V::DT, V::CAP, V::BIAS, 1>), grid, dim3(kSThreads), 0, st, a, s, parts, score_even(a));
  if (parts.n > 1) {
    const hipError_t f = hipGetLastError();
    if (f != hipSuccess) return f;
    const long long n = (long long)a.B * a.Hkv * a.Sk * V::D / 4;
    hipLaunchKernelGGL((score_add_parts<V::D, V::DT>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, parts);
  }
  return hipGetLastError();
}
hipError_t launch_score_fwd_rows(int dt, const ScoreArgs& a, hipStream_t st) {
  return by_variant(dt, a, [&](auto v) { return run_fwd(v, a, st); });
}
hipError_t launch_score_bwd_bf16(int dt, const ScoreArgs& a, void* workspace, hipStream_t st) {
  ScoreStats s;
  ScoreParts parts;
  score_bwd_room(a.B, a.Hq, a.Hkv, a.Sq, a.Sk, a.D, workspace, s, parts);
  return by_variant(dt, a, [&](auto v) { return run_bwd(v, a, s, parts, st); });
}

}  // namespace lx
