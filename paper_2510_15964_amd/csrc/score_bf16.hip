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
// that are not finite are zeroed before they are multiplied (0 * NaN); the result of an own row that attends such a row becomes
// NaN as a whole, so that nothing is hidden.
//
// Softmax in the log2 domain, statistics and accumulators in fp32; P and dS are rounded to the element type once, for the second
// product.
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
// a span per wavefront, written in either case.
__device__ __forceinline__ void spans_of_queries(const ScoreArgs& a, int start, int tile, bool there, int lo, int len, KeySpan* part,
                                                 KeySpan& span, KeySpan& all) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (a.key_lo) {
    span.of(there, lo, len);
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

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------
template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kSThreads, D == 64 ? 4 : 2) void score_fwd(const ScoreArgs a, const int even) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[2][2 * kTileRows * D];   // K tile, V tile
  __shared__ KeySpan part[kSWaves];
  __shared__ unsigned bad_part[kSWaves];
  const QueryWork wk(a, even);
  if (!wk.there) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, half = lane / 32;
  const int hk = wk.hk, q = wk.tile * kOwn + 32 * wave + lane % 32, qc = min(q, a.Sq - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  uint4 qf[D / 16];
  load_own<D>(a.Q, wk.b, wk.h, qc, qf);
  int lo, len;
  key_interval(a, wk.b, qc, start, lo, len);
  KeySpan span, all;
  spans_of_queries(a, start, wk.tile, q < a.Sq, lo, len, part, span, all);

  FastRules<CAP, BIAS> rules;
  rules.template init<true>(a, wk.h);
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
  ScoreRow<D> row;
  row.clear();
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
      attend_tile<2, kTile, D, DT, CAP, BIAS>(tk, off, qf, rules, k0, start + qc, lo, len, !span.covers(k0, kTileRows), row);
      if (bad && (bad & keys_seen(k0, lo, len))) row.weight = __builtin_nanf("");
    }
    lds_barrier();      // the stage is free
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
  int *lo, *len;            // [B, rows]
  KeySpan* span;            // [B, rows / 64]
  int rows;
};
__host__ __device__ inline int stat_rows(int Sq) { return (Sq + kTileRows - 1) / kTileRows * kTileRows; }

template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kSThreads, D == 64 ? (CAP && BIAS ? 3 : 4) : 2) void score_dq(const ScoreArgs a, const ScoreStats st, const int even) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[2][2 * kTileRows * D];   // K tile, V tile
  __shared__ KeySpan part[kSWaves];
  __shared__ unsigned bad_part[kSWaves];
  const QueryWork wk(a, even);
  if (!wk.there) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, half = lane / 32;
  const int hk = wk.hk, q = wk.tile * kOwn + 32 * wave + lane % 32, qc = min(q, a.Sq - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  uint4 qf[D / 16], gf[D / 16], of[D / 16];
  load_own<D>(a.Q, wk.b, wk.h, qc, qf);
  load_own<D>(a.dO, wk.b, wk.h, qc, gf);
  load_own<D>(a.O, wk.b, wk.h, qc, of);
  int lo, len;
  key_interval(a, wk.b, qc, start, lo, len);
  KeySpan span, all;
  spans_of_queries(a, start, wk.tile, q < a.Sq, lo, len, part, span, all);
  if (wk.h == 0) {
    // of the two tiles of 64 queries
    const int tile = 2 * wk.tile + wave / 2;
    KeySpan both = span;
    both.join(part[wave ^ 1]);
    if (wave % 2 == 0 && lane == 0 && tile * kTileRows < st.rows) st.span[(long long)wk.b * (st.rows / kTileRows) + tile] = both;
    if (half == 0 && q < st.rows) {
      st.lo[(long long)wk.b * st.rows + q] = lo;
      st.len[(long long)wk.b * st.rows + q] = q < a.Sq ? len : 0;
    }
  }

  float delta = 0.f;
  {
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
  const float lse2 = none ? INFINITY : lse * kSLog2e - FastRules<CAP, BIAS>::base(a);
  if (none) delta = 0.f;
  if (half == 0 && q < st.rows) {
    st.lse2[head_row * st.rows + q] = q < a.Sq ? lse2 : INFINITY;
    st.delta[head_row * st.rows + q] = q < a.Sq ? -delta : 0.f;
  }
  FastRules<CAP, BIAS> rules;
  rules.template init<true>(a, wk.h);
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
  float gain = a.scale * rules.kDerivative;       // NaN where an attended key's row was cleared
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
    const uint32_t tk = ring0 + stage * kStage, rows = tk + off.rows, tr = tk + off.tr;
    unsigned long long bad = 0;
    if (!all.covers(k0, kTileRows)) bad = join_rows(clear_not_finite<D, DT>(tk), bad_part);
    if (span.touches(k0, kTileRows)) {
      const float far = (float)(start + qc - k0 - 4 * half);
      const bool masked = !span.covers(k0, kTileRows);
      const unsigned long long seen = keys_seen(k0, lo, len);
      if (bad & seen) gain = __builtin_nanf("");
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          s = mfma32<DT>(read_piece<D>(rows, 0, t, kk), qf[kk], s);
          dp = mfma32<DT>(read_piece<D>(rows, kTile, t, kk), gf[kk], dp);
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          float r;
          const float p = __builtin_amdgcn_exp2f(rules.score(s[v], far - (float)(32 * t + acc_row(v)), r) - lse2);
          dp[v] = p * (dp[v] - delta);
          if constexpr (CAP) dp[v] *= rules.derivative(r);
        }
        if (masked) {
          const uint32_t word = (uint32_t)(seen >> (32 * t)) >> (4 * half);
#pragma unroll
          for (int v = 0; v < 16; ++v) dp[v] = or_zero(spread_bit(word, acc_row(v)), dp[v]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint4 p = pack_piece<DT>(dp, j);
#pragma unroll
          for (int ct = 0; ct < D / 32; ++ct) g[ct] = mfma32<DT>(read_piece_tr<D>(tr, 0, t, j, ct), p, g[ct]);
        }
      }
    }
    lds_barrier();
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

// The products of the key side issue a slot at a time, a matrix instruction and the read that fills its operand's registers again, with
// the compiler's scheduler held off between slots: dK, dV, the own rows and a tile of scores are 224 of 256 registers at D = 128,
// and a register in scratch memory costs the transfers ahead.
__device__ __forceinline__ void end_slot() { __builtin_amdgcn_sched_barrier(0); }

template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kSThreads, D == 64 ? 3 : 2) void score_dkv(const ScoreArgs a, const ScoreStats st, const int even) {
  constexpr uint32_t kTile = kTileRows * 2 * D, kStat = kTileRows * 4, kStage = 2 * kTile + 4 * kStat;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[2][kStage];   // Q tile, dO tile, lse2, delta, lo, len
  __shared__ unsigned bad_part[2][kSWaves];
  const ScoreWork wk(a, (a.Sk + kOwn - 1) / kOwn, even);
  if (!wk.there) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), half = lane / 32;
  const int group = a.Hq / a.Hkv, k_wg = wk.z * kOwn, k_wave = k_wg + 32 * wave, k = k_wave + lane % 32, kc = min(k, a.Sk - 1);
  const int start = a.q_start ? a.q_start[wk.b] : a.Sk - a.Sq;
  const KeySpan* spans = st.span + (long long)wk.b * (st.rows / kTileRows);

  uint4 kf[D / 16], vf[D / 16];
  load_own<D>(a.K, wk.b, wk.hk, kc, kf);
  load_own<D>(a.V, wk.b, wk.hk, kc, vf);
  ScoreDma<D> dma;
  dma.init();
  ScoreOff<D> off;
  off.init();
  const uint32_t ring0 = lds_addr(&ring[0][0]);
  QueryWalk walk;
  walk.init(spans, st.rows / kTileRows, k_wg, a.Sk, k_wave, wk.hk * group, group);
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
  float gain = 1.f;       // NaN where an attending query's row was cleared
  FastRules<CAP, BIAS> rules;
  if (walk.there()) issue(0, walk.h, walk.tile());
  int stage = 0, rules_of = -1;
  while (walk.there()) {
    const int h = walk.h, tile = walk.tile(), q0 = tile * kTileRows;
    const unsigned long long bit = 1ull << walk.bit();
    const bool all_wg = walk.all_wg & bit, some = walk.some_wave & bit, masked = !(walk.all_wave & bit);
    if (h != rules_of) rules.template init<true>(a, h), rules_of = h;
    walk.next();
    if (walk.there()) {
      issue(stage ^ 1, walk.h, walk.tile());
      wait_vmcnt<2 * ScoreDma<D>::kPerWave + 1>();
    } else {
      wait_vmcnt<0>();
    }
    lds_barrier();
    const uint32_t tq = ring0 + stage * kStage, tg = tq + kTile, ts = tg + kTile + 16 * half, rows = tq + off.rows, tr = tq + off.tr;
    unsigned long long bad = 0;
    if (!all_wg) {
      bad = join_rows(clear_not_finite<D, DT>(tq), bad_part[0]);
      bad |= join_rows(clear_not_finite<D, DT>(tg), bad_part[1]);
    }
    if (some) {
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
        if (masked)
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
#pragma unroll
        for (int i = 0; i < 2 * kCt; ++i) {
          gv[i % kCt] = mfma32<DT>(ga, p[i / kCt], gv[i % kCt]);
          if (i + 1 < 2 * kCt) ga = read_piece_tr<D>(tr, kTile, t, (i + 1) / kCt, (i + 1) % kCt);
          end_slot();
          gk[i % kCt] = mfma32<DT>(qa, ds[i / kCt], gk[i % kCt]);
          if (i + 1 < 2 * kCt) qa = read_piece_tr<D>(tr, 0, t, (i + 1) / kCt, (i + 1) % kCt);
          end_slot();
        }
      }
    }
    lds_barrier();
    stage ^= 1;
  }
  if (k < a.Sk) {
    store_own<D, DT>(a.dK, wk.b, wk.hk, k, gk, a.scale * rules.kDerivative * gain);
    store_own<D, DT>(a.dV, wk.b, wk.hk, k, gv, gain);
  }
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
size_t score_bwd_bytes(int B, int Hq, int, int Sq, int, int) {
  const size_t rows = stat_rows(Sq);
  return 2 * round_up256(B * (size_t)Hq * rows * 4) + 2 * round_up256(B * rows * 4) + round_up256(B * (rows / kTileRows) * sizeof(KeySpan));
}

template <int D, int DT, bool CAP, bool BIAS>
static hipError_t run_fwd(const ScoreArgs& a, hipStream_t st) {
  ProfScope p(kKScoreFwd, st);
  hipLaunchKernelGGL((score_fwd<D, DT, CAP, BIAS>), dim3(score_grid(a, a.Hq / a.Hkv * ((a.Sq + kOwn - 1) / kOwn))), dim3(kSThreads), 0, st, a, score_even(a));
  return hipGetLastError();
}
template <int D, int DT, bool CAP, bool BIAS>
static hipError_t run_bwd(const ScoreArgs& a, const ScoreStats& s, hipStream_t st) {
  {
    ProfScope p(kKScoreDq, st);
    hipLaunchKernelGGL((score_dq<D, DT, CAP, BIAS>), dim3(score_grid(a, a.Hq / a.Hkv * ((a.Sq + kOwn - 1) / kOwn))), dim3(kSThreads), 0, st, a, s, score_even(a));
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfScope p(kKScoreDkv, st);
  hipLaunchKernelGGL((score_dkv<D, DT, CAP, BIAS>), dim3(score_grid(a, (a.Sk + kOwn - 1) / kOwn)), dim3(kSThreads), 0, st, a, s, score_even(a));
  return hipGetLastError();
}
hipError_t launch_score_fwd_rows(int dt, const ScoreArgs& a, hipStream_t st) {
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
