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
      attend_tile<2, D, DT, CAP, BIAS>(tk, tv, off, qf, rules, k0, start + qc, lo, len, !span.covers(k0, kTileRows), row);
      if (bad && meets(bad, k0, lo, len)) row.weight = __builtin_nanf("");
    }
    lds_barrier();      // the stage is free
  }
  row.sum += __shfl_xor(row.sum, 32);
  row.weight += __shfl_xor(row.weight, 32);
  if (q < a.Sq) {
    store_own<D, DT>(a.O, wk.b, wk.h, q, row.o, row.weight == 0.f ? 0.f : 1.f / row.weight);
    if (a.LSE && half == 0)
      a.LSE[((long long)wk.b * a.Hq + wk.h) * a.Sq + q] = row.sum == 0.f ? -INFINITY : (row.m + __builtin_amdgcn_logf(row.sum)) * kSLn2;
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
  float gain = a.scale;       // NaN where an attended key's row was cleared
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
      if (bad && meets(bad, k0, lo, len)) gain = __builtin_nanf("");
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
          for (int v = 0; v < 16; ++v)
            if ((unsigned)(from + 32 * t + acc_row(v)) >= (unsigned)len) dp[v] = 0.f;
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
  if (q < a.Sq) store_own<D, DT>(a.dQ, wk.b, wk.h, q, g, gain);
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
  float gain = 1.f;       // NaN where an attending query's row was cleared
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
      for (unsigned long long left = bad; left; left &= left - 1) {
        const int r = 4 * (__ffsll((long long)left) - 1);
        if ((unsigned)k - lds_read4(tg + kTile + 2 * kStat + r) < lds_read4(tg + kTile + 3 * kStat + r)) gain = __builtin_nanf("");
      }
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
              if ((unsigned)k - lo[e] >= len[e]) s[v] = dp[v] = 0.f;
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
    store_own<D, DT>(a.dK, wk.b, wk.h, k, gk, a.scale * gain);
    store_own<D, DT>(a.dV, wk.b, wk.h, k, gv, gain);
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
