// Attention of a few queries per sequence over a long cache, 16-bit types: the keys are split among wavefronts, whose results are
// joined by a second launch.
//
// The queries of all heads that share a key head are the columns of one 32x32x16 MFMA (group * Sq rows, in tiles of 32), so the cache
// is read once.  What there is to do is a sequence of units of 32 keys: all pairs (sequence, key head, tile of rows), one after
// the other, each as long as its own keys are; every wavefront takes an equal run of it, whatever the sequences' lengths, and
// so works on the end of one pair, perhaps whole ones, and the beginning of another.  Whole pairs are written at once, parts go
// to the workspace: the sums of a part and its unnormalised output in fp32.  Wavefronts are workgroups of their own: nothing is
// waited for but a wavefront's own transfers.  Bound by memory: 2 * 2 * D bytes per key and key head.
#include "score_tile.h"

namespace lx {

constexpr int kTokenRows = 32, kTokenKeys = 32;
// stages of a wavefront's ring: 32 KB either way, four wavefronts per CU
template <int D>
constexpr int kTokenStages = D == 64 ? 4 : 2;
constexpr int kTokenWaves = 4 * kCUs;
constexpr int kTokenMinUnits = 4;       // fewer units to a wavefront are not worth a part

struct TokenArgs {
  int rows, row_tiles, waves;     // of a pair, tiles of them, wavefronts
  int part_rows;                  // min(rows, 32)
  float* out;                     // [2 waves][part_rows][D]: the part at a wavefront's beginning, the one at its end
  float* stat;                    // [2 waves][part_rows][4]: reference point, sum, sum of the rounded
};

// The sequences' keys, 64 sequences at a time, one a lane.
struct TokenLengths {
  int base, first, units;
  __device__ __forceinline__ void load(const ScoreArgs& a, int from) {
    base = from;
    const int b = from + threadIdx.x % kWave;
    KeySpan s;
    s.of(false, 0, 0);
    if (b < a.B) {
      const int start = a.q_start ? a.q_start[b] : a.Sk - a.Sq;
      for (int q = 0; q < a.Sq; ++q) {
        int lo, len;
        key_interval(a, b, q, start, lo, len);
        KeySpan one;
        one.of(true, lo, len);
        s.join(one);
      }
    }
    first = s.first;
    units = s.end > s.first ? (s.end - s.first + kTokenKeys - 1) / kTokenKeys : 0;
  }
  __device__ __forceinline__ int first_of(int b) const { return __builtin_amdgcn_readlane(first, b - base); }
  __device__ __forceinline__ int units_of(int b) const { return __builtin_amdgcn_readlane(units, b - base); }
  // units of this lane's sequence and those before it in the group, all their pairs
  __device__ __forceinline__ long long upto(int pairs) const {
    long long v = (long long)units * pairs;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const long long w = __shfl_up(v, o);
      if ((int)(threadIdx.x % kWave) >= o) v += w;
    }
    return v;
  }
};
__device__ __forceinline__ long long lane_of(long long v, int l) {
  return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 |
                     (unsigned)__builtin_amdgcn_readlane((int)v, l));
}
// All units; `l` is left at the last group (the only one up to 64 sequences).
__device__ __forceinline__ long long all_units(const ScoreArgs& a, int pairs, TokenLengths& l) {
  long long sum = 0;
  for (int from = 0; from < a.B; from += kWave) {
    l.load(a, from);
    sum += lane_of(l.upto(pairs), kWave - 1);
  }
  return sum;
}
// first unit of wavefront i of n, and the wavefront of a unit
__device__ __forceinline__ long long first_unit(long long i, long long n, long long total) { return i * total / n; }
__device__ __forceinline__ long long wave_of_unit(long long u, long long n, long long total) { return ((u + 1) * n - 1) / total; }

// A place in the sequence of units.
struct TokenPlace {
  TokenLengths l;
  int b, pair, unit;          // sequence, its pair (key head, tile of rows), unit of its keys
  int first, units, pairs;
  __device__ __forceinline__ void seek(const ScoreArgs& a, int n_pairs, const TokenLengths& known, long long at) {
    l = known;
    pairs = n_pairs;
    if (a.B > kWave) l.load(a, 0);
    for (;;) {
      const long long upto = l.upto(pairs), group = lane_of(upto, kWave - 1);
      if (at < group || l.base + kWave >= a.B) {
        const int lane = __ffsll((long long)__ballot(upto > at)) - 1;
        b = l.base + lane;
        first = l.first_of(b), units = l.units_of(b);
        const int in = (int)(at - (lane_of(upto, lane) - (long long)units * pairs));
        pair = in / units;
        unit = in - pair * units;
        return;
      }
      at -= group;
      l.load(a, l.base + kWave);
    }
  }
  __device__ __forceinline__ void next(const ScoreArgs& a) {
    if (++unit < units) return;
    unit = 0;
    if (++pair < pairs) return;
    pair = 0;
    do {
      if (++b >= a.B) return;
      if (b - l.base >= kWave) l.load(a, l.base + kWave);
      first = l.first_of(b), units = l.units_of(b);
    } while (!units);
  }
};

// zeroes what is not finite in a [32 x D] tile, half a row per lane: the rows with any
template <int D, int DT>
__device__ __forceinline__ unsigned clear_not_finite_32(uint32_t tile) {
  constexpr uint32_t kExp = DT == kF16 ? 0x7c007c00u : 0x7f807f80u, kOne = DT == kF16 ? 0x04000400u : 0x00800080u;
  const uint32_t at = tile + threadIdx.x % kWave * D;
  ushort2v top = {0, 0};
#pragma unroll
  for (int i = 0; i < D / 16; ++i) top = top_exponent<kExp>(lds_read16(at + 16 * i), top);
  const bool found = (__builtin_bit_cast(uint32_t, top) + kOne) & 0x80008000u;
  if (found)
#pragma unroll
    for (int i = 0; i < D / 8; ++i) lds_write8(at + 8 * i, make_uint2(0, 0));
  unsigned long long lanes = __ballot(found);
  if (!lanes) return 0;
  lanes |= lanes >> 1;
  unsigned rows = 0;
#pragma unroll
  for (int r = 0; r < 32; ++r) rows |= (unsigned)(lanes >> (2 * r) & 1) << r;
  return rows;
}

template <int D, int DT, bool CAP, bool BIAS>
__global__ __launch_bounds__(kWave, 1) void score_token(const ScoreArgs a, const TokenArgs ta) {
  constexpr int NS = kTokenStages<D>, kSlots = D / 8, kRowsPer = kWave / kSlots, kDma = kTokenKeys / kRowsPer;
  constexpr uint32_t kTile = kTokenKeys * 2 * D, kStage = 2 * kTile;
  __shared__ __attribute__((aligned(1024))) uint16_t ring[NS][2 * kTokenKeys * D];   // K tile, V tile
  const int lane = threadIdx.x, half = lane / 32, wave = blockIdx.x;
  const int group = a.Hq / a.Hkv, pairs = a.Hkv * ta.row_tiles;
  TokenLengths lengths;
  const long long total = all_units(a, pairs, lengths);
  const long long n = min((long long)ta.waves, total);
  if (wave >= n) return;
  const long long u0 = first_unit(wave, n, total), u1 = first_unit(wave + 1, n, total);

  const uint32_t ring0 = lds_addr(&ring[0][0]);
  int dma_row[kDma], dma_slot[kDma];
#pragma unroll
  for (int u = 0; u < kDma; ++u) {
    dma_row[u] = kRowsPer * u + lane / kSlots;
    dma_slot[u] = ((lane % kSlots) ^ score_swz<D>(dma_row[u])) * 16;
  }
  TokenPlace in, at;       // of the transfers, of the computation
  in.seek(a, pairs, lengths, u0);
  at = in;
  long long issued = u0;
  int in_stage = 0;
  auto issue = [&]() {
    const int k0 = in.first + kTokenKeys * in.unit, hk = in.pair / ta.row_tiles, last = a.Sk - 1 - k0;
    const char *k = score_row(a.K, in.b, hk, k0), *v = score_row(a.V, in.b, hk, k0);
    const uint32_t to = ring0 + in_stage * kStage;
#pragma unroll
    for (int u = 0; u < kDma; ++u) dma16(k + (long long)min(dma_row[u], last) * (2 * a.K.ss) + dma_slot[u], to + u * 1024);
#pragma unroll
    for (int u = 0; u < kDma; ++u) dma16(v + (long long)min(dma_row[u], last) * (2 * a.V.ss) + dma_slot[u], to + kTile + u * 1024);
    in_stage = in_stage + 1 == NS ? 0 : in_stage + 1;
    if (++issued < u1) in.next(a);
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (issued < u1) issue();

  ScoreOff<D> off;
  off.init();
  uint4 qf[D / 16];
  ScoreRow<D> row;
  FastRules<CAP, BIAS> rules;
  KeySpan span;
  int h = 0, q = 0, pos = 0, lo = 0, len = 0, from = 0, stage = 0;
  bool there = false, at_start = true;
  for (long long u = u0; u < u1; ++u) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the stage's reads are done
    if (issued < u1) issue();
    if (u == u0 || at.unit == 0) {
      at_start = u == u0;
      from = at.unit;
      const int hk = at.pair / ta.row_tiles, r = (at.pair - hk * ta.row_tiles) * kTokenRows + lane % 32, rc = min(r, ta.rows - 1);
      const int g = rc / a.Sq, start = a.q_start ? a.q_start[at.b] : a.Sk - a.Sq;
      there = r < ta.rows;
      q = rc - g * a.Sq;
      h = hk * group + g;
      pos = start + q;
      key_interval(a, at.b, q, start, lo, len);
      span.of(there, lo, len);
      span = span_of_wave(span);
      load_own<D>(a.Q, at.b, h, q, qf);
      rules.template init<false>(a, h);
      settle(qf);
      row.clear();
    }
    const long long ahead = issued - u - 1;
    if (ahead >= NS - 1) wait_vmcnt<2 * kDma*(NS - 1)>();
    else wait_vmcnt<0>();
    const int k0 = at.first + kTokenKeys * at.unit;
    const uint32_t tk = ring0 + stage * kStage, tv = tk + kTile;
    asm volatile("" ::: "memory");
    const bool masked = !span.covers(k0, kTokenKeys);
    unsigned long long bad = 0;
    if (masked) bad = clear_not_finite_32<D, DT>(tv);
    if (span.touches(k0, kTokenKeys)) attend_tile<1, kTile, D, DT, CAP, BIAS>(tk, off, qf, rules, k0, pos, lo, len, masked, row);
    if (bad && (bad & keys_seen(k0, lo, len))) row.weight = __builtin_nanf("");
    stage = stage + 1 == NS ? 0 : stage + 1;
    if (at.unit + 1 == at.units || u + 1 == u1) {
      const float sum = row.sum + __shfl_xor(row.sum, 32), weight = row.weight + __shfl_xor(row.weight, 32);
      if (from == 0 && at.unit + 1 == at.units) {
        if (there) {
          store_own<D, DT>(a.O, at.b, h, q, row.o, weight == 0.f ? 0.f : 1.f / weight);
          if (a.LSE && half == 0)
            a.LSE[((long long)at.b * a.Hq + h) * a.Sq + q] = sum == 0.f ? -INFINITY : (row.m + rules.base(a) + __builtin_amdgcn_logf(sum)) * kSLn2;
        }
      } else if (there) {
        const long long slot = (2ll * wave + (at_start ? 0 : 1)) * ta.part_rows + lane % 32;
        f32x4* o = (f32x4*)(ta.out + slot * D) + half;
#pragma unroll
        for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            o[8 * ct + 2 * i] = f32x4{row.o[ct][4 * i], row.o[ct][4 * i + 1], row.o[ct][4 * i + 2], row.o[ct][4 * i + 3]};
        if (half == 0) *(f32x4*)(ta.stat + 4 * slot) = f32x4{row.m, sum, weight, 0.f};
      }
    }
    if (u + 1 < u1) at.next(a);
  }
}

// One row of a pair: adds the parts of the wavefronts that worked on it, four lanes groups of 64 at a time.
constexpr int kJoinThreads = 256;
template <int D, int DT>
__global__ __launch_bounds__(kJoinThreads) void score_join(const ScoreArgs a, const TokenArgs ta) {
  __shared__ float part[kJoinThreads / kWave][D + 2];
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  const int pairs = a.Hkv * ta.row_tiles, r = blockIdx.x % ta.rows, hk = blockIdx.x / ta.rows % a.Hkv, b = blockIdx.x / ta.rows / a.Hkv;
  const int pair = hk * ta.row_tiles + r / kTokenRows, h = hk * (a.Hq / a.Hkv) + r / a.Sq, q = r % a.Sq;
  TokenLengths l;
  long long total = 0, before = 0;
  int units = 0;
  for (int from = 0; from < a.B; from += kWave) {
    l.load(a, from);
    const long long upto = l.upto(pairs);
    if (b >= from && b < from + kWave) {
      units = l.units_of(b);
      before = total + lane_of(upto, b - from) - (long long)units * pairs;
    }
    total += lane_of(upto, kWave - 1);
  }
  uint16_t* out = (uint16_t*)const_cast<char*>(score_row(a.O, b, h, q));
  float* lse = a.LSE ? a.LSE + ((long long)b * a.Hq + h) * a.Sq + q : nullptr;
  if (!units) {
    if (threadIdx.x < D) out[threadIdx.x] = 0;
    if (lse && threadIdx.x == 0) *lse = -INFINITY;
    return;
  }
  const long long n = min((long long)ta.waves, total), g0 = before + (long long)pair * units, g1 = g0 + units;
  const long long i0 = wave_of_unit(g0, n, total), i1 = wave_of_unit(g1 - 1, n, total);
  if (i0 == i1) return;          // one wavefront had all of it
  const int parts = (int)(i1 - i0) + 1, row = r % kTokenRows;
  auto slot = [&](int p) {
    return (2 * (i0 + p) + (p == 0 && first_unit(i0, n, total) != g0 ? 1 : 0)) * ta.part_rows + row;
  };
  float m = -INFINITY;
  for (int p = lane; p < parts; p += kWave) m = fmaxf(m, ta.stat[4 * slot(p)]);
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float ref = m == -INFINITY ? 0.f : m;
  float acc[D / 64] = {}, sum = 0.f, weight = 0.f;
#pragma unroll 4
  for (int p = w; p < parts; p += kJoinThreads / kWave) {
    const long long s = slot(p);
    const f32x4 st = *(const f32x4*)(ta.stat + 4 * s);
    const float c = __builtin_amdgcn_exp2f(st[0] - ref);
    sum = fmaf(c, st[1], sum);
    weight = fmaf(c, st[2], weight);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) acc[i] = fmaf(c, ta.out[s * D + lane + 64 * i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i) part[w][lane + 64 * i] = acc[i];
  if (lane == 0) part[w][D] = sum, part[w][D + 1] = weight;
  __syncthreads();
  if (threadIdx.x >= D) return;
  float o = 0.f;
  sum = weight = 0.f;
#pragma unroll
  for (int k = 0; k < kJoinThreads / kWave; ++k) o += part[k][threadIdx.x], sum += part[k][D], weight += part[k][D + 1];
  out[threadIdx.x] = (uint16_t)pack2<DT>(weight == 0.f ? 0.f : o / weight, 0.f);
  if (lse && threadIdx.x == 0) *lse = sum == 0.f ? -INFINITY : (m + (a.cap > 0.f ? a.cap * kSLog2e : 0.f) + __builtin_amdgcn_logf(sum)) * kSLn2;
}

// ---------------------------------------------------------------------------
// Few queries per sequence, and keys enough to split.
static bool by_tokens(int Sq, int Sk) { return Sq <= 16 && Sk > 64; }
static TokenArgs token_args(int B, int Hq, int Hkv, int Sq, int Sk) {
  TokenArgs t = {};
  t.rows = Hq / Hkv * Sq;
  t.row_tiles = (t.rows + kTokenRows - 1) / kTokenRows;
  t.part_rows = t.rows < kTokenRows ? t.rows : kTokenRows;
  const long long most = (long long)B * Hkv * t.row_tiles * ((Sk + kTokenKeys - 1) / kTokenKeys) / kTokenMinUnits;
  t.waves = (int)(most < 1 ? 1 : most < kTokenWaves ? most : kTokenWaves);
  return t;
}
size_t score_fwd_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D) {
  if (!by_tokens(Sq, Sk)) return 0;
  const TokenArgs t = token_args(B, Hq, Hkv, Sq, Sk);
  return round_up256(2 * (size_t)t.waves * t.part_rows * D * 4) + round_up256(2 * (size_t)t.waves * t.part_rows * 16);
}
template <int D, int DT, bool CAP, bool BIAS>
static hipError_t run_token(const ScoreArgs& a, const TokenArgs& t, hipStream_t st) {
  ProfScope p(kKScoreFwd, st);
  hipLaunchKernelGGL((score_token<D, DT, CAP, BIAS>), dim3(t.waves), dim3(kWave), 0, st, a, t);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((score_join<D, DT>), dim3((unsigned)((long long)a.B * a.Hkv * t.rows)), dim3(kJoinThreads), 0, st, a, t);
  return hipGetLastError();
}
hipError_t launch_score_fwd_bf16(int dt, const ScoreArgs& a, void* workspace, hipStream_t st) {
  if (!by_tokens(a.Sq, a.Sk)) return launch_score_fwd_rows(dt, a, st);
  TokenArgs t = token_args(a.B, a.Hq, a.Hkv, a.Sq, a.Sk);
  t.out = (float*)workspace;
  t.stat = (float*)((char*)workspace + round_up256(2 * (size_t)t.waves * t.part_rows * a.D * 4));
  return by_variant(dt, a, [&](auto v) { return run_token<v.D, v.DT, v.CAP, v.BIAS>(a, t, st); });
}

}  // namespace lx
