// Attention of a few queries per sequence over a cache, 16-bit types.
//
// The queries of all heads that share a key head are the columns of one 32x32x16 MFMA (group * Sq rows, in tiles of 32), so the cache
// is read once.  A workgroup works on one pair (sequence and key head, tile of rows) at a time: its wavefronts take tiles of 32
// keys in turn, each with a ring of its own and no barrier, and add up in LDS.  Where there are pairs enough for the chip a
// workgroup has one whole pair.  Otherwise the pairs are one sequence of units of 128 keys, each pair as long as its own keys
// are, of which every workgroup takes an equal run, whatever the sequences' lengths: the end of one pair, perhaps whole ones, the
// beginning of another.  Whole pairs are written at once, parts go to the workspace, sums and unnormalised outputs in fp32, and
// a second launch joins them.
//
// Bound by memory where there is much of it, 2 * 2 * D bytes per key and key head: 256 pairs of 16384 keys, D = 128, 360 us, 6.0 TB/s;
// 32 pairs of up to 32768, capped, 50 us and 4.8 for the join, 5.4 TB/s.  Below that by a wavefront's chain of dependent steps, hence
// eight of them (four, with rings twice as deep: D = 64, 256 pairs of 1024 keys 13.8 us, so 12.7, 128 of 2048 19.3 and 13.9; D = 128, 128
// pairs of 2048 25.2 and 22.8, of lengths up to 4096 39.8 and 32.7, but 128 pairs of up to 128 keys 6.6 and 6.7).
// (Runs of a wavefront instead of a workgroup, 2048 streams of addresses instead of 512: 128 pairs of 16384 keys, D = 64, 153
// us, so 105.)
#include "score_tile.h"

namespace lx {

// Stages of a wavefront's ring, 128 KB for all of them.  With one stage K's half of it is filled again between a tile's products and V's
// behind them.
template <int D>
constexpr int kTokenStages = D == 64 ? 2 : 1;

struct TokenArgs {
  int rows, row_tiles, wgs;       // of a pair, tiles of them, workgroups that share out all units
  int part_rows;                  // min(rows, 32)
  float* out;                     // [2 wgs][part_rows][D]: the part at a workgroup's beginning, the one at its end
  float* stat;                    // [2 wgs][part_rows][4]: reference point, sum, sum of the rounded
};

// The sequences' keys, 64 sequences at a time, one a lane.
struct TokenLengths {
  int base, first, units;
  __device__ __forceinline__ void load(const ScoreArgs& a, int from) {
    base = from;
    const int b = from + threadIdx.x % kWave;
    KeySpan s;
    s.of(false, 0, 0, 0);
    if (b < a.B) {
      const int start = a.q_start ? a.q_start[b] : a.Sk - a.Sq;
      for (int q = 0; q < a.Sq; ++q) {
        int lo, len;
        key_interval(a, b, q, start, lo, len);
        KeySpan one;
        one.of(true, lo, len, 0);
        s.join(one);
      }
    }
    first = s.first;
    units = s.end > s.first ? (s.end - s.first + kTokenStep - 1) / kTokenStep : 0;
  }
  __device__ __forceinline__ int first_of(int b) const { return __builtin_amdgcn_readlane(first, b - base); }
  __device__ __forceinline__ int units_of(int b) const { return __builtin_amdgcn_readlane(units, b - base); }
  // units of this lane's sequence and those before it in the group, all their pairs
  __device__ __forceinline__ int upto(int pairs) const {
    int v = units * pairs;
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // from 1, 2, 4 and 8 lanes before in a row of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // rows 0 and 2's last lane to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // lane 31 to rows 2 and 3
    return v;
  }
};
// All units; `l` is left at the last group (the only one up to 64 sequences).
__device__ __forceinline__ int all_units(const ScoreArgs& a, int pairs, TokenLengths& l) {
  int sum = 0;
  for (int from = 0; from < a.B; from += kWave) {
    l.load(a, from);
    sum += __builtin_amdgcn_readlane(l.upto(pairs), kWave - 1);
  }
  return sum;
}
// How `total` units fall to n workgroups: the first `more` have one more than the others.
struct TokenRuns {
  int each, more;
  __device__ __forceinline__ TokenRuns(int total, int n) : each(total / n), more(total - total / n * n) {}
  __device__ __forceinline__ int first(int i) const { return i * each + min(i, more); }
  __device__ __forceinline__ int of_unit(int u) const {
    const int longer = more * (each + 1);
    return u < longer ? u / (each + 1) : more + (u - longer) / each;
  }
};

// A place in the sequence of units.
struct TokenPlace {
  TokenLengths l;
  int b, pair, unit;          // sequence, its pair (key head, tile of rows), unit of its keys
  int first, units, pairs;
  __device__ __forceinline__ void seek(const ScoreArgs& a, int n_pairs, const TokenLengths& known, int at) {
    l = known;
    pairs = n_pairs;
    if (a.B > kWave) l.load(a, 0);
    for (;;) {
      const int upto = l.upto(pairs), group = __builtin_amdgcn_readlane(upto, kWave - 1);
      if (at < group || l.base + kWave >= a.B) {
        const int lane = __ffsll((long long)__ballot(upto > at)) - 1;
        b = l.base + lane;
        first = l.first_of(b), units = l.units_of(b);
        const int in = at - (__builtin_amdgcn_readlane(upto, lane) - units * pairs);
        pair = in / units;
        unit = in - pair * units;
        return;
      }
      at -= group;
      l.load(a, l.base + kWave);
    }
  }
  __device__ __forceinline__ void next_pair(const ScoreArgs& a) {
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

// The transfers of a [32 x D] tile by one wavefront.
template <int D>
struct TokenDma {
  static constexpr int kSlots = D / 8, kRowsPer = kWave / kSlots, kCount = kTokenKeys / kRowsPer;
  // rows past `last` repeat it
  static __device__ __forceinline__ void issue(uint32_t to, const char* base, long long row_bytes, int last) {
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int u = 0; u < kCount; ++u) {
      const int row = kRowsPer * u + lane / kSlots;
      dma16(base + (long long)min(row, last) * row_bytes + ((lane % kSlots) ^ score_swz<D>(row)) * 16, to + u * 1024);
    }
  }
};
// A lane's row of a pair: query q of head h.
struct TokenRow {
  int h, q, pos, lo, len;
  bool there;
  __device__ __forceinline__ void of(const ScoreArgs& a, const TokenArgs& ta, int b, int pair) {
    const int hk = pair / ta.row_tiles, r = (pair - hk * ta.row_tiles) * kTokenRows + threadIdx.x % 32, rc = min(r, ta.rows - 1), g = rc / a.Sq;
    const int start = a.q_start ? a.q_start[b] : a.Sk - a.Sq;
    there = r < ta.rows;
    q = rc - g * a.Sq;
    h = hk * (a.Hq / a.Hkv) + g;
    pos = start + q;
    key_interval(a, b, q, start, lo, len);
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

__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// PARTS: the workgroup's run of all units; otherwise one pair.
template <int D, int DT, int CAP, bool BIAS, bool PARTS>
__global__ __launch_bounds__(kTokenWaves * kWave, 1) void score_token(const ScoreArgs a, const TokenArgs ta) {
  constexpr int W = kTokenWaves, NS = kTokenStages<D>, kStep = W * kTokenKeys, kDma = TokenDma<D>::kCount;
  constexpr uint32_t kTile = kTokenKeys * 2 * D, kStage = 2 * kTile, kMine = NS * kStage;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[W * kMine];   // K tile, V tile; then a wavefront's sums
  __shared__ __attribute__((aligned(16))) f32x4 stats[W][32];
  const int lane = threadIdx.x % kWave, half = lane / 32, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int pairs = a.Hkv * ta.row_tiles;
  const uint32_t ring0 = lds_addr(ring), mine = ring0 + wave * kMine;
  ScoreOff<D> off;
  off.init();
  int at = 0, end = 1;        // of all units: the next, and the run's end
  TokenPlace place;
  if constexpr (PARTS) {
    TokenLengths lengths;
    const int total = all_units(a, pairs, lengths), n = min(ta.wgs, total), w = blockIdx.x;
    if (w >= n) return;
    const TokenRuns runs(total, n);
    at = runs.first(w), end = runs.first(w + 1);
    place.seek(a, pairs, lengths, at);
  }
  bool at_start = true;
  for (;;) {
    const int b = PARTS ? place.b : blockIdx.x / pairs, pair = PARTS ? place.pair : (int)blockIdx.x - b * pairs, hk = pair / ta.row_tiles;
    TokenRow me;
    me.of(a, ta, b, pair);
    uint4 qf[D / 16];
    load_own<D>(a.Q, b, me.h, me.q, qf);
    KeySpan span;
    span.of(me.there, me.lo, me.len, me.pos);
    span = span_of_wave(span);
    FastRules<CAP, BIAS> rules;
    rules.template init<false>(a, me.h);
    const int from = PARTS ? place.unit : 0, to = PARTS ? min(place.units, from + end - at) : 0;
    const int k_first = PARTS ? place.first + from * kTokenStep : min(span.first, span.end);
    const int k_end = PARTS ? min(span.end, place.first + to * kTokenStep) : span.end;
    const bool whole = !PARTS || (from == 0 && to == place.units);

    int in = k_first + wave * kTokenKeys, in_stage = 0;
    auto issue_k = [&]() { TokenDma<D>::issue(mine + in_stage * kStage, score_row(a.K, b, hk, in), 2 * a.K.ss, a.Sk - 1 - in); };
    auto issue_v = [&]() {      // and on to the next tile
      TokenDma<D>::issue(mine + in_stage * kStage + kTile, score_row(a.V, b, hk, in), 2 * a.V.ss, a.Sk - 1 - in);
      in_stage = in_stage + 1 == NS ? 0 : in_stage + 1;
      in += kStep;
    };
    if (in < k_end) issue_k(), issue_v();
    settle(qf);
    ScoreRow<D> row;
    row.clear();
    auto attend = [&](auto is_linear) {
      constexpr bool linear = decltype(is_linear)::value;
      f32x16 lift = {};
      if constexpr (linear) rules.lift(lift);
      int stage = 0;
      for (int k0 = k_first + wave * kTokenKeys; k0 < k_end; k0 += kStep) {
        const bool more = in < k_end, masked = !span.covers(k0, kTokenKeys);
        const uint32_t tk = mine + stage * kStage;
        unsigned long long bad = 0;
        if constexpr (NS == 2) {
          reads_done();        // of the other stage
          if (more) issue_k(), issue_v(), wait_vmcnt<2 * kDma>();
          else wait_vmcnt<0>();
        } else {
          wait_vmcnt<kDma>();
        }
        asm volatile("" ::: "memory");
        attend_tile<1, kTile, linear, D, DT, CAP, BIAS>(tk, off, qf, rules, lift, k0, me.pos, me.lo, me.len, masked, row, [&] {
          if constexpr (NS == 1) {
            reads_done();
            if (more) issue_k(), wait_vmcnt<kDma>();
            else wait_vmcnt<0>();
            asm volatile("" ::: "memory");
          }
          if (masked) bad = clear_not_finite_32<D, DT>(tk + kTile);
        });
        if (bad && (bad & keys_seen(k0, me.lo, me.len))) row.weight = __builtin_nanf("");
        if constexpr (NS == 1) {
          reads_done();
          if (more) issue_v();
        }
        stage = stage + 1 == NS ? 0 : stage + 1;
      }
    };
    by_linear(rules, span.after, attend);

    // the wavefronts' sums
    row.sum += __shfl_xor(row.sum, 32);
    row.weight += __shfl_xor(row.weight, 32);
    if (half == 0) stats[wave][lane] = f32x4{row.m, row.sum, row.weight, 0.f};
#pragma unroll
    for (int ct = 0; ct < D / 32; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        lds_write16(mine + ((4 * ct + i) * kWave + lane) * 16,
                    __builtin_bit_cast(uint4, f32x4{row.o[ct][4 * i], row.o[ct][4 * i + 1], row.o[ct][4 * i + 2], row.o[ct][4 * i + 3]}));
    lds_barrier();
    float m = -INFINITY, c[W], sum = 0.f, weight = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, stats[w][lane % 32][0]);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const f32x4 s = stats[w][lane % 32];
      c[w] = __builtin_amdgcn_exp2f(s[0] - ref);
      sum = fmaf(c[w], s[1], sum);
      weight = fmaf(c[w], s[2], weight);
    }
    const float norm = weight == 0.f ? 0.f : 1.f / weight;
    uint2* out = (uint2*)const_cast<char*>(score_row(a.O, b, me.h, me.q)) + half;
    const long long slot = PARTS ? (2ll * blockIdx.x + (at_start ? 0 : 1)) * ta.part_rows + lane % 32 : 0;
    f32x4* part = (f32x4*)(ta.out + slot * D) + half;
    if (me.there) {
      // an equal share of the columns to a wavefront
#pragma unroll
      for (int n = 0; n < D / 8 / W; ++n) {
        const int j = wave * (D / 8 / W) + n;
        f32x4 o = {};
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const f32x4 v = __builtin_bit_cast(f32x4, lds_read16(ring0 + w * kMine + (j * kWave + lane) * 16));
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = fmaf(v[e], c[w], o[e]);
        }
        if (whole) out[2 * j] = make_uint2(pack2<DT>(o[0] * norm, o[1] * norm), pack2<DT>(o[2] * norm, o[3] * norm));
        else part[2 * j] = o;
      }
      if (wave == 0 && half == 0) {
        if (!whole) *(f32x4*)(ta.stat + 4 * slot) = f32x4{m, sum, weight, 0.f};
        else if (a.LSE)
          a.LSE[((long long)b * a.Hq + me.h) * a.Sq + me.q] = sum == 0.f ? -INFINITY : (m + rules.base(a) + __builtin_amdgcn_logf(sum)) * kSLn2;
      }
    }
    if constexpr (!PARTS) return;
    at += to - from;
    if (at >= end) return;
    at_start = false;
    place.next_pair(a);
    lds_barrier();       // the rings are free
  }
}

// One row of a pair: adds the parts of the workgroups that worked on it, four at a time.
constexpr int kJoinThreads = 256;
template <int D, int DT>
__global__ __launch_bounds__(kJoinThreads) void score_join(const ScoreArgs a, const TokenArgs ta) {
  __shared__ float part[kJoinThreads / kWave][D + 2];
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  const int pairs = a.Hkv * ta.row_tiles, r = blockIdx.x % ta.rows, hk = blockIdx.x / ta.rows % a.Hkv, b = blockIdx.x / ta.rows / a.Hkv;
  const int pair = hk * ta.row_tiles + r / kTokenRows, h = hk * (a.Hq / a.Hkv) + r / a.Sq, q = r % a.Sq;
  TokenLengths l;
  int total = 0, before = 0, units = 0;
  for (int from = 0; from < a.B; from += kWave) {
    l.load(a, from);
    const int upto = l.upto(pairs);
    if (b >= from && b < from + kWave) {
      units = l.units_of(b);
      before = total + __builtin_amdgcn_readlane(upto, b - from) - units * pairs;
    }
    total += __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  uint16_t* out = (uint16_t*)const_cast<char*>(score_row(a.O, b, h, q));
  float* lse = a.LSE ? a.LSE + ((long long)b * a.Hq + h) * a.Sq + q : nullptr;
  if (!units) {
    if (threadIdx.x < D) out[threadIdx.x] = 0;
    if (lse && threadIdx.x == 0) *lse = -INFINITY;
    return;
  }
  const TokenRuns runs(total, min(ta.wgs, total));
  const int g0 = before + pair * units, i0 = runs.of_unit(g0), i1 = runs.of_unit(g0 + units - 1);
  if (i0 == i1) return;          // one workgroup had all of it
  const int parts = i1 - i0 + 1, row = r % kTokenRows;
  auto slot = [&](int p) { return (2ll * (i0 + p) + (p == 0 && runs.first(i0) != g0 ? 1 : 0)) * ta.part_rows + row; };
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
  if (lse && threadIdx.x == 0) *lse = sum == 0.f ? -INFINITY : (m + cap_base(a.cap) + __builtin_amdgcn_logf(sum)) * kSLn2;
}

// ---------------------------------------------------------------------------
static TokenArgs token_args(int B, int Hq, int Hkv, int Sq, int Sk) {
  TokenArgs t = {};
  t.rows = Hq / Hkv * Sq;
  t.row_tiles = (t.rows + kTokenRows - 1) / kTokenRows;
  t.part_rows = t.rows < kTokenRows ? t.rows : kTokenRows;
  // a workgroup to a CU, two units or more to each
  const long long most = (token_pairs(B, Hq, Hkv, Sq) * ((Sk + kTokenStep - 1) / kTokenStep) + 1) / 2;
  t.wgs = (int)(most < kCUs ? most : kCUs);
  return t;
}
size_t score_fwd_bytes(int B, int Hq, int Hkv, int Sq, int Sk, int D) {
  if (score_route(B, Hq, Hkv, Sq, Sk) != kByParts) return 0;
  const TokenArgs t = token_args(B, Hq, Hkv, Sq, Sk);
  return round_up256(2 * (size_t)t.wgs * t.part_rows * D * 4) + round_up256(2 * (size_t)t.wgs * t.part_rows * 16);
}
template <class V>
static hipError_t run_token(V, const ScoreArgs& a, const TokenArgs& t, bool parts, hipStream_t st) {
  ProfScope p(kKScoreFwd, st);
  if (!parts) {
    hipLaunchKernelGGL((score_token<V::D, V::DT, V::CAP, V::BIAS, false>), dim3((unsigned)token_pairs(a.B, a.Hq, a.Hkv, a.Sq)),
                       dim3(kTokenWaves * kWave), 0, st, a, t);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((score_token<V::D, V::DT, V::CAP, V::BIAS, true>), dim3(t.wgs), dim3(kTokenWaves * kWave), 0, st, a, t);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((score_join<V::D, V::DT>), dim3((unsigned)((long long)a.B * a.Hkv * t.rows)), dim3(kJoinThreads), 0, st, a, t);
  return hipGetLastError();
}
hipError_t launch_score_fwd_bf16(int dt, const ScoreArgs& a, void* workspace, hipStream_t st) {
  const ScoreRoute route = score_route(a.B, a.Hq, a.Hkv, a.Sq, a.Sk);
  if (route == kByRows) return launch_score_fwd_rows(dt, a, st);
  TokenArgs t = token_args(a.B, a.Hq, a.Hkv, a.Sq, a.Sk);
  if (route == kByParts) {
    t.out = (float*)workspace;
    t.stat = (float*)((char*)workspace + round_up256(2 * (size_t)t.wgs * t.part_rows * a.D * 4));
  }
  return by_variant(dt, a, [&](auto v) { return run_token(v, a, t, route == kByParts, st); });
}

}  // namespace lx
