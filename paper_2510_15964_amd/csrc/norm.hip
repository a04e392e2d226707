// Dropout, and the root-mean-square norm of a sum with its residual: h = residual + drop(x), y = h w / sqrt(mean h^2 + eps).
//
// Memory-bound: every input is read once and every output written once, a row stays in registers between the sum of its squares and
// its outputs.  A row belongs to one wavefront up to 1024 elements (no barrier), to four up to 8192, so that a lane holds few runs
// and many rows are on their way: forward, 8192 x 2048 with dropout, 28 us by one wavefront with four runs per lane, 23.6 by four with
// one; backward 50 and 33.  Beyond, sixteen.
//
// Kernels by rocprofv3 (profiles/kernel_stats_more_operators.txt), us, bf16, inputs that are not in the caches: dropout of 8192 x 4096 with a
// residual 37 (201 MB, 5.4 TB/s; the generator hides: 8192 x 8192 without a residual 47.1 at p = 0, 47.7 at 0.1), norm 8192 x 2048 with
// dropout 26 (134 MB, 5.1 TB/s), 8192 x 4096 into 8 bits 50 (236 MB, 4.7 TB/s), backward 8192 x 2048 with dropout 36 and 4.7 (168 MB, 4.6 TB/s).
// Rows that do not lie at multiples of 16 bytes: 8192 x 4095 79 forward (4096: 49) and 109 backward (53), in accesses as wide that cross lines.
#include <type_traits>

#include "../../include/lx.h"
#include "lx_launch.h"
#include "row_plan.h"
#include "rows.h"

namespace lx {

// ---- dropout ---------------------------------------------------------------------------------------

// FLAT: rows follow one another without a gap and hold whole runs, so that a run's number is its place.
template <int DT, bool VEC, bool FLAT>
__global__ __launch_bounds__(256) void dropout_kernel(RowsArgs a, DropArgs drop) {
  using T = ElemT<DT>;
  const Drop g = load_drop(drop);
  const unsigned runs = row_runs(a.d);
  const unsigned long long total = (unsigned long long)a.T * runs;
  const T *X = (const T*)a.in[0], *R = (const T*)a.in[1];
  T* out = (T*)a.out[0];
  for (unsigned long long n = (unsigned long long)blockIdx.x * 256 + threadIdx.x; n < total; n += (unsigned long long)gridDim.x * 256) {
    long long x = (long long)n * 8, r = x, o = x;
    int have = 8;
    if constexpr (!FLAT) {
      const unsigned long long t = total >> 32 ? n / runs : (unsigned)n / runs;
      const int c = (int)(n - t * runs) * 8;
      x = (long long)t * a.is[0] + c, r = (long long)t * a.is[1] + c, o = (long long)t * a.os[0] + c;
      have = a.d - c;
    }
    Run v = load_run<DT, VEC>(X + x, have);
    Run s = {};
    if (R) s = load_run<DT, VEC>(R + r, have);
    if (g.below) g.apply(v, n);
    if (R) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v.v[i] += s.v[i];
    }
    store_run<DT, VEC>(out + o, v, have);
  }
}

// ---- sums over a row -------------------------------------------------------------------------------

// Sums of N numbers over the W wavefronts of a row, the same bits in every lane.  `part`: two sets of W * N floats, used in turn
// (`turn`), so that one barrier per sum is enough.
template <int W, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* part, int turn) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 32; o; o >>= 1) v[i] += __shfl_xor(v[i], o);
  if constexpr (W > 1) {
    float* to = part + turn % 2 * (W * N);
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) to[threadIdx.x / kWave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) v[i] += to[w * N + i];
    }
  }
}
// The largest of a number over the W wavefronts of a row.
template <int W>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* part, int turn) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  if constexpr (W > 1) {
    uint32_t* to = part + turn % 2 * W;
    if (threadIdx.x % kWave == 0) to[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) v = max(v, to[w]);
  }
  return v;
}

// W wavefronts to a row (1: four rows to a workgroup), NR runs to a lane; run number k of a lane is k * 64 W + its place in the row.
template <int W, int NR>
struct Shape {
  static constexpr int kW = W, kRuns = NR, kThreads = W == 1 ? 256 : 64 * W, kRows = W == 1 ? 4 : 1, kLanes = 64 * W, kMost = 8 * kLanes * NR;
};

// The places of a lane's runs: whether it has them, and how many elements the last one holds.
template <class S>
struct Place {
  int at, d;
  __device__ __forceinline__ Place(int d_) : at(S::kW == 1 ? threadIdx.x % kWave : threadIdx.x), d(d_) {}
  __device__ __forceinline__ int col(int k) const { return 8 * (at + k * S::kLanes); }
  __device__ __forceinline__ int have(int k) const { return d - col(k); }
};

// ---- forward ---------------------------------------------------------------------------------------

template <int DT, bool VEC, class S>
__global__ __launch_bounds__(S::kThreads) void norm_fwd(RowsArgs a, DropArgs drop, NormArgs p) {
  using T = ElemT<DT>;
  constexpr int NR = S::kRuns;
  __shared__ float part[2 * 16];
  __shared__ uint32_t tops[2 * 16];
  const Place<S> at(a.d);
  const Drop g = load_drop(drop);
  const T *X = (const T*)a.in[0], *R = (const T*)a.in[1], *weight = (const T*)p.weight;
  T *H = (T*)a.out[0], *Y = (T*)a.out[1];
  const unsigned runs = row_runs(a.d);
  int turn = 0;
  for (long long t = (long long)blockIdx.x * S::kRows + (S::kW == 1 ? threadIdx.x / kWave : 0); t < a.T; t += (long long)gridDim.x * S::kRows, ++turn) {
    Raw<DT> x[NR], r[NR];
    Run h[NR];
    float sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      x[k] = r[k] = Raw<DT>{};
      if (at.have(k) <= 0) continue;
      x[k] = load_raw<DT, VEC>(X + t * a.is[0] + at.col(k), at.have(k));
      if (R) r[k] = load_raw<DT, VEC>(R + t * a.is[1] + at.col(k), at.have(k));
    }
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      h[k] = open<DT>(x[k]);
      if (g.below) g.apply(h[k], (unsigned long long)t * runs + at.col(k) / 8);
      if (R) {
        const Run more = open<DT>(r[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k].v[i] += more.v[i];
      }
    }
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[0] = fmaf(h[k].v[i], h[k].v[i], sum[0]);
    row_sum<S::kW>(sum, part, turn);
    const float scale = 1.f / sqrtf(sum[0] / (float)a.d + p.eps);
    if (H) {
#pragma unroll
      for (int k = 0; k < NR; ++k)
        if (at.have(k) > 0) store_run<DT, VEC>(H + t * a.os[0] + at.col(k), h[k], at.have(k));
    }
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      Run w;
      if (weight && at.have(k) > 0) {
        w = load_run<DT, VEC>(weight + at.col(k), at.have(k));
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k].v[i] *= scale * w.v[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[k].v[i] *= scale;
      }
      if (Y && at.have(k) > 0) store_run<DT, VEC>(Y + t * a.os[1] + at.col(k), h[k], at.have(k));
    }
    if (!p.Y8) continue;
    // 8 bits: a scale per row, or per `group` elements, which are the runs of 4 .. 64 neighbouring lanes.  Sizes are compared
    // as integers: those of infinities and NaN are the largest, so that they reach the scale.
    uint32_t top[NR], all = 0;
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      top[k] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top[k] = max(top[k], __builtin_bit_cast(uint32_t, h[k].v[i]) & 0x7fffffffu);
      if (at.have(k) <= 0) top[k] = 0;
      all = max(all, top[k]);
    }
    const int lanes = p.group / 8;
    if (p.group == a.d) {
      all = row_max<S::kW>(all, tops, turn);
#pragma unroll
      for (int k = 0; k < NR; ++k) top[k] = all;
    } else {
#pragma unroll
      for (int k = 0; k < NR; ++k)
        for (int o = 1; o < lanes; o <<= 1) top[k] = max(top[k], (uint32_t)__shfl_xor((int)top[k], o));
    }
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      // (no smaller than the smallest normal number, whose reciprocal is finite: a row of zeros stays one)
      const float s = __builtin_bit_cast(float, max(__builtin_bit_cast(uint32_t, __builtin_bit_cast(float, top[k]) / 448.f), 0x00800000u));
      const float inv = 1.f / s;
      if (at.have(k) <= 0) continue;
      uint32_t q[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        int u = __builtin_amdgcn_cvt_pk_fp8_f32(h[k].v[4 * i] * inv, h[k].v[4 * i + 1] * inv, 0, false);
        q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(h[k].v[4 * i + 2] * inv, h[k].v[4 * i + 3] * inv, u, true);
      }
      uint8_t* to = p.Y8 + t * a.d + at.col(k);
      if constexpr (VEC) {
        *reinterpret_cast<uint2*>(to) = make_uint2(q[0], q[1]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < at.have(k)) to[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
      }
      if (p.group == a.d) {
        if (k == 0 && at.at == 0) p.scales[t] = s;
      } else if (at.at % lanes == 0) {
        p.scales[t * (a.d / p.group) + at.col(k) / p.group] = s;
      }
    }
  }
}

// ---- backward --------------------------------------------------------------------------------------

// A workgroup of 512 threads (1024 for the widest rows) takes R rows at a time, W wavefronts to a row; the next rows are on their way while
// the sums of these are joined.
template <int W, int NR>
struct BackShape {
  static constexpr int kW = W, kRuns = NR, kThreads = W == 16 ? 1024 : 512, kRows = kThreads / (64 * W), kLanes = 64 * W;
};

// With n = h / rms:  dh = dH + (w dY - n mean(w dY n)) / rms,  dX = drop(dh),  dW = sum over rows of dY n.  Both means are of one
// pass over the row.  A workgroup adds dW of its rows in registers, and leaves a row of partial sums.
template <int DT, bool VEC, class S>
__global__ __launch_bounds__(S::kThreads) void norm_bwd(RowsArgs a, DropArgs drop, NormArgs p) {
  using T = ElemT<DT>;
  constexpr int NR = S::kRuns, W = S::kW, R = S::kRows;
  __shared__ float part[2][R][W][2];
  const int lane = threadIdx.x % S::kLanes, mine = threadIdx.x / S::kLanes, wave = lane / kWave;
  const Drop g = load_drop(drop);
  const T *dY = (const T*)a.in[0], *H = (const T*)a.in[1], *dH = (const T*)a.in[2], *weight = (const T*)p.weight;
  T *dX = (T*)a.out[0], *dR = (T*)a.out[1];
  const unsigned runs = row_runs(a.d);
  int col[NR], have[NR];
  Run dw[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    col[k] = 8 * (lane + k * S::kLanes), have[k] = a.d - col[k];
    dw[k] = Run{};
  }
  // Runs of a row: of H, dY and dH, and w.
  struct Runs {
    Raw<DT> h, dy, dh;
  };
  auto load = [&](Runs& r, int k, long long t) {
    r = Runs{};
    if (have[k] <= 0) return;
    r.h = load_raw<DT, VEC>(H + t * a.is[1] + col[k], have[k]);
    r.dy = load_raw<DT, VEC>(dY + t * a.is[0] + col[k], have[k]);
    if (dH) r.dh = load_raw<DT, VEC>(dH + t * a.is[2] + col[k], have[k]);
  };
  auto load_w = [&](int k) { return weight && have[k] > 0 ? load_raw<DT, VEC>(weight + col[k], have[k]) : Raw<DT>{}; };
  // w dY, and the run's share of the sums of h^2 and w dY h
  auto scaled = [&](const Runs& r, const Raw<DT>& w, Run& h, Run& y, Run& x, float (&sum)[2]) {
    h = open<DT>(r.h), y = open<DT>(r.dy);
    const Run ww = open<DT>(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x.v[i] = weight ? ww.v[i] * y.v[i] : y.v[i];
      sum[0] = fmaf(h.v[i], h.v[i], sum[0]);
      sum[1] = fmaf(x.v[i], h.v[i], sum[1]);
    }
  };
  auto finish = [&](int k, long long t, float scale, float mean, const Run& h, const Run& y, const Run& x, Run out) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float n = h.v[i] * scale;
      out.v[i] += scale * fmaf(-n, mean, x.v[i]);
      dw[k].v[i] = fmaf(y.v[i], n, dw[k].v[i]);
    }
    if (have[k] <= 0) return;
    if (dR) store_run<DT, VEC>(dR + t * a.os[1] + col[k], out, have[k]);
    if (!dX) return;
    if (g.below) g.apply(out, (unsigned long long)t * runs + col[k] / 8);
    store_run<DT, VEC>(dX + t * a.os[0] + col[k], out, have[k]);
  };
  constexpr bool KEEP = W < 16;      // rows of more than 8192 elements, which the registers do not hold, are read again
  Raw<DT> w[KEEP ? NR : 1];
  Runs row[KEEP ? NR : 1];
  const long long stride = (long long)gridDim.x * R;
  long long t = (long long)blockIdx.x * R + mine;
  if constexpr (KEEP) {
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      w[k] = load_w(k);
      if (t < a.T) load(row[k], k, t);
      else row[k] = Runs{};
    }
  }
  int turn = 0;
  for (long long base = (long long)blockIdx.x * R; base < a.T; base += stride, t += stride, turn ^= 1) {
    Run h[KEEP ? NR : 1], x[KEEP ? NR : 1], y[KEEP ? NR : 1], out[KEEP ? NR : 1];
    float sum[2] = {0.f, 0.f};
    if constexpr (KEEP) {
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        scaled(row[k], w[k], h[k], y[k], x[k], sum);
        out[k] = open<DT>(row[k].dh);
      }
#pragma unroll
      for (int k = 0; k < NR; ++k)
        if (t + stride < a.T) load(row[k], k, t + stride);
    } else if (t < a.T) {
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        load(row[0], k, t);
        scaled(row[0], load_w(k), h[0], y[0], x[0], sum);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int o = 32; o; o >>= 1) sum[i] += __shfl_xor(sum[i], o);
    if constexpr (W > 1) {      // (two sets in turn: one barrier per row)
      if (lane % kWave == 0) part[turn][mine][wave][0] = sum[0], part[turn][mine][wave][1] = sum[1];
      lds_barrier();            // (does not wait for the loads)
      sum[0] = sum[1] = 0;
#pragma unroll
      for (int v = 0; v < W; ++v) sum[0] += part[turn][mine][v][0], sum[1] += part[turn][mine][v][1];
    }
    if (t >= a.T) continue;
    const float scale = 1.f / sqrtf(sum[0] / (float)a.d + p.eps);
    const float mean = sum[1] * scale / (float)a.d;      // of w dY n
    if constexpr (KEEP) {
#pragma unroll
      for (int k = 0; k < NR; ++k) finish(k, t, scale, mean, h[k], y[k], x[k], out[k]);
    } else {
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        load(row[0], k, t);
        scaled(row[0], load_w(k), h[0], y[0], x[0], sum);
        finish(k, t, scale, mean, h[0], y[0], x[0], open<DT>(row[0].dh));
      }
    }
  }
  if (!p.dw_part) return;
  float* to = p.dw_part + (long long)blockIdx.x * a.d;
  if constexpr (R == 1) {
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < have[k]) to[col[k] + i] = dw[k].v[i];
  } else {      // the rows' sums, in order
    __shared__ float rows[R - 1][8][S::kLanes];
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      __syncthreads();
      if (mine > 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) rows[mine - 1][i][lane] = dw[k].v[i];
      __syncthreads();
      if (mine == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v = dw[k].v[i];
#pragma unroll
          for (int r = 0; r < R - 1; ++r) v += rows[r][i][lane];
          if (i < have[k]) to[col[k] + i] = v;
        }
      }
    }
  }
}

// dW[c] = the partial sums of column c, in an order that their number fixes: 16 columns to a workgroup, 64 threads to a column.
__global__ __launch_bounds__(1024) void norm_dw_sum(const float* __restrict__ part, int rows, int d, float* __restrict__ dW) {
  __shared__ float sums[64][17];
  const int x = threadIdx.x % 16, y = threadIdx.x / 16, c = blockIdx.x * 16 + x;
  float v = 0;
  if (c < d)
#pragma unroll 8
    for (int r = y; r < rows; r += 64) v += part[(long long)r * d + c];
  sums[y][x] = v;
  __syncthreads();
  // a wavefront to a column: its 64 sums
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  v = sums[lane][w];
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if (lane == 0 && blockIdx.x * 16 + w < d) dW[blockIdx.x * 16 + w] = v;
}

constexpr int kNormBackWorkgroups = 512;      // rows of partial sums
// So few rounds of rows are left to one workgroup, which writes dW itself: a second launch takes longer.
constexpr int kNormBackAlone = 4;

// ---- launches --------------------------------------------------------------------------------------

template <class F>
static hipError_t of_type(int dt, bool vec, F f) {
  using std::integral_constant;
  auto both = [&](auto t) { return vec ? f(t, std::true_type()) : f(t, std::false_type()); };
  if (dt == LX_F32) return both(integral_constant<int, kSingle>());
  return dt == LX_F16 ? both(integral_constant<int, kF16>()) : both(integral_constant<int, kBf16>());
}
// The shapes by width.
template <class F>
static hipError_t of_width(int d, F f) {
  if (d <= 512) return f(Shape<1, 1>());
  if (d <= 1024) return f(Shape<1, 2>());
  if (d <= 2048) return f(Shape<4, 1>());
  if (d <= 4096) return f(Shape<4, 2>());
  if (d <= 8192) return f(Shape<4, 4>());
  return f(Shape<16, 4>());
}
static_assert(Shape<16, 4>::kMost == kNormWidest, "widest row");

hipError_t launch_dropout(int dt, const RowsArgs& a, const DropArgs& drop, bool vec, hipStream_t st) {
  ProfScope prof(kKDropout, st);
  const bool flat = vec && a.is[0] == a.d && (!a.in[1] || a.is[1] == a.d) && a.os[0] == a.d;
  const int grid = dropout_grid(a.T, a.d, kNormWorkgroups * 8);
  return of_type(dt, vec, [&](auto t, auto v) {
    constexpr int DT = decltype(t)::value;
    constexpr bool VEC = decltype(v)::value;
    if (VEC && flat)
      hipLaunchKernelGGL((dropout_kernel<DT, VEC, VEC>), dim3(grid), dim3(256), 0, st, a, drop);
    else
      hipLaunchKernelGGL((dropout_kernel<DT, VEC, false>), dim3(grid), dim3(256), 0, st, a, drop);
    return hipGetLastError();
  });
}

hipError_t launch_norm_fwd(int dt, const RowsArgs& a, const DropArgs& drop, const NormArgs& p, bool vec, hipStream_t st) {
  ProfScope prof(kKNorm, st);
  return of_type(dt, vec, [&](auto t, auto v) {
    return of_width(a.d, [&](auto s) {
      using S = decltype(s);
      const int wgs = (int)(((long long)a.T + S::kRows - 1) / S::kRows), most = kNormWorkgroups * 4;
      hipLaunchKernelGGL((norm_fwd<decltype(t)::value, decltype(v)::value, S>), dim3(wgs < most ? wgs : most), dim3(S::kThreads), 0, st, a, drop, p);
      return hipGetLastError();
    });
  });
}

template <class F>
static hipError_t of_width_back(int d, F f) {
  if (d <= 512) return f(BackShape<1, 1>());
  if (d <= 2048) return f(BackShape<4, 1>());
  if (d <= 4096) return f(BackShape<4, 2>());
  if (d <= 8192) return f(BackShape<8, 2>());
  if (d <= 16384) return f(BackShape<16, 2>());
  return f(BackShape<16, 4>());
}
int norm_bwd_parts(int T, int d) {
  int rows = 0;
  (void)of_width_back(d, [&](auto s) {
    rows = decltype(s)::kRows;
    return hipSuccess;
  });
  const int all = (int)(((long long)T + rows - 1) / rows);
  return all <= kNormBackAlone ? 1 : all < kNormBackWorkgroups ? all : kNormBackWorkgroups;
}
hipError_t launch_norm_bwd(int dt, const RowsArgs& a, const DropArgs& drop, const NormArgs& p, float* dW, bool vec, hipStream_t st) {
  ProfScope prof(kKNormBwd, st);
  const int parts = norm_bwd_parts(a.T, a.d);
  NormArgs q = p;
  if (parts == 1) q.dw_part = dW;
  const hipError_t e = of_type(dt, vec, [&](auto t, auto v) {
    return of_width_back(a.d, [&](auto s) {
      using S = decltype(s);
      hipLaunchKernelGGL((norm_bwd<decltype(t)::value, decltype(v)::value, S>), dim3(parts), dim3(S::kThreads), 0, st, a, drop, q);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess || !dW || parts == 1) return e;
  hipLaunchKernelGGL(norm_dw_sum, dim3((a.d + 15) / 16), dim3(1024), 0, st, p.dw_part, parts, a.d, dW);
  return hipGetLastError();
}

}  // namespace lx
