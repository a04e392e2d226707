// Attention over dense keys with rules on its scores: the plain kernels, for fp32 (the correctness configuration), and the
// key ranges of packed documents.
//
// A wavefront per row: forward and dQ per query, dK/dV per key.  64 keys (queries) at a time, one a lane, each lane making its
// own scores from global memory; then the sums over the pairs that the masks leave, D/64 columns to a lane.  A pair that is
// masked is never added, so what it holds has no effect.  Every sum is in 64 bits, and the mean of dP and
// the softmax's sum stay so from the query side of the backward pass, which makes them from the products, to the key side.
#include "lx_dev.h"
#include "lx_launch.h"

namespace lx {

constexpr int kPlainRows = 4;    // wavefronts, rows, per workgroup

__device__ __forceinline__ const float* row_of(const ScoreTensor& t, int b, int h, long long s) {
  return (const float*)t.p + b * t.sb + h * t.sh + s * t.ss;
}
__device__ __forceinline__ float* out_row(const ScoreTensor& t, int b, int h, long long s) {
  return (float*)const_cast<void*>(t.p) + b * t.sb + h * t.sh + s * t.ss;
}

struct PlainRules {
  long long start;    // position of query 0
  int b;
  const ScoreArgs& a;
  __device__ PlainRules(const ScoreArgs& args, int batch) : b(batch), a(args) {
    start = a.q_start ? a.q_start[b] : (long long)a.Sk - a.Sq;
  }
  // the keys that a query attends: lo .. hi - 1
  __device__ void range(int q, int& lo, int& hi) const {
    lo = 0, hi = a.Sk;
    if (a.causal) hi = (int)max(min((long long)hi, start + q + 1), 0ll);
    if (a.key_lo) {
      lo = max(lo, a.key_lo[(long long)b * a.Sq + q]);
      hi = min(hi, a.key_hi[(long long)b * a.Sq + q]);
    }
  }
  // of a pair's product: the score, and its derivative by the product
  __device__ double score(double dot, int h, int q, int k, double& slope) const {
    double s = dot * (double)a.scale;
    slope = a.scale;
    if (a.cap > 0.f) {
      const double t = tanh(s / (double)a.cap);
      s = t * (double)a.cap;
      slope *= 1.0 - t * t;
    }
    if (a.slopes) s -= (double)a.slopes[h] * (double)llabs(start + q - k);
    return s;
  }
};

template <int D>
__device__ __forceinline__ double dot_row(const float* __restrict__ x, const float* __restrict__ y) {
  double s = 0;
#pragma unroll 8
  for (int d = 0; d < D; ++d) s += (double)x[d] * (double)y[d];
  return s;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ double wave_max(double v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmax(v, __shfl_xor(v, o));
  return v;
}

template <int D>
__global__ __launch_bounds__(64 * kPlainRows) void score_fwd_plain(ScoreArgs a) {
  const int lane = threadIdx.x % kWave, q = blockIdx.x * kPlainRows + threadIdx.x / kWave, h = blockIdx.y, b = blockIdx.z;
  if (q >= a.Sq) return;
  const PlainRules rules(a, b);
  int lo, hi;
  rules.range(q, lo, hi);
  const int hk = h / (a.Hq / a.Hkv);
  const float* qr = row_of(a.Q, b, h, q);
  double m = -INFINITY, l = 0, o[D / 64] = {};
  for (int k0 = lo; k0 < hi; k0 += kWave) {
    const int k = k0 + lane;
    double s = -INFINITY, slope;
    if (k < hi) s = rules.score(dot_row<D>(qr, row_of(a.K, b, hk, k)), h, q, k, slope);
    const double top = fmax(m, wave_max(s)), ref = top == -INFINITY ? 0 : top;
    const double p = k < hi ? exp(s - ref) : 0, scale = exp(m - ref);
    l = l * scale + wave_sum(p);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] *= scale;
    for (int j = 0; j < min(hi - k0, kWave); ++j) {
      const double pj = __shfl(p, j);
      const float* v = row_of(a.V, b, hk, k0 + j);
#pragma unroll
      for (int i = 0; i < D / 64; ++i) o[i] += pj * (double)v[lane + 64 * i];
    }
    m = top;
  }
  float* out = out_row(a.O, b, h, q);
  const bool none = hi <= lo || l == 0;      // (no key, or scores of -inf alone)
#pragma unroll
  for (int i = 0; i < D / 64; ++i) out[lane + 64 * i] = none ? 0.f : (float)(o[i] / l);
  if (a.LSE && lane == 0) a.LSE[((long long)b * a.Hq + h) * a.Sq + q] = none ? -INFINITY : (float)(m + log(l));
}

template <int D>
__global__ __launch_bounds__(64 * kPlainRows) void score_dq_plain(ScoreArgs a) {
  const int lane = threadIdx.x % kWave, q = blockIdx.x * kPlainRows + threadIdx.x / kWave, h = blockIdx.y, b = blockIdx.z;
  if (q >= a.Sq) return;
  const PlainRules rules(a, b);
  int lo, hi;
  rules.range(q, lo, hi);
  const int hk = h / (a.Hq / a.Hkv);
  const float *qr = row_of(a.Q, b, h, q), *dor = row_of(a.dO, b, h, q);
  const long long at = ((long long)b * a.Hq + h) * a.Sq + q;
  // dP less its mean is small next to dP where one key has nearly all the weight.  So the mean and the sum come from the products, not
  // from the rounded O and LSE (two keys, the lesser's weight 1e-3: dQ and dK up to 3e-5 of their norm off), and dP is taken less that
  // of the heaviest key, so that no digits cancel (with the mean itself, in 64 bits: 1e-5 off at a weight of 1e-12, 0.7 at 1e-22).
  // (1 x 512, 4 heads, D = 64, causal, backward: 318 us, 257 from O and LSE.)
  double m = -INFINITY, l = 0, center = 0, delta = 0, g[D / 64] = {};
  if (a.LSE[at] == -INFINITY) hi = lo;
  for (int k0 = lo; k0 < hi; k0 += kWave) {
    const int k = k0 + lane;
    double s = -INFINITY, dp = 0, slope;
    if (k < hi) s = rules.score(dot_row<D>(qr, row_of(a.K, b, hk, k)), h, q, k, slope), dp = dot_row<D>(dor, row_of(a.V, b, hk, k));
    const double here = wave_max(s), top = fmax(m, here), ref = top == -INFINITY ? 0 : top;
    if (here > m) {
      const double next = __shfl(dp, __ffsll(__ballot(s == here)) - 1);
      delta += (center - next) * l;
      center = next;
    }
    const double p = k < hi ? exp(s - ref) : 0, scale = exp(m - ref);
    l = l * scale + wave_sum(p);
    delta = delta * scale + wave_sum(p * (dp - center));
    m = top;
  }
  const double lse = m + log(l);
  if (lo < hi) delta /= l;
  if (lane == 0) a.center[at] = center, a.Delta[at] = delta, a.lse64[at] = lse;
  for (int k0 = lo; k0 < hi; k0 += kWave) {
    const int k = k0 + lane;
    double ds = 0;
    if (k < hi) {
      double slope;
      const double s = rules.score(dot_row<D>(qr, row_of(a.K, b, hk, k)), h, q, k, slope);
      ds = exp(s - lse) * (dot_row<D>(dor, row_of(a.V, b, hk, k)) - center - delta) * slope;
      if (hi - lo == 1) ds *= 0;       // (of one key: zero, and comes out as just that)
    }
    for (int j = 0; j < min(hi - k0, kWave); ++j) {
      const double dj = __shfl(ds, j);
      const float* kr = row_of(a.K, b, hk, k0 + j);
#pragma unroll
      for (int i = 0; i < D / 64; ++i) g[i] += dj * (double)kr[lane + 64 * i];
    }
  }
  float* out = out_row(a.dQ, b, h, q);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) out[lane + 64 * i] = (float)g[i];
}

template <int D>
__global__ __launch_bounds__(64 * kPlainRows) void score_dkv_plain(ScoreArgs a) {
  const int lane = threadIdx.x % kWave, k = blockIdx.x * kPlainRows + threadIdx.x / kWave, hk = blockIdx.y, b = blockIdx.z;
  if (k >= a.Sk) return;
  const PlainRules rules(a, b);
  const float *kr = row_of(a.K, b, hk, k), *vr = row_of(a.V, b, hk, k);
  double gk[D / 64] = {}, gv[D / 64] = {};
  const int group = a.Hq / a.Hkv;
  for (int h = hk * group; h < (hk + 1) * group; ++h)
    for (int q0 = 0; q0 < a.Sq; q0 += kWave) {
      const int q = q0 + lane;
      bool seen = false;
      double p = 0, ds = 0;
      if (q < a.Sq) {
        int lo, hi;
        rules.range(q, lo, hi);
        const long long at = ((long long)b * a.Hq + h) * a.Sq + q;
        seen = lo <= k && k < hi && a.LSE[at] != -INFINITY;
        if (seen) {
          const float *qr = row_of(a.Q, b, h, q), *dor = row_of(a.dO, b, h, q);
          double slope;
          p = exp(rules.score(dot_row<D>(qr, kr), h, q, k, slope) - a.lse64[at]);
          ds = p * (dot_row<D>(dor, vr) - a.center[at] - a.Delta[at]) * slope;
          if (hi - lo == 1) ds *= 0;
        }
      }
      for (unsigned long long left = __ballot(seen); left; left &= left - 1) {
        const int j = __ffsll((long long)left) - 1;
        const double pj = __shfl(p, j), dj = __shfl(ds, j);
        const float *qr = row_of(a.Q, b, h, q0 + j), *dor = row_of(a.dO, b, h, q0 + j);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          gv[i] += pj * (double)dor[lane + 64 * i];
          gk[i] += dj * (double)qr[lane + 64 * i];
        }
      }
    }
  float *ok = out_row(a.dK, b, hk, k), *ov = out_row(a.dV, b, hk, k);
#pragma unroll
  for (int i = 0; i < D / 64; ++i) ok[lane + 64 * i] = (float)gk[i], ov[lane + 64 * i] = (float)gv[i];
}

// A token per thread: bisects the documents' first tokens for its own.
constexpr int kStagedDocs = 2048;
__global__ __launch_bounds__(256) void key_ranges_kernel(int B, int S, const int* __restrict__ begin, const int* __restrict__ end,
                                                         const int* __restrict__ prefix, int n, int causal, int* __restrict__ lo_out,
                                                         int* __restrict__ hi_out) {
  __shared__ int staged[kStagedDocs];
  const long long t = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  // (a search through memory waits for every step of it: 27 documents, 8192 tokens, one call after the other, 2.8 us with a copy)
  const bool here = n <= kStagedDocs;
  if (here)
    for (int i = threadIdx.x; i < n; i += blockDim.x) staged[i] = begin[i];
  __syncthreads();
  if (t >= (long long)B * S) return;
  const int row0 = (int)(t / S) * S;
  int from = 0, to = n;      // documents before `from` begin at t or earlier, those from `to` on later
  while (from < to) {
    const int mid = (from + to) / 2;
    if ((here ? staged[mid] : begin[mid]) <= t) from = mid + 1;
    else to = mid;
  }
  int lo = 0, hi = 0;
  if (from > 0 && t < end[from - 1]) {
    const int d0 = begin[from - 1], d1 = min(end[from - 1], row0 + S);
    lo = max(d0, row0);
    hi = d1;
    if (causal) {
      hi = (int)t + 1;
      if (prefix) hi = (int)max((long long)hi, min((long long)d1, (long long)d0 + prefix[from - 1]));
    }
    lo -= row0;
    hi -= row0;
  }
  lo_out[t] = lo;
  hi_out[t] = hi;
}

template <int D>
static hipError_t plain_fwd(const ScoreArgs& a, hipStream_t st) {
  ProfScope p(kKScoreFwd, st);
  hipLaunchKernelGGL(score_fwd_plain<D>, dim3((a.Sq + kPlainRows - 1) / kPlainRows, a.Hq, a.B), dim3(64 * kPlainRows), 0, st, a);
  return hipGetLastError();
}
template <int D>
static hipError_t plain_bwd(const ScoreArgs& a, hipStream_t st) {
  {
    ProfScope p(kKScoreDq, st);
    hipLaunchKernelGGL(score_dq_plain<D>, dim3((a.Sq + kPlainRows - 1) / kPlainRows, a.Hq, a.B), dim3(64 * kPlainRows), 0, st, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  ProfScope p(kKScoreDkv, st);
  hipLaunchKernelGGL(score_dkv_plain<D>, dim3((a.Sk + kPlainRows - 1) / kPlainRows, a.Hkv, a.B), dim3(64 * kPlainRows), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_score_fwd_plain(const ScoreArgs& a, hipStream_t st) { return a.D == 64 ? plain_fwd<64>(a, st) : plain_fwd<128>(a, st); }
hipError_t launch_score_bwd_plain(const ScoreArgs& a, hipStream_t st) { return a.D == 64 ? plain_bwd<64>(a, st) : plain_bwd<128>(a, st); }

hipError_t launch_key_ranges(int B, int S, const int* begin, const int* end, const int* prefix, int n, int causal, int* lo, int* hi,
                             hipStream_t st) {
  ProfScope p(kKKeyRanges, st);
  hipLaunchKernelGGL(key_ranges_kernel, dim3((unsigned)(((long long)B * S + 255) / 256)), dim3(256), 0, st, B, S, begin, end, prefix, n,
                     causal, lo, hi);
  return hipGetLastError();
}

}  // namespace lx
