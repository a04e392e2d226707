// Global norm of many gradients and clipping, in two launches for any number of tensors.
//
// The set is cut into pieces of one tensor each, listed in the device table, and the pieces are dealt to a fixed number of
// workgroups.  The first launch leaves a sum of squares per workgroup, in 64 bits (the squares of what fp32 holds overflow fp32);
// every workgroup of the second adds those sums, in the same order, and scales its pieces, the ones read last first, since
// they are the likeliest to be still in the caches, past which it writes.  Memory-bound; nothing is added by atomics.
//
// 200 tensors, 740 MB, scaled in place: 472 us, 4.7 TB/s for reading twice and writing once (cached stores 488); 48 of fp32 gradients,
// 63 MB, which the caches hold between the launches, 33; 24 of 1.5 MB together 8.2, two launches.
#include "lx_dev.h"
#include "../../include/lx.h"
#include "lx_launch.h"

namespace lx {

constexpr int kClipThreads = 256;

template <class F>
__device__ __forceinline__ void of_type(int dt, F f) {
  if (dt == LX_F32) f(std::integral_constant<int, 2>());
  else if (dt == LX_F16) f(std::integral_constant<int, kF16>());
  else f(std::integral_constant<int, kBf16>());
}
// DT: kBf16, kF16, or 2 for float
template <int DT>
struct Elem {
  static constexpr int kSize = DT == 2 ? 4 : 2, kRun = 16 / kSize;
  using T = std::conditional_t<DT == 2, float, uint16_t>;
  static __device__ __forceinline__ float load(T x) {
    if constexpr (DT == 2) return x;
    else return to_f32<DT>(x);
  }
  static __device__ __forceinline__ T store(float x) {
    if constexpr (DT == 2) return x;
    else return (T)pack2<DT>(x, 0.f);
  }
  static __device__ __forceinline__ void open(const uint4& u, float (&v)[kRun]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == 2) v[i] = __builtin_bit_cast(float, w[i]);
      else v[2 * i] = to_f32<DT>(w[i] & 0xffff), v[2 * i + 1] = to_f32<DT>(w[i] >> 16);
    }
  }
  static __device__ __forceinline__ uint4 close(const float (&v)[kRun]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == 2) w[i] = __builtin_bit_cast(uint32_t, v[i]);
      else w[i] = pack2<DT>(v[2 * i], v[2 * i + 1]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
// A piece: [from, to) of its tensor; `runs` runs of 16 aligned bytes from `first` on, single elements before and after.
struct Piece {
  long long from, to, first;
  int runs;
  template <int DT>
  __device__ __forceinline__ void of(const GradEntry& e, int piece) {
    using E = Elem<DT>;
    from = (long long)(piece - e.first_piece) * kGradPiece;
    to = min(e.n, from + kGradPiece);
    const uintptr_t at = (uintptr_t)e.in + from * E::kSize;
    first = min(to, from + (long long)((16 - at % 16) % 16 / E::kSize));
    runs = (int)((to - first) / E::kRun);
  }
};
__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kClipThreads / kWave; ++w) v += part[w];
  return v;
}

__global__ __launch_bounds__(kClipThreads) void grad_squares(const GradEntry* __restrict__ table, const int* __restrict__ entry_of, int pieces,
                                                             double* __restrict__ sums) {
  __shared__ double part[kClipThreads / kWave];
  double sum = 0;
  int next = (int)blockIdx.x < pieces ? entry_of[blockIdx.x] : 0;      // (read a piece ahead: 134 us for 740 MB, so 129)
  for (int p = blockIdx.x; p < pieces; p += gridDim.x) {
    const GradEntry e = table[next];
    if (p + (int)gridDim.x < pieces) next = entry_of[p + gridDim.x];
    of_type(e.dt, [&](auto dt) {
      using E = Elem<decltype(dt)::value>;
      Piece w;
      w.of<decltype(dt)::value>(e, p);
      const typename E::T* in = (const typename E::T*)e.in;
      const uint4* v = (const uint4*)(in + w.first);
#pragma unroll 4
      for (int i = threadIdx.x; i < w.runs; i += kClipThreads) {
        float x[E::kRun];
        E::open(v[i], x);
#pragma unroll
        for (int k = 0; k < E::kRun; ++k) sum = fma((double)x[k], (double)x[k], sum);
      }
      const long long rest = w.first + (long long)w.runs * E::kRun;
      for (long long i = w.from + threadIdx.x; i < w.first; i += kClipThreads) sum += (double)E::load(in[i]) * (double)E::load(in[i]);
      for (long long i = rest + threadIdx.x; i < w.to; i += kClipThreads) sum += (double)E::load(in[i]) * (double)E::load(in[i]);
    });
  }
  sum = block_sum(sum, part);
  if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kClipThreads) void grad_scale(const GradEntry* __restrict__ table, const int* __restrict__ entry_of, int pieces,
                                                           const double* __restrict__ sums, int n_sums, float max_norm, float* __restrict__ norm_out) {
  __shared__ double part[kClipThreads / kWave];
  double total = 0;
  for (int i = threadIdx.x; i < n_sums; i += kClipThreads) total += sums[i];
  total = sqrt(block_sum(total, part));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)total;
  const bool keep = total <= (double)max_norm;
  const float c = keep ? 1.f : (float)((double)max_norm / total);
  for (int p = pieces - 1 - (int)blockIdx.x; p >= 0; p -= gridDim.x) {
    const GradEntry e = table[entry_of[p]];
    if (!e.out || (keep && e.out == e.in)) continue;
    of_type(e.dt, [&](auto dt) {
      using E = Elem<decltype(dt)::value>;
      Piece w;
      w.of<decltype(dt)::value>(e, p);
      const typename E::T* in = (const typename E::T*)e.in;
      typename E::T* out = (typename E::T*)e.out;
      const uint4* v = (const uint4*)(in + w.first);
      if (((uintptr_t)(out + w.first)) % 16 == 0) {
        uint4* o = (uint4*)(out + w.first);
#pragma unroll 4
        for (int i = threadIdx.x; i < w.runs; i += kClipThreads) {
          float x[E::kRun];
          E::open(v[i], x);
#pragma unroll
          for (int k = 0; k < E::kRun; ++k) x[k] *= c;
          __builtin_nontemporal_store(__builtin_bit_cast(u32x4, E::close(x)), (u32x4*)(o + i));
        }
      } else {
        for (long long i = w.first + threadIdx.x; i < w.first + (long long)w.runs * E::kRun; i += kClipThreads) out[i] = E::store(E::load(in[i]) * c);
      }
      const long long rest = w.first + (long long)w.runs * E::kRun;
      for (long long i = w.from + threadIdx.x; i < w.first; i += kClipThreads) out[i] = E::store(E::load(in[i]) * c);
      for (long long i = rest + threadIdx.x; i < w.to; i += kClipThreads) out[i] = E::store(E::load(in[i]) * c);
    });
  }
}

hipError_t launch_grad_norm_clip(const GradEntry* table, int n_tensors, int pieces, float max_norm, float* norm, double* sums, hipStream_t st) {
  ProfScope p(kKClip, st);
  const int* entry_of = (const int*)(table + n_tensors);
  const int wgs = pieces < kGradSums ? pieces : kGradSums;
  if (pieces > 0) {
    hipLaunchKernelGGL(grad_squares, dim3(wgs), dim3(kClipThreads), 0, st, table, entry_of, pieces, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(grad_scale, dim3(wgs > 0 ? wgs : 1), dim3(kClipThreads), 0, st, table, entry_of, pieces, sums, wgs, max_norm, norm);
  return hipGetLastError();
}

}  // namespace lx
