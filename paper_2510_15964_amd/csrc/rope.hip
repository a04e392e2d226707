// Rotary positions and their table.
//
// A thread turns the same E pairs (two runs of E elements, or one of E / 2 pairs) of several heads of one token: the table's
// cosines and sines are read once per token, not once per head, and the loads of the heads do not wait for each other.
// Memory-bound: every element is read and written once, as runs of up to 16 bytes.  4 x 2048 tokens, 32 and 32 heads, D = 128, bf16:
// 268 MB in 49 us, 5.4 TB/s, fp32 112 and 4.8; a few tokens 5 us, a launch.  Runs of single elements, where half of what is turned is odd,
// are bound by the number of accesses: 126 of 128 in place 57 us.
#include "lx_dev.h"
#include "../../include/lx.h"
#include "lx_launch.h"

namespace lx {

constexpr int kRopeThreads = 256;
struct F32Type { using T = float; static __device__ float load(float x) { return x; } static __device__ float store(float x) { return x; } };
struct Bf16Type {
  using T = uint16_t;
  static __device__ float load(uint16_t x) { return to_f32<kBf16>(x); }
  static __device__ uint16_t store(float x) { return (uint16_t)pack2<kBf16>(x, 0.f); }
};
struct F16Type {
  using T = uint16_t;
  static __device__ float load(uint16_t x) { return to_f32<kF16>(x); }
  static __device__ uint16_t store(float x) { return (uint16_t)pack2<kF16>(x, 0.f); }
};

// N elements that lie together, one access
template <class T, int N>
struct Run {
  T v[N];
  static __device__ __forceinline__ Run from(const T* p) {
    Run r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
  }
  __device__ __forceinline__ void to(T* p) const { __builtin_memcpy(p, this, sizeof *this); }
};

// What the threads of a token do: runs of pairs, then runs of the elements that stay (none where in and out are the same).
struct RopeGrid {
  int turned, tail, tail_run;      // runs of E, runs of tail_run elements
  int heads_per_wg;
};

template <class Ty, int E, int LAYOUT>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a, const RopeGrid g) {
  using T = typename Ty::T;
  using R = Run<T, E>;
  const unsigned per_token = g.turned + g.tail;
  const unsigned i = blockIdx.x * kRopeThreads + threadIdx.x, token = i / per_token, run = i - token * per_token;
  if (token >= (unsigned)a.B * a.S) return;
  const int b = token / a.S, s = token - b * a.S;
  const int h0 = blockIdx.y * g.heads_per_wg, h1 = min(h0 + g.heads_per_wg, a.t[0].heads + (a.n > 1 ? a.t[1].heads : 0));
  auto at = [&](int h, const T*& in, T*& out) {
    const bool first = h < a.t[0].heads;
    const RopeTensor& t = a.t[first ? 0 : 1];
    const int hh = first ? h : h - a.t[0].heads;
    in = (const T*)t.in + b * t.is[0] + hh * t.is[1] + s * t.is[2];
    out = (T*)t.out + b * t.os[0] + hh * t.os[1] + s * t.os[2];
  };
  const T* in;
  T* out;
  // The loads of four heads come first: one that follows a store would not be moved before it.
  auto copy = [&](auto of) {
    using C = Run<T, decltype(of)::value>;
    const int c = a.rot + (run - g.turned) * decltype(of)::value;
    for (int h = h0; h < h1; h += 4) {
      C x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        at(min(h + j, h1 - 1), in, out);
        x[j] = C::from(in + c);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (h + j >= h1) break;
        at(h + j, in, out);
        x[j].to(out + c);
      }
    }
  };
  if (run >= (unsigned)g.turned) {
    if constexpr (sizeof(T) == 2)
      if (g.tail_run == 8) return copy(std::integral_constant<int, 8>());
    if (g.tail_run == 4) return copy(std::integral_constant<int, 4>());
    if (g.tail_run == 2) return copy(std::integral_constant<int, 2>());
    return copy(std::integral_constant<int, 1>());
  }
  const int p = a.positions ? a.positions[token] : s, hr = a.rot / 2;
  constexpr bool kHalf = LAYOUT == LX_ROPE_HALF, kTwo = kHalf || E == 1;      // kTwo: x and y in runs of their own
  constexpr int P = kTwo ? E : E / 2;     // pairs
  const int pair0 = run * P, cx = kHalf ? pair0 : 2 * pair0, cy = kHalf ? hr + pair0 : cx + 1;
  const bool known = p >= 0 && p < a.n_pos;
  const float* row = a.table + (long long)(known ? p : 0) * a.rot + pair0;
  Run<float, P> co = Run<float, P>::from(row), si = Run<float, P>::from(row + hr);
#pragma unroll
  for (int k = 0; k < P; ++k) {
    if (!known) co.v[k] = si.v[k] = __builtin_nanf("");
    if (a.inverse) si.v[k] = -si.v[k];
  }
  for (int h = h0; h < h1; h += 4) {
    R x[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      at(min(h + j, h1 - 1), in, out);
      x[j] = R::from(in + cx);
      if constexpr (kTwo) y[j] = R::from(in + cy);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (h + j >= h1) break;
      at(h + j, in, out);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        T& u = x[j].v[kTwo ? k : 2 * k];
        T& w = kTwo ? y[j].v[k] : x[j].v[2 * k + 1];
        const float fx = Ty::load(u), fy = Ty::load(w);
        u = Ty::store(fx * co.v[k] - fy * si.v[k]);
        w = Ty::store(fx * si.v[k] + fy * co.v[k]);
      }
      x[j].to(out + cx);
      if constexpr (kTwo) y[j].to(out + cy);
    }
  }
}

__global__ __launch_bounds__(kRopeThreads) void rope_table_kernel(int rot, int n_pos, double base, int kind, double factor, double trained,
                                                                  double low, double high, double gain, float* __restrict__ table) {
  const int hr = rot / 2;
  const long long i = (long long)blockIdx.x * kRopeThreads + threadIdx.x;
  if (i >= (long long)n_pos * hr) return;
  const int p = (int)(i / hr), k = (int)(i - (long long)p * hr);
  if (kind == LX_ROPE_BASE) base *= pow(factor, (double)rot / (rot - 2));
  double f = pow(base, -2.0 * k / rot);
  if (kind == LX_ROPE_LINEAR) f /= factor;
  if (kind == LX_ROPE_PARTS) {
    const double turns = trained * f / 6.283185307179586, w = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
    f *= w + (1.0 - w) / factor;
  }
  double sn, cs;
  sincos(p * f, &sn, &cs);
  table[(long long)p * rot + k] = (float)(gain * cs);
  table[(long long)p * rot + hr + k] = (float)(gain * sn);
}

// Runs as wide as the sizes, the strides and the addresses allow: 16, 8 or 4 bytes, or element by element.  `length` of them from
// element `at` on.  (16 bytes at any address and what is left pair by pair instead: half of 126 and of 62 elements in place, bf16, 57 and
// 30 us, so 77 and 43.)
static int run_elements(const RopeArgs& a, int at, int length, int size) {
  for (int e = 16 / size; e > 1; e /= 2) {
    if (e * size < 4) break;
    bool ok = at % e == 0 && length % e == 0;
    for (int i = 0; i < a.n && ok; ++i) {
      const RopeTensor& t = a.t[i];
      ok = ((uintptr_t)t.in | (uintptr_t)t.out) % (e * size) == 0;
      for (int k = 0; k < 3; ++k) ok = ok && t.is[k] % e == 0 && t.os[k] % e == 0;
    }
    if (ok) return e;
  }
  return 1;
}
template <class Ty, int E>
static hipError_t run_rope(int layout, const RopeArgs& a, hipStream_t st) {
  bool in_place = true;
  for (int i = 0; i < a.n; ++i) in_place = in_place && a.t[i].in == a.t[i].out;
  RopeGrid g;
  g.turned = layout == LX_ROPE_HALF || E == 1 ? a.rot / 2 / E : a.rot / E;
  g.tail_run = run_elements(a, a.rot, a.D - a.rot, sizeof(typename Ty::T));
  g.tail = in_place ? 0 : (a.D - a.rot) / g.tail_run;
  const int heads = a.t[0].heads + (a.n > 1 ? a.t[1].heads : 0);
  const long long wgs = ((long long)a.B * a.S * (g.turned + g.tail) + kRopeThreads - 1) / kRopeThreads;
  // As many heads to a thread, whose cosines and sines are read once, as leave two workgroups to a CU (eight: 3 x 900 tokens, 12 and 12
  // heads, D = 256, bf16, in place 13.0 us, so 10.8; half of it turned 8.0 and 6.7).
  g.heads_per_wg = (int)lora_clamp((int)((long long)heads * wgs / (2 * kCUs)), 8);
  const dim3 grid((unsigned)wgs, (heads + g.heads_per_wg - 1) / g.heads_per_wg);
  if (layout == LX_ROPE_HALF)
    hipLaunchKernelGGL((rope_kernel<Ty, E, LX_ROPE_HALF>), grid, dim3(kRopeThreads), 0, st, a, g);
  else
    hipLaunchKernelGGL((rope_kernel<Ty, E, LX_ROPE_INTERLEAVED>), grid, dim3(kRopeThreads), 0, st, a, g);
  return hipGetLastError();
}
template <class Ty>
static hipError_t by_run(int layout, const RopeArgs& a, hipStream_t st) {
  const int e = run_elements(a, 0, layout == LX_ROPE_HALF ? a.rot / 2 : a.rot, sizeof(typename Ty::T));
  if constexpr (sizeof(typename Ty::T) == 2)
    if (e == 8) return run_rope<Ty, 8>(layout, a, st);
  return e == 4 ? run_rope<Ty, 4>(layout, a, st) : e == 2 ? run_rope<Ty, 2>(layout, a, st) : run_rope<Ty, 1>(layout, a, st);
}
hipError_t launch_rope(int dt, int layout, const RopeArgs& a, hipStream_t st) {
  ProfScope p(kKRope, st);
  if (dt == LX_F32) return by_run<F32Type>(layout, a, st);
  return dt == LX_F16 ? by_run<F16Type>(layout, a, st) : by_run<Bf16Type>(layout, a, st);
}
hipError_t launch_rope_table(int rot, int n_pos, double base, int kind, double factor, double trained, double low, double high, double gain,
                             float* table, hipStream_t st) {
  ProfScope p(kKRope, st);
  const long long n = (long long)n_pos * (rot / 2);
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + kRopeThreads - 1) / kRopeThreads)), dim3(kRopeThreads), 0, st, rot, n_pos, base, kind,
                     factor, trained, low, high, gain, table);
  return hipGetLastError();
}

}  // namespace lx
