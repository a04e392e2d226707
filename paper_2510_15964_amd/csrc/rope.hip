// Rotary positions and their table.
//
// A thread turns the same E pairs (two runs of E elements, or one of E / 2 pairs) of several heads of one token: the table's
// cosines and sines are read once per token, not once per head, and the loads of the heads do not wait for each other.
// Memory-bound: every element is read and written once, as runs of up to 16 bytes.  4 x 2048 tokens, 32 and 32 heads, D = 128, bf16:
// 268 MB in 61 us with the launch, 4.4 TB/s (a copy 5.1); 16 tokens 5.7, a launch; 3 x 1021, 12 and 12 heads, D = 64, half of it turned,
// pairs side by side, fp32: 9.2.
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

// E elements that lie together: one access of E * sizeof(T) bytes
template <class T, int E>
struct alignas(E * sizeof(T)) Run {
  T v[E];
};

struct RopeGrid {
  int turned, tail;      // runs per token and head: of pairs, and of the elements that stay (0 where in and out are the same)
  int heads_per_wg;
};

template <class Ty, int E, int LAYOUT>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeArgs a, const RopeGrid g) {
  using T = typename Ty::T;
  const unsigned per_token = g.turned + g.tail;
  const unsigned long long i = (unsigned long long)blockIdx.x * kRopeThreads + threadIdx.x;
  const unsigned token = (unsigned)(i / per_token), run = (unsigned)(i % per_token);
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
  if (run >= (unsigned)g.turned) {
    const int c = a.rot + (run - g.turned) * E;
    for (int h = h0; h < h1; ++h) {
      at(h, in, out);
      *(Run<T, E>*)(out + c) = *(const Run<T, E>*)(in + c);
    }
    return;
  }
  const int p = a.positions ? a.positions[token] : s, hr = a.rot / 2;
  constexpr int P = LAYOUT == LX_ROPE_HALF || E == 1 ? E : E / 2;     // pairs
  const int pair0 = run * P;
  float co[P], si[P];
  const bool known = p >= 0 && p < a.n_pos;
  const float* row = a.table + (long long)(known ? p : 0) * a.rot + pair0;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    co[k] = known ? row[k] : __builtin_nanf("");
    si[k] = known ? row[hr + k] : __builtin_nanf("");
    if (a.inverse) si[k] = -si[k];
  }
#pragma unroll 4
  for (int h = h0; h < h1; ++h) {
    at(h, in, out);
    if constexpr (LAYOUT == LX_ROPE_HALF) {
      const Run<T, E> x = *(const Run<T, E>*)(in + pair0), y = *(const Run<T, E>*)(in + hr + pair0);
      Run<T, E> u, w;
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const float fx = Ty::load(x.v[k]), fy = Ty::load(y.v[k]);
        u.v[k] = Ty::store(fx * co[k] - fy * si[k]);
        w.v[k] = Ty::store(fx * si[k] + fy * co[k]);
      }
      *(Run<T, E>*)(out + pair0) = u;
      *(Run<T, E>*)(out + hr + pair0) = w;
    } else if constexpr (E == 1) {       // a pair, element by element
      const float fx = Ty::load(in[2 * pair0]), fy = Ty::load(in[2 * pair0 + 1]);
      out[2 * pair0] = Ty::store(fx * co[0] - fy * si[0]);
      out[2 * pair0 + 1] = Ty::store(fx * si[0] + fy * co[0]);
    } else {
      const Run<T, E> x = *(const Run<T, E>*)(in + 2 * pair0);
      Run<T, E> u;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const float fx = Ty::load(x.v[2 * k]), fy = Ty::load(x.v[2 * k + 1]);
        u.v[2 * k] = Ty::store(fx * co[k] - fy * si[k]);
        u.v[2 * k + 1] = Ty::store(fx * si[k] + fy * co[k]);
      }
      *(Run<T, E>*)(out + 2 * pair0) = u;
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

// Runs as wide as the sizes, the strides and the addresses allow: 16, 8 or 4 bytes, or element by element.
static int run_elements(const RopeArgs& a, int layout, int size) {
  for (int e = 16 / size; e > 1; e /= 2) {
    if (e * size < 4) break;
    bool ok = (layout == LX_ROPE_HALF ? a.rot / 2 : a.rot) % e == 0 && (a.D - a.rot) % e == 0;
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
static void run_rope(int layout, const RopeArgs& a, const RopeGrid& g, hipStream_t st) {
  const int heads = a.t[0].heads + (a.n > 1 ? a.t[1].heads : 0);
  const long long wgs = ((long long)a.B * a.S * (g.turned + g.tail) + kRopeThreads - 1) / kRopeThreads;
  const dim3 grid((unsigned)wgs, (heads + g.heads_per_wg - 1) / g.heads_per_wg);
  if (layout == LX_ROPE_HALF)
    hipLaunchKernelGGL((rope_kernel<Ty, E, LX_ROPE_HALF>), grid, dim3(kRopeThreads), 0, st, a, g);
  else
    hipLaunchKernelGGL((rope_kernel<Ty, E, LX_ROPE_INTERLEAVED>), grid, dim3(kRopeThreads), 0, st, a, g);
}
hipError_t launch_rope(int dt, int layout, const RopeArgs& a, hipStream_t st) {
  ProfScope p(kKRope, st);
  const int size = dt == LX_F32 ? 4 : 2, e = run_elements(a, layout, size);
  bool in_place = true;
  for (int i = 0; i < a.n; ++i) in_place = in_place && a.t[i].in == a.t[i].out;
  RopeGrid g;
  g.turned = layout == LX_ROPE_HALF ? a.rot / 2 / e : e == 1 ? a.rot / 2 : a.rot / e;
  g.tail = in_place ? 0 : (a.D - a.rot) / e;
  const int heads = a.t[0].heads + (a.n > 1 ? a.t[1].heads : 0);
  const long long wgs = ((long long)a.B * a.S * (g.turned + g.tail) + kRopeThreads - 1) / kRopeThreads;
  // as many heads to a thread as leave eight workgroups to a CU: a thread per head reads the table again, one for all leaves CUs idle
  g.heads_per_wg = (int)lora_clamp((int)((long long)heads * wgs / (8 * kCUs)), 8);
  if (dt == LX_F32) {
    if (e == 4) run_rope<F32Type, 4>(layout, a, g, st);
    else if (e == 2) run_rope<F32Type, 2>(layout, a, g, st);
    else run_rope<F32Type, 1>(layout, a, g, st);
  } else if (dt == LX_F16) {
    if (e == 8) run_rope<F16Type, 8>(layout, a, g, st);
    else if (e == 4) run_rope<F16Type, 4>(layout, a, g, st);
    else if (e == 2) run_rope<F16Type, 2>(layout, a, g, st);
    else run_rope<F16Type, 1>(layout, a, g, st);
  } else {
    if (e == 8) run_rope<Bf16Type, 8>(layout, a, g, st);
    else if (e == 4) run_rope<Bf16Type, 4>(layout, a, g, st);
    else if (e == 2) run_rope<Bf16Type, 2>(layout, a, g, st);
    else run_rope<Bf16Type, 1>(layout, a, g, st);
  }
  return hipGetLastError();
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
