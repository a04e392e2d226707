// Rows of elements in runs of eight, and the counter-based generator of dropout.
#pragma once
#include <type_traits>

#include "lx_dev.h"

namespace lx {

constexpr int kSingle = 2;      // DT of float elements, beside kBf16 and kF16

template <int DT>
using ElemT = std::conditional_t<DT == kSingle, float, uint16_t>;

// A run: eight consecutive elements of a row as floats.  VEC: whole runs at multiples of 16 bytes; otherwise at any address of an element,
// whole ones in as wide accesses as the others, `n` elements of a row's last one one by one, the others zero.
struct Run {
  float v[8];
};
// ... and as they lie in memory, which takes half the registers in 16 bits.
template <int DT>
struct Raw {
  u32x4 w[DT == kSingle ? 2 : 1];
};
struct __attribute__((packed, aligned(2))) Loose16 {
  u32x4 w;
};
template <int DT, bool VEC>
__device__ __forceinline__ Raw<DT> load_raw(const ElemT<DT>* p, int n) {
  Raw<DT> r;
  if (VEC || n >= 8) {
#pragma unroll
    for (int i = 0; i < (DT == kSingle ? 2 : 1); ++i) {
      if constexpr (VEC) r.w[i] = reinterpret_cast<const u32x4*>(p)[i];
      else r.w[i] = reinterpret_cast<const Loose16*>(p)[i].w;
    }
  } else if constexpr (DT == kSingle) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i / 4][i % 4] = i < n ? __builtin_bit_cast(uint32_t, p[i]) : 0u;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[0][i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  }
  return r;
}
template <int DT>
__device__ __forceinline__ Run open(const Raw<DT>& u) {
  Run r;
  if constexpr (DT == kSingle) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = __builtin_bit_cast(float, (uint32_t)u.w[i / 4][i % 4]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[2 * i] = to_f32<DT>(u.w[0][i] & 0xffff), r.v[2 * i + 1] = to_f32<DT>(u.w[0][i] >> 16);
  }
  return r;
}
template <int DT, bool VEC>
__device__ __forceinline__ Run load_run(const ElemT<DT>* p, int n) {
  return open<DT>(load_raw<DT, VEC>(p, n));
}
template <int DT, bool VEC>
__device__ __forceinline__ void store_run(ElemT<DT>* p, const Run& r, int n) {
  Raw<DT> u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == kSingle) {
      u.w[0][i] = __builtin_bit_cast(uint32_t, r.v[i]);
      u.w[1][i] = __builtin_bit_cast(uint32_t, r.v[4 + i]);
    } else {
      u.w[0][i] = pack2<DT>(r.v[2 * i], r.v[2 * i + 1]);
    }
  }
  if (VEC || n >= 8) {
#pragma unroll
    for (int i = 0; i < (DT == kSingle ? 2 : 1); ++i) {
      if constexpr (VEC) reinterpret_cast<u32x4*>(p)[i] = u.w[i];
      else reinterpret_cast<Loose16*>(p)[i].w = u.w[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i >= n) continue;
      if constexpr (DT == kSingle) p[i] = r.v[i];
      else p[i] = (uint16_t)(u.w[0][i / 2] >> 16 * (i % 2));
    }
  }
}

// Dropout's numbers: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011).  A call yields 128 bits, sixteen for each element of a run: a share of 2^-16 is as fine as a training run needs, and one call
// for 16 bytes in and 16 out stays hidden behind them.
struct Drop {
  uint32_t key0, key1, site, step;
  uint32_t below;     // dropped where the number is below this; 0: none is
  float factor;       // of what is kept
  __device__ __forceinline__ void numbers(unsigned long long run, uint32_t (&w)[4]) const {
    uint32_t x0 = (uint32_t)run, x1 = (uint32_t)(run >> 32), x2 = site, x3 = step, k0 = key0, k1 = key1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t a = (uint64_t)0xD2511F53u * x0, b = (uint64_t)0xCD9E8D57u * x2;
      const uint32_t y0 = (uint32_t)(b >> 32) ^ x1 ^ k0, y2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
      x1 = (uint32_t)b, x3 = (uint32_t)a, x0 = y0, x2 = y2;
      k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    w[0] = x0, w[1] = x1, w[2] = x2, w[3] = x3;
  }
  // What a dropped element holds has no effect.
  __device__ __forceinline__ void apply(Run& r, unsigned long long run) const {
    uint32_t w[4];
    numbers(run, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
      r.v[i] = u < below ? 0.f : r.v[i] * factor;
    }
  }
};
// {seed, step} lie on the device, so that a captured graph can advance them.
__device__ __forceinline__ Drop load_drop(const DropArgs& a) {
  Drop d = {0, 0, (uint32_t)a.site, 0, a.below, a.factor};
  if (a.below) {
    const unsigned long long seed = (unsigned long long)a.rng[0];
    d.key0 = (uint32_t)seed, d.key1 = (uint32_t)(seed >> 32), d.step = (uint32_t)a.rng[1];
  }
  return d;
}

}  // namespace lx
