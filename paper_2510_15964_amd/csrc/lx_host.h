// Host helpers of the C-ABI files.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <cstdio>
#include <cstdlib>

#include "../../include/lx.h"
#include "lx_launch.h"   // kBf16 / kF16

namespace lx {

// LX_LOG=1: one line per call on stderr (read once; any other value: silent)
inline bool log_on() {
  static const bool on = [] {
    const char* v = std::getenv("LX_LOG");
    return v && v[0] == '1';
  }();
  return on;
}
#define LX_LOGF(...)                          \
  do {                                        \
    if (log_on()) {                           \
      std::fprintf(stderr, "[lx] " __VA_ARGS__); \
      std::fputc('\n', stderr);               \
    }                                         \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t esize(lx_dtype dt) { return dt == LX_F32 ? 4 : 2; }
inline bool is16(lx_dtype dt) { return dt == LX_BF16 || dt == LX_F16; }
inline int dt16(lx_dtype dt) { return dt == LX_F16 ? kF16 : kBf16; }   // element type of the 16-bit kernels

}  // namespace lx
