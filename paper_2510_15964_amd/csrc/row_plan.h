// Runs of eight elements of a row, and how many workgroups dropout takes for them.  Plain C++ for host and device.
#pragma once
#include "ffn_plan.h"

namespace lx {

// (d up to 2^31 - 1, whose sum with 7 is no int)
LX_HD unsigned row_runs(int d) { return ((unsigned)d + 7) / 8; }
// Workgroups of 256 threads, a run to a thread, each of which takes several where there are more than `most`.
inline int dropout_grid(int T, int d, int most) {
  const unsigned long long wgs = ((unsigned long long)T * row_runs(d) + 255) / 256;
  return wgs < (unsigned long long)most ? (int)wgs : most;
}

}  // namespace lx
