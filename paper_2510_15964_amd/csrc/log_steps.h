// Exponentials exp(y), y <= 0, in 16 bits as numbers of steps of their logarithm.  Plain C++ for host and device.
//
// Half precision has 11 bits for 29 powers of two and nothing below the 40th: of logits that are 28 and more below the largest one nothing
// would be left, although bfloat16 holds their gradients.  A logarithm in equal steps has the same relative error everywhere; in 2^16 steps for all
// that bfloat16 holds, 126 powers of two, it would be 2^-10.6.  So there are two kinds of steps: 1/720 of a power of two down to 2^-79.2, off by 2^-11.02
// at most, as half precision is, and below four times that, off by 2^-9.02.  What is below 2^-126.5 is 0.
#pragma once
#include <math.h>

#include "ffn_plan.h"

namespace lx {

constexpr float kStepTop = 65535.f;                         // of 1
constexpr float kFineSteps = 720.f, kCoarseSteps = 180.f;   // to a power of two
constexpr float kCoarseTop = 22785.f;                       // where the coarse line meets 1: the lines cross at step 8535
// Added to a number below 2^23 it leaves that number's nearest whole one in the lowest bits.
constexpr float kWhole = 8388608.f;

// The step of exp(y) as the lowest 16 bits of a float's.  NaN: any step.
LX_HD float log_step(float y) {
  constexpr float kLog2e = 1.4426950408889634f;
  return fmaxf(fmaxf(fmaf(y, kFineSteps * kLog2e, kWhole + kStepTop), fmaf(y, kCoarseSteps * kLog2e, kWhole + kCoarseTop)), kWhole);
}
// The power of two that step s stands for; 0 stands for 0.
LX_HD float step_log2(unsigned s) {
  const float f = (float)s;
  return s == 0 ? -INFINITY : fminf((f - kStepTop) * (1.f / kFineSteps), (f - kCoarseTop) * (1.f / kCoarseSteps));
}

}  // namespace lx
