// The loss over a vocabulary: launches, shared by the host code (lx_block_api.hip), vocab.hip and vocab_plain.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vocab_plan.h"

namespace lx {

struct VocabArgs {
  int T, d, V, dt;                // dt: kBf16 or kF16
  const uint16_t* X;
  long long xs;
  const uint16_t* W;              // [V, d] contiguous
  const int* targets;
  const float* weights;           // may be null
  float *loss, *lse;              // lse may be null
  uint16_t* dX;                   // may be null
  long long dxs;
  void* dW;                       // may be null
  int dw_f32;
};

// ... in single precision (vocab_plain.hip)
struct PlainVocabArgs {
  int T, d, V;
  const float* X;
  long long xs;
  const float* W;
  const int* targets;
  const float* weights;
  float *loss, *lse, *dX;
  long long dxs;
  float* dW;
};

// One piece after the other on the stream; `ws` holds room's bytes.
hipError_t launch_vocab_loss(const VocabArgs& a, const VocabRoom& room, void* ws, hipStream_t st);
hipError_t launch_vocab_loss_plain(const PlainVocabArgs& a, const VocabRoom& room, void* ws, hipStream_t st);

}  // namespace lx
