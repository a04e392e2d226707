// The loss over a vocabulary: sizes, workspace and launches, shared by the host code (lx_block_api.hip) and vocab.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "lx_chip.h"

namespace lx {

constexpr int kVocabTile = 256;                 // tokens, and rows of the vocabulary, of a workgroup's product
constexpr int kVocabPieceMost = 65536;          // tokens of a piece, each of whose workgroups counts the targets before its own
constexpr size_t kVocabPieceBytes = (size_t)1 << 30;   // of a piece's probabilities, where the library chooses

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

// A piece's part of the workspace, for up to `rows` tokens (a multiple of kVocabTile).
struct VocabRoom {
  size_t head, list, target, weight, at, stats, x, tail, p, part, dw, bytes;
  int rows, units;       // units: columns of statistics per token
  long long ldp;         // elements between rows of the probabilities
};
inline size_t vocab_align(size_t x) { return (x + 255) & ~(size_t)255; }
inline VocabRoom vocab_room(int rows, int T, int d, int V, bool grads, bool dw, bool dw_f32) {
  VocabRoom r = {};
  const size_t tiles = ((size_t)V + kVocabTile - 1) / kVocabTile, n = (size_t)rows;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += vocab_align(bytes);
    return here;
  };
  r.rows = rows;
  r.units = (int)tiles * 4;      // (of 128 or 64 columns)
  r.ldp = (long long)tiles * kVocabTile;
  r.head = take(256);
  r.list = take(n * 4);
  r.target = take(n * 4);
  r.weight = take(n * 4);
  r.at = take(n * 4);
  r.stats = take(n * r.units * 8);
  r.x = take(n * d * 2);
  r.tail = take((size_t)64 * d * 2);
  if (grads) {
    r.p = take(n * r.ldp * 2);
    r.part = take((size_t)kCUs * kVocabTile * kVocabTile * 4);
  }
  if (dw && !dw_f32 && T > rows) r.dw = take((size_t)V * d * 4);
  r.bytes = at;
  return r;
}
// Tokens of a piece: the whole call, or as many as fit kVocabPieceBytes, in pieces of equal length.
inline int vocab_rows(int T, int V, bool grads) {
  const long long row = ((long long)V + kVocabTile - 1) / kVocabTile * (grads ? kVocabTile * 2 : 32);
  long long most = (long long)(kVocabPieceBytes / (size_t)row) / kVocabTile * kVocabTile;
  most = most < kVocabTile ? kVocabTile : most > kVocabPieceMost ? kVocabPieceMost : most;
  const long long pieces = (T + most - 1) / most, even = (T + pieces - 1) / pieces;
  return (int)((even + kVocabTile - 1) / kVocabTile * kVocabTile);
}

// One piece after the other on the stream; `ws` holds room's bytes.
hipError_t launch_vocab_loss(const VocabArgs& a, const VocabRoom& room, void* ws, hipStream_t st);

}  // namespace lx
