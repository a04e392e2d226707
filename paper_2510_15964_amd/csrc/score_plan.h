// Which kernel a forward call of attention with rules on its scores takes.  Plain C++, without the device's headers.
#pragma once
#include "lx_chip.h"

namespace lx {

constexpr int kTileRows = 64;                   // rows of a streamed tile, by rows
constexpr int kTokenRows = 32, kTokenKeys = 32;
constexpr int kTokenStep = 4 * kTokenKeys;      // a unit
constexpr int kTokenWaves = 8;                  // wavefronts of a workgroup, one workgroup per CU
constexpr long long kMostPairs = ((1ll << 32) - 1) / (64 * kTokenWaves);      // a workgroup each: a launch counts its threads in 32 bits

// By rows with more than 16 queries (a tile of 32 rows then reads the keys once for few heads), up to one tile of keys, and with more
// pairs than a launch by pairs may have.  By pairs / by parts, us, one query, lengths equal: 1024 keys, D = 64, 1 pair 7.9 / 10.4, 128
// pairs 8.9 / 13.2, 512 pairs 25 / 29; 4096 keys 18 / 11, 23 / 30, 94 / 101; 16384 keys 62 / 12, 118 / 105, 365 / 395; D = 128, 1024 keys
// 10.6 / 12, 14.4 / 19, 43 / 49; 4096 keys 39 / 12, 40 / 50, 190 / 192; 256 pairs of 16384 keys 376 / 381.  With lengths from a tenth up
// whole pairs are up to 45 % faster below 4096 keys and up to 20 % slower above (D = 64, 512 pairs of 16384 251 / 228; 128 94 / 68).
enum ScoreRoute { kByRows, kByPairs, kByParts };
inline long long token_pairs(int B, int Hq, int Hkv, int Sq) {
  return (long long)B * Hkv * ((Hq / Hkv * (long long)Sq + kTokenRows - 1) / kTokenRows);
}
inline ScoreRoute score_route(int B, int Hq, int Hkv, int Sq, int Sk) {
  if (Sq > 16 || Sk <= kTileRows) return kByRows;
  const long long pairs = token_pairs(B, Hq, Hkv, Sq);
  if (pairs > kMostPairs) return kByRows;
  // (units are counted in 32 bits)
  if (pairs * (Sk / kTokenStep + 1) > 0x7fffffff) return kByPairs;
  return Sk <= 1024 || pairs >= kCUs || (pairs >= kCUs / 2 && Sk <= 4096) ? kByPairs : kByParts;
}

}  // namespace lx
