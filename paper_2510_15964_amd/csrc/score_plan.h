// Which kernel a forward call of attention with rules on its scores takes.  Plain C++, without the device's headers.
#pragma once
#include "lx_chip.h"

namespace lx {

constexpr int kTileRows = 64;                   // rows of a streamed tile, by rows
constexpr int kTokenRows = 32, kTokenKeys = 32;
constexpr int kTokenStep = 4 * kTokenKeys;      // a unit
constexpr int kTokenWaves = 8;                  // wavefronts of a workgroup, one workgroup per CU
constexpr long long kMostPairs = ((1ll << 32) - 1) / (64 * kTokenWaves);      // a workgroup each: a launch counts its threads in 32 bits

// By rows with more than 16 queries, up to one tile of keys, and with more pairs than a launch by pairs may have.  By pairs / by parts,
// us, one query, lengths equal: 1024 keys, D = 64, 1 pair 8.4 / 10.6, 128 pairs 9.2 / 12.5, 512 pairs 26 / 29; 4096 keys 21 / 11, 23 / 29,
// 94 / 99; 16384 keys 74 / 12, 102 / 96, 348 / 356; D = 128, 1024 keys 11.6 / 11.9, 15 / 20, 44 / 46; 4096 keys 32 / 13, 41 / 46, 183 /
// 185; 256 pairs of 16384 keys 360 / 366.  With lengths from a tenth up, which the host does not know, whole pairs are up to 50 % faster
// below 4096 keys and up to 10 % slower above (D = 64, 512 pairs of 16384 242 / 221).
// By rows / by parts, D = 128, 8 key heads of 4 query heads: 1 sequence of 32768 keys, 1 to 128 queries 433 - 440; 1 query 29, 16 35, 17 70,
// 64 109, 128 222; 16 sequences of 4096, 16 queries 124 / 106, 17 123 / 148, 64 129 / 548.  Keys are read once for every 32 rows of a
// key head, so that parts lose where rows fill the chip.  The limit of 16 is the number at which they still win for many sequences; one
// sequence would gain up to some hundred queries, for which the rule would have to look at the number of workgroups.
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
