// Which kernel a forward call of attention with rules on its scores takes (csrc/score_plan.h), as C functions.
#include "../paper_2510_15964_amd/csrc/score_plan.h"

extern "C" {
int route(int B, int Hq, int Hkv, int Sq, int Sk) { return lx::score_route(B, Hq, Hkv, Sq, Sk); }
long long threads_by_pairs(int B, int Hq, int Hkv, int Sq) { return lx::token_pairs(B, Hq, Hkv, Sq) * lx::kTokenWaves * 64; }
}
