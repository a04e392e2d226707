// Runs and workgroups of the calls over rows (csrc/row_plan.h), as C functions.
#include "../paper_2510_15964_amd/csrc/row_plan.h"

extern "C" {
unsigned runs(int d) { return lx::row_runs(d); }
int grid(int T, int d, int most) { return lx::dropout_grid(T, d, most); }
}
