// Host entry points over the grid of the 8-bit row kernels
// (pk_rows_i8_launch.hpp) for the CPU tests.
#include "../paper_1904_05347_amd/csrc/pk_rows_i8_launch.hpp"

extern "C" {

int64_t shim_most_rows() { return pk::kMostRows; }
int shim_rows_group(int team) { return pk::rows_group(team); }
int64_t shim_rows_groups(int64_t rows, int team) { return pk::rows_groups(rows, team); }

}  // extern "C"
