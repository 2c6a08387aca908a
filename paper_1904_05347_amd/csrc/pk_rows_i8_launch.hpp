// pk_rows_i8_launch.hpp -- how the rows of one launch of the 8-bit row kernels
// are laid over work-groups.  Plain integer arithmetic, which the CPU tests
// evaluate too.
#pragma once

#include <stdint.h>

namespace pk {

// Rows of one launch: with the most work-items a row, 1024, its grid has 2^31,
// and a launch takes fewer than 2^32.
constexpr int64_t kMostRows = 1 << 21;

// Work-items of a work-group whose rows have `team` (64, 256, 512 or 1024) each,
// and the work-groups of that many rows.
constexpr int rows_group(int team) { return team < 256 ? 256 : team; }
constexpr int64_t rows_groups(int64_t rows, int team)
{
    const int a_group = rows_group(team) / team;
    return (rows + a_group - 1) / a_group;
}

}  // namespace pk
