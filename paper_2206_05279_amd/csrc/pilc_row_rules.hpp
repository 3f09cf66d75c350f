// How rows are counted where a workgroup goes from row to row.  Code that needs no HIP header.  There may be up to 2^32 - 1 rows: a
// sum of a row's number and a step does not always fit.
#pragma once
#include <cstdint>

namespace pilc {

// The next of a workgroup's rows, `step` further on; false, and `row` as it is, where there is none up to `last`.
constexpr bool next_row(uint32_t &row, uint32_t step, uint32_t last)
{
    if (last - row < step) return false;
    row += step;
    return true;
}

constexpr uint32_t div_up(uint32_t a, uint32_t b) { return a / b + (a % b != 0); }

}  // namespace pilc
