// Rows of a block of work, in plain C++ (host and device).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define AIF_HD __host__ __device__
#else
#define AIF_HD
#endif

namespace aif {

// Of the rows row0 .. row0 + most - 1 (row0 >= 0, most >= 0) those before `end`: any number that a caller's offsets may hold, so compared before anything is
// subtracted or narrowed.
AIF_HD inline int rows_before(int64_t end, int64_t row0, int most) { return end <= row0 ? 0 : end - row0 < most ? (int)(end - row0) : most; }

}  // namespace aif
