// Tensor maps of byte matrices.
#pragma once

#include <cuda.h>

namespace eat {

// [planes][rows][cols] bytes (cols a multiple of 16), in boxes of box_rows rows of 128 bytes of one plane,
// 128-byte swizzle, zeros outside.  rank: 3, or 2 for a matrix of one plane; the copies through a map have
// as many coordinates as its rank (any other number is an illegal instruction).
bool encode_bytes(CUtensorMap* m, int rank, const void* ptr, long long cols, long long rows,
                  long long planes, int box_rows);

}  // namespace eat
