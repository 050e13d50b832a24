// How far a product's loads may reach into a matrix.  Plain arithmetic: the host compiles
// it too.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rmm {

// Bytes from the first element of a matrix of `rows` rows of `cols` bf16, ld elements
// apart, to the end of its last row (vec: of the 16 bytes that hold it; base and ld are
// then multiples of 16 bytes).  A tile's columns past the last one read what follows
// them, the next row or padding; behind the last row nothing need follow, as where the
// matrix is some columns of a wider one.
__host__ __device__ inline int64_t span_bytes(int64_t rows, int64_t ld, int64_t cols, bool vec = true) {
    return ((rows - 1) * ld + (vec ? (cols + 7) / 8 * 8 : cols)) * 2;
}

}  // namespace rmm
