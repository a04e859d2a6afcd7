// Offsets of the linear layer's stores: the arithmetic that keeps them in the output, shared by the
// kernel and the host's check of it.
#pragma once
#include <stdint.h>

namespace cham {

// Scalar offset of the row `row` rows behind a lane's first one, in a tile of `records` bytes.  The
// range check compares the lane's offset with `records` less this one, in 32 bits: it stops at
// `records`, where every lane is dropped, else the difference would wrap in a tile of few rows.
__host__ __device__ inline uint32_t row_offset(uint32_t row, uint32_t row_bytes, uint32_t records) {
    return row * row_bytes < records ? row * row_bytes : records;
}

}  // namespace cham
