// Layout of the operands of the 8-bit matrix product, shared by the quantiser and the product.
//
// Codes: row major, rows of `cols` bytes padded with zero codes to a multiple of 16.
// Scales: E8M0 bytes (2^(byte - 127)).  128 rows x 4 blocks (512 columns) are a tile of 512 bytes,
// in the order in which the tensor cores' scale memory takes them: byte
//     16 (row mod 32) + 4 ((row mod 128) / 32) + (block mod 4)
// of tile (row / 128, block / 4); the tiles of 128 rows follow one another along the columns.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace lgn {

constexpr uint64_t kFp8MaxDim = 1ull << 30;

__host__ __device__ __forceinline__ uint64_t fp8_pitch(uint64_t cols) { return (cols + 15) & ~15ull; }

// Index of the 32-bit word with the scales of blocks 4 grp .. 4 grp + 3 of a row.
__host__ __device__ __forceinline__ uint64_t fp8_scale_word(uint32_t row, uint32_t grp, uint32_t groups) {
    return ((uint64_t)(row >> 7) * groups + grp) * 128 + (row & 31) * 4 + ((row >> 5) & 3);
}

}  // namespace lgn
