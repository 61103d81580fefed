// Layout of the scales of 8-bit floating point codes, shared by the quantizers that write them and the product that reads them.
#pragma once

#include <stdint.h>

namespace qb {

// Codes [R][Kp] (Kp a multiple of 128), one byte per row and block of 128 along K.  Four consecutive blocks of a row are one
// 32-bit word, the words of 128 rows lie in the order in which tensor memory takes them (512 bytes that one copy
// instruction moves: word of row r at 16 * (r % 32) + 4 * (r % 128 / 32)), these pieces along K first.
__host__ __device__ __forceinline__ int64_t fp8_scale_words(int64_t Kp) { return (Kp + 511) / 512; }
__host__ __device__ __forceinline__ int64_t fp8_scale_offset(int64_t row, int64_t block, int64_t words) {
  return ((row >> 7) * words + (block >> 2)) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4 + (block & 3);
}

}  // namespace qb
