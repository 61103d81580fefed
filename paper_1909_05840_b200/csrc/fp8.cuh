// Layout of the scales of 8-bit floating point codes, shared by the quantizers that write them and the product that reads them, and what
// the quantizers read of rows of any alignment.
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

// Rows that do not begin at a multiple of four elements are read by the aligned quads that have something of them.  Of a segment of
// `width` columns from element `base` of x on, the off-th of its aligned quad, lane l takes the quads at base + at(l) while at(l) <
// left (what the row has from base on); one lane takes the quad behind the segment, which its last columns need where off is not 0.
__host__ __device__ __forceinline__ int fp8_quad_at(int j, int lane, int off) { return j * 128 + lane * 4 - off; }
__host__ __device__ __forceinline__ bool fp8_needs_behind(int width, int off, int left) { return off != 0 && width - off < left; }
// May such a quad of the segments at base .. last_base have elements that lie before x or behind its n?  Those segments are read element by
// element.
__host__ __device__ __forceinline__ bool fp8_at_edge(int64_t base, int64_t last_base, int left, int width, int64_t n) {
  return base < 4 || n - last_base < (left < width ? left : width) + 4;
}

}  // namespace qb
