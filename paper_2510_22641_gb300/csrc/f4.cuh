// 4-bit floats with a scale per 16 columns and one per row: the byte order of packed rows.
#pragma once

#include "lowbit.cuh"

namespace ssd {

// A record is 128 rows x 256 columns.  Codes: 128 bytes a row, a column's code in the low nibble of its byte where the
// column is even, the row's eight 16-byte units in the order of the 128-byte swizzle (unit ^ row % 8), so that a copy
// of the bytes is an operand of tcgen05.mma.  Scales: e4m3, 512 bytes per 64 columns, row r's four at
// (r % 32) * 16 + r / 32 * 4: 32 lanes of four words, as tensor memory holds the scales of 128 rows.
constexpr int kF4Rows = 128, kF4Cols = 256, kF4Group = 16;
constexpr int kF4CodeBytes = kF4Rows * kF4Cols / 2, kF4Record = kF4CodeBytes + kF4Rows * kF4Cols / kF4Group;

__host__ __device__ __forceinline__ int f4_chunks(int k) { return (k + kF4Cols - 1) / kF4Cols; }
__host__ __device__ __forceinline__ int64_t f4_scales_at(int rows, int k) {  // byte of the row scales
  return static_cast<int64_t>((rows + kF4Rows - 1) / kF4Rows) * f4_chunks(k) * kF4Record;
}
// Byte of 16 columns' codes (8 bytes' aligned half of a unit) and of a group's scale in a record.
__host__ __device__ __forceinline__ int f4_code_byte(int row, int col) {
  return row * 128 + (((col >> 5) ^ (row & 7)) << 4) + (col >> 1 & 15);
}
__host__ __device__ __forceinline__ int f4_scale_byte(int row, int col) {
  return kF4CodeBytes + (col >> 6) * 512 + (row & 31) * 16 + (row >> 5) * 4 + (col >> 4 & 3);
}

ssd_status f4_check_shape(int rows, int k);
ssd_status f4_pack_rows(const char* what, const void* x, int type, int rows, int k, int64_t x_row, void* packed,
                        cudaStream_t s);

}  // namespace ssd
