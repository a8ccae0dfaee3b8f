// The stored form of a matrix in 8-bit integers.
//
// Every row has one scale; a value is a signed byte times it.  Rows are padded with zeros to whole chunks of 128 bytes, so that
// the products know no tails in the summed dimension and every row begins on a cache line:
//   codes   [rows][chunks * 128] bytes;
//   scales  [rows] floats behind them.
#pragma once

#include "fh_mx.hpp"

namespace fh {

constexpr int kQ8Chunk = 128;
constexpr int64_t kQ8MostSummed = ((int64_t)1 << 17) - 1;       // (-128)^2 times as many stay below 2^31

inline __host__ __device__ int64_t q8_chunks(int64_t cols) { return (cols + kQ8Chunk - 1) / kQ8Chunk; }
inline bool q8_shape_ok(int64_t rows, int64_t cols) { return mx_shape_ok(rows, cols); }
inline uint64_t q8_codes_bytes(int64_t rows, int64_t cols) { return (uint64_t)rows * (uint64_t)q8_chunks(cols) * kQ8Chunk; }
inline uint64_t q8_bytes(int64_t rows, int64_t cols) { return cols > 0 ? q8_codes_bytes(rows, cols) + (uint64_t)rows * 4u : 0u; }

}  // namespace fh
