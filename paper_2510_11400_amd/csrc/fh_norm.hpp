// What layer norm and the quantiser that follows it share: the row's statistics applied to one value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fedhybrid.h"
#include "fh_mx.hpp"

namespace fh {

// y of one value, x less the mean, in this order everywhere, so that a row's and a column's stored form of a norm's output come
// from the same bits.
__device__ __forceinline__ float norm_value(float d, float rstd, float w, float b) { return __builtin_fmaf(d * rstd, w, b); }

// A norm ahead of the quantiser; weight and bias may be null (1 and 0).
struct NormArgs {
    const void*  weight;
    const void*  bias;
    int32_t      p_dtype;
    float        eps;
    float*       mean;
    float*       rstd;
};
__device__ __forceinline__ float parameter(const void* p, int32_t dtype, int64_t i, float otherwise)
{
    if (!p) return otherwise;
    return dtype == FH_F32 ? static_cast<const float*>(p)[i] : value(static_cast<const Bf16*>(p)[i]);
}

// Layer norm of rows to y (dense), to `codes` (by rows), or the statistics alone where both are null.
hipError_t launch_layer_norm(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t x_stride, const NormArgs& n,
                             void* y, int64_t y_stride, void* codes, hipStream_t s);
// Layer norm to codes by columns, and by rows too where by_rows is not null, in one pass over rows that fit.
bool norm_blocks_fit(int32_t dtype, int64_t rows, int64_t cols);
hipError_t launch_norm_blocks(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t x_stride, const NormArgs& n, void* by_rows,
                              void* by_columns, hipStream_t s);
// The quantiser over tiles of 256 rows, with or without a norm whose statistics are known; either form may be null.  `sums` (without a
// norm): mx_tile_rows(rows) rows of partial sums of x's columns, or null.
inline int64_t mx_tile_rows(int64_t rows) { return (rows + 255) / 256; }
hipError_t launch_mx_tiles(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t x_stride, const NormArgs* n, float* sums,
                           bool stochastic, uint64_t seed, uint64_t tensor_id, void* by_rows, void* by_columns, hipStream_t s);
// Rows of partial sums added up: row i's k-th of `count` vectors begins at partial + (i * count + k) * cols, their sums go to
// first (k = 0) and second (k = 1), of p_dtype; either may be null.
hipError_t launch_join(const float* partial, int64_t parts, int64_t cols, int32_t count, int32_t p_dtype, void* first, void* second, hipStream_t s);

// fh_layer_norm_backward with a dy of its own type: b.dtype or FH_F32.
fh_status norm_backward(const fh_norm_backward& b, int32_t dy_dtype, hipStream_t s);

// The host's checks of a matrix in rows: `elements` from its pointer on are read or written.
inline bool is_aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool is_dtype(int d) { return d == FH_F32 || d == FH_BF16; }
inline size_t dtype_size(int d) { return d == FH_F32 ? 4u : 2u; }
inline uint64_t strided_elements(int64_t rows, int64_t cols, int64_t stride)
{
    return rows > 0 && cols > 0 ? (uint64_t)(rows - 1) * (uint64_t)stride + (uint64_t)cols : 0u;
}
constexpr int64_t kMostStride = (int64_t)1 << 31;

}  // namespace fh
