// Microscaled 4-bit storage: quantisation by rows, by columns or both, and its inverse.
#include "fh_norm.hpp"

namespace fh {
namespace {

constexpr int kThreads = 256;

// ---- by rows, nearest: 8 values a lane, one row's chunk of 256 for half a wave ------------
// Bound by the read: 2 or 4 bytes in, 17/32 out a value.
template <typename T>
__global__ __launch_bounds__(kThreads) void mx_rows_kernel(const T* x, int64_t rows, int64_t cols, int64_t stride, MxStore to, int64_t units)
{
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const bool write = unit < units;
    const int64_t row = write ? unit / to.chunks : 0, chunk = write ? unit - row * to.chunks : 0;
    const int64_t first = chunk * kMxChunk + (threadIdx.x & 31) * 8;
    float v[8];
    load8(x + row * stride + first, cols - first, v);
    mx_write8(to, row, first, v, write);
}

// ---- tiles: blocks along the columns, along the rows, or both ------------------------------
// A wave holds 32 rows x 128 columns, a lane two columns of all 32 rows: a column's block is the lane's own registers, a
// row's block the 16 lanes of a DPP row.  Eight waves make 256 rows, so that the codes of a column, gathered in LDS, leave
// as whole lines of 128 bytes.  The random bits of eight rows of a column are one Philox block, which the lane computes for
// itself whatever the tensor's width.
__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

constexpr int kTileRows = 256, kTileCols = 128, kTileThreads = 512;

template <typename T, bool NORM, bool STOCHASTIC>
__global__ __launch_bounds__(kTileThreads) void mx_tiles_kernel(const T* x, int64_t rows, int64_t cols, int64_t stride, NormArgs n,
                                                                uint32_t k0, uint32_t k1, uint32_t id0, uint32_t id1,
                                                                MxStore by_rows, MxStore by_columns, uint32_t col_tiles)
{
    __shared__ u32x4 s_codes[kTileCols * 8];
    __shared__ uint32_t s_scales[kTileCols * 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col_tile = blockIdx.x % col_tiles, row_tile = blockIdx.x / col_tiles;
    const int64_t r0 = row_tile * kTileRows + wave * 32;
    const int64_t c0 = col_tile * kTileCols + lane * 2;
    const bool in0 = c0 < cols, in1 = c0 + 1 < cols;

    float v0[32], v1[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v0[i] = v1[i] = 0.0f;
        if (r0 + i < rows) {                                     // uniform
            const T* p = x + (r0 + i) * stride + c0;
            if (in1) {
                if constexpr (sizeof(T) == 4) {
                    const f32x2 w = *reinterpret_cast<const f32x2_a4*>(p);
                    v0[i] = w.x; v1[i] = w.y;
                } else {
                    const uint32_t w = *reinterpret_cast<const u32_a2*>(p);
                    v0[i] = bf16_lo(w); v1[i] = bf16_hi(w);
                }
            } else if (in0) v0[i] = value(*p);
        }
    }
    if constexpr (NORM) {
        const float w0 = in0 ? parameter(n.weight, n.p_dtype, c0, 1.0f) : 0.0f, b0 = in0 ? parameter(n.bias, n.p_dtype, c0, 0.0f) : 0.0f;
        const float w1 = in1 ? parameter(n.weight, n.p_dtype, c0 + 1, 1.0f) : 0.0f, b1 = in1 ? parameter(n.bias, n.p_dtype, c0 + 1, 0.0f) : 0.0f;
        // lane i of the wave fetches row i's statistics; rows past the last stay zeros, whatever the bias
        const int64_t mine = r0 + (lane & 31);
        const float means = mine < rows ? n.mean[mine] : 0.0f, rstds = mine < rows ? n.rstd[mine] : 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float mean = lane_value(means, i), rstd = lane_value(rstds, i);
            const bool row_in = r0 + i < rows;
            v0[i] = row_in && in0 ? norm_value(v0[i], mean, rstd, w0, b0) : 0.0f;
            v1[i] = row_in && in1 ? norm_value(v1[i], mean, rstd, w1, b1) : 0.0f;
        }
    }
    // 65535 - h of row 8g + i: half-word i of not_h[.][g]
    u32x4 not_h0[4], not_h1[4];
    if constexpr (STOCHASTIC) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint64_t at = (uint64_t)((r0 >> 3) + g) * (uint64_t)cols + (uint64_t)c0;
            not_h0[g] = philox4x32_10_complement((uint32_t)at, (uint32_t)(at >> 32), id0, id1, k0, k1);
            const uint64_t bt = at + 1;
            not_h1[g] = philox4x32_10_complement((uint32_t)bt, (uint32_t)(bt >> 32), id0, id1, k0, k1);
        }
    }
    auto half = [](const u32x4 (&w)[4], int i) -> uint32_t {
        const uint32_t word = w[i >> 3][(i & 7) >> 1];
        return i & 1 ? word >> 16 : word & 0xFFFFu;
    };

    if (by_columns.codes) {
        uint32_t t0 = 0, t1 = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) { t0 = umax(t0, abs_bits(v0[i])); t1 = umax(t1, abs_bits(v1[i])); }
        const uint32_t s0 = mx_scale_byte(t0), s1 = mx_scale_byte(t1);
        u32x4 q0, q1;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t a = 0, b = 0;
            if constexpr (STOCHASTIC) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a |= mx_stochastic(v0[8 * w + i], s0, half(not_h0, 8 * w + i)) << (4 * i);
                    b |= mx_stochastic(v1[8 * w + i], s1, half(not_h1, 8 * w + i)) << (4 * i);
                }
            } else {
                a = mx_nearest<0>(a, v0[8 * w], v0[8 * w + 1], s0);
                a = mx_nearest<1>(a, v0[8 * w + 2], v0[8 * w + 3], s0);
                a = mx_nearest<2>(a, v0[8 * w + 4], v0[8 * w + 5], s0);
                a = mx_nearest<3>(a, v0[8 * w + 6], v0[8 * w + 7], s0);
                b = mx_nearest<0>(b, v1[8 * w], v1[8 * w + 1], s1);
                b = mx_nearest<1>(b, v1[8 * w + 2], v1[8 * w + 3], s1);
                b = mx_nearest<2>(b, v1[8 * w + 4], v1[8 * w + 5], s1);
                b = mx_nearest<3>(b, v1[8 * w + 6], v1[8 * w + 7], s1);
            }
            q0[w] = s0 == 255u ? 0u : a;
            q1[w] = s1 == 255u ? 0u : b;
        }
        // a column's eight pieces are turned by the column pair, so that the lanes' writes meet all banks
        const int turned = wave ^ (lane & 7);
        s_codes[(2 * lane) * 8 + turned] = q0;
        s_codes[(2 * lane + 1) * 8 + turned] = q1;
        // [column/32][wave/4][column%32][wave%4], as the stored form has it
        uint8_t* bytes = reinterpret_cast<uint8_t*>(s_scales);
        const int at = (lane >> 4) * 256 + (wave >> 2) * 128 + (wave & 3);
        bytes[at + ((2 * lane) & 31) * 4] = (uint8_t)s0;
        bytes[at + ((2 * lane + 1) & 31) * 4] = (uint8_t)s1;
        __syncthreads();
        const int64_t first = col_tile * kTileCols;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = threadIdx.x + i * kTileThreads, c = id >> 3, piece = id & 7;
            if (first + c < by_columns.rows)
                *reinterpret_cast<u32x4*>(by_columns.codes + (first + c) * (by_columns.chunks * 128) + row_tile * 128 + piece * 16) =
                    s_codes[c * 8 + (piece ^ ((c >> 1) & 7))];
        }
        if (threadIdx.x < 256) {
            const int64_t group = (first >> 5) + (threadIdx.x >> 6);
            if (group * 32 < by_columns.rows)
                *reinterpret_cast<uint32_t*>(by_columns.scales + ((group * by_columns.chunks + row_tile) << 8) + (threadIdx.x & 63) * 4) =
                    s_scales[threadIdx.x];
        }
    }

    if (by_rows.codes) {
        const int quad = lane & 3;
        const uint32_t pick1 = lane & 1 ? 0x03070105u : 0x06020400u;      // {b1,a1,b3,a3} : {a0,b0,a2,b2}, b the neighbour's
        const uint32_t pick2 = lane & 2 ? 0x03020706u : 0x05040100u;
        uint32_t kept0 = 1, kept1 = 1;                                    // scales of rows lane%16 and 16 + lane%16
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            uint32_t word = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t s = mx_scale_byte(row_max(umax(abs_bits(v0[i + k]), abs_bits(v1[i + k]))));
                uint32_t byte;
                if constexpr (STOCHASTIC)
                    byte = mx_stochastic(v0[i + k], s, half(not_h0, i + k)) | mx_stochastic(v1[i + k], s, half(not_h1, i + k)) << 4;
                else
                    byte = mx_nearest<0>(0, v0[i + k], v1[i + k], s) & 0xFFu;
                word |= (s == 255u ? 0u : byte) << (8 * k);
                if (i + k < 16) kept0 = (lane & 15) == i + k ? s : kept0;
                else kept1 = (lane & 15) == i + k - 16 ? s : kept1;
            }
            // four rows' bytes of a column pair to a row's bytes of four column pairs, within each quad of lanes
            word = __builtin_amdgcn_perm(dpp<kQuadXor1>(word), word, pick1);
            word = __builtin_amdgcn_perm(dpp<kQuadXor2>(word), word, pick2);
            const int64_t row = r0 + i + quad;
            if (row < rows)
                *reinterpret_cast<uint32_t*>(by_rows.codes + row * (by_rows.chunks * 128) + col_tile * (kTileCols / 2) + (lane >> 2) * 4) = word;
        }
        const int64_t block = col_tile * 4 + (lane >> 4), row = r0 + (lane & 15);
        if (row < rows) by_rows.scales[mx_scale_at(row, block, by_rows.chunks)] = (uint8_t)kept0;
        if (row + 16 < rows) by_rows.scales[mx_scale_at(row + 16, block, by_rows.chunks)] = (uint8_t)kept1;
    }
}

// ---- back ---------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kThreads) void mx_restore_kernel(MxStore from, int64_t cols, T* out, int64_t stride, int64_t units)
{
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (unit >= units) return;
    const int64_t row = unit / from.chunks, chunk = unit - row * from.chunks;
    const int64_t first = chunk * kMxChunk + (threadIdx.x & 31) * 8;
    if (first >= cols) return;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(from.codes + row * (from.chunks * 128) + (first >> 1));
    const uint32_t s = from.scales[mx_scale_at(row, first >> 5, from.chunks)];
    // byte 0 is 2^-127, byte 255 no number; the product is exact but for numbers over the largest
    const float scale = __builtin_bit_cast(float, s == 0u ? 0x00400000u : s == 255u ? 0x7FC00000u : s << 23);
    float v[8];
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    v[0] = a.x * scale; v[1] = a.y * scale; v[2] = b.x * scale; v[3] = b.y * scale;
    v[4] = c.x * scale; v[5] = c.y * scale; v[6] = d.x * scale; v[7] = d.y * scale;
    store8(out + row * stride + first, cols - first, v);
}

template <typename T>
hipError_t rows_of(const void* x, int64_t rows, int64_t cols, int64_t stride, const MxStore& to, hipStream_t s)
{
    const int64_t units = rows * to.chunks, groups = (units + kThreads / 32 - 1) / (kThreads / 32);
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((mx_rows_kernel<T>), dim3((uint32_t)groups), dim3(kThreads), 0, s, static_cast<const T*>(x), rows, cols, stride, to, units);
    return hipGetLastError();
}

template <typename T, bool NORM, bool STOCHASTIC>
hipError_t tiles_of(const void* x, int64_t rows, int64_t cols, int64_t stride, const NormArgs& n, uint64_t seed, uint64_t id,
                    const MxStore& by_rows, const MxStore& by_columns, hipStream_t s)
{
    // columns up to a whole chunk where rows are stored, rows up to a whole chunk where columns are
    const int64_t col_tiles = by_rows.codes ? 2 * by_rows.chunks : (cols + kTileCols - 1) / kTileCols;
    const int64_t row_tiles = (rows + kTileRows - 1) / kTileRows;
    if (col_tiles * row_tiles > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((mx_tiles_kernel<T, NORM, STOCHASTIC>), dim3((uint32_t)(col_tiles * row_tiles)), dim3(kTileThreads), 0, s,
                       static_cast<const T*>(x), rows, cols, stride, n, (uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)id,
                       (uint32_t)(id >> 32), by_rows, by_columns, (uint32_t)col_tiles);
    return hipGetLastError();
}

template <typename T>
hipError_t restore_of(const MxStore& from, int64_t rows, int64_t cols, void* out, int64_t stride, hipStream_t s)
{
    const int64_t units = rows * from.chunks, groups = (units + kThreads / 32 - 1) / (kThreads / 32);
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((mx_restore_kernel<T>), dim3((uint32_t)groups), dim3(kThreads), 0, s, from, cols, static_cast<T*>(out), stride, units);
    return hipGetLastError();
}

// Where a stored form is wanted: its buffer's checks.
fh_status check_store(const void* p, size_t cap, int64_t rows, int64_t cols)
{
    if (!p) return FH_OK;
    if (!is_aligned(p, 16)) return FH_ERR_ALIGNMENT;
    if (cap < mx_bytes(rows, cols)) return FH_ERR_BUFFER_TOO_SMALL;
    return FH_OK;
}

fh_status check_input(const void* x, int x_dtype, int64_t rows, int64_t cols, int64_t stride, int32_t rounding, const void* by_rows,
                      size_t by_rows_cap, const void* by_columns, size_t by_columns_cap)
{
    if (!is_dtype(x_dtype)) return FH_ERR_BAD_DTYPE;
    if (rounding != FH_ROUND_NEAREST && rounding != FH_ROUND_STOCHASTIC) return FH_ERR_BAD_ROUND;
    if (!mx_shape_ok(rows, cols) || stride < cols || stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (rows == 0 || cols == 0) return FH_OK;
    if (!x || (!by_rows && !by_columns)) return FH_ERR_NULL;
    if (!is_aligned(x, dtype_size(x_dtype))) return FH_ERR_ALIGNMENT;
    const fh_status s = check_store(by_rows, by_rows_cap, rows, cols);
    return s != FH_OK ? s : check_store(by_columns, by_columns_cap, cols, rows);
}

}  // namespace

hipError_t launch_mx_tiles(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, const NormArgs* n, bool stochastic,
                           uint64_t seed, uint64_t id, const MxStore& by_rows, const MxStore& by_columns, hipStream_t s)
{
    const NormArgs none = {};
    if (dtype == FH_F32) {
        if (n) return stochastic ? tiles_of<float, true, true>(x, rows, cols, stride, *n, seed, id, by_rows, by_columns, s)
                                 : tiles_of<float, true, false>(x, rows, cols, stride, *n, seed, id, by_rows, by_columns, s);
        return stochastic ? tiles_of<float, false, true>(x, rows, cols, stride, none, seed, id, by_rows, by_columns, s)
                          : tiles_of<float, false, false>(x, rows, cols, stride, none, seed, id, by_rows, by_columns, s);
    }
    if (n) return stochastic ? tiles_of<Bf16, true, true>(x, rows, cols, stride, *n, seed, id, by_rows, by_columns, s)
                             : tiles_of<Bf16, true, false>(x, rows, cols, stride, *n, seed, id, by_rows, by_columns, s);
    return stochastic ? tiles_of<Bf16, false, true>(x, rows, cols, stride, none, seed, id, by_rows, by_columns, s)
                      : tiles_of<Bf16, false, false>(x, rows, cols, stride, none, seed, id, by_rows, by_columns, s);
}

}  // namespace fh

extern "C" {

size_t fh_mx_bytes(int64_t rows, int64_t cols) { return fh::mx_shape_ok(rows, cols) ? (size_t)fh::mx_bytes(rows, cols) : 0; }

size_t fh_mx_scales_offset(int64_t rows, int64_t cols) { return fh::mx_shape_ok(rows, cols) ? (size_t)fh::mx_codes_bytes(rows, cols) : 0; }

fh_status fh_mx_quantize(const void* x, fh_dtype x_dtype, int64_t rows, int64_t cols, int64_t row_stride, int32_t rounding,
                         uint64_t seed, uint64_t tensor_id, void* by_rows, size_t by_rows_cap, void* by_columns,
                         size_t by_columns_cap, void* stream)
{
    using namespace fh;
    const fh_status st = check_input(x, x_dtype, rows, cols, row_stride, rounding, by_rows, by_rows_cap, by_columns, by_columns_cap);
    if (st != FH_OK || rows == 0 || cols == 0) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const MxStore to = mx_store(by_rows, rows, cols), turned = mx_store(by_columns, cols, rows);
    hipError_t e;
    if (by_columns || rounding == FH_ROUND_STOCHASTIC)
        e = launch_mx_tiles(x, x_dtype, rows, cols, row_stride, nullptr, rounding == FH_ROUND_STOCHASTIC, seed, tensor_id, to, turned, s);
    else
        e = x_dtype == FH_F32 ? rows_of<float>(x, rows, cols, row_stride, to, s) : rows_of<Bf16>(x, rows, cols, row_stride, to, s);
    return e == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

fh_status fh_mx_dequantize(const void* stored, size_t stored_cap, int64_t rows, int64_t cols, fh_dtype out_dtype, void* out,
                           int64_t row_stride, size_t out_cap, void* stream)
{
    using namespace fh;
    if (!is_dtype(out_dtype)) return FH_ERR_BAD_DTYPE;
    if (!mx_shape_ok(rows, cols) || row_stride < cols || row_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (rows == 0 || cols == 0) return FH_OK;
    if (!stored || !out) return FH_ERR_NULL;
    if (!is_aligned(stored, 16) || !is_aligned(out, dtype_size(out_dtype))) return FH_ERR_ALIGNMENT;
    if (stored_cap < mx_bytes(rows, cols) || out_cap < strided_elements(rows, cols, row_stride) * dtype_size(out_dtype))
        return FH_ERR_BUFFER_TOO_SMALL;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const MxStore from = mx_store(const_cast<void*>(stored), rows, cols);
    const hipError_t e = out_dtype == FH_F32 ? restore_of<float>(from, rows, cols, out, row_stride, s)
                                             : restore_of<Bf16>(from, rows, cols, out, row_stride, s);
    return e == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

fh_status fh_layer_norm_mx(const void* x, fh_dtype x_dtype, int64_t rows, int64_t cols, int64_t row_stride, const void* weight,
                           const void* bias, fh_dtype p_dtype, float eps, int32_t rounding, uint64_t seed, uint64_t tensor_id,
                           void* by_rows, size_t by_rows_cap, void* by_columns, size_t by_columns_cap, void* mean, void* rstd, void* stream)
{
    using namespace fh;
    if (!is_dtype(p_dtype)) return FH_ERR_BAD_DTYPE;
    if (!(eps >= 0.0f)) return FH_ERR_BAD_PARAM;
    if (cols < 1) return FH_ERR_BAD_SHAPE;
    const fh_status st = check_input(x, x_dtype, rows, cols, row_stride, rounding, by_rows, by_rows_cap, by_columns, by_columns_cap);
    if (st != FH_OK || rows == 0) return st;
    const bool tiles = by_columns || rounding == FH_ROUND_STOCHASTIC;
    if (tiles && (!mean || !rstd)) return FH_ERR_NULL;
    if (!is_aligned(mean, 4) || !is_aligned(rstd, 4) || (weight && !is_aligned(weight, dtype_size(p_dtype))) ||
        (bias && !is_aligned(bias, dtype_size(p_dtype)))) return FH_ERR_ALIGNMENT;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const MxStore to = mx_store(by_rows, rows, cols), turned = mx_store(by_columns, cols, rows), none = {};
    const NormArgs n = {weight, bias, p_dtype, eps, static_cast<float*>(mean), static_cast<float*>(rstd)};
    if (launch_layer_norm(x, x_dtype, rows, cols, row_stride, n, nullptr, 0, tiles ? none : to, s) != hipSuccess) return FH_ERR_LAUNCH;
    if (!tiles) return FH_OK;
    return launch_mx_tiles(x, x_dtype, rows, cols, row_stride, &n, rounding == FH_ROUND_STOCHASTIC, seed, tensor_id, to, turned, s) == hipSuccess
               ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
