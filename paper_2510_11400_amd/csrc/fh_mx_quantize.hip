// Microscaled 4-bit storage: quantisation by rows, by columns or both, and its inverse.
#include <type_traits>

#include "fh_norm.hpp"

namespace fh {
namespace {

constexpr int kThreads = 256;

// ---- by rows, nearest, and back: a chunk of a row is half a wave's, 8 values a lane --------------
// A workgroup takes one chunk of eight (four) rows, the grid is (chunks, rows / 8, and a third dimension where that passes the second's
// limit): no thread divides.  With a division of 64 bits in every thread the kernels, which have little else to do, took a third longer.
// Bound by memory: 2 or 4 bytes a value on the plain side, 17/32 on the stored one.
constexpr int64_t kMostGridY = 65535;
template <int LANES>
__device__ __forceinline__ int64_t row_of_thread() { return ((int64_t)blockIdx.z * kMostGridY + blockIdx.y) * (kThreads / LANES) + threadIdx.x / LANES; }
// part(first row, grid) for all rows, of which a workgroup takes kThreads / lanes.
template <typename F>
hipError_t by_rows_and_chunks(int64_t rows, int64_t chunks, int lanes, F part)
{
    const int64_t each = kThreads / lanes;
    return in_parts((rows + each - 1) / each, chunks * kThreads, [&](int64_t first, int64_t groups) {
        const int64_t z = (groups + kMostGridY - 1) / kMostGridY;
        return part(first * each, dim3((uint32_t)chunks, (uint32_t)(z > 1 ? kMostGridY : groups), (uint32_t)z));
    });
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mx_rows_kernel(const T* x, int64_t rows, int64_t cols, int64_t stride, MxStore to, int64_t first_row)
{
    const int64_t row = first_row + row_of_thread<32>(), first = (int64_t)blockIdx.x * kMxChunk + (threadIdx.x & 31) * 8;
    const bool write = row < rows;
    float v[8];
    load8(x + (write ? row : 0) * stride + first, write ? cols - first : 0, v);
    mx_write8(to, row, first, v, write);
}

// ---- tiles: blocks along the columns, along the rows, or both ------------------------------
// A wave holds 32 rows x 256 bytes.  It reads them by 16 bytes a lane, eight values of a row each, whose blocks are quads
// of lanes, and passes them through LDS to have the 32 values of a column in one lane (two columns in bf16), whose block is
// the lane's own registers: with columns in the lanes from the start a row's block would be 16 lanes wide, which took four
// times the instructions.  Eight waves make 256 rows, so that the codes of a column, gathered in LDS, leave as whole lines
// of 128 bytes.  The random bits of eight rows of a column are one Philox block, computed where the column is and handed to
// the rows through LDS as well.
constexpr int kTileRows = 256 /* mx_tile_rows */, kTileThreads = 512;
constexpr int kWaveBytes = 32 * 256 + 16;          // the 16 turn the waves' areas, so that a gather of all eight meets all banks
template <typename T> constexpr int kTileCols = 256 / (int)sizeof(T);

// A linear layer's bias has the sums of its output gradient's columns for gradient: they come with that gradient's codes, from the lanes
// that hold the columns, a row of partial sums a tile, where a pass of their own read 8192 x 2304 once more.
struct SumArgs { float* sums; uint32_t first_tile; };          // tiles of the launches before
struct TileNormArgs { const void *weight, *bias; const float *mean, *rstd; int32_t p_dtype; uint32_t first_tile; };
template <typename T, bool NORM, bool STOCHASTIC>
__global__ __launch_bounds__(kTileThreads, STOCHASTIC && sizeof(T) == 2 ? 2 : 4) void mx_tiles_kernel(const T* x, int64_t rows, int64_t cols, int64_t stride,
                                                                   std::conditional_t<NORM, TileNormArgs, SumArgs> n,
                                                                   uint32_t k0, uint32_t k1, uint32_t id0, uint32_t id1,
                                                                   uint8_t* rows_form, uint8_t* columns_form, uint32_t col_tiles, uint32_t tiles)
{
    const MxStore by_rows = mx_store(rows_form, rows, cols), by_columns = mx_store(columns_form, cols, rows);
    constexpr int kCols = kTileCols<T>, kLanes = kCols / 8, kAtOnce = 64 / kLanes, kGroups = 32 / kAtOnce, kEach = kCols / 64;
    __shared__ __attribute__((aligned(16))) uint8_t s_area[8 * kWaveBytes];
    __shared__ uint32_t s_scales[kCols * 2];
    __shared__ __attribute__((aligned(16))) uint8_t s_row_scales[8][kCols];                   // a wave's: [row][block]
    __shared__ __attribute__((aligned(16))) f32x2 s_stats[NORM ? 8 : 1][32];   // mean and 1 / deviation of a wave's rows
    __shared__ float s_sums[NORM ? 1 : 8][NORM ? 1 : kCols];                   // of a wave's rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // In fp32 a row's codes leave by 32 bytes a tile, so an XCD takes a run of neighbours, whose parts of a line meet in its L2
    // (8192 x 8192, both forms: 86 -> 71 us); the halves of bf16 lose by it (48 -> 50).
    const uint32_t at = n.first_tile + (sizeof(T) == 4 ? run_of(blockIdx.x, tiles) : blockIdx.x);
    const int64_t col_tile = at % col_tiles, row_tile = at / col_tiles;
    const int64_t r0 = row_tile * kTileRows + wave * 32, c0 = col_tile * kCols;
    const bool whole = r0 + 32 <= rows && c0 + kCols <= cols;
    uint8_t* area = s_area + wave * kWaveBytes;

    // as rows: lane (row % kAtOnce, column / 8)
    const int64_t row_c = c0 + (lane % kLanes) * 8;
    Run<T> run[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int64_t row = r0 + g * kAtOnce + lane / kLanes;
        run[g].load(x + (row < rows ? row : 0) * stride + row_c, row < rows ? cols - row_c : 0);
    }
    if constexpr (NORM) {
        const int64_t row = r0 + (lane & 31) < rows ? r0 + (lane & 31) : rows - 1;
        s_stats[wave][lane & 31] = f32x2{n.mean[row], n.rstd[row]};
        asm volatile("" ::: "memory");
    }
    // 65535 - h of the lane's columns: half-word i of a block is row 8g + i's
    u32x4 not_h[kEach][4];
    if constexpr (STOCHASTIC) {
#pragma unroll
        for (int e = 0; e < kEach; ++e)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint64_t at = (uint64_t)((r0 >> 3) + g) * (uint64_t)cols + (uint64_t)(c0 + lane * kEach + e);
                not_h[e][g] = philox4x32_10_complement((uint32_t)at, (uint32_t)(at >> 32), id0, id1, k0, k1);
            }
    }
    auto half = [&](int e, int i) -> uint32_t {
        const uint32_t word = not_h[e][i >> 3][(i & 7) >> 1];
        return i & 1 ? word >> 16 : word & 0xFFFFu;
    };

    bool by_lane = columns_form != nullptr;                      // the columns are wanted in the lanes
    if constexpr (!NORM) by_lane = by_lane || n.sums;
    if (by_lane) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < Run<T>::kWords; i += 4)
                *reinterpret_cast<u32x4*>(area + (g * kAtOnce + lane / kLanes) * 256 + (lane % kLanes) * (8 * sizeof(T)) + i * 4) =
                    u32x4{run[g].w[i], run[g].w[i + 1], run[g].w[i + 2], run[g].w[i + 3]};
    }
    const auto put = [&](int64_t row, int in_area, uint32_t codes, uint32_t s) {
        if (row < rows && row_c < by_rows.chunks * kMxChunk)
            *reinterpret_cast<uint32_t*>(by_rows.codes + row * (by_rows.chunks * 128) + (row_c >> 1)) = s == 255u ? 0u : codes;
        if ((lane & 3) == 0) s_row_scales[wave][in_area * (kCols / 32) + (lane % kLanes) / 4] = (uint8_t)s;
    };
    // the rows' form, from the registers
    auto write_rows = [&]() {
        if constexpr (STOCHASTIC) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if constexpr (kEach == 2) *reinterpret_cast<uint32_t*>(area + i * 256 + lane * 4) = half(0, i) | half(1, i) << 16;
                else *reinterpret_cast<uint16_t*>(area + i * 128 + lane * 2) = (uint16_t)half(0, i);
            }
            asm volatile("" ::: "memory");
        }
        float w[8], b[8];
        if constexpr (NORM) {
#pragma unroll
            for (int i = 0; i < 8; ++i) { w[i] = 1.0f; b[i] = 0.0f; }
            if (n.p_dtype == FH_F32) {
                if (n.weight) load8(static_cast<const float*>(n.weight) + row_c, cols - row_c, w);
                if (n.bias) load8(static_cast<const float*>(n.bias) + row_c, cols - row_c, b);
            } else {
                if (n.weight) load8(static_cast<const Bf16*>(n.weight) + row_c, cols - row_c, w);
                if (n.bias) load8(static_cast<const Bf16*>(n.bias) + row_c, cols - row_c, b);
            }
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int in_area = g * kAtOnce + lane / kLanes;
            const int64_t row = r0 + in_area;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = run[g].at(i);
            if constexpr (NORM) {
                const f32x2 st = s_stats[wave][in_area];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = norm_value(v[i] - st.x, st.y, w[i], b[i]);
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = row_c + i < cols ? v[i] : 0.0f;
                }
            }
            if constexpr (STOCHASTIC) {
                const u32x4 u = *reinterpret_cast<const u32x4*>(area + in_area * (kCols * 2) + (lane % kLanes) * 16);
                uint32_t top = 0, codes = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = umax(top, abs_bits(v[i]));
                const uint32_t s = mx_scale_byte(quad_max(top));
#pragma unroll
                for (int i = 0; i < 8; ++i) codes |= mx_stochastic(v[i], s, i & 1 ? u[i / 2] >> 16 : u[i / 2] & 0xFFFFu) << (4 * i);
                put(row, in_area, codes, s);
            } else {
                uint32_t s;
                const uint32_t codes = mx_codes8(v, s);
                put(row, in_area, codes, s);
            }
        }
        asm volatile("" ::: "memory");                           // the scales of 32 rows are next to each other in the stored form
        if (lane < 32 && r0 + lane < rows && c0 < by_rows.chunks * kMxChunk) {
            uint8_t* to = by_rows.scales + mx_scale_at(r0 + lane, c0 >> 5, by_rows.chunks);
            if constexpr (kCols == 128) *reinterpret_cast<uint32_t*>(to) = reinterpret_cast<const uint32_t*>(s_row_scales[wave])[lane];
            else *reinterpret_cast<uint16_t*>(to) = reinterpret_cast<const uint16_t*>(s_row_scales[wave])[lane];
        }
    };
    // Random bits are made where the columns are, and reach the rows through the area that the columns leave; without them
    // the rows come first, which frees their registers.
    if (!STOCHASTIC && rows_form) write_rows();
    if (by_lane) {
        asm volatile("" ::: "memory");                           // a wave's own LDS accesses are in order
        u32x4 q[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {                        // one column at a time: both at once do not fit 128 registers
            __builtin_amdgcn_sched_barrier(0);
            const int c = lane * kEach + e;
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(area + i * 256 + lane * 4);
                if constexpr (sizeof(T) == 4) v[i] = __builtin_bit_cast(float, w);
                else v[i] = e ? bf16_hi(w) : bf16_lo(w);
            }
            asm volatile("" ::: "memory");
            if constexpr (NORM) {
                const bool in = c0 + c < cols;
                const float w = in ? parameter(n.weight, n.p_dtype, c0 + c, 1.0f) : 0.0f, b = in ? parameter(n.bias, n.p_dtype, c0 + c, 0.0f) : 0.0f;
#pragma unroll
                for (int i = 0; i < 32; i += 2) {                // two rows' statistics by one read, the same for all lanes
                    const f32x4 st = *reinterpret_cast<const f32x4*>(&s_stats[wave][i]);
                    v[i] = norm_value(v[i] - st.x, st.y, w, b);
                    v[i + 1] = norm_value(v[i + 1] - st.z, st.w, w, b);
                }
                if (!whole) {                                    // zeros stay zeros, whatever the bias
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = in && r0 + i < rows ? v[i] : 0.0f;
                }
            }
            if constexpr (!NORM) {
                if (n.sums) {
                    float sum[4] = {};
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[i & 3] += v[i];
                    s_sums[wave][c] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                }
            }
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) top = umax(top, abs_bits(v[i]));
            const uint32_t s = mx_scale_byte(top);
            if constexpr (STOCHASTIC) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t a = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) a |= mx_stochastic(v[8 * w + i], s, half(e, 8 * w + i)) << (4 * i);
                    q[e][w] = s == 255u ? 0u : a;
                }
            } else {
                q[e] = mx_codes32(v, s);
            }
            // [column/32][wave/4][column%32][wave%4], as the stored form has it
            reinterpret_cast<uint8_t*>(s_scales)[(c >> 5) * 256 + (wave >> 2) * 128 + (c & 31) * 4 + (wave & 3)] = (uint8_t)s;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) *reinterpret_cast<u32x4*>(area + (lane * kEach + e) * 16) = q[e];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCols * 8 / kTileThreads; ++i) {
            const int id = threadIdx.x + i * kTileThreads, c = id >> 3, piece = id & 7;
            if (columns_form && c0 + c < cols)
                *reinterpret_cast<u32x4*>(by_columns.codes + (c0 + c) * (by_columns.chunks * 128) + row_tile * 128 + piece * 16) =
                    *reinterpret_cast<const u32x4*>(s_area + piece * kWaveBytes + c * 16);
        }
        if constexpr (!NORM) {
            if (n.sums && threadIdx.x < kCols && c0 + threadIdx.x < cols) {
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) sum += s_sums[w][threadIdx.x];
                n.sums[row_tile * cols + c0 + threadIdx.x] = sum;
            }
        }
        if (columns_form && threadIdx.x < kCols * 2) {
            const int64_t group = (c0 >> 5) + (threadIdx.x >> 6);
            if (group * 32 < cols)
                *reinterpret_cast<uint32_t*>(by_columns.scales + ((group * by_columns.chunks + row_tile) << 8) + (threadIdx.x & 63) * 4) =
                    s_scales[threadIdx.x];
        }
        if (STOCHASTIC && rows_form) __syncthreads();        // the random bits go where the codes were
    }

    if (STOCHASTIC && rows_form) write_rows();
}

// 16 bytes of output a lane and row: 4 values in fp32, 8 in bf16; ROWS neighbouring rows a lane (a power of two: their scales are in one group).
template <typename T, int ROWS>
__global__ __launch_bounds__(kThreads) void mx_restore_kernel(MxStore from, int64_t rows, int64_t cols, T* out, int64_t stride, int64_t first_row)
{
    constexpr int kEach = 16 / (int)sizeof(T), kLanes = kMxChunk / kEach;
    const int64_t row = first_row + row_of_thread<kLanes>() * ROWS, first = (int64_t)blockIdx.x * kMxChunk + (threadIdx.x % kLanes) * kEach;
    if (row >= rows || first >= cols) return;
    const uint8_t* at = from.codes + row * (from.chunks * 128) + (first >> 1);
    const uint8_t* at_scale = from.scales + mx_scale_at(row, first >> 5, from.chunks);
    const int here = rows - row < ROWS ? (int)(rows - row) : ROWS;
    uint32_t codes[ROWS], s[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int q = r < here ? r : 0;
        if constexpr (kEach == 8) codes[r] = *reinterpret_cast<const uint32_t*>(at + q * (from.chunks * 128));
        else codes[r] = *reinterpret_cast<const uint16_t*>(at + q * (from.chunks * 128));
        s[r] = at_scale[q * 4];
    }
    T* to = out + row * stride + first;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        // byte 0 is 2^-127, byte 255 no number; the product is exact but for numbers over the largest
        const float scale = __builtin_bit_cast(float, s[r] == 0u ? 0x00400000u : s[r] == 255u ? 0x7FC00000u : s[r] << 23);
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 1);
        if (r >= here) return;
        if constexpr (kEach == 8) {
            const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[r], 1.0f, 3);
            const float v[8] = {a.x * scale, a.y * scale, b.x * scale, b.y * scale, c.x * scale, c.y * scale, d.x * scale, d.y * scale};
            store8(to + r * stride, cols - first, v);
        } else {
            const float v[4] = {a.x * scale, a.y * scale, b.x * scale, b.y * scale};
            store4(to + r * stride, cols - first, v);
        }
    }
}

template <typename T>
hipError_t rows_of(const void* x, int64_t rows, int64_t cols, int64_t stride, const MxStore& to, hipStream_t s)
{
    return by_rows_and_chunks(rows, to.chunks, 32, [&](int64_t first, dim3 grid) {
        return launch(mx_rows_kernel<T>, grid, dim3(kThreads), s, static_cast<const T*>(x), rows, cols, stride, to, first);
    });
}

template <typename T, bool NORM, bool STOCHASTIC>
hipError_t tiles_of(const void* x, int64_t rows, int64_t cols, int64_t stride, std::conditional_t<NORM, TileNormArgs, SumArgs> n, uint64_t seed, uint64_t id,
                    void* by_rows, void* by_columns, hipStream_t s)
{
    // columns up to a whole chunk where rows are stored, rows up to a whole chunk where columns are
    const int64_t width = by_rows ? mx_chunks(cols) * kMxChunk : cols, col_tiles = (width + kTileCols<T> - 1) / kTileCols<T>;
    const int64_t row_tiles = mx_tile_rows(rows);
    if (col_tiles * row_tiles > INT32_MAX) return hipErrorInvalidValue;
    return in_parts(col_tiles * row_tiles, kTileThreads, [&](int64_t first, int64_t tiles) {
        n.first_tile = (uint32_t)first;
        return launch(mx_tiles_kernel<T, NORM, STOCHASTIC>, dim3((uint32_t)tiles), dim3(kTileThreads), s,
                      static_cast<const T*>(x), rows, cols, stride, n, (uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)id,
                      (uint32_t)(id >> 32), static_cast<uint8_t*>(by_rows), static_cast<uint8_t*>(by_columns), (uint32_t)col_tiles, (uint32_t)tiles);
    });
}

template <typename T, int ROWS>
hipError_t restore_by(const MxStore& from, int64_t rows, int64_t cols, void* out, int64_t stride, hipStream_t s)
{
    return by_rows_and_chunks((rows + ROWS - 1) / ROWS, from.chunks, sizeof(T) == 4 ? 64 : 32, [&](int64_t first, dim3 grid) {
        return launch(mx_restore_kernel<T, ROWS>, grid, dim3(kThreads), s, from, rows, cols, static_cast<T*>(out), stride, first * ROWS);
    });
}
// Four rows a lane once there are workgroups enough: addresses and bounds are worked out once for them (fp32, one row and four: 30000 x 2048
// 61.3 and 55.4 us, 100000 x 64 14.1 and 9.8, but 8192 x 1024 7.2 and 7.5, 1000 x 4095 5.3 and 5.5; bf16 33.5 and 32.6, 8.2 and 6.8, 5.2 and 5.2, 3.8 and 4.1).
template <typename T>
hipError_t restore_of(const MxStore& from, int64_t rows, int64_t cols, void* out, int64_t stride, hipStream_t s)
{
    return rows * from.chunks > 65536 ? restore_by<T, 4>(from, rows, cols, out, stride, s) : restore_by<T, 1>(from, rows, cols, out, stride, s);
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

hipError_t launch_mx_tiles(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t stride, const NormArgs* n, float* sums,
                           bool stochastic, uint64_t seed, uint64_t id, void* by_rows, void* by_columns, hipStream_t s)
{
    const SumArgs none = {sums, 0};
    const TileNormArgs norm = n ? TileNormArgs{n->weight, n->bias, n->mean, n->rstd, n->p_dtype, 0} : TileNormArgs{};
    if (dtype == FH_F32) {
        if (n) return stochastic ? tiles_of<float, true, true>(x, rows, cols, stride, norm, seed, id, by_rows, by_columns, s)
                                 : tiles_of<float, true, false>(x, rows, cols, stride, norm, seed, id, by_rows, by_columns, s);
        return stochastic ? tiles_of<float, false, true>(x, rows, cols, stride, none, seed, id, by_rows, by_columns, s)
                          : tiles_of<float, false, false>(x, rows, cols, stride, none, seed, id, by_rows, by_columns, s);
    }
    if (n) return stochastic ? tiles_of<Bf16, true, true>(x, rows, cols, stride, norm, seed, id, by_rows, by_columns, s)
                             : tiles_of<Bf16, true, false>(x, rows, cols, stride, norm, seed, id, by_rows, by_columns, s);
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
    hipError_t e;
    if (by_columns || rounding == FH_ROUND_STOCHASTIC)
        e = launch_mx_tiles(x, x_dtype, rows, cols, row_stride, nullptr, nullptr, rounding == FH_ROUND_STOCHASTIC, seed, tensor_id, by_rows, by_columns, s);
    else
        e = x_dtype == FH_F32 ? rows_of<float>(x, rows, cols, row_stride, mx_store(by_rows, rows, cols), s)
                                : rows_of<Bf16>(x, rows, cols, row_stride, mx_store(by_rows, rows, cols), s);
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
    const NormArgs n = {weight, bias, p_dtype, eps, static_cast<float*>(mean), static_cast<float*>(rstd)};
    if (by_columns && rounding == FH_ROUND_NEAREST && norm_blocks_fit(x_dtype, rows, cols))
        return launch_norm_blocks(x, x_dtype, rows, cols, row_stride, n, by_rows, by_columns, s) == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
    if (launch_layer_norm(x, x_dtype, rows, cols, row_stride, n, nullptr, 0, tiles ? nullptr : by_rows, s) != hipSuccess) return FH_ERR_LAUNCH;
    if (!tiles) return FH_OK;
    return launch_mx_tiles(x, x_dtype, rows, cols, row_stride, &n, nullptr, rounding == FH_ROUND_STOCHASTIC, seed, tensor_id, by_rows, by_columns, s) == hipSuccess
               ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
