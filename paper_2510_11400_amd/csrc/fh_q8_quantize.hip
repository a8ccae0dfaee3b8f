// Storage in 8-bit integers with a scale per row, and its inverse.
#include "fh_norm.hpp"
#include "fh_q8.hpp"

namespace fh {
namespace {

// The scale of a row and the factor that its values are multiplied by, from the largest magnitude's bits.  Both are one
// correctly rounded division; the factor is at most 127 * 2^100, so no product overflows.
__device__ __forceinline__ void q8_scale(uint32_t top, float& scale, float& factor)
{
    const float t = __builtin_bit_cast(float, top);
    const bool number = top < 0x7F800000u, some = number && t >= 0x1p-100f;
    scale = some ? t / 127.0f : number ? 0.0f : __builtin_nanf("");
    factor = some ? 127.0f / t : 0.0f;
}
// Four codes.  Adding 1.5 * 2^23 rounds a number below 2^22 to a whole one, ties to even, and leaves it in the sum's low bits.  In a row
// without a scale the factor is 0 and NaN or infinity times it is NaN: its codes are 0 by the mask.
__device__ __forceinline__ uint32_t q8_codes4(float a, float b, float c, float d, float factor, uint32_t mask)
{
    const auto bits = [&](float v) { return __builtin_bit_cast(uint32_t, v * factor + 12582912.0f); };
    const uint32_t low = __builtin_amdgcn_perm(bits(b), bits(a), 0x0C0C0400u), high = __builtin_amdgcn_perm(bits(d), bits(c), 0x04000C0Cu);
    return (low | high) & mask;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = quad_max(v);
    v = umax(v, dpp<kHalfMirror>(v));
    v = umax(v, dpp<kRowMirror>(v));
    float a, b;
    self_swap<16>(__builtin_bit_cast(float, v), a, b);
    v = umax(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
    self_swap<32>(__builtin_bit_cast(float, v), a, b);
    return umax(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}

// THREADS threads to a row, RUNS runs of eight values to a thread, which stay in registers between the largest magnitude and the codes: the
// row is read once.  LOOPS: rows of any length, which are read a second time for the codes (from the caches as a rule).  The memory bounds many
// rows: 8192 of 2048 in bf16 are read and written in 8.9 us, 5.7 TB/s, part of it out of the memory-side cache; a launch bounds few of them.
template <typename T, int THREADS, int RUNS, bool LOOPS>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void q8_quantize_kernel(const T* x, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes, float* scales,
                                                                                  uint32_t pitch, uint32_t first)
{
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1, kWaves = THREADS / 64, kStep = THREADS * 8;
    const int thread = threadIdx.x % THREADS;
    const int64_t row = ((int64_t)first + blockIdx.x) * kRows + threadIdx.x / THREADS;
    if (row >= rows) return;                                     // whole waves; with more than one wave a row there is a row for every workgroup
    const T* from = x + row * stride;
    Run<T> v[RUNS];
    uint32_t top = 0;
    const auto look = [&](const Run<T>& r) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = umax(top, abs_bits(r.at(e)));
    };
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        const int64_t c = (int64_t)i * kStep + thread * 8;
        v[i].load(from + c, cols - c);
    }
#pragma unroll
    for (int i = 0; i < RUNS; ++i) look(v[i]);
    if constexpr (LOOPS)
        for (int64_t c = (int64_t)RUNS * kStep + thread * 8; c < cols; c += kStep) {
            Run<T> r;
            r.load(from + c, cols - c);
            look(r);
        }
    top = wave_max(top);
    if constexpr (kWaves > 1) {
        __shared__ uint32_t s_top[kWaves];
        if (threadIdx.x % 64 == 0) s_top[threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = umax(top, s_top[w]);
    }
    float scale, factor;
    q8_scale(top, scale, factor);
    const uint32_t mask = top < 0x7F800000u ? 0xFFFFFFFFu : 0u;
    uint8_t* to = codes + row * pitch;
    const auto store = [&](const Run<T>& r, int64_t c) {
        if (c < pitch)
            *reinterpret_cast<u32x2*>(to + c) = u32x2{q8_codes4(r.at(0), r.at(1), r.at(2), r.at(3), factor, mask),
                                                      q8_codes4(r.at(4), r.at(5), r.at(6), r.at(7), factor, mask)};
    };
#pragma unroll
    for (int i = 0; i < RUNS; ++i) store(v[i], (int64_t)i * kStep + thread * 8);
    if constexpr (LOOPS)
        for (int64_t c = (int64_t)RUNS * kStep + thread * 8; c < pitch; c += kStep) {
            Run<T> r;
            r.load(from + c, cols - c);
            store(r, c);
        }
    if (thread == 0) scales[row] = scale;
}

// Eight values a thread; `runs` of them make a row.  Bound by the memory: 8192 x 2048 to bf16 take 9.5 us, 5.3 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void q8_dequantize_kernel(const uint8_t* codes, const float* scales, uint32_t rows, uint32_t cols, uint32_t pitch, uint32_t runs,
                                                            T* out, int64_t stride)
{
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, row = at / runs, c = (at - row * runs) * 8;
    if (row >= rows) return;
    const u32x2 w = *reinterpret_cast<const u32x2*>(codes + (int64_t)row * pitch + c);
    const float scale = scales[row];
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t four = e < 4 ? w.x : w.y;
        v[e] = (float)(int8_t)(four >> (8 * (e & 3))) * scale;
    }
    store8(out + row * stride + c, (int64_t)cols - c, v);
}

template <typename T, int THREADS, int RUNS, bool LOOPS = false>
hipError_t quantize_by(const T* x, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes, float* scales, hipStream_t s)
{
    constexpr int kThreads = THREADS < 256 ? 256 : THREADS;
    const int64_t groups = (rows + kThreads / THREADS - 1) / (kThreads / THREADS);
    return in_parts(groups, kThreads, [&](int64_t first, int64_t count) {
        return launch(q8_quantize_kernel<T, THREADS, RUNS, LOOPS>, dim3((uint32_t)count), dim3(kThreads), s, x, rows, cols, stride, codes, scales,
                      (uint32_t)(q8_chunks(cols) * kQ8Chunk), (uint32_t)first);
    });
}
// Threads and runs, by what they took (us, 64 threads x 1, 2, 4, 8 runs | 256 x 1, 2, 4 | 1024 x 1, 2; bf16, fp32 alike):
//        1 x 2048     -     -   2.11   2.41 |  1.88   1.90   2.16 |  1.98   2.24        8192 x  512   3.34  3.58  4.36   6.31 |  6.10   7.97  10.79 | 18.12  24.78
//     1024 x 2048     -     -   2.62   3.03 |  2.88   3.00   3.49 |  4.21   5.12        8192 x 1024     -   4.28  4.96   6.81 |  6.69   8.23  11.08 | 18.36  25.15
//        1 x 4096     -     -     -    2.83 |    -    1.93   2.26 |  1.94   2.30        8192 x 2048     -     -   8.85  10.33 | 10.48  10.84  12.78 | 19.95  26.43
//     1024 x 8192     -     -     -      -  |    -      -    4.51 |  5.52   6.09        8192 x 4096     -     -     -   18.46 |    -   16.35  17.31 | 22.24  27.45
// A workgroup's rows wait for nothing in one wave each; beyond 2048 values a wave's row is too long a chain of loads and codes, and few rows are quicker by
// four waves from 1024 values on.  Longer rows than 8192 take 1024 threads' loop: 8192 x 16384 70.8, by 256 threads' loop 82.8; one row of 32768 3.9 and 7.7.
template <typename T>
hipError_t quantize_of(const T* x, int64_t rows, int64_t cols, int64_t stride, uint8_t* codes, float* scales, hipStream_t s)
{
    if (cols <= 512) return quantize_by<T, 64, 1>(x, rows, cols, stride, codes, scales, s);
    if (cols <= 1024) return quantize_by<T, 64, 2>(x, rows, cols, stride, codes, scales, s);
    if (cols <= 2048)
        return rows >= 512 ? quantize_by<T, 64, 4>(x, rows, cols, stride, codes, scales, s) : quantize_by<T, 256, 1>(x, rows, cols, stride, codes, scales, s);
    if (cols <= 4096) return quantize_by<T, 256, 2>(x, rows, cols, stride, codes, scales, s);
    if (cols <= 8192) return quantize_by<T, 256, 4>(x, rows, cols, stride, codes, scales, s);
    return quantize_by<T, 1024, 2, true>(x, rows, cols, stride, codes, scales, s);
}
template <typename T>
hipError_t dequantize_of(const uint8_t* codes, const float* scales, int64_t rows, int64_t cols, T* out, int64_t stride, hipStream_t s)
{
    const int64_t runs = (cols + 7) / 8, pitch = q8_chunks(cols) * kQ8Chunk, most = (int64_t)kLaunchThreads / runs;
    for (int64_t first = 0; first < rows; first += most) {
        const int64_t some = rows - first < most ? rows - first : most;
        const hipError_t e = launch(q8_dequantize_kernel<T>, dim3((uint32_t)((some * runs + 255) / 256)), dim3(256), s, codes + first * pitch, scales + first, (uint32_t)some,
                                    (uint32_t)cols, (uint32_t)pitch, (uint32_t)runs, out + first * stride, stride);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace fh

extern "C" {

size_t fh_q8_bytes(int64_t rows, int64_t cols) { return fh::q8_shape_ok(rows, cols) ? fh::q8_bytes(rows, cols) : 0; }
size_t fh_q8_scales_offset(int64_t rows, int64_t cols) { return fh::q8_shape_ok(rows, cols) ? fh::q8_codes_bytes(rows, cols) : 0; }

fh_status fh_q8_quantize(const void* x, fh_dtype x_dtype, int64_t rows, int64_t cols, int64_t row_stride, void* stored, size_t stored_cap, void* stream)
{
    using namespace fh;
    if (!is_dtype(x_dtype)) return FH_ERR_BAD_DTYPE;
    if (!q8_shape_ok(rows, cols) || row_stride < cols || row_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (rows == 0 || cols == 0) return FH_OK;
    if (!x || !stored) return FH_ERR_NULL;
    if (!is_aligned(x, dtype_size(x_dtype)) || !is_aligned(stored, 16)) return FH_ERR_ALIGNMENT;
    if (stored_cap < q8_bytes(rows, cols)) return FH_ERR_BUFFER_TOO_SMALL;
    uint8_t* codes = static_cast<uint8_t*>(stored);
    float* scales = reinterpret_cast<float*>(codes + q8_codes_bytes(rows, cols));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = x_dtype == FH_F32 ? quantize_of(static_cast<const float*>(x), rows, cols, row_stride, codes, scales, s)
                                           : quantize_of(static_cast<const Bf16*>(x), rows, cols, row_stride, codes, scales, s);
    return e == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

fh_status fh_q8_dequantize(const void* stored, size_t stored_cap, int64_t rows, int64_t cols, fh_dtype out_dtype, void* out, int64_t row_stride, size_t out_cap,
                           void* stream)
{
    using namespace fh;
    if (!is_dtype(out_dtype)) return FH_ERR_BAD_DTYPE;
    if (!q8_shape_ok(rows, cols) || row_stride < cols || row_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (rows == 0 || cols == 0) return FH_OK;
    if (!stored || !out) return FH_ERR_NULL;
    if (!is_aligned(stored, 16) || !is_aligned(out, dtype_size(out_dtype))) return FH_ERR_ALIGNMENT;
    if (stored_cap < q8_bytes(rows, cols) || out_cap < strided_elements(rows, cols, row_stride) * dtype_size(out_dtype)) return FH_ERR_BUFFER_TOO_SMALL;
    const uint8_t* codes = static_cast<const uint8_t*>(stored);
    const float* scales = reinterpret_cast<const float*>(codes + q8_codes_bytes(rows, cols));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = out_dtype == FH_F32 ? dequantize_of(codes, scales, rows, cols, static_cast<float*>(out), row_stride, s)
                                             : dequantize_of(codes, scales, rows, cols, static_cast<Bf16*>(out), row_stride, s);
    return e == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
