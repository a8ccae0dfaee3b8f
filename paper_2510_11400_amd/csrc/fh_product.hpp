// Matrix products out[i][j] = sum_k A[i][k] B[j][k] of rows that lie in chunks of 128 bytes, and what becomes of the sums before they
// are stored: scales and a bias, the gated projection, or that one's backward pass.
//
// One kernel serves 8-bit integers, bf16 and fp32, because a chunk is 128 bytes of a row for each of them: 128, 64 or 32 values.  A lane of the
// 32 x 32 matrix instructions brings 16 bytes of row lane % 32 of each operand; which of a chunk's values meet in one instruction does not
// matter as long as both operands agree.
#pragma once

#include "fh_activation.hpp"
#include "fh_matrix.hpp"
#include "fh_q8.hpp"

namespace fh {

constexpr uint32_t kChunkBytes = 128;

typedef int    i32x4 __attribute__((ext_vector_type(4)));
typedef int    i32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The operands' types: lane (r = lane % 32, h = lane / 32) gets the outputs [8 (i/4) + 4 h + i % 4][r], the first index the first operand's row.
struct OfQ8 {
    typedef i32x16 Sums;                                         // whole numbers: exact in any order
    typedef int Sum;
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};
struct OfBf16 {
    typedef f32x16 Sums;
    typedef float Sum;
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct OfF32 {
    typedef f32x16 Sums;
    typedef float Sum;
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};

// What is made of the sums.
enum class Made : int32_t {
    linear,                            // sum (scaled) + bias
    gated,                             // act(gate) * up, each a sum (scaled) + bias; half of a tile's rows of B are the gate's, half those of up
    gated_backward                     // the gradients of gate and up from that of their result
};

struct ProductArgs {
    const uint8_t *a, *b, *b2;         // b2: up, where b is the gate
    const void    *bias, *bias2;       // may be null
    void*          out;
    int64_t        stride;             // of out, in elements
    uint32_t       a_pitch, b_pitch, b2_pitch;                   // bytes from row to row
    uint32_t       chunks;             // of a row
    uint32_t       m, n;               // rows of out, columns of out
    uint32_t       m_tiles, n_tiles;
    uint32_t       first;              // workgroup of the launches before this one, or from a workgroup's tile to its next one
    int16_t        bias_dtype, act;
};
static_assert(sizeof(ProductArgs) <= 112, "longer arguments are enqueued a microsecond later");
struct BackwardArgs : ProductArgs {    // out: the gate's gradients, and `up_at` columns further those of up
    const void*    dh;
    int64_t        dh_stride;
    int64_t        up_at;
    float*         sums;               // [m_tiles][2][n] sums of the columns over the tile's rows, or null
};
template <Made MADE> struct ArgsOf { typedef ProductArgs type; };
template <> struct ArgsOf<Made::gated_backward> { typedef BackwardArgs type; };

// A stored matrix in 8-bit integers has its rows' scales behind them.  No chunks: the sums are 0 and there are no scales.
template <typename OP>
__device__ __forceinline__ float scale_of(const uint8_t* codes, uint32_t rows, uint32_t pitch, uint32_t chunks, uint32_t row)
{
    if constexpr (!OP::kScaled) return 1.0f;
    else return chunks ? reinterpret_cast<const float*>(codes + (int64_t)rows * pitch)[row] : 0.0f;
}
// A sum as the value that it stands for.
template <typename OP>
__device__ __forceinline__ float made_of(typename OP::Sum sum, float scales, float bias)
{
    if constexpr (OP::kScaled) return (float)sum * scales + bias;
    else return sum + bias;
}

template <typename T> __device__ __forceinline__ void load4(const T* p, int64_t n, float (&v)[4])
{
    Run<T, 4> r;
    r.load(p, n);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = r.at(e);
}

// ---- the sum split over a workgroup's waves, through LDS -----------------------------------------
// (32 MT) x (32 NT) sums a workgroup; each wave multiplies every WAVES-th chunk by itself, with an area of LDS of its own and no
// barrier: a chunk's rows come as whole lines into the area, from there to registers, and while those are multiplied the next chunk's
// come.  The waves' sums are joined in LDS in the waves' order.
template <typename OP, Made MADE, typename T, int MT, int NT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void product_waves_kernel(typename ArgsOf<MADE>::type p)
{
    constexpr int kRowsA = MT * 32, kRowsB = NT * 32, kPad = kRowsB + 4;
    constexpr bool kPair = MADE != Made::linear;
    constexpr int kCols = kPair ? kRowsB / 2 : kRowsB;           // columns of the tile
    constexpr uint32_t kCodes = (kRowsA + kRowsB) * kChunkBytes, kSums = kRowsA * kPad * 4, kArea = kCodes > kSums ? kCodes : kSums;
    constexpr int kThreads = WAVES * 64, kRuns = kCols / 4, kSteps = kRowsA * kRuns / kThreads;
    static_assert(kRowsA * kRuns % kThreads == 0 && kThreads % kRuns == 0, "a thread stays with its columns");
    __shared__ __attribute__((aligned(16))) uint8_t s_area[WAVES * kArea];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t i, j;
    in_bands(p.first + blockIdx.x, p.m_tiles, p.n_tiles, i, j);
    const uint32_t i0 = i * kRowsA, j0 = j * kCols;
    // rows past the last are the last one, so that every address is inside
    const uint32_t rows_a = p.m - i0 < kRowsA ? p.m - i0 : kRowsA, rows_b = p.n - j0 < kCols ? p.n - j0 : kCols;
    const uint32_t width = p.chunks * kChunkBytes;
    const u32x4 from_a = buffer_of(p.a + (int64_t)i0 * p.a_pitch, (rows_a - 1) * p.a_pitch + width);
    const u32x4 from_b = buffer_of(p.b + (int64_t)j0 * p.b_pitch, (rows_b - 1) * p.b_pitch + width);
    const u32x4 from_b2 = kPair ? buffer_of(p.b2 + (int64_t)j0 * p.b2_pitch, (rows_b - 1) * p.b2_pitch + width) : from_b;
    const uint32_t piece = ((lane & 7) ^ (lane >> 4)) * 16;      // turned by half the row's number, 4 more for every other eight rows
    uint32_t at_a[MT * 4], at_b[NT * 4];
#pragma unroll
    for (int t = 0; t < MT * 4; ++t) {
        const uint32_t r = t * 8 + (lane >> 3);
        at_a[t] = (r < rows_a ? r : rows_a - 1) * p.a_pitch + (piece ^ (t & 1) * 64);
    }
#pragma unroll
    for (int t = 0; t < NT * 4; ++t) {
        const uint32_t r = (t * 8 + (lane >> 3)) % kCols, pitch = t * 8 < kCols ? p.b_pitch : p.b2_pitch;
        at_b[t] = (r < rows_b ? r : rows_b - 1) * pitch + (piece ^ (t & 1) * 64);
    }
    uint8_t* area = s_area + wave * kArea;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_area + wave * kArea;
    const auto load = [&](uint32_t chunk) {
#pragma unroll
        for (int t = 0; t < MT * 4; ++t) to_lds(lds + t * 1024, from_a, at_a[t], chunk * kChunkBytes);
#pragma unroll
        for (int t = 0; t < NT * 4; ++t) to_lds(lds + kRowsA * kChunkBytes + t * 1024, t * 8 < kCols ? from_b : from_b2, at_b[t], chunk * kChunkBytes);
    };
    const int h = lane >> 5, r = lane & 31, turned = (h * 4) ^ (lane >> 1 & 7);
    typename OP::Sums c[MT][NT] = {};
    uint32_t k = wave;
    if (k < p.chunks) load(k);
    while (k < p.chunks) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        u32x4 fa[4][MT], fb[4][NT];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint8_t* from = area + (uint32_t)(turned ^ q) * 16 + r * kChunkBytes;
#pragma unroll
            for (int t = 0; t < NT; ++t) fb[q][t] = *reinterpret_cast<const u32x4*>(from + kRowsA * kChunkBytes + t * 4096);
#pragma unroll
            for (int t = 0; t < MT; ++t) fa[q][t] = *reinterpret_cast<const u32x4*>(from + t * 4096);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the area may be written again
        k += WAVES;
        if (k < p.chunks) load(k);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int x = 0; x < MT; ++x)
#pragma unroll
                for (int y = 0; y < NT; ++y) c[x][y] = OP::multiply(fb[q][y], fa[q][x], c[x][y]);
    }
    // this wave's area is its own still
    typedef typename OP::Sum Sum;
    typedef Sum Sum4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<Sum4*>(area + ((x * 32 + r) * kPad + y * 32 + 2 * e + 4 * h) * 4) = Sum4{c[x][y][e], c[x][y][e + 1], c[x][y][e + 2], c[x][y][e + 3]};
    __syncthreads();
    const auto sum_at = [&](int row, int col) {
        Sum4 sum = *reinterpret_cast<const Sum4*>(s_area + (row * kPad + col) * 4);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += *reinterpret_cast<const Sum4*>(s_area + w * kArea + (row * kPad + col) * 4);
        return sum;
    };
    const int col = threadIdx.x % kRuns * 4;
    const uint32_t at = j0 + col;
    float bias[4], bias2[4], scales[4], scales2[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool inside = at + e < p.n;
        bias[e] = inside ? parameter(p.bias, p.bias_dtype, at + e, 0.0f) : 0.0f;
        scales[e] = inside ? scale_of<OP>(p.b, p.n, p.b_pitch, p.chunks, at + e) : 0.0f;
        bias2[e] = kPair && inside ? parameter(p.bias2, p.bias_dtype, at + e, 0.0f) : 0.0f;
        scales2[e] = kPair && inside ? scale_of<OP>(p.b2, p.n, p.b2_pitch, p.chunks, at + e) : 0.0f;
    }
    float sums[2][4] = {};
    const int64_t left = (int64_t)p.n - at;
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
        const int row = (t * kThreads + threadIdx.x) / kRuns;
        const uint32_t i = i0 + row;
        if (i >= p.m) continue;
        const float mine = scale_of<OP>(p.a, p.m, p.a_pitch, p.chunks, i);
        const Sum4 sum = sum_at(row, col);
        float v[4];
        if constexpr (!kPair) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = made_of<OP>(sum[e], mine * scales[e], bias[e]);
            store4(static_cast<T*>(p.out) + (int64_t)i * p.stride + at, left, v);
        } else {
            const Sum4 sum2 = sum_at(row, kCols + col);
            float gate[4], up[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gate[e] = made_of<OP>(sum[e], mine * scales[e], bias[e]);
                up[e] = made_of<OP>(sum2[e], mine * scales2[e], bias2[e]);
            }
            if constexpr (MADE == Made::gated) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = activated(gate[e], p.act) * up[e];
                store4(static_cast<T*>(p.out) + (int64_t)i * p.stride + at, left, v);
            } else {
                float dh[4], dup[4];
                load4(static_cast<const T*>(p.dh) + (int64_t)i * p.dh_stride + at, left, dh);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Activated a = activated_both(gate[e], p.act);
                    v[e] = dh[e] * up[e] * a.slope;
                    dup[e] = dh[e] * a.value;
                    sums[0][e] += v[e];
                    sums[1][e] += dup[e];
                }
                T* to = static_cast<T*>(p.out) + (int64_t)i * p.stride + at;
                store4(to, left, v);
                store4(to + p.up_at, left, dup);
            }
        }
    }
    if constexpr (MADE == Made::gated_backward) {
        if (!p.sums) return;
        __syncthreads();
        float* s_sums = reinterpret_cast<float*>(s_area);        // [threads / kRuns][2][kCols]
#pragma unroll
        for (int u = 0; u < 2; ++u)
            *reinterpret_cast<f32x4*>(s_sums + ((threadIdx.x / kRuns * 2 + u) * kCols + col)) = f32x4{sums[u][0], sums[u][1], sums[u][2], sums[u][3]};
        __syncthreads();
        for (int t = threadIdx.x; t < 2 * kCols; t += kThreads) {
            float v = 0.0f;
            for (int g = 0; g < kThreads / kRuns; ++g) v += s_sums[g * 2 * kCols + t];
            const uint32_t c = t % kCols;
            if (j0 + c < p.n) p.sums[((int64_t)i * 2 + t / kCols) * p.n + j0 + c] = v;
        }
    }
}

template <typename OP, Made MADE, typename T, int MT, int NT, int WAVES>
hipError_t product_waves(typename ArgsOf<MADE>::type p, hipStream_t s)
{
    constexpr uint32_t kCols = NT * (MADE == Made::linear ? 32 : 16);
    p.m_tiles = (p.m + MT * 32 - 1) / (MT * 32);
    p.n_tiles = (p.n + kCols - 1) / kCols;
    const int64_t groups = (int64_t)p.m_tiles * p.n_tiles;
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    return in_parts(groups, WAVES * 64, [&](int64_t first, int64_t count) {
        p.first = (uint32_t)first;
        return launch(product_waves_kernel<OP, MADE, T, MT, NT, WAVES>, dim3((uint32_t)count), dim3(WAVES * 64), s, p);
    });
}

}  // namespace fh
