// Matrix products out[i][j] = sum_k A[i][k] B[j][k] of rows that lie in chunks of 128 bytes, and what becomes of the sums before they
// are stored: scales and a bias, the gated projection, or that one's backward pass.
//
// One kernel serves 8-bit integers, bf16 and fp32, because a chunk is 128 bytes of a row for each of them: 128, 64 or 32 values.  A lane of the
// 32 x 32 matrix instructions brings 16 bytes of row lane % 32 of each operand; which of a chunk's values meet in one instruction does not
// matter as long as both operands agree.
#pragma once

#include "fh_activation.hpp"
#include "fh_matrix.hpp"
#include "fh_product_plan.hpp"
#include "fh_q8.hpp"

namespace fh {

constexpr uint32_t kChunkBytes = 128;

typedef int    i32x4 __attribute__((ext_vector_type(4)));
typedef int    i32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The operands' types: lane (r = lane % 32, h = lane / 32) gets the outputs [8 (i/4) + 4 h + i % 4][r], the first index the first operand's row.
struct OfQ8 {
    static constexpr uint32_t kSize = 1;
    static constexpr int kSteps = 1;                            // matrix instructions of a product of 16 bytes a lane
    typedef i32x16 Sums;                                         // whole numbers: exact in any order
    typedef int Sum;
    static constexpr bool kScaled = true;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};
struct OfBf16 {
    static constexpr uint32_t kSize = 2;
    static constexpr int kSteps = 1;                            // matrix instructions of a product of 16 bytes a lane
    typedef f32x16 Sums;
    typedef float Sum;
    static constexpr bool kScaled = false;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct OfF32 {
    static constexpr uint32_t kSize = 4;
    static constexpr int kSteps = 4;                            // matrix instructions of a product of 16 bytes a lane
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
    void*          out;                // parts > 1: float [parts][m][n]
    int64_t        stride;             // of out, in elements
    uint32_t       a_pitch, b_pitch, b2_pitch;                   // bytes from row to row
    uint32_t       chunks;             // of a row
    uint32_t       tail;               // bytes of a row's last chunk: a multiple of 16
    uint32_t       parts, chunks_each; // workgroups that share a tile's sum, chunks of each
    uint32_t       m, n;               // rows of out, columns of out
    uint32_t       m_tiles, n_tiles;
    uint32_t       first;              // workgroup of the launches before this one, or from a workgroup's tile to its next one
    int16_t        bias_dtype, act;
};
static_assert(sizeof(ProductArgs) <= 112, "longer arguments are enqueued a microsecond later");
struct BackwardArgs : ProductArgs {    // out: the gate's gradients, and `up_at` columns further those of up; zeros from column n to up_at
    const void*    dh;
    int64_t        dh_stride;
    int64_t        up_at;
    int64_t        rest_at;            // columns from a gradient to the rest of its rounding; 0: there are none (tiles through LDS know none)
    float*         sums;               // [m_tiles][2][n] sums of the columns over the tile's rows, or null
};
struct TurnedArgs;
template <typename Args> struct has_gap { static constexpr bool value = false; };
template <> struct has_gap<TurnedArgs> { static constexpr bool value = true; };
struct TurnedArgs : ProductArgs {      // products with an operand that lies by columns: its rows are the summed dimension
    uint32_t       summed;             // rows of a and b where they lie so
    uint32_t       split;              // chunks that b has; b2 goes on behind them
    uint32_t       halves;             // 1: every chunk twice in turn, of b the same, of a at a + rest the second time; 0 (in tiles through LDS always): once
    uint32_t       rest;
    uint32_t       gap_from, gap;      // so many rows of out from there on are left out, those behind them move up
};
// The row of out that row i's outputs go to; false where they go nowhere.
template <typename Args>
__device__ __forceinline__ bool out_row(const Args& p, uint32_t i, uint32_t& to)
{
    to = i;
    if constexpr (has_gap<Args>::value) {
        if (i >= p.gap_from) {
            to = i - p.gap;
            return i >= p.gap_from + p.gap && i < p.m;
        }
    }
    return i < p.m;
}
// How an operand lies: its rows by the summed dimension, or the summed dimension's rows by it.
enum class Lies { rows, columns };
template <Made MADE, Lies B> struct ArgsOf { typedef ProductArgs type; };
template <> struct ArgsOf<Made::gated_backward, Lies::rows> { typedef BackwardArgs type; };
template <> struct ArgsOf<Made::linear, Lies::columns> { typedef TurnedArgs type; };

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

// A buffer that is the same in all lanes, where the compiler has worked it out in vector registers.
__device__ __forceinline__ u32x4 in_scalars(u32x4 b)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __builtin_amdgcn_readfirstlane(b[i]);
    return b;
}

// An operand that lies by columns, in LDS: the rows of a chunk (64 of bf16, 32 of fp32) one behind the other, COLS columns of each, 128 * COLS bytes as
// by rows.  In row k the pieces of 16 bytes are turned by turn(k), so that what a wave reads at a time meets all banks: of bf16 four rows
// of 64 bytes (a transposing read gives a lane four rows of its column), of fp32 one row for each half of the wave.
template <typename OP, int COLS>
struct ByColumns {
    static constexpr int kReads = OP::kSize == 2 ? 2 : 4;        // instructions of a read
    static constexpr uint32_t kRow = COLS * OP::kSize, kPieces = kRow / 16, kRows = kChunkBytes / OP::kSize;   // bytes, pieces of a row; rows of a chunk
    static __device__ __forceinline__ uint32_t turn(uint32_t k)
    {
        if constexpr (OP::kSize == 2) return kPieces >= 16 ? (k & 3) << 2 : kPieces == 8 ? (k & 2) << 1 : 0;
        else return kPieces >= 16 ? (k >> 4 & 1) << 3 : 0;
    }
    // Where a lane's 16 bytes at `at` of the operand's LDS come from: row and byte of the row.
    static __device__ __forceinline__ uint32_t row_of(uint32_t at) { return at / kRow; }
    static __device__ __forceinline__ uint32_t byte_of(uint32_t at) { return ((at % kRow / 16) ^ turn(row_of(at))) * 16; }
    // 16 bytes a lane of 32 columns from `col` on: summed rows (4 h + quarter) of the chunk's eighths.
    static __device__ __forceinline__ u32x4 read(const uint8_t* s, uint32_t col, int quarter, int lane)
    {
        if constexpr (OP::kSize == 2) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            const uint32_t i = lane & 15, k = (lane >> 5) * 32 + (i >> 2), piece = (col >> 3) + (lane >> 4 & 1) * 2 + (i >> 1 & 1);
            const uint8_t* from = s + k * kRow + (piece ^ turn(k)) * 16 + (i & 1) * 8 + quarter * 8 * kRow;
            const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)from);
            const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(from + 4 * kRow));
            const u32x2 a = __builtin_bit_cast(u32x2, low), b = __builtin_bit_cast(u32x2, high);
            return u32x4{a.x, a.y, b.x, b.y};
        } else {
            const uint32_t k = (lane >> 5) * 16, c = col + (lane & 31);
            const uint8_t* from = s + k * kRow + ((c >> 2) ^ turn(k)) * 16 + (c & 3) * 4 + quarter * 4 * kRow;
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const uint32_t*>(from + e * kRow);
            return v;
        }
    }
    // The buffer of rows `row` to `end`, of which `rows` exist, from column `col` of `cols` on, whose last 16 bytes are whole: what is past the rows is
    // read as zeros, past the columns as zeros or another row's.
    static __device__ __forceinline__ u32x4 buffer(const uint8_t* p, uint32_t pitch, uint32_t row, uint32_t end, uint32_t rows, uint32_t col, uint32_t cols)
    {
        const uint32_t last = end < rows ? end : rows, left = row >= last ? 0u : last - row;
        return in_scalars(buffer_of(p + (int64_t)row * pitch + (int64_t)col * OP::kSize, left ? (left - 1) * pitch + ((cols - col) * OP::kSize + 15) / 16 * 16 : 0u));
    }
};

template <typename T> __device__ __forceinline__ void load4(const T* p, int64_t n, float (&v)[4])
{
    Run<T, 4> r;
    r.load(p, n);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = r.at(e);
}

// What is left of four values by their rounding to bf16; nothing where the rounded one is no number.
__device__ __forceinline__ void rests(float (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float rest = v[e] - __builtin_bit_cast(float, bf16_pair(v[e], v[e]) << 16);
        v[e] = __builtin_fabsf(rest) < __builtin_inff() ? rest : 0.0f;
    }
}

// Four parameters from column `col` of `n` on, zeros where there are none: by one load, of either type.
__device__ __forceinline__ void parameter4(const void* p, int32_t dtype, int64_t col, int64_t n, float (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = 0.0f;
    if (!p) return;
    if (dtype == FH_F32) load4(static_cast<const float*>(p) + col, n - col, v);
    else load4(static_cast<const Bf16*>(p) + col, n - col, v);
}

// ---- the sum split over a workgroup's waves, through LDS -----------------------------------------
// (32 MT) x (32 NT) sums a workgroup; each wave multiplies every WAVES-th chunk by itself, with an area of LDS of its own and no
// barrier: a chunk's rows come as whole lines into the area, from there to registers, and while those are multiplied the next chunk's
// come.  The waves' sums are joined in LDS in the waves' order.  Small products are bound by the launch and by a wave's chain of chunks, each a trip to the
// memory, which the split shortens (8 bits, 512 x 768 x 768: two chunks a wave at most, 4.1 us, 2 of them the launch's), larger ones by reads of
// operands that a tile of 32 or 64 uses little of (2048 x 2048 x 768 12.1 us, by squares of 128 9.7).
template <typename OP, Made MADE, Lies LA, Lies LB, typename T, int MT, int NT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void product_waves_kernel(typename ArgsOf<MADE, LB>::type p)
{
    constexpr int kRowsA = MT * 32, kRowsB = NT * 32, kPad = kRowsB + 4;
    constexpr bool kPair = MADE != Made::linear;
    constexpr int kCols = kPair ? kRowsB / 2 : kRowsB;           // columns of the tile
    constexpr uint32_t kCodes = (kRowsA + kRowsB) * kChunkBytes, kSums = kRowsA * kPad * 4, kArea = kCodes > kSums ? kCodes : kSums;
    constexpr int kThreads = WAVES * 64, kRuns = kCols / 4, kSteps = (kRowsA * kRuns + kThreads - 1) / kThreads;
    typedef ByColumns<OP, kRowsA> ColumnsA;
    typedef ByColumns<OP, kRowsB> ColumnsB;
    static_assert(kThreads % kRuns == 0, "a thread stays with its columns");
    __shared__ __attribute__((aligned(16))) uint8_t s_area[WAVES * kArea];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t number = p.first + blockIdx.x, tiles = p.m_tiles * p.n_tiles, share = p.parts > 1 ? number / tiles : 0;
    uint32_t i, j;
    in_bands(number - share * tiles, p.m_tiles, p.n_tiles, i, j);
    const uint32_t i0 = i * kRowsA, j0 = j * kCols;
    const uint32_t piece = ((lane & 7) ^ (lane >> 4)) * 16;      // turned by half the row's number, 4 more for every other eight rows
    const uint32_t width = (p.chunks - 1) * kChunkBytes + p.tail;
    // rows past the last are the last one, so that every address is inside; pieces past a row's end are past the buffer's, which reads as zeros
    u32x4 from_a, from_b, from_b2;
    uint32_t at_a[MT * 4], at_b[NT * 4];
    if constexpr (LA == Lies::rows) {
        const uint32_t rows_a = p.m - i0 < kRowsA ? p.m - i0 : kRowsA;
        from_a = buffer_of(p.a + (int64_t)i0 * p.a_pitch, (rows_a - 1) * p.a_pitch + width);
#pragma unroll
        for (int t = 0; t < MT * 4; ++t) {
            const uint32_t r = t * 8 + (lane >> 3);
            at_a[t] = (r < rows_a ? r : rows_a - 1) * p.a_pitch + (piece ^ (t & 1) * 64);
        }
    } else {
#pragma unroll
        for (int t = 0; t < MT * 4; ++t) at_a[t] = ColumnsA::row_of(t * 1024 + lane * 16) * p.a_pitch + ColumnsA::byte_of(t * 1024 + lane * 16);
    }
    if constexpr (LB == Lies::rows) {
        const uint32_t row_b = j0 < p.n ? j0 : p.n - 1, rows_b = p.n - row_b < kCols ? p.n - row_b : kCols;
        from_b = buffer_of(p.b + (int64_t)row_b * p.b_pitch, (rows_b - 1) * p.b_pitch + width);
        from_b2 = kPair ? buffer_of(p.b2 + (int64_t)row_b * p.b2_pitch, (rows_b - 1) * p.b2_pitch + width) : from_b;
#pragma unroll
        for (int t = 0; t < NT * 4; ++t) {
            const uint32_t r = (t * 8 + (lane >> 3)) % kCols, pitch = t * 8 < kCols ? p.b_pitch : p.b2_pitch;
            at_b[t] = (r < rows_b ? r : rows_b - 1) * pitch + (piece ^ (t & 1) * 64);
        }
    }
    uint8_t* area = s_area + wave * kArea;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_area + wave * kArea;
    constexpr uint32_t kNowhere = 1u << 31;                      // past the end of any buffer here
    const auto load = [&](uint32_t chunk) {
        const bool cut = chunk + 1 == p.chunks && p.tail < kChunkBytes;
        uint32_t mine = chunk, rest = 0;                         // chunk of the operands, bytes of a in front of it
        if constexpr (LB == Lies::columns) {
            mine = chunk >> p.halves;
            rest = chunk & p.halves ? p.rest : 0;
        }
        if constexpr (LA == Lies::rows) {
            const uint32_t moved = mine * kChunkBytes + rest;
#pragma unroll
            for (int t = 0; t < MT * 4; ++t)
                to_lds(lds + t * 1024, from_a, cut && (piece ^ (t & 1) * 64) >= p.tail ? kNowhere : at_a[t], moved);
        } else {
            from_a = ColumnsA::buffer(p.a + rest, p.a_pitch, mine * ColumnsA::kRows, (mine + 1) * ColumnsA::kRows, p.summed, i0, p.m);
#pragma unroll
            for (int t = 0; t < MT * 4; ++t) to_lds(lds + t * 1024, from_a, at_a[t], 0);
        }
        if constexpr (LB == Lies::rows) {
#pragma unroll
            for (int t = 0; t < NT * 4; ++t)
                to_lds(lds + kRowsA * kChunkBytes + t * 1024, t * 8 < kCols ? from_b : from_b2, cut && (piece ^ (t & 1) * 64) >= p.tail ? kNowhere : at_b[t],
                       chunk * kChunkBytes);
        } else {
            const bool second = mine >= p.split;
            const uint32_t pitch = second ? p.b2_pitch : p.b_pitch;
            const uint32_t row = (second ? mine - p.split : mine) * ColumnsB::kRows;
            from_b = ColumnsB::buffer(second ? p.b2 : p.b, pitch, row, row + ColumnsB::kRows, p.summed, j0, p.n);
#pragma unroll
            for (int t = 0; t < NT * 4; ++t)
                to_lds(lds + kRowsA * kChunkBytes + t * 1024, from_b, ColumnsB::row_of(t * 1024 + lane * 16) * pitch + ColumnsB::byte_of(t * 1024 + lane * 16), 0);
        }
    };
    const int h = lane >> 5, r = lane & 31, turned = (h * 4) ^ (lane >> 1 & 7);
    typename OP::Sums c[MT][NT] = {};
    uint32_t k = share * p.chunks_each + wave;
    const uint32_t end = p.chunks - share * p.chunks_each < p.chunks_each ? p.chunks : (share + 1) * p.chunks_each;
    if (k < end) load(k);
    while (k < end) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        u32x4 fa[4][MT], fb[4][NT];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint8_t* from = area + (uint32_t)(turned ^ q) * 16 + r * kChunkBytes;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (LB == Lies::rows) fb[q][t] = *reinterpret_cast<const u32x4*>(from + kRowsA * kChunkBytes + t * 4096);
                else fb[q][t] = ColumnsB::read(area + kRowsA * kChunkBytes, t * 32, q, lane);
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (LA == Lies::rows) fa[q][t] = *reinterpret_cast<const u32x4*>(from + t * 4096);
                else fa[q][t] = ColumnsA::read(area, t * 32, q, lane);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the area may be written again
        k += WAVES;
        if (k < end) load(k);
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
    parameter4(p.bias, p.bias_dtype, at, p.n, bias);
    parameter4(kPair ? p.bias2 : nullptr, p.bias_dtype, at, p.n, bias2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bool inside = at + e < p.n;
        scales[e] = inside ? scale_of<OP>(p.b, p.n, p.b_pitch, p.chunks, at + e) : 0.0f;
        scales2[e] = kPair && inside ? scale_of<OP>(p.b2, p.n, p.b2_pitch, p.chunks, at + e) : 0.0f;
    }
    float sums[2][4] = {};
    const int64_t left = (int64_t)p.n - at;
#pragma unroll
    for (int t = 0; t < kSteps; ++t) {
        const int row = (t * kThreads + threadIdx.x) / kRuns;
        const uint32_t i = i0 + row;
        if (row >= kRowsA || i >= p.m) continue;
        const float mine = scale_of<OP>(p.a, p.m, p.a_pitch, p.chunks, i);
        const Sum4 sum = sum_at(row, col);
        float v[4];
        if constexpr (!kPair) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = made_of<OP>(sum[e], mine * scales[e], bias[e]);
            uint32_t to;
            if (out_row(p, i, to)) store4(static_cast<T*>(p.out) + (int64_t)share * p.m * p.n + (int64_t)to * p.stride + at, left, v);
        } else {
            const Sum4 sum2 = sum_at(row, kCols + col);
            float gate[4], up[4], dup[4], slopes[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                gate[e] = made_of<OP>(sum[e], mine * scales[e], bias[e]);
                up[e] = made_of<OP>(sum2[e], mine * scales2[e], bias2[e]);
            }
            if constexpr (MADE == Made::gated) {
                activate(gate, p.act, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] *= up[e];
                store4(static_cast<T*>(p.out) + (int64_t)i * p.stride + at, left, v);
            } else {
                float dh[4], act[4];
                load4(static_cast<const T*>(p.dh) + (int64_t)i * p.dh_stride + at, left, dh);
                activate(gate, p.act, act, slopes);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = e < left ? dh[e] * up[e] * slopes[e] : 0.0f;
                    dup[e] = e < left ? dh[e] * act[e] : 0.0f;
                    sums[0][e] += v[e];
                    sums[1][e] += dup[e];
                }
                T* to = static_cast<T*>(p.out) + (int64_t)i * p.stride + at;
                store4(to, p.up_at - at, v);
                store4(to + p.up_at, p.up_at - at, dup);
                if (sizeof(T) == 2 && p.rest_at) {
                    rests(v);
                    rests(dup);
                    store4(to + p.rest_at, p.up_at - at, v);
                    store4(to + p.rest_at + p.up_at, p.up_at - at, dup);
                }
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

// The tiles of a product in squares (or halves of them, for a pair) of `side` sums.
template <Made MADE, typename Args>
int64_t tiles_of(Args& p, uint32_t side)
{
    const uint32_t cols = MADE == Made::linear ? side : side / 2;
    uint32_t n = p.n;
    if constexpr (MADE == Made::gated_backward) n = (uint32_t)p.up_at;   // the zeros behind the last column are written too
    p.m_tiles = (p.m + side - 1) / side;
    p.n_tiles = (n + cols - 1) / cols;
    return (int64_t)p.m_tiles * p.n_tiles;
}
template <typename OP, Made MADE, Lies LA, Lies LB, typename T, int MT, int NT, int WAVES>
hipError_t product_waves(typename ArgsOf<MADE, LB>::type p, hipStream_t s)
{
    static_assert(MT == NT, "squares");
    const int64_t groups = tiles_of<MADE>(p, MT * 32) * p.parts;
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    return in_parts(groups, WAVES * 64, [&](int64_t first, int64_t count) {
        p.first = (uint32_t)first;
        return launch(product_waves_kernel<OP, MADE, LA, LB, T, MT, NT, WAVES>, dim3((uint32_t)count), dim3(WAVES * 64), s, p);
    });
}

// A wave's (32 MT) x 64 sums to what is made of them.  Sixteen rows at a time go through 4 KiB of LDS, so that a lane has eight of a row: of a linear product
// neighbours, of a pair four of the gate and the same four of up.  The formulas, which are long, stand here once for eight passes, and what a
// row brings (its scale, dh) is read a pass ahead.
template <typename OP, Made MADE, typename T, int MT, int NT, typename Args>
__device__ __forceinline__ void tile_epilogue(const Args& p, T* out, const typename OP::Sums (&c)[MT][NT], uint8_t* s_area, uint32_t i0, uint32_t j0, int lane)
{
    constexpr bool kPair = MADE != Made::linear;
    typedef typename OP::Sum Sum;
    typedef Sum Sum4 __attribute__((ext_vector_type(4)));
    const int row16 = lane & 15, upper = lane >> 4 & 1, half = lane >> 5, piece = lane & 7, mine = lane >> 3;
    const uint32_t col = j0 + piece * (kPair ? 4 : 8);           // and of the second four
    const uint32_t col2 = kPair ? col : col + 4;
    const int64_t left = (int64_t)p.n - col;
    float bias[2][4], scales[2][4];
    parameter4(p.bias, p.bias_dtype, col, p.n, bias[0]);
    parameter4(kPair ? p.bias2 : p.bias, p.bias_dtype, col2, p.n, bias[1]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t inside = col + e < p.n ? col + e : p.n - 1, inside2 = col2 + e < p.n ? col2 + e : p.n - 1;
        scales[0][e] = scale_of<OP>(p.b, p.n, p.b_pitch, p.chunks, inside);
        scales[1][e] = scale_of<OP>(kPair ? p.b2 : p.b, p.n, kPair ? p.b2_pitch : p.b_pitch, p.chunks, inside2);
    }
    struct OfRow { float scale; f32x4 dh; };
    const auto of_row = [&](int row, OfRow& r) {
        const uint32_t i = i0 + row;
        r.scale = OP::kScaled ? scale_of<OP>(p.a, p.m, p.a_pitch, p.chunks, i < p.m ? i : p.m - 1) : 1.0f;
        if constexpr (MADE == Made::gated_backward) {
            float dh[4];
            load4(static_cast<const T*>(p.dh) + (int64_t)i * p.dh_stride + col, i < p.m ? left : 0, dh);
            r.dh = f32x4{dh[0], dh[1], dh[2], dh[3]};
        }
    };
    float sums[2][4] = {};
    OfRow next[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) of_row(t * 8 + mine, next[t]);
#pragma clang loop unroll(disable)
    for (int pass = 0; pass < 2 * MT; ++pass) {
#pragma unroll
        for (int x = 0; x < MT; ++x)
            if (x == pass >> 1 && upper == (pass & 1)) {
#pragma unroll
                for (int y = 0; y < NT; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *reinterpret_cast<Sum4*>(s_area + row16 * 256 + ((y * 8 + 2 * e + half) ^ row16) * 16) =
                            Sum4{c[x][y][4 * e], c[x][y][4 * e + 1], c[x][y][4 * e + 2], c[x][y][4 * e + 3]};
            }
        asm volatile("" ::: "memory");                           // a wave's own LDS accesses are in order
        OfRow now[2];
        Sum4 sum[2][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int row = t * 8 + mine;
            now[t] = next[t];
#pragma unroll
            for (int u = 0; u < 2; ++u) sum[t][u] = *reinterpret_cast<const Sum4*>(s_area + row * 256 + ((kPair ? u * 8 + piece : piece * 2 + u) ^ row) * 16);
        }
        asm volatile("" ::: "memory");
        if (pass + 1 < 2 * MT) {
#pragma unroll
            for (int t = 0; t < 2; ++t) of_row((pass + 1) * 16 + t * 8 + mine, next[t]);
        }
        float first[8], second[8], act[8], slopes[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int t = e / 4;
            first[e] = made_of<OP>(sum[t][0][e % 4], now[t].scale * scales[0][e % 4], bias[0][e % 4]);
            second[e] = made_of<OP>(sum[t][1][e % 4], now[t].scale * scales[1][e % 4], bias[1][e % 4]);
        }
        if constexpr (MADE == Made::gated) activate(first, p.act, act);
        if constexpr (MADE == Made::gated_backward) activate(first, p.act, act, slopes);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t i = i0 + pass * 16 + t * 8 + mine;
            float v[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = t * 4 + e;
                if constexpr (MADE == Made::linear) {
                    v[e] = first[at];
                    w[e] = second[at];
                } else if constexpr (MADE == Made::gated) {
                    v[e] = act[at] * second[at];
                } else {
                    const bool inside = i < p.m && e < left;     // the others' sums are of no rows
                    v[e] = inside ? now[t].dh[e] * second[at] * slopes[at] : 0.0f;
                    w[e] = inside ? now[t].dh[e] * act[at] : 0.0f;
                    sums[0][e] += v[e];
                    sums[1][e] += w[e];
                }
            }
            uint32_t row;
            const bool some = out_row(p, i, row);
            T* to = out + (int64_t)row * p.stride + col;
            if constexpr (MADE == Made::linear) {
                const float both[8] = {v[0], v[1], v[2], v[3], w[0], w[1], w[2], w[3]};
                store8(to, some ? left : 0, both);
            } else if constexpr (MADE == Made::gated) {
                store4(to, some ? left : 0, v);
            } else {
                const int64_t most = some ? p.up_at - col : 0;
                store4(to, most, v);
                store4(to + p.up_at, most, w);
            }
        }
    }
    if constexpr (MADE == Made::gated_backward) {
        if (!p.sums || i0 >= p.m) return;
        // over the eight lanes that have the same columns
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float s = sums[u][e], a, b;
                s += dpp<0x128>(s);                              // row_ror:8
                self_swap<16>(s, a, b);
                s = a + b;
                self_swap<32>(s, a, b);
                sums[u][e] = a + b;
            }
        if (mine == 0) {
            float* to = p.sums + (int64_t)(i0 / (MT * 32)) * 2 * p.n + col;
            store4(to, left, sums[0]);
            store4(to + p.n, left, sums[1]);
        }
    }
}

// ---- large products: tiles through LDS -----------------------------------------------------------
// B x B sums of a tile, a chunk at a time; a workgroup of 2 x WN waves, each with B/2 x 64 sums, takes one tile after another.  Two stages of LDS: while one
// is multiplied the next is on its way, and a stage is handed over before its last quarter, which is in registers by then, so that the matrix
// unit works across the barrier.  A row's eight pieces of 16 bytes are turned by half the row's number (the loads take them from turned
// addresses), so that sixteen lanes reading the same piece of sixteen rows meet all 64 banks.
// The chunks of the next tile follow those of the last without a gap: a tile's outputs go through LDS of their own, and since memory
// operations are counted in their order and the loads are sent before the outputs are, the next wait is for the loads alone.
// Of a pair's 64 columns of a wave the first 32 are the gate's and the others the same columns of up, so that both sums of an output are one wave's.
// Measured, one call among others (a trace has gaps between them and varies more): 8 bits, 8192 x 8192 x 4096, 240 to 255 us, 2.2 to 2.3 POP/s; bf16, pairs of
// 4096 x 8192 x 4096, 450 us, 1.22 PFLOP/s, and 8192 x 2048 x 768, 56 us.  The large ones are bound by the card's power: the matrix unit is busy 56 to 61 % of the
// cycles, and the busier it is kept the further the clock falls (1.93 to 1.86 GHz); without the loads 377 of 450 us were left.  In the last a tile has 12 chunks,
// and the second of two rounds of tiles has nothing to hide its outputs behind.
template <typename OP, Made MADE, Lies LA, Lies LB, typename T, int B, int WN>
__global__ __launch_bounds__(2 * WN * 64, B > 128 ? 1 : 2) void product_tile_kernel(typename ArgsOf<MADE, LB>::type p)
{
    constexpr bool kPair = MADE != Made::linear;
    constexpr int kWaves = 2 * WN, MT = B / 64, NT = 2, kCols = kPair ? B / 2 : B;
    constexpr uint32_t kOfA = B * kChunkBytes, kStage = 2 * kOfA;
    constexpr int kStores = MT * 4 * (MADE == Made::gated_backward || (MADE == Made::linear && sizeof(T) == 4) ? 2 : 1);   // of a whole tile, a wave's
    typedef ByColumns<OP, B> Columns;
    static_assert(kWaves * 32 == B && WN * 64 == B, "a wave loads 32 rows of each operand, and has 64 columns");
    __shared__ __attribute__((aligned(16))) uint8_t s_stage[2 * kStage + kWaves * 4096];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;

    const uint32_t squares = p.m_tiles * p.n_tiles, tiles = squares * p.parts, xcd = blockIdx.x & 7;
    const uint32_t end_tile = run_of(xcd, tiles) + (tiles >> 3) + (xcd < (tiles & 7) ? 1 : 0);
    const auto share_of = [&](uint32_t tile) { return p.parts > 1 ? tile / squares : 0u; };
    const auto corner = [&](uint32_t tile, uint32_t& i0, uint32_t& j0) {
        in_bands(tile - share_of(tile) * squares, p.m_tiles, p.n_tiles, i0, j0);
        i0 *= B;
        j0 *= kCols;
    };
    const auto end_of = [&](uint32_t share) { return p.chunks - share * p.chunks_each < p.chunks_each ? p.chunks : (share + 1) * p.chunks_each; };

    // what is loaded next: a chunk of a tile, in this wave 4 KiB of each operand: 32 rows, or as much of its columns.  (64 rows of one operand a
    // wave: products by columns 2.7 % slower, the backward pass of 4096 x 4096 -> 8192 in bf16 1457 us and 1418 on one card; by rows alike within 1 %.)
    const uint32_t width = (p.chunks - 1) * kChunkBytes + p.tail;
    uint32_t next_tile = run_of(blockIdx.x, tiles), next_chunk = 0, next_end = 0, next_i = 0, next_j = 0;
    const bool of_up = kPair && (wave & 1);                      // a pair's rows of B are by turns 32 of the gate and 32 of up
    const uint32_t pitch_b = of_up ? p.b2_pitch : p.b_pitch;
    u32x4 from_a = {}, from_b = {};
    const auto aim = [&]() {
        corner(next_tile, next_i, next_j);
        const uint32_t share = share_of(next_tile);
        next_chunk = share * p.chunks_each;
        next_end = end_of(share);
        // rows past the last are past the buffer's end: zeros are read for them, and nothing of theirs is stored
        const auto rows_of = [&](const uint8_t* base, uint32_t row0, uint32_t all, uint32_t row_pitch) {
            const uint32_t rows = row0 >= all ? 0u : all - row0 < 32u ? all - row0 : 32u;
            return buffer_of(base + (int64_t)(rows ? row0 : 0u) * row_pitch, rows ? (rows - 1) * row_pitch + width : 0u);
        };
        if constexpr (LA == Lies::rows) from_a = rows_of(p.a, next_i + wave * 32, p.m, p.a_pitch);
        if constexpr (LB == Lies::rows) from_b = rows_of(of_up ? p.b2 : p.b, next_j + (kPair ? wave / 2 : wave) * 32, p.n, pitch_b);
    };
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_stage;
    // Four loads of an operand from one buffer, neighbours `step` bytes apart, every other one with its pieces turned another way.  Where no tile is left
    // the buffers are empty.
    struct Loads { u32x4 from; uint32_t at[2], step, moved, to; };
    const auto next_rows = [&](u32x4 from, uint32_t pitch, uint32_t l) {
        constexpr uint32_t kNowhere = 1u << 31;                  // past the end of any buffer here: zeros
        const uint32_t limit = next_chunk + 1 == p.chunks ? p.tail : kChunkBytes, piece = ((l & 7) ^ (l >> 4)) * 16;
        return Loads{from, {(piece < limit ? piece : kNowhere) + (l >> 3) * pitch, ((piece ^ 64) < limit ? piece ^ 64 : kNowhere) + (l >> 3) * pitch}, 8 * pitch,
                     next_chunk * kChunkBytes, 0};
    };
    const auto next_columns = [&](const uint8_t* base, uint32_t pitch, uint32_t chunk, uint32_t summed, uint32_t col, uint32_t all, uint32_t l) {
        const uint32_t place = wave * 4096;
        return Loads{Columns::buffer(base, pitch, chunk * Columns::kRows + Columns::row_of(place), (chunk + 1) * Columns::kRows, summed, col, all),
                     {Columns::row_of(l * 16) * pitch + Columns::byte_of(place + l * 16), Columns::row_of(l * 16) * pitch + Columns::byte_of(place + 1024 + l * 16)},
                     Columns::row_of(1024) * pitch, 0, 0};
    };
    struct Load { Loads a, b; };
    const auto next_load = [&](uint32_t stage) {
        Load n;
        uint32_t l = lane;
        asm("" : "+v"(l));                                       // offsets made here, not registers kept
        if constexpr (LA == Lies::rows) n.a = next_rows(from_a, p.a_pitch, l);
        else n.a = next_columns(p.a, p.a_pitch, next_chunk, next_tile < end_tile ? p.summed : 0u, next_i, p.m, l);
        if constexpr (LB == Lies::rows) {
            n.b = next_rows(from_b, pitch_b, l);
        } else {
            const bool second = next_chunk >= p.split;
            n.b = next_columns(second ? p.b2 : p.b, second ? p.b2_pitch : p.b_pitch, second ? next_chunk - p.split : next_chunk, next_tile < end_tile ? p.summed : 0u,
                               next_j, p.n, l);
        }
        n.a.from = in_scalars(n.a.from);
        n.b.from = in_scalars(n.b.from);
        n.a.to = lds + stage + wave * 4096;
        n.b.to = lds + stage + kOfA + wave * 4096;
        return n;
    };
    const auto load_piece = [&](const Load& n, int t) {
        const Loads& o = t < 4 ? n.a : n.b;
        to_lds(o.to + t % 4 * 1024, o.from, o.at[t & 1] + t % 4 * o.step, o.moved);
    };
    const auto loaded = [&]() {
        if (++next_chunk != next_end) return;
        next_tile += p.first;
        if (next_tile < end_tile) {
            aim();
        } else {
            from_a = u32x4{from_a.x, from_a.y, 0, from_a.w};
            from_b = u32x4{from_b.x, from_b.y, 0, from_b.w};
        }
    };
    const auto load = [&](uint32_t stage) {
        const Load n = next_load(stage);
#pragma unroll
        for (int t = 0; t < 8; ++t) load_piece(n, t);
        loaded();
    };

    const int h = lane >> 5, r = lane & 31, turned = (h * 4) ^ (lane >> 1 & 7);
    const uint32_t read_a = (wm * MT * 32 + r) * kChunkBytes, read_b = kOfA + (wn * NT * 32 + r) * kChunkBytes;
    u32x4 fa[2][MT], fb[2][NT];
    const auto read = [&](uint32_t stage, int quarter, int to) {
        const uint8_t* at_piece = s_stage + stage + (uint32_t)(turned ^ quarter) * 16;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if constexpr (LA == Lies::rows) fa[to][t] = *reinterpret_cast<const u32x4*>(at_piece + read_a + t * 4096);
            else fa[to][t] = Columns::read(s_stage + stage, (wm * MT + t) * 32, quarter, lane);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (LB == Lies::rows) fb[to][t] = *reinterpret_cast<const u32x4*>(at_piece + read_b + t * 4096);
            else fb[to][t] = Columns::read(s_stage + stage + kOfA, (wn * NT + t) * 32, quarter, lane);
        }
    };
    typename OP::Sums c[MT][NT];
    // Sums run along b's rows within a lane.
    const auto product = [&](int which, int number) {
        const int x = number / NT, y = number % NT;
        c[x][y] = OP::multiply(fb[which][y], fa[which][x], c[x][y]);
    };
    // A quarter's products while the next quarter is read, a read or two to a matrix instruction: left to itself the compiler sends the reads late and waits.
    constexpr int kReads = MT * (LA == Lies::rows ? 1 : Columns::kReads) + NT * (LB == Lies::rows ? 1 : Columns::kReads), kSteps = MT * NT * OP::kSteps;
    const auto multiply = [&](int which) {
#pragma unroll
        for (int number = 0; number < MT * NT; ++number) product(which, number);
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
            if ((step + 1) * kReads / kSteps > step * kReads / kSteps) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if ((step + 1) * kReads / kSteps > step * kReads / kSteps + 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
    };
    uint32_t tile = next_tile, stage = 0;
    bool behind = false;                                         // outputs were sent after the load that is waited for
    if (tile >= end_tile) return;
    aim();
    load(0);
    load(kStage);
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");             // the first stage's are older
    __syncthreads();
#pragma clang loop unroll(disable)
    for (; tile < end_tile; tile += p.first) {
        uint32_t i0, j0;
        corner(tile, i0, j0);
        const uint32_t share = share_of(tile), begin = share * p.chunks_each, end = end_of(share);
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
            for (int y = 0; y < NT; ++y) c[x][y] = typename OP::Sums{};
        read(stage, 0, 0);
#pragma clang loop unroll(disable)
        for (uint32_t k = begin; k < end; ++k) {
            __builtin_amdgcn_sched_barrier(0);
            read(stage, 1, 1);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            read(stage, 2, 0);
            multiply(1);
            __builtin_amdgcn_sched_barrier(0);
            read(stage, 3, 1);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            // this wave has read all of this stage, and its part of the next has arrived
            if (behind) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kStores) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            behind = false;
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const Load n = next_load(stage);
            stage = kStage - stage;
            read(stage, 0, 0);                                   // after the last chunk the next tile's: read again behind the epilogue, which needs the registers
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                load_piece(n, t);
#pragma unroll
                for (int number = t * MT * NT / 8; number < (t + 1) * MT * NT / 8; ++number) product(1, number);
                __builtin_amdgcn_sched_barrier(0);
            }
            loaded();
        }
        tile_epilogue<OP, MADE, T, MT, NT>(p, static_cast<T*>(p.out) + (int64_t)share * p.m * p.n, c, s_stage + 2 * kStage + wave * 4096, i0 + wm * MT * 32, j0 + wn * (kPair ? 32 : 64),
                                           lane);
        behind = i0 + B <= p.m && j0 + kCols <= p.n;
        if constexpr (has_gap<typename ArgsOf<MADE, LB>::type>::value) behind = behind && !p.gap;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // the empty loads behind the last tile go to LDS too, which is another workgroup's next
}

template <typename OP, Made MADE, Lies LA, Lies LB, typename T, int B, int WN>
hipError_t product_tiles(typename ArgsOf<MADE, LB>::type p, hipStream_t s)
{
    const int64_t tiles = tiles_of<MADE>(p, B) * p.parts, held = B > 128 ? 256 : 512;     // what the card holds at a time
    if (tiles * 8 > INT32_MAX) return hipErrorInvalidValue;
    const uint32_t grid = (uint32_t)(tiles < held ? tiles : held);
    p.first = (grid + 7) / 8;
    return launch(product_tile_kernel<OP, MADE, LA, LB, T, B, WN>, dim3(grid), dim3(2 * WN * 64), s, p);
}

// ---- few rows: what counts is how fast the rows of B come ----------------------------------------
// Up to 16 rows x 16 columns (of a pair both) a workgroup; its waves take 256 bytes of every row in turn, straight from memory to the registers that the
// 16 x 16 matrix instructions want: lane (r = lane % 16, g = lane / 16) brings 16 bytes of row r, every fourth piece.  The waves' sums are joined in LDS in
// the waves' order.  Rows may lie at any alignment of their elements: `tail` is exact here.  A pair of 8192 x 4096 in 8 bits comes at 5.2 TB/s, the launch left
// out; workgroups of 4 and of 16 waves were slower (14.8 us; 17.4 and 17.9).
template <typename OP> struct Sums16;
template <> struct Sums16<OfQ8> {
    typedef i32x4 Sums;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
    }
};
template <> struct Sums16<OfBf16> {
    typedef f32x4 Sums;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Sums16<OfF32> {
    typedef f32x4 Sums;
    static __device__ __forceinline__ Sums multiply(u32x4 a, u32x4 b, Sums c)
    {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    }
};
// The bytes from `at` on of a row of `width`, zeros behind its end.
template <typename OP>
__device__ __forceinline__ u32x4 end_of_row(const uint8_t* row, uint32_t at, uint32_t width)
{
    u32x4 v = {};
    if (at + 16 <= width) return *reinterpret_cast<const u32x4_a2*>(row + at);
    if constexpr (OP::kSize == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (at + 4 * i < width) v[i] = *reinterpret_cast<const uint32_t*>(row + at + 4 * i);
    } else {                                                     // rows of bytes are whole pieces
#pragma unroll
        for (int i = 0; i < 8; ++i) if (at + 2 * i < width) v[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(row + at + 2 * i) << (16 * (i & 1));
    }
    return v;
}
template <typename OP, Made MADE, typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void product_rows_kernel(ProductArgs p)
{
    constexpr bool kPair = MADE != Made::linear;
    constexpr int kBoth = kPair ? 2 : 1, kThreads = WAVES * 64, kValues = 256;
    typedef typename OP::Sum Sum;
    typedef typename Sums16<OP>::Sums Sums;
    __shared__ __attribute__((aligned(16))) Sum s_sums[WAVES][kBoth][16][20];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const uint32_t j0 = (p.first + blockIdx.x) * 16, width = p.chunks ? (p.chunks - 1) * kChunkBytes + p.tail : 0u;
    // rows past the last are the last one
    const int64_t row = j0 + r < p.n ? j0 + r : p.n - 1;
    const uint8_t* b[kBoth];
    b[0] = p.b + row * p.b_pitch + g * 16;
    if constexpr (kPair) b[1] = p.b2 + row * p.b2_pitch + g * 16;
    const uint8_t* a = p.a + (int64_t)((uint32_t)r < p.m ? r : p.m - 1) * p.a_pitch + g * 16;
    // what a thread's output takes beside the sums, on its way meanwhile
    static_assert(kThreads >= kValues, "an output a thread");
    const uint32_t out_row = threadIdx.x / 16, out_col = threadIdx.x % 16, i = out_row, j = j0 + out_col;
    const bool mine = threadIdx.x < kValues && i < p.m && j < p.n;
    float bias[kBoth], scales[kBoth];
    if (mine) {
        const float scale = scale_of<OP>(p.a, p.m, p.a_pitch, p.chunks, i);
        bias[0] = parameter(p.bias, p.bias_dtype, j, 0.0f);
        scales[0] = scale_of<OP>(p.b, p.n, p.b_pitch, p.chunks, j) * scale;
        if constexpr (kPair) {
            bias[1] = parameter(p.bias2, p.bias_dtype, j, 0.0f);
            scales[1] = scale_of<OP>(p.b2, p.n, p.b2_pitch, p.chunks, j) * scale;
        }
    }
    Sums c[kBoth] = {};
    struct Pieces { u32x4 a[4], b[4][kBoth]; };
    const auto load = [&](uint32_t k, Pieces& q) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int y = 0; y < kBoth; ++y) q.b[t][y] = *reinterpret_cast<const u32x4_a2*>(b[y] + k + t * 64);
            q.a[t] = *reinterpret_cast<const u32x4_a2*>(a + k + t * 64);
        }
    };
    const auto multiply = [&](const Pieces& q) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int y = 0; y < kBoth; ++y) c[y] = Sums16<OP>::multiply(q.b[t][y], q.a[t], c[y]);
    };
    uint32_t k = wave * 256;
    constexpr uint32_t kStep = WAVES * 256;
    if (k + 256 <= width) {
        Pieces now;
        load(k, now);
        k += kStep;
        while (k + 256 <= width) {                               // the next pieces are sent for before these are multiplied
            Pieces next;
            load(k, next);
            __builtin_amdgcn_sched_barrier(0);
            multiply(now);
            now = next;
            k += kStep;
        }
        multiply(now);
    }
    if (k < width) {
#pragma clang loop unroll(disable)
        for (uint32_t t = 0; t < 4; ++t) {
            const uint32_t at = k + t * 64 + g * 16;
            const u32x4 fa = end_of_row<OP>(a - g * 16, at, width);
#pragma unroll
            for (int y = 0; y < kBoth; ++y) c[y] = Sums16<OP>::multiply(end_of_row<OP>(b[y] - g * 16, at, width), fa, c[y]);
        }
    }
    // a lane has columns 4 g .. of row r
#pragma unroll
    for (int y = 0; y < kBoth; ++y) *reinterpret_cast<Sums*>(&s_sums[wave][y][r][g * 4]) = c[y];
    __syncthreads();
    if (!mine) return;
    float v[kBoth];
#pragma unroll
    for (int y = 0; y < kBoth; ++y) {
        Sum sum = s_sums[0][y][out_row][out_col];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += s_sums[w][y][out_row][out_col];
        v[y] = made_of<OP>(sum, scales[y], bias[y]);
    }
    if constexpr (kPair) {
        const float gate[1] = {v[0]};
        float act[1];
        activate(gate, p.act, act);
        v[0] = act[0] * v[1];
    }
    store1(static_cast<T*>(p.out) + (int64_t)i * p.stride + j, v[0]);
}
template <typename OP, Made MADE, typename T>
hipError_t product_rows(ProductArgs p, hipStream_t s)
{
    constexpr int kWaves = 8;
    if (p.m > kMostFewRows) return hipErrorInvalidValue;
    return in_parts(((int64_t)p.n + 15) / 16, kWaves * 64, [&](int64_t first, int64_t count) {
        p.first = (uint32_t)first;
        return launch(product_rows_kernel<OP, MADE, T, kWaves>, dim3((uint32_t)count), dim3(kWaves * 64), s, p);
    });
}

template <typename OP, Made MADE, typename T, Lies LA = Lies::rows, Lies LB = Lies::rows>
hipError_t product_by(ProductTile tile, const typename ArgsOf<MADE, LB>::type& p, hipStream_t s)
{
    switch (tile) {
        case ProductTile::waves32: return product_waves<OP, MADE, LA, LB, T, 1, 1, 4>(p, s);
        case ProductTile::waves32_wide: return product_waves<OP, MADE, LA, LB, T, 1, 1, 8>(p, s);
        case ProductTile::waves64: return product_waves<OP, MADE, LA, LB, T, 2, 2, 4>(p, s);
        case ProductTile::square128: return product_tiles<OP, MADE, LA, LB, T, 128, 2>(p, s);
        case ProductTile::square256: break;
    }
    return product_tiles<OP, MADE, LA, LB, T, 256, 4>(p, s);
}

}  // namespace fh
