// Layer norm, its backward pass, and the form that writes 4-bit codes.
#include <type_traits>

#include "fh_norm.hpp"

namespace fh {
namespace {

// Columns up to which a row is held in registers: by a wave, and by a workgroup of 1024.
constexpr int64_t kWaveCols = 2048, kGroupCols = 16384;

// The sums of v and of u over the T threads that share a row (a workgroup's rows are T threads each).  `s_pairs` holds two
// values per wave; the calls of a workgroup take its two halves in turn, so that one barrier a call is enough: a wave writes a half
// again only after the barrier of the call between, which every wave enters when it has read that half.
template <int T>
__device__ __forceinline__ void row_sums(float& v, float& u, f32x2 (&s_pairs)[2][16], int turn)
{
    constexpr int kLanes = T < 64 ? T : 64;
    v = lane_sum<kLanes>(v);
    u = lane_sum<kLanes>(u);
    if constexpr (T > 64) {
        f32x2* sums = s_pairs[turn & 1];
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = f32x2{v, u};
        __syncthreads();
        const f32x2* mine = sums + threadIdx.x / T * (T / 64);
        v = u = 0.0f;
        for (int w = 0; w < T / 64; ++w) { v += mine[w].x; u += mine[w].y; }
    }
}

// Mean and sum of squares about it of a row whose T threads hold `sum` of its values, and whose squares about any mean
// `about(mean)` gives.  Each wave takes the squares about its own mean, and one barrier brings the waves' sums and squares
// together: with n_w values of mean m_w in wave w the squares about the row's mean m are sum_w (squares_w + n_w (m_w - m)^2), which
// costs no digits either.  `s_counts`: n_w; `s_waves`: each wave's sum, squares and mean.
template <int T, typename About>
__device__ __forceinline__ void row_moments(float sum, float columns, float& mean, float& squares, About about, f32x4 (&s_waves)[2][16],
                                            const float (&s_counts)[16], int turn)
{
    if constexpr (T <= 64) {
        mean = lane_sum<T>(sum) / columns;
        squares = lane_sum<T>(about(mean));
    } else {
        const int wave = threadIdx.x >> 6;
        const float all = lane_sum<64>(sum), count = s_counts[wave % (T / 64)];
        const float own = count > 0.0f ? all / count : 0.0f;
        const float inside = lane_sum<64>(about(own));
        // With two waves a row the divisions are made again: a mean more in registers costs their kernels a wave a SIMD (4096 x 4096 bf16
        // 14.6 -> 17.7 us); with more it is one more value of the wave's (64 x 8192 5.6 -> 4.5, 2047 x 8193 fp32 30.8 -> 28.5).
        using Sums = std::conditional_t<T == 128, f32x2, f32x4>;
        Sums* waves = reinterpret_cast<Sums*>(s_waves[turn & 1]);
        if ((threadIdx.x & 63) == 0) {
            if constexpr (T == 128) waves[wave] = f32x2{all, inside};
            else waves[wave] = f32x4{all, inside, own, count};
        }
        __syncthreads();
        const Sums* mine = waves + threadIdx.x / T * (T / 64);
        float total = 0.0f;
#pragma unroll 4
        for (int w = 0; w < T / 64; ++w) total += mine[w].x;
        mean = total / columns;
        squares = 0.0f;
#pragma unroll 4
        for (int w = 0; w < T / 64; ++w) {
            float n, m;
            if constexpr (T == 128) {
                n = s_counts[w];
                m = n > 0.0f ? mine[w].x / n : mean;
            } else {
                n = mine[w].w;
                m = n > 0.0f ? mine[w].z : mean;
            }
            const float d = m - mean;
            squares += __builtin_fmaf(n * d, d, mine[w].y);
        }
    }
}

// ---- forward: a row in the registers of T threads, NV runs of eight values each ------------
// Where the rows go: dense (MX false: y and its row stride), or as codes.
struct NormOut { void* y; uint8_t* scales; int64_t stride_or_chunks; };

// A workgroup stays, with the parameters of its threads' columns in registers, and takes rows a grid apart, the next one on its way
// while one is worked on: with a workgroup a row the parameters came from L2 for every row, up to four times the bytes of a
// bf16 row (8192 x 768 bf16: 9.6 us).  The rows have columns in every run, so that only the last runs can end early.
template <int THREADS> constexpr int kNormGroup = THREADS <= 64 ? 256 : THREADS;     // threads of a workgroup
template <typename T, int THREADS, int NV, bool MX>
__global__ __launch_bounds__(kNormGroup<THREADS>) void norm_rows_kernel(const T* x, int64_t rows, int64_t cols, int64_t x_stride,
                                                                                  NormArgs n, NormOut to, int32_t groups)
{
    constexpr int kRows = kNormGroup<THREADS> / THREADS, kWhole = NV - 1;
    __shared__ __attribute__((aligned(16))) f32x4 s_waves[2][16];
    __shared__ float s_counts[16];                               // columns of a row's waves
    const int t = threadIdx.x % THREADS, part = threadIdx.x / THREADS;
    Run<T> next[NV];
    auto load = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t first = ((int64_t)k * THREADS + t) * 8;
            next[k].load(x + (row < rows ? row : 0) * x_stride + first, row < rows ? cols - first : 0);
        }
    };
    load((int64_t)blockIdx.x * kRows + part);
    if constexpr (THREADS > 64) {
        if (threadIdx.x < THREADS / 64) {
            const int64_t end = cols - (int64_t)kWhole * THREADS * 8 - threadIdx.x * 512;      // of the last run
            s_counts[threadIdx.x] = (float)(kWhole * 512 + (end < 0 ? 0 : end < 512 ? end : 512));
        }
        __syncthreads();
    }
    float w[NV][8], b[NV][8];
    int left[NV];                                                // columns of a run
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int64_t first = ((int64_t)k * THREADS + t) * 8;
        left[k] = (int)(cols - first < 0 ? 0 : cols - first < 8 ? cols - first : 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) { w[k][i] = 1.0f; b[k][i] = 0.0f; }
        if (n.p_dtype == FH_F32) {
            if (n.weight) load8(static_cast<const float*>(n.weight) + first, left[k], w[k]);
            if (n.bias) load8(static_cast<const float*>(n.bias) + first, left[k], b[k]);
        } else {
            if (n.weight) load8(static_cast<const Bf16*>(n.weight) + first, left[k], w[k]);
            if (n.bias) load8(static_cast<const Bf16*>(n.bias) + first, left[k], b[k]);
        }
    }
    const int64_t step = (int64_t)groups * kRows;
    const float columns = (float)cols;
    int turn = 0;
    for (int64_t start = (int64_t)blockIdx.x * kRows; start < rows; start += step, ++turn) {
        const int64_t row = start + part;
        const bool write = row < rows;
        float v[NV][8];
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[k][i] = next[k].at(i);
                sum += v[k][i];
            }
        if (start + step < rows) load(row + step);
        // the squares of what is left, so that a mean far from zero costs no digits
        const auto about = [&](float m) {
            float squares = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = k < kWhole || i < left[k] ? v[k][i] - m : 0.0f;
                    squares = __builtin_fmaf(d, d, squares);
                }
            return squares;
        };
        float mean, squares;
        row_moments<THREADS>(sum, columns, mean, squares, about, s_waves, s_counts, turn);
        const float rstd = 1.0f / __builtin_sqrtf(squares / columns + n.eps);
        if (write && t == 0) {
            if (n.mean) n.mean[row] = mean;
            if (n.rstd) n.rstd[row] = rstd;
        }
        if (!to.y) continue;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t first = ((int64_t)k * THREADS + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = norm_value(v[k][i] - mean, rstd, w[k][i], b[k][i]);
            if constexpr (!MX) {
                if (write) store8(static_cast<T*>(to.y) + row * to.stride_or_chunks + first, left[k], v[k]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] = k < kWhole || i < left[k] ? v[k][i] : 0.0f;
                mx_write8(MxStore{static_cast<uint8_t*>(to.y), to.scales, to.stride_or_chunks}, row, first, v[k],
                          write && first < to.stride_or_chunks * kMxChunk);
            }
        }
    }
}

// Rows that do not fit: the row is read three times, from the caches after the first.
template <typename T, bool MX>
__global__ __launch_bounds__(1024) void norm_long_rows_kernel(const T* x, int64_t cols, int64_t x_stride, NormArgs n, NormOut to)
{
    __shared__ f32x2 s_pairs[2][16];
    const int64_t row = blockIdx.x;
    const T* p = x + row * x_stride;
    const int64_t end = mx_chunks(cols) * kMxChunk;             // whole waves have the same number of turns
    float sum = 0.0f, v[8];
    for (int64_t first = threadIdx.x * 8; first < cols; first += 8192) {
        load8(p + first, cols - first, v);
        for (int i = 0; i < 8; ++i) sum += v[i];
    }
    float none = 0.0f;
    row_sums<1024>(sum, none, s_pairs, 0);
    const float mean = sum / (float)cols;
    float squares = 0.0f;
    for (int64_t first = threadIdx.x * 8; first < cols; first += 8192) {
        load8(p + first, cols - first, v);
        for (int i = 0; i < 8; ++i) {
            const float d = first + i < cols ? v[i] - mean : 0.0f;
            squares = __builtin_fmaf(d, d, squares);
        }
    }
    row_sums<1024>(squares, none, s_pairs, 1);
    const float rstd = 1.0f / __builtin_sqrtf(squares / (float)cols + n.eps);
    if (threadIdx.x == 0) {
        if (n.mean) n.mean[row] = mean;
        if (n.rstd) n.rstd[row] = rstd;
    }
    if (!to.y) return;
    for (int64_t start = 0; start < end; start += 8192) {       // every lane takes every turn: quads work together
        const int64_t first = start + threadIdx.x * 8;
        load8(p + first, cols - first, v);
        for (int i = 0; i < 8; ++i) {
            const int64_t c = first + i;
            v[i] = c < cols ? norm_value(v[i] - mean, rstd, parameter(n.weight, n.p_dtype, c, 1.0f), parameter(n.bias, n.p_dtype, c, 0.0f)) : 0.0f;
        }
        if constexpr (!MX) store8(static_cast<T*>(to.y) + row * to.stride_or_chunks + first, cols - first, v);
        else mx_write8(MxStore{static_cast<uint8_t*>(to.y), to.scales, to.stride_or_chunks}, row, first, v, first < end);
    }
}

// ---- forward to codes by columns: blocks of 32 rows -----------------------------------------
// A block of a column is 32 rows, so a workgroup that has all of 32 rows writes both forms from one pass over x: it takes a row's
// statistics and codes from registers as above, leaves the row in LDS, and then has its columns in the lanes.  With a kernel for the
// statistics and the tiles behind it x was read twice and a launch more was waited for: bf16 64 x 768 12.6 -> 8.6 us, 8192 x 768 16.3 -> 11.5,
// 8192 x 2048 26.7 -> 20.5, 32768 x 256 17.4 -> 18.8, fp32 8192 x 1024 18.5 -> 13.5.  Bound by arithmetic, some fifteen instructions a value and form.
// A column's 16 bytes of a block are an eighth of a line: neighbours run on one XCD, in whose L2 the line is put together.
template <typename T, int LANES, int NV>
__global__ __launch_bounds__(1024) void norm_blocks_kernel(const T* x, int64_t rows, int64_t cols, int64_t x_stride, NormArgs n, uint8_t* rows_form,
                                                           uint8_t* columns_form)
{
    constexpr int kAtOnce = 1024 / LANES, kTurns = 32 / kAtOnce, kRow = NV * LANES * 8, kWhole = NV - 1;
    __shared__ __attribute__((aligned(16))) T s_rows[32 * kRow];
    __shared__ __attribute__((aligned(16))) f32x2 s_stats[32];   // mean and 1 / deviation
    const MxStore by_rows = mx_store(rows_form, rows, cols), by_columns = mx_store(columns_form, cols, rows);
    const int64_t block = run_of(blockIdx.x, gridDim.x), r0 = block * 32;
    const int t = threadIdx.x % LANES, part = threadIdx.x / LANES;
    const float columns = (float)cols;
    Run<T> run[kTurns][NV];
#pragma unroll
    for (int u = 0; u < kTurns; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t row = r0 + u * kAtOnce + part, first = (k * LANES + t) * 8;
            run[u][k].load(x + (row < rows ? row : 0) * x_stride + first, row < rows ? cols - first : 0);
        }
    float mean[kTurns], rstd[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int in_block = u * kAtOnce + part;
        const int64_t row = r0 + in_block;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += run[u][k].at(i);
#pragma unroll
            for (int i = 0; i < Run<T>::kWords; i += 4)
                *reinterpret_cast<u32x4*>(reinterpret_cast<uint32_t*>(s_rows + in_block * kRow + (k * LANES + t) * 8) + i) =
                    u32x4{run[u][k].w[i], run[u][k].w[i + 1], run[u][k].w[i + 2], run[u][k].w[i + 3]};
        }
        mean[u] = lane_sum<LANES>(sum) / columns;
        float squares = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = k < kWhole || (k * LANES + t) * 8 + i < cols ? run[u][k].at(i) - mean[u] : 0.0f;
                squares = __builtin_fmaf(d, d, squares);
            }
        rstd[u] = 1.0f / __builtin_sqrtf(lane_sum<LANES>(squares) / columns + n.eps);
        if (t == 0) {
            s_stats[in_block] = f32x2{mean[u], rstd[u]};
            if (row < rows) {
                n.mean[row] = mean[u];
                n.rstd[row] = rstd[u];
            }
        }
    }
    if (rows_form) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int first = (k * LANES + t) * 8, left = (int)cols - first;
            float w[8], b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) { w[i] = 1.0f; b[i] = 0.0f; }
            if (n.p_dtype == FH_F32) {
                if (n.weight) load8(static_cast<const float*>(n.weight) + first, left, w);
                if (n.bias) load8(static_cast<const float*>(n.bias) + first, left, b);
            } else {
                if (n.weight) load8(static_cast<const Bf16*>(n.weight) + first, left, w);
                if (n.bias) load8(static_cast<const Bf16*>(n.bias) + first, left, b);
            }
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                const int64_t row = r0 + u * kAtOnce + part;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float y = norm_value(run[u][k].at(i) - mean[u], rstd[u], w[i], b[i]);
                    v[i] = k < kWhole || i < left ? y : 0.0f;
                }
                mx_write8(by_rows, row, first, v, row < rows && first < by_rows.chunks * kMxChunk);
            }
        }
    }
    __syncthreads();
    const bool whole = r0 + 32 <= rows;
    for (int c = threadIdx.x; c < cols; c += 1024) {
        const float w = parameter(n.weight, n.p_dtype, c, 1.0f), b = parameter(n.bias, n.p_dtype, c, 0.0f);
        float v[32];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 32; i += 2) {                        // two rows' statistics by one read, the same for all lanes
            const f32x4 st = *reinterpret_cast<const f32x4*>(&s_stats[i]);
            v[i] = norm_value(value(s_rows[i * kRow + c]) - st.x, st.y, w, b);
            v[i + 1] = norm_value(value(s_rows[(i + 1) * kRow + c]) - st.z, st.w, w, b);
        }
        if (!whole) {                                            // rows past the last: zeros, whatever the bias
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = r0 + i < rows ? v[i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) top = umax(top, abs_bits(v[i]));
        const uint32_t s = mx_scale_byte(top);
        *reinterpret_cast<u32x4*>(by_columns.codes + c * (by_columns.chunks * 128) + block * 16) = mx_codes32(v, s);
        by_columns.scales[mx_scale_at(c, block, by_columns.chunks)] = (uint8_t)s;
    }
}

// ---- backward ------------------------------------------------------------------------------
struct NormBackwardArgs {
    const void*  dy;
    const void*  x;
    const float* mean;
    const float* rstd;
    const void*  weight;
    void*        dx;                   // may be null
    float*       partial;              // [workgroups][2][cols]: sums of dy * x^ and of dy; may be null
    int64_t      dy_stride, x_stride, dx_stride, rows, cols;
    int32_t      p_dtype;
    int32_t      groups;               // workgroups
};

// A workgroup takes ROWS rows at a time, a grid apart, THREADS threads each, NV runs of four columns a thread (with eight, a row of 768
// left a quarter of the lanes idle, and the arithmetic of some 17 instructions a value is what binds rows of bf16).  Every
// thread keeps the sums of its columns in registers; at the end the rows' sums are added up in LDS, all at once (by runs of
// columns it took two barriers a run and sum: 8192 x 768 bf16 13.7 -> 12.4 us), and the workgroup leaves one row of partial sums, for norm_join_kernel.
// dy is of type G: T, or float where it is a product that has not been rounded to T.
template <typename T, typename G, int THREADS, int NV, int ROWS>
__global__ __launch_bounds__(THREADS * ROWS) void norm_backward_kernel(NormBackwardArgs a)
{
    constexpr bool kAhead = sizeof(G) == 2 || NV < (THREADS < 1024 ? 8 : 4);   // the next row's loads before this row's sums: as registers allow
    constexpr int kWidth = THREADS * 4;
    __shared__ f32x2 s_pairs[2][16];
    __shared__ __attribute__((aligned(16))) float s_join[ROWS > 1 ? ROWS * 2 * NV * kWidth : 4];
    // the weight, read again for every row: in registers it would push the next row's loads out of them
    __shared__ __attribute__((aligned(16))) float s_weight[NV * kWidth];
    const int t = threadIdx.x % THREADS, part = threadIdx.x / THREADS;
    Run<T, 4> next_x[NV];
    Run<G, 4> next_g[NV];
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto load = [&](int64_t row) {                               // nothing of a row past the last
        const bool here = row < a.rows;
        const int64_t at = here ? row : 0;
        next_mean = here ? a.mean[at] : 0.0f;
        next_rstd = here ? a.rstd[at] : 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t first = (int64_t)k * kWidth + t * 4;
            next_x[k].load(static_cast<const T*>(a.x) + at * a.x_stride + first, here ? a.cols - first : 0);
            next_g[k].load(static_cast<const G*>(a.dy) + at * a.dy_stride + first, here ? a.cols - first : 0);
        }
    };
    if constexpr (kAhead) load((int64_t)blockIdx.x * ROWS + part);
    const auto stage_weight = [&](const auto* p) {               // all loads ahead of the first store (one value at a time: 3 x 14488 fp32 11.8 us, now 9.8)
        using P = std::remove_cv_t<std::remove_reference_t<decltype(*p)>>;
        constexpr int kRuns = NV * THREADS, kTimes = (kRuns + THREADS * ROWS - 1) / (THREADS * ROWS);
        Run<P, 4> run[kTimes];
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            const int at = (threadIdx.x + i * THREADS * ROWS) * 4;
            run[i].load(p + at, at < kRuns * 4 ? a.cols - at : 0);
        }
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            const int at = (threadIdx.x + i * THREADS * ROWS) * 4;
            if (at < kRuns * 4) *reinterpret_cast<f32x4*>(s_weight + at) = f32x4{run[i].at(0), run[i].at(1), run[i].at(2), run[i].at(3)};
        }
    };
    if (!a.weight) {
        for (int c = threadIdx.x; c < NV * kWidth; c += THREADS * ROWS) s_weight[c] = c < a.cols ? 1.0f : 0.0f;
    } else if (a.p_dtype == FH_F32) stage_weight(static_cast<const float*>(a.weight));
    else stage_weight(static_cast<const Bf16*>(a.weight));
    __syncthreads();
    f32x4 dw[NV] = {}, db[NV] = {};
    const float share = 1.0f / (float)a.cols;
    const int64_t step = (int64_t)a.groups * ROWS;
    int turn = 0;
    for (int64_t start = (int64_t)blockIdx.x * ROWS; start < a.rows; start += step, ++turn) {
        const int64_t row = start + part;
        const bool here = row < a.rows;
        if constexpr (!kAhead) load(row);
        f32x4 h[NV], g[NV];
        const float mean = next_mean, rstd = next_rstd;
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) { h[k][i] = next_x[k].at(i); g[k][i] = next_g[k].at(i); }
        if constexpr (kAhead) {
            if (start + step < a.rows) load(row + step);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(s_weight + k * kWidth + t * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {                        // where there is no column or row: g is 0, and rstd without a row
                h[k][i] = (h[k][i] - mean) * rstd;
                dw[k][i] = __builtin_fmaf(g[k][i], h[k][i], dw[k][i]);
                db[k][i] += g[k][i];
                g[k][i] *= w[i];
                s1 += g[k][i];
                s2 = __builtin_fmaf(g[k][i], h[k][i], s2);
            }
        }
        if (a.dx) {
            row_sums<THREADS>(s1, s2, s_pairs, turn);
            s1 *= share * rstd;
            s2 *= share * rstd;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int64_t first = (int64_t)k * kWidth + t * 4;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __builtin_fmaf(g[k][i], rstd, -__builtin_fmaf(h[k][i], s2, s1));
                if (here) store4(static_cast<T*>(a.dx) + row * a.dx_stride + first, a.cols - first, v);
            }
        }
    }
    if (!a.partial) return;
    float* to = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t first = (int64_t)k * kWidth + t * 4;
            const f32x4 v = which ? db[k] : dw[k];
            if constexpr (ROWS == 1) {
                const float u[4] = {v.x, v.y, v.z, v.w};
                store4(to + which * a.cols + first, a.cols - first, u);
            } else {
                *reinterpret_cast<f32x4*>(s_join + (part * 2 + which) * (NV * kWidth) + first) = v;
            }
        }
    if constexpr (ROWS > 1) {
        __syncthreads();
#pragma unroll
        for (int which = 0; which < 2; ++which)
            for (int c = threadIdx.x; c < a.cols; c += THREADS * ROWS) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) sum += s_join[(r * 2 + which) * (NV * kWidth) + c];
                to[which * a.cols + c] = sum;
            }
    }
}

// Rows that do not fit: dx by a workgroup a row, which reads the row twice; the columns' sums by a kernel of their own.
template <typename T, typename G>
__global__ __launch_bounds__(1024) void norm_backward_long_rows_kernel(NormBackwardArgs a)
{
    __shared__ f32x2 s_pairs[2][16];
    const int64_t row = blockIdx.x;
    const T* px = static_cast<const T*>(a.x) + row * a.x_stride;
    const G* pg = static_cast<const G*>(a.dy) + row * a.dy_stride;
    const float mean = a.mean[row], rstd = a.rstd[row], share = 1.0f / (float)a.cols;
    float x[8], g[8], s1 = 0.0f, s2 = 0.0f;
    for (int64_t first = threadIdx.x * 8; first < a.cols; first += 8192) {
        load8(px + first, a.cols - first, x);
        load8(pg + first, a.cols - first, g);
        for (int i = 0; i < 8; ++i) {
            const float gw = first + i < a.cols ? g[i] * parameter(a.weight, a.p_dtype, first + i, 1.0f) : 0.0f;
            s1 += gw;
            s2 = __builtin_fmaf(gw, (x[i] - mean) * rstd, s2);
        }
    }
    row_sums<1024>(s1, s2, s_pairs, 0);
    s1 *= share;
    s2 *= share;
    for (int64_t first = threadIdx.x * 8; first < a.cols; first += 8192) {
        load8(px + first, a.cols - first, x);
        load8(pg + first, a.cols - first, g);
        for (int i = 0; i < 8; ++i) {
            const float gw = first + i < a.cols ? g[i] * parameter(a.weight, a.p_dtype, first + i, 1.0f) : 0.0f;
            g[i] = rstd * (gw - s1 - (x[i] - mean) * rstd * s2);
        }
        store8(static_cast<T*>(a.dx) + row * a.dx_stride + first, a.cols - first, g);
    }
}
template <typename T, typename G>
__global__ __launch_bounds__(256) void norm_column_sums_kernel(NormBackwardArgs a, int64_t rows_each, uint32_t col_groups)
{
    const int64_t first = ((int64_t)(blockIdx.x % col_groups) * 256 + threadIdx.x) * 8, part = blockIdx.x / col_groups;
    if (first >= a.cols) return;
    float x[8], g[8], dw[8] = {}, db[8] = {};
    const int64_t end = part * rows_each + rows_each < a.rows ? part * rows_each + rows_each : a.rows;
    for (int64_t row = part * rows_each; row < end; ++row) {
        load8(static_cast<const T*>(a.x) + row * a.x_stride + first, a.cols - first, x);
        load8(static_cast<const G*>(a.dy) + row * a.dy_stride + first, a.cols - first, g);
        const float mean = a.mean[row], rstd = a.rstd[row];
        for (int i = 0; i < 8; ++i) {
            dw[i] = __builtin_fmaf(g[i], (x[i] - mean) * rstd, dw[i]);
            db[i] += g[i];
        }
    }
    float* to = a.partial + part * 2 * a.cols;
    store8(to + first, a.cols - first, dw);
    store8(to + a.cols + first, a.cols - first, db);
}

// Rows of partial sums added up in an order of their number alone: 64 columns of one of the `count` sums a workgroup, a sixteenth of
// 256 rows at a time a wave, whose loads are all on their way at once: up to 256 rows the kernel takes little more than one of them.
constexpr int kMostParts = 256;
template <typename P>
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* partial, int64_t parts, int64_t cols, int32_t count, P* first, P* second, uint32_t first_group)
{
    constexpr int kEach = kMostParts / 16;
    __shared__ float s_part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t group = first_group + blockIdx.x;
    const int32_t which = count == 2 ? group & 1 : 0;
    const int64_t c = (int64_t)(count == 2 ? group >> 1 : group) * 64 + lane;
    const float* from = partial + which * cols + (c < cols ? c : 0);
    float sum = 0.0f;
    for (int64_t start = 0; start < parts; start += kMostParts) {
        float v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {                        // rows past the last: the run's first, for nothing
            const int64_t row = start + wave + 16 * i;
            v[i] = from[(row < parts ? row : start) * count * cols];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = start + wave + 16 * i < parts ? v[i] : 0.0f;
#pragma unroll
        for (int half = kEach / 2; half > 0; half /= 2)
#pragma unroll
            for (int i = 0; i < half; ++i) v[i] += v[i + half];
        sum += v[0];
    }
    s_part[wave][lane] = sum;
    __syncthreads();
    P* to = which ? second : first;
    if (wave == 0 && c < cols && to) {
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < 16; ++w) all += s_part[w][lane];
        store1(to + c, all);
    }
}

// ---- launches ------------------------------------------------------------------------------
template <typename T, int THREADS, int NV, bool MX>
hipError_t norm_of(const void* x, int64_t rows, int64_t cols, int64_t xs, const NormArgs& n, const NormOut& to, hipStream_t s)
{
    // workgroups that stay: what 256 compute units hold, by the threads that NV runs' registers allow on one
    constexpr int kThreads = kNormGroup<THREADS>, kRows = kThreads / THREADS, kHeld = NV == 1 ? 2048 : NV == 2 ? 1280 : NV == 3 ? 1024 : 768;
    constexpr int64_t kStay = kHeld < kThreads ? 256 : 256 * (kHeld / kThreads);
    int64_t groups = (rows + kRows - 1) / kRows;
    if (groups > kStay) groups = kStay;
    return launch(norm_rows_kernel<T, THREADS, NV, MX>, dim3((uint32_t)groups), dim3(kThreads), s, static_cast<const T*>(x), rows, cols,
                       xs, n, to, (int32_t)groups);
}
template <typename T, bool MX>
hipError_t norm_any(const void* x, int64_t rows, int64_t cols, int64_t xs, const NormArgs& n, const NormOut& to, hipStream_t s)
{
    // narrow rows share a wave; codes are written for 256 columns at least, which takes 32 lanes
    if constexpr (!MX) {
        if (cols <= 64) return norm_of<T, 8, 1, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= 128) return norm_of<T, 16, 1, MX>(x, rows, cols, xs, n, to, s);
    }
    if (cols <= 256) return norm_of<T, 32, 1, MX>(x, rows, cols, xs, n, to, s);
    if (cols <= 512) return norm_of<T, 64, 1, MX>(x, rows, cols, xs, n, to, s);
    if (cols <= 1024) return norm_of<T, 64, 2, MX>(x, rows, cols, xs, n, to, s);
    if (cols <= 1536) return norm_of<T, 64, 3, MX>(x, rows, cols, xs, n, to, s);
    if (cols <= kWaveCols) return norm_of<T, 64, 4, MX>(x, rows, cols, xs, n, to, s);
    // Codes of somewhat longer rows by a wave each, where there are many.  By a wave and by two, us, for 1100, 1500, 1800, 3000, 8192, 20000 rows:
    //   2100 columns bf16  6.9 6.7  7.1 6.8  7.2  9.7  12.3 12.5  22.0 26.3  41.8 51.6   fp32  6.0 5.8  6.7 6.1  6.7 8.4  11.3 12.1  19.9 22.8  47.8 50.6
    //   2560               6.2 6.0  6.3 6.1  6.6  8.2  11.0 11.3  18.4 21.4  34.9 42.6         5.8 5.6  6.2 6.2  7.3 8.6  11.6 11.6  19.9 22.1  51.2 53.7
    //   2600               7.1 6.2  7.2 6.4  7.5  8.8  12.7 11.9  21.2 22.2  38.6 44.2         6.4 5.8  7.1 6.6  7.8 9.0  12.7 12.3  21.3 23.0  54.6 55.2
    //   3000               7.1 6.2  7.3 6.5  7.6  9.0  13.5 12.3  21.8 22.4  44.4 46.4         6.9 6.1  7.7 7.2  8.5 9.5  13.2 12.6  22.4 24.2  60.1 60.0
    // (Dense rows gain nothing by it: 8192 x 2304 bf16 18.2 by two waves, 19.2 by one.)
    if constexpr (MX) {
        if (rows > 1536 && cols <= 2560) return norm_of<T, 64, 5, MX>(x, rows, cols, xs, n, to, s);
        if (rows > 1536 && cols <= 3072) return norm_of<T, 64, 6, MX>(x, rows, cols, xs, n, to, s);
    }
    if (rows <= 256) {                                           // no more than a row a compute unit: all the threads it can use
        if (cols <= 4096) return norm_of<T, 512, 1, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= 8192) return norm_of<T, 1024, 1, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= kGroupCols) return norm_of<T, 1024, 2, MX>(x, rows, cols, xs, n, to, s);
    } else {
        if (cols <= 3072) return norm_of<T, 128, 3, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= 4096) return norm_of<T, 128, 4, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= 6144) return norm_of<T, 256, 3, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= 8192) return norm_of<T, 256, 4, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= 12288) return norm_of<T, 512, 3, MX>(x, rows, cols, xs, n, to, s);
        if (cols <= kGroupCols) return norm_of<T, 512, 4, MX>(x, rows, cols, xs, n, to, s);
    }
    return in_parts(rows, 1024, [&](int64_t first, int64_t count) {        // parts of 2^21 rows: whole groups of 32 rows' scales
        NormArgs of = n;
        if (of.mean) of.mean += first;
        if (of.rstd) of.rstd += first;
        NormOut there = to;
        if (to.y) there.y = static_cast<uint8_t*>(to.y) + (MX ? first * (to.stride_or_chunks * 128) : first * to.stride_or_chunks * (int64_t)sizeof(T));
        if (MX && to.y) there.scales = to.scales + first / 32 * (to.stride_or_chunks * 256);
        return launch(norm_long_rows_kernel<T, MX>, dim3((uint32_t)count), dim3(1024), s, static_cast<const T*>(x) + first * xs, cols, xs, of, there);
    });
}

// Threads that share a row of the backward pass, runs of four columns a thread, rows that a workgroup takes at a time (as many as
// their registers allow; with few rows the workgroups are smaller, so that there are more of them), workgroups, each of which
// leaves a row of partial sums.
struct BackwardShape { int32_t threads, runs, rows; };
inline BackwardShape backward_shape(int64_t rows, int64_t cols)
{
    int32_t threads = cols <= 64 ? 16 : cols <= 128 ? 32 : cols <= kWaveCols ? 64 : cols <= 4096 ? 256 : 1024;
    int32_t runs = (int32_t)((cols + threads * 4 - 1) / (threads * 4));
    if (threads == 64 && runs > 4) runs = runs > 6 ? 8 : 6;
    else if (threads == 256) runs = 4;
    const int32_t most = threads == 64 && runs > 4 ? 512 : runs == 4 ? 768 : 1024;
    const bool few = rows * threads <= 128 * 1024 && threads <= 256;
    return BackwardShape{threads, runs, threads == 1024 ? 1 : (few ? 256 : most) / threads};
}
inline int64_t backward_groups(int64_t rows, int64_t cols)
{
    const int64_t each = backward_shape(rows, cols).rows, groups = (rows + each - 1) / each;
    return groups < kMostParts ? groups : kMostParts;
}

template <typename T, typename G, int THREADS, int NV, int ROWS>
hipError_t backward_of(const NormBackwardArgs& a, int64_t groups, hipStream_t s)
{
    return launch(norm_backward_kernel<T, G, THREADS, NV, ROWS>, dim3((uint32_t)groups), dim3(THREADS * ROWS), s, a);
}
template <typename T, typename G>
hipError_t backward_any(const NormBackwardArgs& a, int64_t* parts, hipStream_t s)
{
    const int64_t groups = a.groups;
    *parts = groups;
    if (a.cols <= kGroupCols) {
        const BackwardShape b = backward_shape(a.rows, a.cols);
        const bool few = b.threads * b.rows == 256;
        switch (b.threads * 16 + b.runs) {
            case 16 * 16 + 1: return few ? backward_of<T, G, 16, 1, 16>(a, groups, s) : backward_of<T, G, 16, 1, 64>(a, groups, s);
            case 32 * 16 + 1: return few ? backward_of<T, G, 32, 1, 8>(a, groups, s) : backward_of<T, G, 32, 1, 32>(a, groups, s);
            case 64 * 16 + 1: return few ? backward_of<T, G, 64, 1, 4>(a, groups, s) : backward_of<T, G, 64, 1, 16>(a, groups, s);
            case 64 * 16 + 2: return few ? backward_of<T, G, 64, 2, 4>(a, groups, s) : backward_of<T, G, 64, 2, 16>(a, groups, s);
            case 64 * 16 + 3: return few ? backward_of<T, G, 64, 3, 4>(a, groups, s) : backward_of<T, G, 64, 3, 16>(a, groups, s);
            case 64 * 16 + 4: return few ? backward_of<T, G, 64, 4, 4>(a, groups, s) : backward_of<T, G, 64, 4, 12>(a, groups, s);
            case 64 * 16 + 6: return few ? backward_of<T, G, 64, 6, 4>(a, groups, s) : backward_of<T, G, 64, 6, 8>(a, groups, s);
            case 64 * 16 + 8: return few ? backward_of<T, G, 64, 8, 4>(a, groups, s) : backward_of<T, G, 64, 8, 8>(a, groups, s);
            case 256 * 16 + 4: return few ? backward_of<T, G, 256, 4, 1>(a, groups, s) : backward_of<T, G, 256, 4, 3>(a, groups, s);
            case 1024 * 16 + 2: return backward_of<T, G, 1024, 2, 1>(a, groups, s);
            case 1024 * 16 + 3: return backward_of<T, G, 1024, 3, 1>(a, groups, s);
            default: return backward_of<T, G, 1024, 4, 1>(a, groups, s);
        }
    }
    if (a.partial) {                                             // first: dx may be dy itself
        const int64_t each = (a.rows + groups - 1) / groups, col_groups = (a.cols + 2047) / 2048;
        *parts = (a.rows + each - 1) / each;
        const hipError_t e = launch(norm_column_sums_kernel<T, G>, dim3((uint32_t)(col_groups * *parts)), dim3(256), s, a, each, (uint32_t)col_groups);
        if (e != hipSuccess) return e;
    }
    if (!a.dx) return hipSuccess;
    return in_parts(a.rows, 1024, [&](int64_t first, int64_t count) {
        NormBackwardArgs of = a;
        of.x = static_cast<const T*>(a.x) + first * a.x_stride;
        of.dy = static_cast<const G*>(a.dy) + first * a.dy_stride;
        of.dx = static_cast<T*>(a.dx) + first * a.dx_stride;
        of.mean += first;
        of.rstd += first;
        return launch(norm_backward_long_rows_kernel<T, G>, dim3((uint32_t)count), dim3(1024), s, of);
    });
}
bool norm_shape_ok(int64_t rows, int64_t cols) { return mx_shape_ok(rows, cols) && cols >= 1; }

}  // namespace

hipError_t launch_join(const float* partial, int64_t parts, int64_t cols, int32_t count, int32_t p_dtype, void* first, void* second, hipStream_t s)
{
    return in_parts((cols + 63) / 64 * count, 1024, [&](int64_t begin, int64_t groups) {
        const dim3 grid((uint32_t)groups), block(1024);
        const uint32_t b = (uint32_t)begin;
        if (p_dtype == FH_F32) return launch(norm_join_kernel<float>, grid, block, s, partial, parts, cols, count, static_cast<float*>(first), static_cast<float*>(second), b);
        return launch(norm_join_kernel<Bf16>, grid, block, s, partial, parts, cols, count, static_cast<Bf16*>(first), static_cast<Bf16*>(second), b);
    });
}

// Rows of which 32 fit in LDS, and no more threads than a launch may have (2^32).
bool norm_blocks_fit(int32_t dtype, int64_t rows, int64_t cols) { return cols <= (dtype == FH_F32 ? 1024 : 2048) && mx_chunks(rows) < (1 << 19); }

hipError_t launch_norm_blocks(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t x_stride, const NormArgs& n, void* by_rows,
                              void* by_columns, hipStream_t s)
{
    const auto of = [&](auto kernel, auto typed) {
        return launch(kernel, dim3((uint32_t)(mx_chunks(rows) * 8)), dim3(1024), s, typed, rows, cols, x_stride, n, static_cast<uint8_t*>(by_rows),
                      static_cast<uint8_t*>(by_columns));
    };
    if (dtype == FH_F32) {
        const float* p = static_cast<const float*>(x);
        return cols <= 256 ? of(norm_blocks_kernel<float, 32, 1>, p) : cols <= 512 ? of(norm_blocks_kernel<float, 64, 1>, p) : of(norm_blocks_kernel<float, 64, 2>, p);
    }
    const Bf16* p = static_cast<const Bf16*>(x);
    return cols <= 256 ? of(norm_blocks_kernel<Bf16, 32, 1>, p) : cols <= 512 ? of(norm_blocks_kernel<Bf16, 64, 1>, p)
         : cols <= 1024 ? of(norm_blocks_kernel<Bf16, 64, 2>, p) : cols <= 1536 ? of(norm_blocks_kernel<Bf16, 64, 3>, p) : of(norm_blocks_kernel<Bf16, 64, 4>, p);
}

hipError_t launch_layer_norm(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t xs, const NormArgs& n, void* y, int64_t ys,
                             void* codes, hipStream_t s)
{
    if (codes) {
        const MxStore m = mx_store(codes, rows, cols);
        const NormOut to = {m.codes, m.scales, m.chunks};
        return dtype == FH_F32 ? norm_any<float, true>(x, rows, cols, xs, n, to, s) : norm_any<Bf16, true>(x, rows, cols, xs, n, to, s);
    }
    const NormOut to = {y, nullptr, ys};
    return dtype == FH_F32 ? norm_any<float, false>(x, rows, cols, xs, n, to, s) : norm_any<Bf16, false>(x, rows, cols, xs, n, to, s);
}

fh_status norm_backward(const fh_norm_backward& b, int32_t dy_dtype, hipStream_t s)
{
    if (!is_dtype(b.dtype) || !is_dtype(b.p_dtype) || (dy_dtype != b.dtype && dy_dtype != FH_F32)) return FH_ERR_BAD_DTYPE;
    if (!norm_shape_ok(b.rows, b.cols) || b.dy_stride < b.cols || b.x_stride < b.cols || b.dx_stride < b.cols ||
        b.dy_stride > kMostStride || b.x_stride > kMostStride || b.dx_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    const bool sums = b.dweight || b.dbias;
    if (b.rows > 0 && (!b.dy || !b.x || !b.mean || !b.rstd)) return FH_ERR_NULL;
    const size_t size = dtype_size(b.dtype), p_size = dtype_size(b.p_dtype);
    if (!is_aligned(b.dy, dtype_size(dy_dtype)) || !is_aligned(b.x, size) || !is_aligned(b.dx, size) || !is_aligned(b.weight, p_size) ||
        !is_aligned(b.dweight, p_size) || !is_aligned(b.dbias, p_size) || !is_aligned(b.mean, 4) || !is_aligned(b.rstd, 4) ||
        !is_aligned(b.workspace, 16)) return FH_ERR_ALIGNMENT;
    if (b.dx && b.dx_cap < strided_elements(b.rows, b.cols, b.dx_stride) * size) return FH_ERR_BUFFER_TOO_SMALL;
    if (sums && b.rows > 0) {
        if (!b.workspace) return FH_ERR_NULL;
        if (b.workspace_cap < fh_layer_norm_backward_workspace_bytes(b.rows, b.cols)) return FH_ERR_BUFFER_TOO_SMALL;
    }
    float* partial = sums ? static_cast<float*>(b.workspace) : nullptr;
    int64_t parts = 0;
    if (b.rows > 0 && (b.dx || sums)) {
        const NormBackwardArgs a = {b.dy, b.x, static_cast<const float*>(b.mean), static_cast<const float*>(b.rstd), b.weight, b.dx, partial,
                                    b.dy_stride, b.x_stride, b.dx_stride, b.rows, b.cols, b.p_dtype,
                                    (int32_t)backward_groups(b.rows, b.cols)};
        const hipError_t e = b.dtype == FH_F32 ? backward_any<float, float>(a, &parts, s)
                           : dy_dtype == FH_F32 ? backward_any<Bf16, float>(a, &parts, s) : backward_any<Bf16, Bf16>(a, &parts, s);
        if (e != hipSuccess) return FH_ERR_LAUNCH;
    }
    if (!sums) return FH_OK;                                     // no rows: sums of nothing, which are written all the same
    return launch_join(partial, parts, b.cols, 2, b.p_dtype, b.dweight, b.dbias, s) == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

}  // namespace fh

extern "C" {

fh_status fh_layer_norm(const void* x, fh_dtype dtype, int64_t rows, int64_t cols, int64_t x_stride, const void* weight, const void* bias,
                        fh_dtype p_dtype, float eps, void* y, int64_t y_stride, size_t y_cap, void* mean, void* rstd, void* stream)
{
    using namespace fh;
    if (!is_dtype(dtype) || !is_dtype(p_dtype)) return FH_ERR_BAD_DTYPE;
    if (!norm_shape_ok(rows, cols) || x_stride < cols || y_stride < cols || x_stride > kMostStride || y_stride > kMostStride)
        return FH_ERR_BAD_SHAPE;
    if (!(eps >= 0.0f)) return FH_ERR_BAD_PARAM;
    if (rows == 0) return FH_OK;
    if (!x || !y) return FH_ERR_NULL;
    if (!is_aligned(x, dtype_size(dtype)) || !is_aligned(y, dtype_size(dtype)) || !is_aligned(weight, dtype_size(p_dtype)) ||
        !is_aligned(bias, dtype_size(p_dtype)) || !is_aligned(mean, 4) || !is_aligned(rstd, 4)) return FH_ERR_ALIGNMENT;
    if (y_cap < strided_elements(rows, cols, y_stride) * dtype_size(dtype)) return FH_ERR_BUFFER_TOO_SMALL;
    const NormArgs n = {weight, bias, p_dtype, eps, static_cast<float*>(mean), static_cast<float*>(rstd)};
    return launch_layer_norm(x, dtype, rows, cols, x_stride, n, y, y_stride, nullptr, static_cast<hipStream_t>(stream)) == hipSuccess
               ? FH_OK : FH_ERR_LAUNCH;
}

size_t fh_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    if (!fh::norm_shape_ok(rows, cols)) return 0;
    return (size_t)fh::backward_groups(rows, cols) * 2u * (size_t)cols * 4u;
}

fh_status fh_layer_norm_backward(const fh_norm_backward* b, void* stream)
{
    return b ? fh::norm_backward(*b, b->dtype, static_cast<hipStream_t>(stream)) : FH_ERR_NULL;
}

}  // extern "C"
