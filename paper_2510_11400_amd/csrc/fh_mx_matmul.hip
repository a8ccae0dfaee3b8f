// The product of two microscaled matrices: out[i][j] = sum_k A[i][k] B[j][k] + bias[j].
#include "fh_matrix.hpp"
#include "fh_mx_plan.hpp"

namespace fh {
namespace {

constexpr int64_t kMostSummed = (int64_t)1 << 24;   // a row's codes are addressed with 32 bits

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
    const uint8_t *a, *a_scales;       // m rows
    const uint8_t *b, *b_scales;       // n rows
    int64_t        m, n;
    const void*    bias;               // may be null
    void*          out;                // parts > 1: float [parts][m][n]
    int64_t        stride;
    int32_t        chunks;             // of the rows of both
    int32_t        chunks_each;        // of a workgroup's part of the sum
    int32_t        parts;              // workgroups that share a tile's sum
    int32_t        bias_dtype;
    uint32_t       m_tiles, n_tiles;
    uint32_t       step;               // from a workgroup's tile to its next one
    uint32_t       first;              // workgroup of the launches before this one
};
static_assert(sizeof(ProductArgs) <= 112, "longer arguments are enqueued a microsecond later");

// v_mfma_scale_f32_32x32x64_f8f6f4: lane (r = lane % 32, h = lane / 32) brings 32 values of row r of each operand, and gets
// the outputs [8 (i/4) + 4 h + i % 4][r].  Of a chunk's
// eight blocks a lane takes 4h .. 4h+3, in four instructions, whose scales are the bytes of one word.  From registers alone it measured 5.3 to 5.7 PFLOP/s on
// operands of all kinds (7.2 on zeros), the 16 x 16 x 128 form 6.8 to 7.1 (8.8) with eight accumulators; the kernels have not been built on that one.
template <int BYTE>
__device__ __forceinline__ f32x16 mx_mfma32(u32x4 a, u32x4 b, uint32_t sa, uint32_t sb, f32x16 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
}

// ---- few tiles: the sum split over a workgroup's waves, through LDS --------------------------------
// (32 MT) x (32 NT) outputs a workgroup; each wave multiplies a run of chunks by itself, with an area of LDS of its own and no barrier:
// a chunk's rows come as whole lines into the area, from there to registers, and while those are multiplied the next chunk's
// come.  The waves' sums are joined in LDS in the waves' order.
template <typename T, int MT, int NT, int WAVES, bool RUNS>
__global__ __launch_bounds__(WAVES * 64) void mx_waves_kernel(ProductArgs p)
{
    constexpr int kRowsA = MT * 32, kRowsB = NT * 32, kPad = kRowsB + 4;
    constexpr uint32_t kCodes = (kRowsA + kRowsB) * 128, kScales = (kRowsA + kRowsB) * 8;
    constexpr uint32_t kSums = kRowsA * kPad * 4, kArea = kCodes + kScales > kSums ? kCodes + kScales : kSums;
    static_assert(kScales <= 1024, "one load brings the scales");
    __shared__ __attribute__((aligned(16))) uint8_t s_area[WAVES * kArea];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles = p.m_tiles * p.n_tiles, number = p.first + blockIdx.x, part = RUNS ? 0 : number / tiles;
    uint32_t i, j;
    if constexpr (RUNS) {                                        // 0.2 us of divisions in a row: where it pays
        in_bands(run_of(number, tiles), p.m_tiles, p.n_tiles, i, j);
    } else {
        const uint32_t tile = number - part * tiles;
        i = tile / p.n_tiles;
        j = tile % p.n_tiles;
    }
    const int64_t i0 = (int64_t)i * kRowsA, j0 = (int64_t)j * kRowsB;
    const uint32_t pitch = (uint32_t)p.chunks * 128, scale_pitch = (uint32_t)p.chunks * 256;
    // rows past the last are the last one, so that every address is inside
    const int rows_a = (int)(p.m - i0 < kRowsA ? p.m - i0 : kRowsA), rows_b = (int)(p.n - j0 < kRowsB ? p.n - j0 : kRowsB);
    const u32x4 from_a = buffer_of(p.a + i0 * pitch, rows_a * pitch), from_b = buffer_of(p.b + j0 * pitch, rows_b * pitch);
    const uint32_t piece = ((lane & 7) ^ (lane >> 4)) * 16;      // turned by half the row's number, 4 more for every other eight rows
    uint32_t at_a[MT * 4], at_b[NT * 4];
#pragma unroll
    for (int t = 0; t < MT * 4; ++t) {
        const int r = t * 8 + (lane >> 3);
        at_a[t] = (r < rows_a ? r : rows_a - 1) * pitch + (piece ^ (t & 1) * 64);
    }
#pragma unroll
    for (int t = 0; t < NT * 4; ++t) {
        const int r = t * 8 + (lane >> 3);
        at_b[t] = (r < rows_b ? r : rows_b - 1) * pitch + (piece ^ (t & 1) * 64);
    }
    const uint32_t groups_a = (rows_a + 31) / 32, groups_b = (rows_b + 31) / 32;
    const u32x4 from_sa = buffer_of(p.a_scales + (i0 >> 5) * scale_pitch, groups_a * scale_pitch);
    const u32x4 from_sb = buffer_of(p.b_scales + (j0 >> 5) * scale_pitch, groups_b * scale_pitch);
    const uint32_t group = lane >> 4, group_b = group - MT;
    const bool of_a = group < MT, of_b = !of_a && group_b < NT;
    const uint32_t at_scales = (of_a ? (group < groups_a ? group : groups_a - 1) : (group_b < groups_b ? group_b : groups_b - 1)) * scale_pitch + (lane & 15) * 16;
    uint8_t* area = s_area + wave * kArea;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_area + wave * kArea;
    auto load = [&](uint32_t chunk) {
        if (of_a) to_lds(lds + kCodes, from_sa, at_scales, chunk * 256);
        if (of_b) to_lds(lds + kCodes, from_sb, at_scales, chunk * 256);
#pragma unroll
        for (int t = 0; t < MT * 4; ++t) to_lds(lds + t * 1024, from_a, at_a[t], chunk * 128);
#pragma unroll
        for (int t = 0; t < NT * 4; ++t) to_lds(lds + kRowsA * 128 + t * 1024, from_b, at_b[t], chunk * 128);
    };
    const int h = lane >> 5, r = lane & 31, turned = (h * 4) ^ (lane >> 1 & 7);
    const uint32_t chunks = (uint32_t)p.chunks, begin = part * (uint32_t)p.chunks_each;
    const uint32_t end = begin + (uint32_t)p.chunks_each < chunks ? begin + (uint32_t)p.chunks_each : chunks;
    f32x16 c[MT][NT] = {};
    uint32_t k = begin + wave;
    if (k < end) load(k);
    while (k < end) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        u32x4 fa[4][MT], fb[4][NT];
        uint32_t sa[MT], sb[NT];
#pragma unroll
        for (int t = 0; t < MT; ++t) sa[t] = *reinterpret_cast<const uint32_t*>(area + kCodes + t * 256 + h * 128 + r * 4);
#pragma unroll
        for (int t = 0; t < NT; ++t) sb[t] = *reinterpret_cast<const uint32_t*>(area + kCodes + (MT + t) * 256 + h * 128 + r * 4);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint8_t* from = area + (uint32_t)(turned ^ q) * 16 + r * 128;
#pragma unroll
            for (int t = 0; t < NT; ++t) fb[q][t] = *reinterpret_cast<const u32x4*>(from + kRowsA * 128 + t * 4096);
#pragma unroll
            for (int t = 0; t < MT; ++t) fa[q][t] = *reinterpret_cast<const u32x4*>(from + t * 4096);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the area may be written again
        k += WAVES;
        if (k < end) load(k);
#define FH_QUARTER(Q)                                                                                             \
        _Pragma("unroll") for (int x = 0; x < MT; ++x) _Pragma("unroll") for (int y = 0; y < NT; ++y)             \
            c[x][y] = mx_mfma32<Q>(fb[Q][y], fa[Q][x], sb[y], sa[x], c[x][y]);
        FH_QUARTER(0) FH_QUARTER(1) FH_QUARTER(2) FH_QUARTER(3)
#undef FH_QUARTER
    }
    // this wave's area is its own still
#pragma unroll
    for (int x = 0; x < MT; ++x)
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(area + ((x * 32 + r) * kPad + y * 32 + 2 * i + 4 * h) * 4) = f32x4{c[x][y][i], c[x][y][i + 1], c[x][y][i + 2], c[x][y][i + 3]};
    __syncthreads();
    for (int at = threadIdx.x; at < kRowsA * kRowsB / 4; at += WAVES * 64) {
        const int row = at / (kRowsB / 4), col = at % (kRowsB / 4) * 4;
        f32x4 sum = *reinterpret_cast<const f32x4*>(s_area + (row * kPad + col) * 4);
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += *reinterpret_cast<const f32x4*>(s_area + w * kArea + (row * kPad + col) * 4);
        const int64_t i = i0 + row, j = j0 + col;
        if (i >= p.m) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum[e] + (j + e < p.n ? parameter(p.bias, p.bias_dtype, j + e, 0.0f) : 0.0f);
        store4(static_cast<T*>(p.out) + (int64_t)part * p.m * p.n + i * p.stride + j, p.n - j, v);
    }
}

// ---- large products: tiles through LDS ----------------------------------------------------------
// B x B outputs of a tile, a chunk of 256 summed values at a time; a workgroup of 2 x WN waves, each with B/2 x 64 outputs, takes one
// tile after another.  Two stages of LDS: while one is multiplied the next is on its way, and a stage is handed over before its last
// quarter, which is in registers by then, so that the matrix unit works across the barrier.  A row's eight pieces of 16 bytes
// are turned by half the row's number (the loads take them from turned addresses), so that sixteen lanes reading the same
// piece of sixteen rows meet all 64 banks.
// The chunks of the next tile follow those of the last without a gap.  A wave's outputs are turned into rows in the part of the free stage that
// the wave itself loads, so it needs no barrier before it loads there again; that load is sent before the outputs are, because
// memory operations are counted in their order and the next wait is for the load alone.
template <typename T, int B, int WN>
__global__ __launch_bounds__(2 * WN * 64, B > 128 ? 1 : 2) void mx_tile_kernel(ProductArgs p)
{
    constexpr int kWaves = 2 * WN, kHalf = kWaves / 2, MT = B / 64, NT = 2;
    constexpr uint32_t kCodes = 2 * B * 128, kStage = kCodes + 2 * B * 8;
    constexpr int kRun = 16 / sizeof(T), kLanes = 64 / kRun, kRows = 64 / kLanes, kStores = MT * 32 / kRows;
    static_assert(kHalf * 64 == B && WN * 64 == B, "a wave loads 64 rows of one operand, and has 64 columns");
    __shared__ __attribute__((aligned(16))) uint8_t s_stage[2 * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;

    const uint32_t tiles = p.m_tiles * p.n_tiles, xcd = blockIdx.x & 7;
    const uint32_t end_tile = run_of(xcd, tiles) + (tiles >> 3) + (xcd < (tiles & 7) ? 1 : 0);
    const auto corner = [&](uint32_t tile, int64_t& i0, int64_t& j0) {
        uint32_t i, j;
        in_bands(tile, p.m_tiles, p.n_tiles, i, j);
        i0 = (int64_t)i * B;
        j0 = (int64_t)j * B;
    };

    // what is loaded next: a chunk of a tile, in this wave 64 rows of one operand and with it maybe the scales of 128
    const bool of_b = wave >= kHalf, loads_scales = wave % kHalf < kHalf / 2;
    const int part = wave % kHalf;
    const uint32_t pitch = (uint32_t)p.chunks * 128, scale_pitch = (uint32_t)p.chunks * 256, end = (uint32_t)p.chunks;
    uint32_t next_tile = run_of(blockIdx.x, tiles), next_chunk = 0;
    u32x4 from, from_scales;
    const uint32_t at = (part * 64 + (lane >> 3)) * pitch + ((lane & 7) ^ (lane >> 4)) * 16, at_scales = (part * 4 + (lane >> 4)) * scale_pitch + (lane & 15) * 16;
    const auto aim = [&]() {
        int64_t i0, j0;
        corner(next_tile, i0, j0);
        const int64_t row0 = of_b ? j0 : i0, left = (of_b ? p.n : p.m) - row0;
        const int rows = left < B ? (int)left : B, groups = (rows + 31) / 32;
        // rows past the last are past the buffer's end: nothing is read for them, and nothing of theirs is stored
        from = buffer_of((of_b ? p.b : p.a) + row0 * pitch, (uint32_t)rows * pitch);
        from_scales = buffer_of((of_b ? p.b_scales : p.a_scales) + (row0 >> 5) * scale_pitch, (uint32_t)groups * scale_pitch);
    };
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_stage;
    const uint32_t lds_scales = kCodes + (of_b ? B * 8 : 0) + part * 1024;
    const auto load = [&](uint32_t stage) {
        if (next_tile >= end_tile) return;
        if (loads_scales) to_lds(lds + stage + lds_scales, from_scales, at_scales, next_chunk * 256);
        uint32_t row_at = at;
        asm("" : "+v"(row_at));                                  // seven sums made here, not seven registers kept
#pragma unroll
        for (int t = 0; t < 8; ++t) to_lds(lds + stage + wave * 8192 + t * 1024, from, (row_at ^ (t & 1) * 64) + t * 8 * pitch, next_chunk * 128);
        if (++next_chunk == end) {
            next_chunk = 0;
            next_tile += p.step;
            if (next_tile < end_tile) aim();
        }
    };

    const int h = lane >> 5, r = lane & 31, turned = (h * 4) ^ (lane >> 1 & 7);
    const uint32_t read_a = (wm * MT * 32 + r) * 128, read_b = B * 128 + (wn * NT * 32 + r) * 128;
    const uint32_t read_sa = kCodes + wm * MT * 256 + h * 128 + r * 4, read_sb = kCodes + B * 8 + wn * NT * 256 + h * 128 + r * 4;
    u32x4 fa[2][MT], fb[2][NT];
    uint32_t sa[MT], sb[NT], next_sa[MT], next_sb[NT];
    const auto read = [&](uint32_t stage, int quarter, int to) {
        const uint8_t* at_piece = s_stage + stage + (uint32_t)(turned ^ quarter) * 16;
#pragma unroll
        for (int t = 0; t < MT; ++t) fa[to][t] = *reinterpret_cast<const u32x4*>(at_piece + read_a + t * 4096);
#pragma unroll
        for (int t = 0; t < NT; ++t) fb[to][t] = *reinterpret_cast<const u32x4*>(at_piece + read_b + t * 4096);
    };
    const auto read_scales = [&](uint32_t stage, uint32_t (&ua)[MT], uint32_t (&ub)[NT]) {
#pragma unroll
        for (int t = 0; t < MT; ++t) ua[t] = *reinterpret_cast<const uint32_t*>(s_stage + stage + read_sa + t * 256);
#pragma unroll
        for (int t = 0; t < NT; ++t) ub[t] = *reinterpret_cast<const uint32_t*>(s_stage + stage + read_sb + t * 256);
    };
    // Outputs run along b's rows within a lane.  A read of LDS goes with every two matrix instructions.
#define FH_QUARTER(Q, WHICH)                                                                                      \
    _Pragma("unroll") for (int x = 0; x < MT; ++x) _Pragma("unroll") for (int y = 0; y < NT; ++y)                 \
        c[x][y] = mx_mfma32<Q>(fb[WHICH][y], fa[WHICH][x], sb[y], sa[x], c[x][y]);                                \
    _Pragma("unroll") for (int z = 0; z < MT + NT; ++z) {                                                         \
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                                                        \
        __builtin_amdgcn_sched_group_barrier(0x008, MT * NT / (MT + NT), 0);                                      \
    }
    uint32_t tile = next_tile, stage = 0;
    bool behind = false;                                         // outputs were sent after the load that is waited for
    aim();
    load(0);
    if (next_tile < end_tile) {
        load(kStage);
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");         // the first stage's are older
    } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    read(stage, 0, 0);
    read_scales(stage, sa, sb);
    T* out = static_cast<T*>(p.out);
#pragma clang loop unroll(disable)
    for (; tile < end_tile; tile += p.step) {
        int64_t i0, j0;
        corner(tile, i0, j0);
        float bias_here = 0.0f;
        f32x16 c[MT][NT] = {};
#pragma clang loop unroll(disable)
        for (uint32_t k = 0; k < end; ++k) {
            if (k + 1 == end && p.bias) {
                const int64_t j = j0 + wn * 64 + lane;
                bias_here = parameter(p.bias, p.bias_dtype, j < p.n ? j : p.n - 1, 0.0f);
            }
            read(stage, 1, 1);
            FH_QUARTER(0, 0)
            read(stage, 2, 0);
            FH_QUARTER(1, 1)
            read(stage, 3, 1);
            FH_QUARTER(2, 0)
            // this wave has read all of this stage, and its part of the next has arrived
            if (behind) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(kStores) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            behind = false;
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (k + 1 < end) load(stage);
            stage = kStage - stage;
            read(stage, 0, 0);                                   // after the last chunk: of no use, and inside
            read_scales(stage, next_sa, next_sb);
            FH_QUARTER(3, 1)
#pragma unroll
            for (int t = 0; t < MT; ++t) sa[t] = next_sa[t];
#pragma unroll
            for (int t = 0; t < NT; ++t) sb[t] = next_sb[t];
        }

        // 32 rows at a time through this wave's 8 KiB of the stage that is free, to runs of 16 bytes a lane
        int l = lane;
        asm("" : "+v"(l));                                       // what is worked out from it is not kept in registers meanwhile
        const int mine = l / kLanes, piece = l % kLanes, row32 = l & 31, half = l >> 5;
        uint8_t* s_out = s_stage + (kStage - stage) + wave * 8192;
        if (p.bias) {
#pragma unroll
            for (int y = 0; y < NT; ++y)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float b = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute((y * 32 + i / 4 * 8 + half * 4 + i % 4) * 4, __builtin_bit_cast(int, bias_here)));
#pragma unroll
                    for (int x = 0; x < MT; ++x) c[x][y][i] += b;
                }
        }
        u32x4 v[kStores];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
#pragma unroll
            for (int y = 0; y < NT; ++y)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x16& o = c[x][y];
                    if constexpr (sizeof(T) == 2) {              // rows of 128 bytes; the upper sixteen have the halves of a piece exchanged
                        const uint32_t at_piece = (uint32_t)((y * 4 + i) ^ (row32 >> 1 & 7)) * 16 + (uint32_t)(half ^ row32 >> 4) * 8;
                        *reinterpret_cast<u32x2*>(s_out + row32 * 128 + at_piece) = u32x2{bf16_pair(o[4 * i], o[4 * i + 1]), bf16_pair(o[4 * i + 2], o[4 * i + 3])};
                    } else {
                        const uint32_t at_piece = (uint32_t)((y * 8 + 2 * i + half) ^ (row32 & 15)) * 16;
                        *reinterpret_cast<f32x4*>(s_out + row32 * 256 + at_piece) = f32x4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
                    }
                }
            asm volatile("" ::: "memory");                       // a wave's own LDS accesses are in order
#pragma unroll
            for (int t = 0; t < 32 / kRows; ++t) {
                const int from_row = t * kRows + mine;
                const uint32_t turn = sizeof(T) == 2 ? from_row >> 1 & 7 : from_row & 15;
                const u32x4 w = *reinterpret_cast<const u32x4*>(s_out + from_row * (kLanes * 16) + (piece ^ turn) * 16);
                v[x * (32 / kRows) + t] = sizeof(T) == 2 && t * kRows >= 16 ? u32x4{w.z, w.w, w.x, w.y} : w;
            }
            asm volatile("" ::: "memory");
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load(kStage - stage);
        const int64_t row = i0 + wm * MT * 32 + mine, col = j0 + wn * 64 + piece * kRun;
        T* to = out + row * p.stride + col;
        if (i0 + B <= p.m && j0 + B <= p.n) {
#pragma unroll
            for (int t = 0; t < kStores; ++t) *reinterpret_cast<u32x4_a2*>(to + (int64_t)(t * kRows) * p.stride) = v[t];
            behind = true;
        } else {
            const int rows = p.m - row < B ? (int)(p.m - row) : B, cols = p.n - col < kRun ? (int)(p.n - col) : kRun;
#pragma unroll
            for (int t = 0; t < kStores; ++t) {
                int some = t * kRows < rows ? cols : 0;
                asm("" : "+v"(some));                            // its masks are not kept in registers either
                store_packed(to + (int64_t)(t * kRows) * p.stride, some, v[t]);
            }
        }
    }
#undef FH_QUARTER
}

// The parts of a split sum added up in their order.
template <typename T>
__global__ __launch_bounds__(256) void mx_join_kernel(const float* parts, int64_t m, int64_t n, int32_t count, const void* bias, int32_t bias_dtype,
                                                      T* out, int64_t stride, uint32_t runs)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / runs, col = (at - row * runs) * 4;
    if (row >= m) return;
    float v[4] = {};
    for (int32_t k = 0; k < count; ++k) {
        const float* from = parts + ((int64_t)k * m + row) * n + col;
        if (col + 4 <= n) {
            const f32x4 w = *reinterpret_cast<const f32x4_a4*>(from);
            for (int i = 0; i < 4; ++i) v[i] += w[i];
        } else {
            for (int i = 0; i < 4; ++i) if (col + i < n) v[i] += from[i];
        }
    }
    for (int i = 0; i < 4; ++i)
        if (col + i < n) store1(out + row * stride + col + i, v[i] + parameter(bias, bias_dtype, col + i, 0.0f));
}

// ---- launches -----------------------------------------------------------------------------------
template <typename T, int MT, int NT, int WAVES, bool RUNS = false>
hipError_t waves_of(ProductArgs p, hipStream_t s)
{
    const int64_t m_tiles = (p.m + MT * 32 - 1) / (MT * 32), n_tiles = (p.n + NT * 32 - 1) / (NT * 32), groups = m_tiles * n_tiles * p.parts;
    if (groups > INT32_MAX) return hipErrorInvalidValue;
    p.m_tiles = (uint32_t)m_tiles;
    p.n_tiles = (uint32_t)n_tiles;
    return in_parts(groups, WAVES * 64, [&](int64_t first, int64_t count) {
        p.first = (uint32_t)first;
        return launch(mx_waves_kernel<T, MT, NT, WAVES, RUNS>, dim3((uint32_t)count), dim3(WAVES * 64), s, p);
    });
}
template <typename T, int B, int WN>
hipError_t squares_of(ProductArgs p, hipStream_t s)
{
    const int64_t m_tiles = (p.m + B - 1) / B, n_tiles = (p.n + B - 1) / B;
    if (m_tiles * n_tiles * 8 > INT32_MAX) return hipErrorInvalidValue;
    const int64_t groups = B > 128 ? 256 : 512;                  // what the card holds at a time
    p.m_tiles = (uint32_t)m_tiles;
    p.n_tiles = (uint32_t)n_tiles;
    const uint32_t grid = (uint32_t)(m_tiles * n_tiles < groups ? m_tiles * n_tiles : groups);
    p.step = (grid + 7) / 8;
    return launch(mx_tile_kernel<T, B, WN>, dim3(grid), dim3(2 * WN * 64), s, p);
}
template <typename T>
hipError_t product_of(const ProductArgs& p, const Plan& plan, float* workspace, hipStream_t s)
{
    switch (plan.tile) {
        case Tile::square256: return squares_of<T, 256, 4>(p, s);
        case Tile::square128: return squares_of<T, 128, 2>(p, s);
        case Tile::waves64: return tiles_in_runs(p.m, p.n, p.chunks) ? waves_of<T, 2, 2, 4, true>(p, s) : waves_of<T, 2, 2, 4>(p, s);
        case Tile::waves32: return waves_of<T, 1, 1, 4>(p, s);
        case Tile::waves32_wide: break;
    }
    if (plan.parts == 1) return waves_of<T, 1, 1, 8>(p, s);
    ProductArgs q = p;
    q.out = workspace;
    q.stride = p.n;
    q.bias = nullptr;
    const hipError_t e = waves_of<float, 1, 1, 8>(q, s);
    if (e != hipSuccess) return e;
    const int64_t runs = (p.n + 3) / 4, groups = (p.m * runs + 255) / 256;
    return launch(mx_join_kernel<T>, dim3((uint32_t)groups), dim3(256), s, workspace, p.m, p.n, p.parts, p.bias, p.bias_dtype,
                       static_cast<T*>(p.out), p.stride, (uint32_t)runs);
}

}  // namespace
}  // namespace fh

extern "C" {

size_t fh_mx_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (!fh::mx_shape_ok(m, k) || !fh::mx_shape_ok(n, k) || k > fh::kMostSummed || m == 0 || n == 0) return 0;
    const fh::Plan plan = fh::plan_of(m, n, fh::mx_chunks(k));
    return plan.parts > 1 ? (size_t)plan.parts * (size_t)m * (size_t)n * 4u : 0;
}

fh_status fh_mx_matmul(const fh_mx_product* q, void* stream)
{
    using namespace fh;
    if (!q) return FH_ERR_NULL;
    if (!is_dtype(q->out_dtype) || !is_dtype(q->bias_dtype)) return FH_ERR_BAD_DTYPE;
    if (!mx_shape_ok(q->m, q->k) || !mx_shape_ok(q->n, q->k) || q->k > kMostSummed || q->stride < q->n || q->stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (q->reserved != 0) return FH_ERR_BAD_PARAM;
    if (q->m == 0 || q->n == 0) return FH_OK;
    if (!q->out || (q->k > 0 && (!q->a || !q->b))) return FH_ERR_NULL;
    const size_t size = dtype_size(q->out_dtype);
    if (!is_aligned(q->a, 16) || !is_aligned(q->b, 16) || !is_aligned(q->out, size) || !is_aligned(q->bias, dtype_size(q->bias_dtype)) ||
        !is_aligned(q->workspace, 16)) return FH_ERR_ALIGNMENT;
    if (q->a_cap < mx_bytes(q->m, q->k) || q->b_cap < mx_bytes(q->n, q->k) || q->out_cap < strided_elements(q->m, q->n, q->stride) * size)
        return FH_ERR_BUFFER_TOO_SMALL;
    const size_t workspace = fh_mx_matmul_workspace_bytes(q->m, q->n, q->k);
    if (workspace && !q->workspace) return FH_ERR_NULL;
    if (q->workspace_cap < workspace) return FH_ERR_BUFFER_TOO_SMALL;
    const Plan plan = plan_of(q->m, q->n, mx_chunks(q->k));
    const MxStore a = mx_store(const_cast<void*>(q->a), q->m, q->k), b = mx_store(const_cast<void*>(q->b), q->n, q->k);
    const ProductArgs p = {a.codes, a.scales, b.codes, b.scales, q->m, q->n, q->bias, q->out, q->stride, (int32_t)a.chunks,
                           (int32_t)plan.chunks_each, plan.parts, q->bias_dtype, 0, 0, 0, 0};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    float* w = static_cast<float*>(q->workspace);
    const hipError_t e = q->out_dtype == FH_F32 ? product_of<float>(p, plan, w, s) : product_of<Bf16>(p, plan, w, s);
    return e == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
