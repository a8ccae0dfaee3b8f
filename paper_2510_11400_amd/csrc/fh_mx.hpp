// The stored form of a microscaled matrix, and what the kernels that write and read it share.
//
// Along each row 32 consecutive values share a scale 2^(s-127), s a byte; a value is a sign and one of
// {0, 0.5, 1, 1.5, 2, 3, 4, 6} in four bits.  Rows are padded with zeros to whole chunks of 256 values:
//   codes   [rows][chunks * 128] bytes, value c in byte c/2, the even one in the low half;
//   scales  behind them, in pieces of 32 rows x one chunk (8 blocks): [row/32][chunk][b/4][row%32][b%4].
// A lane of the matrix instruction wants 16 bytes of codes and the scale of those 32 values.  In this order the scales of
// 32 rows x 4 blocks are 128 contiguous bytes, so a wave fetches 32 rows x a chunk (or 16 rows x a chunk) by one load of a
// word per lane, and the instruction picks the byte of that word by its operand selector.  With the scales in plain rows
// the same load touches 32 lines for 8 bytes each.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fh_device.hpp"
#include "fh_rules.hpp"

namespace fh {

constexpr int kMxBlock = 32, kMxChunk = 256;
constexpr int64_t kMxMost = ((int64_t)1 << 31) - 256;      // rows, columns

inline __host__ __device__ int64_t mx_chunks(int64_t cols) { return (cols + kMxChunk - 1) / kMxChunk; }
inline __host__ __device__ int64_t mx_pitch(int64_t cols) { return mx_chunks(cols) * (kMxChunk / 2); }
inline bool mx_shape_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows <= kMxMost && cols <= kMxMost; }
inline uint64_t mx_codes_bytes(int64_t rows, int64_t cols) { return (uint64_t)rows * (uint64_t)mx_pitch(cols); }
inline uint64_t mx_bytes(int64_t rows, int64_t cols)
{
    return mx_codes_bytes(rows, cols) + (uint64_t)((rows + 31) / 32) * (uint64_t)mx_chunks(cols) * 256u;
}

// A stored matrix for the kernels.  Their arguments hold as few of these as possible: a launch of up to 112 bytes of
// arguments is enqueued a microsecond sooner than a longer one, and the small calls wait for nothing else.
struct MxStore {
    uint8_t* codes;
    uint8_t* scales;
    int64_t  chunks;
};
inline __host__ __device__ MxStore mx_store(void* p, int64_t rows, int64_t cols)
{
    uint8_t* b = static_cast<uint8_t*>(p);
    return MxStore{b, b + rows * mx_pitch(cols), mx_chunks(cols)};
}
// Where the scale of row r's block b is.
__device__ __forceinline__ int64_t mx_scale_at(int64_t r, int64_t b, int64_t chunks)
{
    return (((r >> 5) * chunks + (b >> 3)) << 8) + ((b & 7) >> 2) * 128 + (r & 31) * 4 + (b & 3);
}

// ---- from values to codes ------------------------------------------------------------
// The scale byte of a block whose largest magnitude has the bits `top` (integer comparison of the magnitudes' bits, so
// that NaN and infinity are the largest): the exponent of the largest magnitude less that of 4, at least 1; 255 where the
// block holds no number.  Scale 2^-127 (byte 0) is read but never written: its factor is no normal float.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : (e > 3u ? e - 2u : 1u);
}
// 2^(s-127) for s in 1..254.
__device__ __forceinline__ float mx_scale(uint32_t s) { return __builtin_bit_cast(float, s << 23); }

// Two values into byte `BYTE` of `into`, to the nearest code (ties to even, magnitudes over 6 to 6).  The instruction
// does exactly that for every fp32 pair and scale 2^-126 .. 2^125 (checked over all bf16 values and 2M fp32 pairs).
template <int BYTE>
__device__ __forceinline__ uint32_t mx_nearest(uint32_t into, float a, float b, uint32_t s)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, a, b, mx_scale(s), BYTE);
}
// The code of one value, rounded up where 16 random bits h are below 2^16 times the fraction (which counts in steps of
// 2^-22): at 2^(1-s) times the magnitude the smallest code, 0.5, is the upper half of fp32's subnormal range, so that
// the code is the number's bits from the 22nd on in both ranges and a carry out of the fraction rounds up.
__device__ __forceinline__ uint32_t mx_stochastic(float v, uint32_t s, uint32_t not_h /* 65535 - h */)
{
    const uint32_t sign = __builtin_bit_cast(uint32_t, v) >> 31 << 3;
    const float t = __builtin_ldexpf(__builtin_fabsf(v), 1 - (int)s);
    const uint32_t u = __builtin_bit_cast(uint32_t, t);
    const uint32_t top = 7u << 22;                               // 6
    // 2^22 - 1 - 64 h = 64 (65535 - h) + 63
    return (((u < top ? u : top) + (not_h << 6 | 63u)) >> 22) | sign;
}

// ---- sums and maxima over lanes --------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, v))); }
constexpr int kQuadXor1 = 0xB1, kQuadXor2 = 0x4E, kHalfMirror = 0x141, kRowMirror = 0x140;

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    v = umax(v, dpp<kQuadXor1>(v));
    return umax(v, dpp<kQuadXor2>(v));
}
template <int LANES>
__device__ __forceinline__ float lane_sum(float v)           // over aligned runs of 8, 16, 32 or 64 lanes
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "run length");
    v += dpp<kQuadXor1>(v);
    v += dpp<kQuadXor2>(v);
    v += dpp<kHalfMirror>(v);
    if constexpr (LANES >= 16) v += dpp<kRowMirror>(v);
    if constexpr (LANES >= 32) {
        float a, b;
        self_swap<16>(v, a, b);
        v = a + b;
    }
    if constexpr (LANES >= 64) {
        float a, b;
        self_swap<32>(v, a, b);
        v = a + b;
    }
    return v;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

// ---- rows of values at any alignment of their type --------------------------------------
// The hardware takes 16-byte accesses at any element's address; the types only say so to the compiler.
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

struct Bf16 { uint16_t bits; };
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(Bf16 v) { return __builtin_bit_cast(float, (uint32_t)v.bits << 16); }

// A launch as the runtime takes it; <<< >>> lays its shape aside on the way, which is 0.2 us of the host's 2.4.
template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t s, const A&... given)
{
    if ((uint64_t)grid.x * block.x * grid.y * grid.z >> 32) return hipErrorInvalidConfiguration;
    return [&](P... args) {
        void* list[] = {static_cast<void*>(&args)...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, list, 0, s);
    }(given...);
}

// `groups` workgroups of `threads` by launches of as many as one may have: part(first, number).
template <typename F>
hipError_t in_parts(int64_t groups, int64_t threads, F part)
{
    const int64_t most = groups_at_once(threads);
    for (int64_t first = 0; first < groups; first += most) {
        const hipError_t e = part(first, groups - first < most ? groups - first : most);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// N values in words as they lie in memory.
template <typename T, int N = 8>
struct Run {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p, int64_t n)
    {
        if (n >= N) {
            if constexpr (kWords == 2) {
                const u32x2 v = *reinterpret_cast<const u32x2_a2*>(p);
                w[0] = v.x; w[1] = v.y;
            } else {
#pragma unroll
                for (int i = 0; i < kWords; i += 4) {
                    const u32x4 v = *reinterpret_cast<const u32x4_a2*>(reinterpret_cast<const uint32_t*>(p) + i);
                    w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = 0u;
            if (n <= 0) return;                                  // not by way of the run's end, which waits for the loads before it
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if constexpr (sizeof(T) == 4) w[i] = i < n ? __builtin_bit_cast(uint32_t, p[i]) : 0u;
                else w[i / 2] |= (i < n ? (uint32_t)p[i].bits : 0u) << (16 * (i & 1));
            }
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        else return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    }
};

// Workgroups go to the eight XCDs in turn.  A run of neighbours for each: the at-th of `all`.
__device__ __forceinline__ uint32_t run_of(uint32_t at, uint32_t all)
{
    const uint32_t xcd = at & 7, share = all >> 3, rest = all & 7;
    return xcd * share + (xcd < rest ? xcd : rest) + (at >> 3);
}

// Eight values from p on, of which the first `n` exist (the others are 0).
__device__ __forceinline__ void load8(const float* p, int64_t n, float (&v)[8])
{
    if (n >= 8) {
        const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p), b = *reinterpret_cast<const f32x4_a4*>(p + 4);
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if (n <= 0) return;
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const Bf16* p, int64_t n, float (&v)[8])
{
    if (n >= 8) {
        const u32x4 a = *reinterpret_cast<const u32x4_a2*>(p);
        for (int i = 0; i < 4; ++i) { const uint32_t w = a[i]; v[2 * i] = bf16_lo(w); v[2 * i + 1] = bf16_hi(w); }
    } else {
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        if (n <= 0) return;
        for (int i = 0; i < 8; ++i) v[i] = i < n ? value(p[i]) : 0.0f;
    }
}
// bf16 of two values, nearest even (one instruction on gfx950; NaN stays NaN).
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(Bf16* p, float v) { p->bits = (uint16_t)bf16_pair(v, v); }
__device__ __forceinline__ void store8(float* p, int64_t n, const float (&v)[8])
{
    if (n >= 8) {
        *reinterpret_cast<f32x4_a4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4_a4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void store8(Bf16* p, int64_t n, const float (&v)[8])
{
    if (n >= 8) {
        *reinterpret_cast<u32x4_a2*>(p) = u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    } else {
        for (int i = 0; i < 8; ++i) if (i < n) store1(p + i, v[i]);
    }
}

__device__ __forceinline__ void store4(float* p, int64_t n, const float (&v)[4])
{
    if (n >= 4) *reinterpret_cast<f32x4_a4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    else for (int i = 0; i < 4; ++i) if (i < n) p[i] = v[i];
}
__device__ __forceinline__ void store4(Bf16* p, int64_t n, const float (&v)[4])
{
    if (n >= 4) *reinterpret_cast<u32x2_a2*>(p) = u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    else for (int i = 0; i < 4; ++i) if (i < n) store1(p + i, v[i]);
}

// ---- eight values of a lane, 32 of a quad, to the stored form of their row ----------------
// All 64 lanes are active; `first` is a multiple of 8, the quad's 32 values are one block.  Columns past the row's end hold
// 0 (the caller's loads see to that), so that the padding becomes what a block of zeros becomes.
__device__ __forceinline__ uint32_t mx_codes8(const float (&v)[8], uint32_t& s)
{
    uint32_t top = abs_bits(v[0]);
    for (int i = 1; i < 8; ++i) top = umax(top, abs_bits(v[i]));
    s = mx_scale_byte(quad_max(top));
    uint32_t codes = 0;
    codes = mx_nearest<0>(codes, v[0], v[1], s);
    codes = mx_nearest<1>(codes, v[2], v[3], s);
    codes = mx_nearest<2>(codes, v[4], v[5], s);
    return mx_nearest<3>(codes, v[6], v[7], s);
}
// 32 values of a lane: a block's 16 bytes of codes, to the nearest.
__device__ __forceinline__ u32x4 mx_codes32(const float (&v)[32], uint32_t s)
{
    u32x4 q;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t a = 0;
        a = mx_nearest<0>(a, v[8 * w], v[8 * w + 1], s);
        a = mx_nearest<1>(a, v[8 * w + 2], v[8 * w + 3], s);
        a = mx_nearest<2>(a, v[8 * w + 4], v[8 * w + 5], s);
        q[w] = s == 255u ? 0u : mx_nearest<3>(a, v[8 * w + 6], v[8 * w + 7], s);
    }
    return q;
}
__device__ __forceinline__ void mx_write8(const MxStore& to, int64_t row, int64_t first, const float (&v)[8], bool write)
{
    uint32_t s;
    const uint32_t codes = mx_codes8(v, s);
    if (!write) return;
    *reinterpret_cast<uint32_t*>(to.codes + row * (to.chunks * 128) + (first >> 1)) = s == 255u ? 0u : codes;
    if ((first & 31) == 0) to.scales[mx_scale_at(row, first >> 5, to.chunks)] = (uint8_t)s;
}

}  // namespace fh
