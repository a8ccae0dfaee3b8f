// What the matrix products share: loads that go straight into LDS, the order of tiles, stores of a row's last values.
#pragma once

#include "fh_norm.hpp"

namespace fh {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// 16 bytes a lane from a buffer straight into LDS, at `lds` + 16 * lane.  Written out because the compiler would wait for all
// of them before every later read of LDS, the other stage's too.  No register is written; the caller waits by
// s_waitcnt vmcnt before the barrier that hands the stage over.
__device__ __forceinline__ void to_lds(uint32_t lds, u32x4 from, uint32_t offset, uint32_t moved)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(from), "s"(__builtin_amdgcn_readfirstlane(moved)) : "memory", "m0");
}
__device__ __forceinline__ u32x4 buffer_of(const uint8_t* p, uint32_t bytes)
{
    const uint64_t at = (uint64_t)p;
    return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, 0x00020000u};
}

// Tiles in bands of eight columns, so that what an XCD works on at a time shares rows of both operands in its L2.
__device__ __forceinline__ void in_bands(uint32_t tile, uint32_t m_tiles, uint32_t n_tiles, uint32_t& i, uint32_t& j)
{
    const uint32_t band = tile / (8 * m_tiles), first = band * 8, wide = n_tiles - first < 8 ? n_tiles - first : 8, in_band = tile - first * m_tiles;
    i = in_band / wide;
    j = first + in_band - i * wide;
}

// Of 16 bytes of outputs those that are before a row's end.
template <typename T>
__device__ __forceinline__ void store_packed(T* p, int n, u32x4 v)
{
    constexpr int kRun = 16 / sizeof(T);
    if (n >= kRun) *reinterpret_cast<u32x4_a2*>(p) = v;
    else {
#pragma unroll
        for (int i = 0; i < kRun; ++i)
            if (i < n) {
                const uint32_t w = v[i * (int)sizeof(T) / 4];    // a value of its own: bit_cast of a vector's element takes element 0 whichever is asked for
                if constexpr (sizeof(T) == 4) p[i] = __builtin_bit_cast(float, w);
                else p[i].bits = (uint16_t)(w >> (16 * (i & 1)));
            }
    }
}

}  // namespace fh
