// Tiles of 16-bit matrices in LDS and the operands read from them.
#pragma once
#include "ffops_device.h"

namespace ffops {

// A tile of rows of D elements, read along the rows (16 bytes per lane, 32 rows) or transposed (4 x 16 blocks).  The 16-byte
// chunk c of row r lies at chunk c ^ spread(r) of its row, which puts 16 rows' chunk c, and four rows' four neighbouring
// chunks, into different banks (a bank line of 256 bytes holds one row of 128 elements or two of 64).  Rows of 256 elements are only read transposed.
template <int D>
static __device__ __forceinline__ int spread(int r)
{
    static_assert(D == 64 || D == 128 || D == 256, "row lengths in use");
    if constexpr (D == 64) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
    else if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return (r & 3) << 2;
}

// rows 0 .. ROWS-1 of a tile whose row r starts at base + r * stride, by WAVES waves, asynchronously; rows from `rows` on, and
// chunks from `chunks` on, become zeros
template <int ROWS, int D, int WAVES>
static __device__ __forceinline__ void stage(lds_char* dst, const char* base, int64_t stride, int rows, int chunks)
{
    constexpr int CH = D / 8, PER = ROWS * CH / 64 / WAVES;
    static_assert(PER >= 1, "every wave stages something");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
#pragma unroll
    for (int n = 0; n < PER; ++n) {
        const int at = (n * WAVES + wave) * 64, r = (at + lane) / CH, c = (lane % CH) ^ spread<D>(r);
        const char* src = base + r * stride + c * 16;
        load_lds16(r < rows && c < chunks ? src : (const char*)&zero16, dst + at * 16);
    }
}

// operand: row r0 + lane % 32 of a tile, elements 16 * step + 8 * (lane / 32) + e
template <class T, int D>
static __device__ __forceinline__ typename T::vec8 along(const lds_char* tile, int r0, int step)
{
    const int lane = threadIdx.x % 64, r = r0 + lane % 32;
    return read8<T>(tile + r * D * 2 + (((step * 2 + lane / 32) ^ spread<D>(r)) * 16));
}

// operand: element d0 + lane % 32 of the rows r0 + 8 * (e / 4) + 4 * (lane / 32) + e % 4 (the order of a product's registers), or,
// IN_ORDER, r0 + 8 * (lane / 32) + e (the order of `along`)
template <class T, int D, bool IN_ORDER = false>
static __device__ __forceinline__ typename T::vec8 across(const lds_char* tile, int r0, int d0)
{
    constexpr int HALF = IN_ORDER ? 8 : 4, HI = IN_ORDER ? 4 : 8;
    const int lane = threadIdx.x % 64, i = lane % 16, r = r0 + HALF * (lane / 32) + i / 4;
    const int chunk = d0 / 8 + 2 * ((lane / 16) % 2) + (i % 4) / 2;
    const lds_char* lo = tile + r * D * 2 + ((chunk ^ spread<D>(r)) * 16) + (i % 2) * 8;
    const lds_char* hi = tile + (r + HI) * D * 2 + ((chunk ^ spread<D>(r + HI)) * 16) + (i % 2) * 8;
    return read8_tr<T>(lo, hi);
}

}  // namespace ffops
