// Tiles of 16-bit matrices in LDS and the operands read from them.
#pragma once
#include "ffops_device.h"

namespace ffops {

// A tile of rows of D elements, read along the rows (16 bytes per lane, 32 rows) or transposed (4 x 16 blocks).  The 16-byte
// chunk c of row r lies at chunk c ^ spread(r) of its row, which puts 16 rows' chunk c, and four rows' four neighbouring
// chunks, into different banks (a bank line of 256 bytes holds one row of 128 elements or two of 64).  Rows of 256 elements are only read transposed,
// rows r .. r + 3 and r + 8 .. r + 11 and two chunks of each at a time.  A 16-byte read serves lanes 0-3, 12-15, 20-23 and 24-27 together, then
// the other sixteen of a half wave; where lanes 16-31 ask for the neighbouring chunk (16x16x32 products), rows 0-3 and 12-15 have to lie in
// pairs of chunks that rows 4-11 leave free: hence the order 0, 2, 3, 1 of row fours in rows of 64 elements.
template <int D>
static __device__ __forceinline__ int spread(int r)
{
    static_assert(D == 32 || D == 64 || D == 128 || D == 256, "row lengths in use");
    if constexpr (D == 32) return (((r >> 2) & 1) << 1) ^ (((r >> 3) & 1) * 3);
    else if constexpr (D == 64) return (((r >> 1) & 1) << 2) | ((((r >> 2) & 1) << 1) ^ (((r >> 3) & 1) * 3));
    else if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return ((r & 3) << 2) | (((r >> 3) & 1) << 1);
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

// The same for tiles without zeros: where each of this lane's loads starts, relative to the tile's base, is worked out once.  Rows and
// chunks that do not exist are replaced by the last ones (what a product makes of them belongs to no element of the result).  The row stride times
// ROWS has to fit 32 bits.
template <int ROWS, int D, int WAVES>
struct Stager {
    static constexpr int CH = D / 8, PER = ROWS * CH / 64 / WAVES;
    uint32_t off[PER];

    __device__ __forceinline__ void init(int64_t stride, int rows, int chunks)
    {
        const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const int at = (n * WAVES + wave) * 64, r = (at + lane) / CH, c = (lane % CH) ^ spread<D>(r);
            off[n] = (uint32_t)min(r, rows - 1) * (uint32_t)stride + min(c, chunks - 1) * 16;
        }
    }

    // base is uniform; load n of PER
    __device__ __forceinline__ void load_one(lds_char* dst, const char* base, int n) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        load_lds16(base, off[n], dst + (n * WAVES + wave) * 1024);
    }
    __device__ __forceinline__ void load(lds_char* dst, const char* base) const
    {
#pragma unroll
        for (int n = 0; n < PER; ++n) load_one(dst, base, n);
    }
};

// operand: row r0 + lane % 32 of a tile, elements 16 * step + 8 * (lane / 32) + e
template <class T, int D>
static __device__ __forceinline__ typename T::vec8 along(const lds_char* tile, int r0, int step)
{
    const int lane = threadIdx.x % 64, r = r0 + lane % 32;
    return read8<T>(tile + r * D * 2 + (((step * 2 + lane / 32) ^ spread<D>(r)) * 16));
}

// operand: element d0 + lane % 32 of the rows r0 + 8 * (e / 4) + 4 * (lane / 32) + e % 4, the order of a product's registers
template <class T, int D>
static __device__ __forceinline__ typename T::vec8 across(const lds_char* tile, int r0, int d0)
{
    const int lane = threadIdx.x % 64, i = lane % 16, r = r0 + 4 * (lane / 32) + i / 4;
    const int chunk = d0 / 8 + 2 * ((lane / 16) % 2) + (i % 4) / 2;
    const lds_char* lo = tile + r * D * 2 + ((chunk ^ spread<D>(r)) * 16) + (i % 2) * 8;
    const lds_char* hi = tile + (r + 8) * D * 2 + ((chunk ^ spread<D>(r + 8)) * 16) + (i % 2) * 8;
    return read8_tr<T>(lo, hi);
}

// operands of the 16x16x32 product: row (element) at + lane % 16 of a tile, k = 32 * step + 8 * (lane / 16) + e
template <class T, int D>
static __device__ __forceinline__ typename T::vec8 along16(const lds_char* tile, int at, int step)
{
    const int lane = threadIdx.x % 64, r = at + lane % 16;
    return read8<T>(tile + r * D * 2 + (((step * 4 + lane / 16) ^ spread<D>(r)) * 16));
}

template <class T, int D>
static __device__ __forceinline__ typename T::vec8 across16(const lds_char* tile, int step, int at)
{
    const int lane = threadIdx.x % 64, i = lane % 16, r = step * 32 + 8 * (lane / 16) + i / 4, chunk = at / 8 + (i % 4) / 2;
    const lds_char* lo = tile + r * D * 2 + ((chunk ^ spread<D>(r)) * 16) + (i % 2) * 8;
    const lds_char* hi = tile + (r + 4) * D * 2 + ((chunk ^ spread<D>(r + 4)) * 16) + (i % 2) * 8;
    return read8_tr<T>(lo, hi);
}

// The order of what stands before it in its block: N products of which every one needs READS reads of LDS, read AHEAD products before they are
// used, and OTHER other instructions after each product
template <int N, int READS, int AHEAD, int OTHER>
static __device__ __forceinline__ void interleave()
{
    __builtin_amdgcn_sched_group_barrier(0x100, READS * AHEAD, 0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (n + AHEAD < N) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        if (OTHER) __builtin_amdgcn_sched_group_barrier(0x002, OTHER, 0);
    }
}

}  // namespace ffops
