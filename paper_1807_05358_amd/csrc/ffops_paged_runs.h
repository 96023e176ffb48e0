// How attention over a paged cache deals its work, and where in the cache it looks: plain arithmetic, for the kernels and for the host.
#pragma once
#include <algorithm>
#include <cstdint>

#ifdef __HIP__
#define FFOPS_BOTH __host__ __device__ inline
#else
#define FFOPS_BOTH inline
#endif

namespace ffops {

constexpr int TILE = 32;                    // positions of a tile
constexpr uint32_t TILES_OF_RUN = 8;        // no run is shorter where sequences are cut
constexpr uint32_t ENTRY = 8;               // what a run takes to begin with a sequence and to end with it, in tiles

// The tiles of all sequences, each with ENTRY tiles that there are not before its own, make one list, `all` long, which is dealt in runs, one behind the other, the first ones a tile longer where it does not come out even.  Runs in use: none is
// shorter than TILES_OF_RUN tiles.
struct Runs {
    uint32_t n;
    uint32_t longer;        // runs of each + 1 tiles
    int64_t each;
    FFOPS_BOTH int64_t begin(uint32_t run) const { return run * each + (run < longer ? run : longer); }
    // the run that holds a tile
    FFOPS_BOTH uint32_t of(int64_t tile) const
    {
        const int64_t first = longer * (each + 1);
        return tile < first ? quotient(tile, each + 1) : longer + quotient(tile - first, each);
    }
    static FFOPS_BOTH uint32_t quotient(int64_t a, int64_t b)      // the wide division takes a hundred instructions
    {
        return (uint64_t)(a | b) >> 32 ? (uint32_t)((uint64_t)a / (uint64_t)b) : (uint32_t)a / (uint32_t)b;
    }
};
// the places of a sequence of nk positions in the list
FFOPS_BOTH uint32_t tiles_of(int nk) { return ((uint32_t)nk + TILE - 1) / TILE; }
FFOPS_BOTH uint32_t places_of(int nk) { return nk ? ENTRY + tiles_of(nk) : 0; }

FFOPS_BOTH Runs runs_used(uint32_t runs, int64_t all)
{
    const int64_t most = (all + TILES_OF_RUN - 1) / TILES_OF_RUN;
    Runs r;
    r.n = most < 1 ? 1 : most < (int64_t)runs ? (uint32_t)most : runs;
    r.each = (uint64_t)all >> 32 ? (int64_t)((uint64_t)all / r.n) : (int64_t)((uint32_t)all / r.n);
    r.longer = (uint32_t)(all - r.each * r.n);
    return r;
}

// A run that begins or ends inside a sequence leaves a part of its sum: in slot 2 x where the sequence began in another run, in 2 x + 1 where it begins here and goes on in another.
FFOPS_BOTH uint32_t slot_of(uint32_t run, bool begins_here) { return 2 * run + (begins_here ? 1 : 0); }

// The 16 positions from `at` of a sequence of nk (at least one): the table's entry for them and their place in that page.  Behind the last position: those of the last one.
FFOPS_BOTH uint32_t entry_of(int at, int nk, uint32_t page_log2) { return (uint32_t)(at < nk ? at : nk - 1) >> page_log2; }
FFOPS_BOTH uint32_t place_of(int at, int nk, uint32_t page) { return (uint32_t)(at < nk ? at : nk - 1) & (page - 1) & ~15u; }

// Runs of a key head, or none: then a block takes a sequence.  blocks: key heads times blocks of columns, of one sequence.  Cutting takes a second kernel, 3 to 5 us, and pays where blocks are few and sequences long, or of
// different lengths: 1 x 8 heads of 4096 positions, bf16, 39 us whole, 20 cut, of 1024 18 and 20; 32 x 16 heads of up to 4000 113 and 91, all of 4000 176 and 179, all of 1000 41 and 44; 64 x 16 heads of 300 29 and 31, of up to 4000
// 195 and 187.
inline uint32_t runs_of(uint64_t blocks, uint64_t batch, uint64_t positions)
{
    if (positions <= 1024 || blocks * batch >= 1024 || (blocks * batch >= 512 && positions <= 2048)) return 0;
    const uint64_t tiles = (positions + TILE - 1) / TILE;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(512 / blocks, (tiles * batch + TILES_OF_RUN - 1) / TILES_OF_RUN));
}

}  // namespace ffops
