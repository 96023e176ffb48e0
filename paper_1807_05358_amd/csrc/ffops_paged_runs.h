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

// The tiles of all sequences make one list, `all` long, of which run x takes the x-th part.  Runs in use: none is shorter than TILES_OF_RUN tiles.
FFOPS_BOTH uint32_t runs_used(uint32_t runs, int64_t all)
{
    const int64_t n = (all + TILES_OF_RUN - 1) / TILES_OF_RUN;
    return n < 1 ? 1 : n < (int64_t)runs ? (uint32_t)n : runs;
}
FFOPS_BOTH int64_t run_begin(uint32_t run, uint32_t runs, int64_t all) { return (int64_t)run * all / runs; }

// the run that holds a tile
FFOPS_BOTH uint32_t run_of(int64_t tile, uint32_t runs, int64_t all)
{
    uint32_t r = (uint32_t)(tile * runs / all);
    while (run_begin(r + 1, runs, all) <= tile) ++r;
    while (run_begin(r, runs, all) > tile) --r;
    return r;
}

// A run that begins or ends inside a sequence leaves a part of its sum: in slot 2 x where the sequence began in another run, in 2 x + 1 where it begins here and goes on in another.
FFOPS_BOTH uint32_t slot_of(uint32_t run, bool begins_here) { return 2 * run + (begins_here ? 1 : 0); }

// The 16 positions from `at` of a sequence of nk (at least one): the table's entry for them and their place in that page.  Behind the last position: those of the last one.
FFOPS_BOTH uint32_t entry_of(int at, int nk, uint32_t page_log2) { return (uint32_t)(at < nk ? at : nk - 1) >> page_log2; }
FFOPS_BOTH uint32_t place_of(int at, int nk, uint32_t page) { return (uint32_t)(at < nk ? at : nk - 1) & (page - 1) & ~15u; }

// Runs of a key head, or none: then a block takes a sequence.  Sequences are cut where they alone do not fill the device.  others: key heads times blocks of columns.
inline uint32_t runs_of(uint64_t others, uint64_t batch, uint64_t positions)
{
    const uint64_t tiles = (positions + TILE - 1) / TILE;
    if (tiles <= 8 || others * batch >= 4096) return 0;
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(1024 / others, (tiles * batch + TILES_OF_RUN - 1) / TILES_OF_RUN));
}

}  // namespace ffops
