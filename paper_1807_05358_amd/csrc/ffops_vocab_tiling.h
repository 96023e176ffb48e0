// How the products of the vocabulary's loss are cut.
#pragma once
#include <algorithm>
#include <cstdint>

namespace ffops {

// How a product of m x n over k is cut: the largest tile of which there are enough, k split where that is allowed into no less than 512 of it and into no more than 16,
// and none much longer than the shorter side.  256 x 256 tiles are half as fast again as others per product once they run, and take 20 us before and after that:
// dx of 3328 x 28040 x 1096 with 195 blocks of them 208 us, 128 x 128 321 us; dw with k = 207 114 us, 64 x 64 87 us.  128 x 128 read half as
// much as 64 x 64: 300 x 8000 x 1024 60 us for all, 64 x 64 66 us.
struct Tiling {
    uint32_t tile, ms, ns, splits;
    uint32_t blocks() const { return ms * ns; }
};

inline Tiling tiling_of(uint64_t m, uint64_t n, uint64_t k, bool split)
{
    const auto ceil_div = [](uint64_t a, uint64_t b) { return (a + b - 1) / b; };
    Tiling t = {};
    for (uint32_t tile : {256u, 128u, 64u}) {
        const uint64_t tiles = ceil_div(m, tile) * ceil_div(n, tile), places = tile == 256 ? 256 : tile == 128 ? 512 : 768;      // one, two and three on a unit, by their LDS
        const uint64_t splits = split && tiles ? std::max<uint64_t>(1, std::min<uint64_t>({places / tiles, k / 512, 16})) : 1;
        t = {tile, (uint32_t)ceil_div(m, tile), (uint32_t)ceil_div(n, tile), (uint32_t)splits};
        if (tile == 64 || (tiles * splits >= (tile == 256 ? 160 : 256) && tile <= (std::min(m, n) + 63) / 64 * 64 && (tile < 256 || k >= 512))) break;
    }
    return t;
}

constexpr uint64_t PIECE_BYTES = 256ull << 20;      // gradient of the logits of a piece: what the last-level cache holds

// words of a piece of the backward pass
inline uint32_t piece_of(uint32_t rows, uint32_t vocab)
{
    const uint64_t fit = PIECE_BYTES / 2 / std::max(1u, rows) / 256 * 256;
    return (uint32_t)std::min<uint64_t>(((uint64_t)vocab + 255) / 256 * 256, std::max<uint64_t>(fit, 256));
}

}  // namespace ffops
