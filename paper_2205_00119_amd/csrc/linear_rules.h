// How a product is cut into tiles and parts: rules on sizes alone, host code.
#pragma once

#include <cstddef>

namespace mics {

constexpr size_t kLinearWorkspace = size_t{64} << 20;      // the parts of a product take no more
constexpr size_t kTile = 128;
constexpr size_t ceil_div(size_t a, size_t b) { return a / b + (a % b ? 1 : 0); }

// Parts into which the sum over k is cut.
constexpr int linear_splits(size_t m, size_t n, size_t k)
{
    if (m == 0 || n == 0 || k == 0) return 1;
    const size_t tiles = ceil_div(m, kTile) * ceil_div(n, kTile);
    if (tiles >= 256) return 1;
    size_t s = 512 / tiles;
    const size_t most = ceil_div(k, 256);
    if (s > most) s = most;
    while (s > 1 && s * m > kLinearWorkspace / 4 / n) --s;
    return s < 1 ? 1 : (int)s;
}

}  // namespace mics
