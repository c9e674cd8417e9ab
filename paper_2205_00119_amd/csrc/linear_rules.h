// How a product is cut into tiles and parts: rules on sizes, an element's width, strides, alignment and whether blocks of a checkpoint
// have to stay whole, host code.
#pragma once

#include <algorithm>
#include <cstddef>

namespace mics {

constexpr size_t ceil_div(size_t a, size_t b) { return a / b + (a % b ? 1 : 0); }

constexpr size_t kLinearWorkspace = size_t{64} << 20;      // the parts of a product take no more
constexpr size_t kFewRows = 32;                            // up to here the kernel of few rows
constexpr size_t kCUs = 256;

struct ProductShape {
    size_t m, n, k, width;                                 // width: bytes of an element
    bool a_turned, b_turned;
    bool a_on_16, b_on_16;                                 // every chunk of 16 bytes lies on 16 (on_16)
    bool chunks;                                           // rows hold whole chunks, offsets fit 31 bits (in_chunks)
    bool blocks;                                           // a workgroup has to hold whole blocks of 64 columns
};

// `whole` tiles have one workgroup each, the `shared` ones behind them `splits`, of `depth` tiles of k (128 bytes) each.
// Operands that are copied first, so that they lie on 16 bytes, take a_copy and b_copy bytes.
struct ProductPlan {
    bool few;
    size_t bm, bn, whole, shared, splits, depth;
    size_t a_copy, b_copy;
};
constexpr size_t parts_bytes(const ProductPlan& p) { return p.splits > 1 ? p.shared * p.splits * p.bm * p.bn * 4 : 0; }
// Parts, copies, and what the first copy's place on 16 bytes may take.
constexpr size_t workspace_of(const ProductPlan& p) { return parts_bytes(p) + (p.a_copy + p.b_copy ? p.a_copy + p.b_copy + 16 : 0); }
// k of operands that are both copied: zeros fill it up to whole tiles.
constexpr size_t copy_k(size_t k, size_t width) { return ceil_div(k * width, 128) * 128 / width; }
// Elements of a row of a copy.
constexpr size_t copy_stride(size_t row, size_t width) { return ceil_div(row * width, 16) * 16 / width; }

// What a cut into tiles of `tile` rows and columns takes in ns, with the best number of parts for the tiles of the last round.
// slow: what a tile of k takes against operands on 16 bytes.  Measured (us): a tile of k for all workgroups that fit, 256 x 256, one on
// a compute unit, 1.45 (4096 x 8192 x 4096 bf16 191), 128 x 128, two on one, 0.9 (2048 x 4096 x 4096 62.5), one on one 0.56
// (4096 x 8192 x 1024 78); 320 tiles of 128 x 128 with k = 5120 63.5, in three parts each 71; beginning and end of a tile 5 and 3.5.
// In 32 bits, of 128 x 128, two on one 3.66 (2048 x 4096 x 4096 468) and one on one 1.95, of 64 x 64 0.69 to 1.95 with one to four
// (input gradient 154 x 5120 x 5120 in one part 113, in three 92; of 128 x 128 in three 118), of 32 x 128 as much (in five 75).
// The ends are one figure whatever is stored, which is too little where results of 32 bits end a short sum of 16-bit elements: weight
// gradient 1003 x 2563 x 1285 off 16 bytes 18 by this, 25.8 measured.
struct TileCost {
    ProductPlan plan;
    double ns;
};
inline TileCost cost_of_tiles(const ProductShape& s, size_t bm, size_t bn, size_t room, double slow)
{
    const size_t tiles = ceil_div(s.m, bm) * ceil_div(s.n, bn), size = bm * bn, depths = ceil_div(s.k, 128 / s.width);
    const bool large = bm == 256, small = bm < 128;
    const double ends = large ? 5000 : 3500;
    const size_t slots = large ? kCUs : small ? 4 * kCUs : 2 * kCUs;
    // with one, two, three and four workgroups on a compute unit
    const double four[4] = {690, 1060, 1500, 1950}, two[2] = {1950, 3660};
    auto tile_of_k = [&](size_t units) {
        if (large) return 1450 * slow;
        if (s.width == 4) return (small ? four : two)[ceil_div(units, kCUs) - 1] * slow;
        return (units <= kCUs ? 560 : 662 + 238 * (double)(units - kCUs) / kCUs) * slow;       // what all share counts too
    };
    auto rounds = [&](size_t units, size_t depth) {
        const size_t rest = units % slots;
        return (units / slots) * (depth * tile_of_k(slots) + ends) + (rest ? depth * tile_of_k(rest) + ends : 0);
    };
    TileCost best{{false, bm, bn, tiles, 0, 1, depths, 0, 0}, rounds(tiles, depths)};
    for (const size_t shared : {tiles % slots, tiles % slots + slots}) {
        if (shared == 0 || shared > tiles) continue;
        for (size_t splits = 2; splits <= 64 && splits <= depths; ++splits) {
            const size_t units = shared * splits, depth = ceil_div(depths, splits);
            if (units > 2 * slots || units * size * 4 > room) break;
            if (ceil_div(depths, depth) < splits) continue;
            // the parts are written and read, and a second launch
            const double ns = rounds(tiles - shared, depths) + rounds(units, depth) + units * size * 8 / 5000.0 + 5000;
            if (ns < best.ns) best = {{false, bm, bn, tiles - shared, shared, splits, depth, 0, 0}, ns};
        }
    }
    return best;
}

inline ProductPlan plan_product(const ProductShape& s)
{
    const size_t depths = ceil_div(s.k, 128 / s.width);
    if (s.m == 0) return {false, 128, 128, 0, 0, 1, depths, 0, 0};
    if (s.m <= kFewRows && !s.a_turned && s.chunks && depths && (s.b_turned || s.b_on_16)) {
        const size_t bm = s.m <= 16 ? 16 : 32;
        const size_t bn = s.b_turned ? 256 / s.width : s.blocks ? 64 : 16;
        const size_t tiles = ceil_div(s.n, bn);
        size_t splits = 1, depth = depths;
        // Few columns: enough workgroups for the memory's latency.  us, one part / several, 16 rows: 16384 x 1024 bf16 30.6 / 13.3,
        // 20480 x 5120 72 / 49, 16384 x 1 20 / 7.3, 2560 x 256 f32 11.5 / 7.5.  Of shorter k, or with a workgroup for every compute unit,
        // the join takes what that saves: 5120 x 2560 bf16 11.5 / 12.5, 8192 x 4096 17.1 / 19.7, 16384 x 4096 31.3 / 34.5 (256 tiles of k;
        // the line of 320 is between this and 20480 x 5120), 4096 x 4096 f32 19.6 / 20.0; 16384 x 4096 f32 88.9 / 83.3 is above it.
        // Workgroups of 64 columns are a quarter as many, and parts would pay from shorter k on than these lines, measured with 16
        // columns, let them: with a checkpoint 16 x 5120 x 2560 bf16 25.8 / 12.5, 16 x 4096 x 4096 20.9 / 13.4; where the lines do,
        // 16 x 8192 x 4096 38.1 / 20.5, 16 x 16384 x 1024 72 / 13.5, 16 x 10240 x 2560 f32 91 / 32.6; 16 x 2560 x 10240 15.6 / 21.0.
        if (tiles < 2 * kCUs && (s.b_turned || depths >= (tiles < kCUs ? 256 / s.width : 320))) {
            splits = s.b_turned ? std::min(2 * kCUs / tiles, ceil_div(depths, 8))
                                : std::min({std::max<size_t>(ceil_div(2 * kCUs, tiles), 4), ceil_div(depths, 16), size_t{32}});
            depth = ceil_div(depths, splits);
            splits = ceil_div(depths, depth);
        }
        return {true, bm, bn, splits > 1 ? 0 : tiles, splits > 1 ? tiles : 0, splits, depth, 0, 0};
    }
    auto best = [&](size_t room, double slow_128, double slow_256) {           // 0: no tiles of 256 x 256
        TileCost small = cost_of_tiles(s, 128, 128, room, slow_128);
        if (s.width == 4 && s.chunks) {                    // smaller tiles, since idle rows and columns cost as much as others
            for (const size_t bm : {64, 32}) {
                if (bm == 32 && s.a_turned) continue;      // its swizzle takes rows of 64
                const TileCost other = cost_of_tiles(s, bm, 4096 / bm, room, slow_128);
                if (other.ns < small.ns) small = other;
            }
            return small;
        }
        if (!s.chunks || slow_256 == 0) return small;
        const TileCost large = cost_of_tiles(s, 256, 256, room, slow_256);
        return large.ns <= small.ns ? large : small;
    };
    const bool off = s.chunks && !(s.a_on_16 && s.b_on_16);
    if (!off) return best(kLinearWorkspace, 1, 1).plan;
    // Loads off 16 bytes take the L1 cache twice the time and more.  us, so / copied first: 128 x 128, 2047 x 5121 x 2561 133 / 92, its
    // gradients 107 / 86 and 103 / 80, 300 x 2047 x 5121 36.2 / 35.9; 256 x 256, 4095 x 3001 x 3003 107 / 83, 4095 x 8193 x 4095 256 / 254.
    // Both turned, 256 x 256 takes 1.8 times as long as on 16 bytes, and 128 x 128 is faster.  32-bit products are bound by the matrix
    // instructions.
    const TileCost own = s.width == 4 ? best(kLinearWorkspace, 1.1, 0) : best(kLinearWorkspace, 1.6, s.a_turned ? 0 : 1.45);
    const size_t k = s.a_on_16 || s.b_on_16 ? s.k : copy_k(s.k, s.width);
    const size_t a = s.a_on_16 ? 0 : (s.a_turned ? k * copy_stride(s.m, s.width) : s.m * copy_stride(k, s.width)) * s.width;
    const size_t b = s.b_on_16 ? 0 : (s.b_turned ? k * copy_stride(s.n, s.width) : s.n * copy_stride(k, s.width)) * s.width;
    if (a > kLinearWorkspace || b > kLinearWorkspace || a + b + 16 > kLinearWorkspace) return own.plan;
    TileCost copied = best(kLinearWorkspace - a - b - 16, 1, 1);
    copied.ns += (a + b) / 3000.0 + 4000;
    if (copied.ns >= own.ns) return own.plan;
    copied.plan.a_copy = a;
    copied.plan.b_copy = b;
    return copied.plan;
}

// Of every type and alignment.
inline size_t most_workspace(size_t m, size_t n, size_t k, bool a_turned, bool b_turned)
{
    size_t most = 0;
    for (const size_t width : {2, 4})
        for (int flags = 0; flags < 16; ++flags)
            most = std::max(most, workspace_of(plan_product({m, n, k, width, a_turned, b_turned, (flags & 1) != 0, (flags & 2) != 0,
                                                             (flags & 4) != 0, (flags & 8) != 0})));
    return most;
}

}  // namespace mics
