// How log probabilities and their gradient are launched: workgroups that share a row, lanes, vectors in flight, paths past the
// caches.  Host code without HIP, so that its answers are tested where there is no GPU.  Every rule has both sides measured beside it
// (us, one MI355X).
#pragma once

#include <algorithm>
#include <cstddef>

namespace mics {
namespace {

constexpr int kCandidates = 2048;           // keys that a workgroup ranks
constexpr size_t kRowVec = 8;               // logits of a vector

// Workgroups that share a row: as many as there are compute units for it, none with fewer than 16384 logits (8192 / so / 32768 /
// 65536: 4 x 131072 bf16, 8 alternatives 13.0 / 12.6 / 12.8 / 14.9; 8 x 150000 with entropy 7.8 / 7.8 / 9.3 / 11.2; 32 x 128000, 5
// alternatives 13.2 / 12.8 / 15.4 / 17.6; 1 x 32000 7.6 / 4.5 / 4.5 / 4.5: the second launch and the join have to be paid for), and no
// more keys than the join ranks.
inline int splits_of(size_t rows, size_t vocab, int top)
{
    constexpr size_t kRowUnits = 256, kLeast = 16384;
    if (rows == 0 || rows >= kRowUnits) return 1;
    return (int)std::max<size_t>(1, std::min<size_t>({kRowUnits / rows, vocab / kLeast, 64, (size_t)kCandidates / std::max(top, 1)}));
}

// Logits that no cache holds (256 MB of Infinity Cache) are read past the caches: 4096 x 65536 bf16 97.0 us, so 83.2; where
// they may still be in one it costs 9 % (1024 x 50001 f32, 205 MB, 36.9 / 40.2).
constexpr size_t kUncached = size_t{256} << 20;
// A gradient that no cache keeps for its reader is stored past them: 4096 x 65536 bf16 171.7 us, so 165.8.
constexpr size_t kUnkept = size_t{224} << 20;

struct LogProbsShape {
    int splits;            // workgroups of a row
    unsigned chunk;        // vectors of one of them
    int lanes, flight;     // of a workgroup; vectors of a lane that are in flight
    bool uncached;
};
// 1024 lanes only where there is a compute unit for every workgroup (500 x 50001 f32, 5 alternatives: 256 lanes 22.3 us,
// 1024 lanes 43.9) and enough for each lane, less where it saves the join (1 x 32000 bf16 256 lanes 5.0, 1024 lanes 4.5;
// 4 x 131072 in eight parts 12.4 / 13.2); two vectors in flight instead of four in short rows (8192 x 5000 bf16 24.7 / 26.0;
// 3475 x 9296 binary16, 20 alternatives, 38.4 / 44.1).
inline LogProbsShape logprobs_shape(size_t rows, size_t vocab, int top, size_t width)
{
    const unsigned vecs = (unsigned)((vocab + kRowVec - 1) / kRowVec);
    LogProbsShape s{splits_of(rows, vocab, top), 0, 256, 4, false};
    s.chunk = (vecs + s.splits - 1) / s.splits;
    if (rows * s.splits <= 256 && s.chunk >= (s.splits == 1 ? 2048u : 4096u)) s.lanes = 1024;
    else if (s.chunk < (top ? 2048u : 1024u)) s.flight = 2;
    else s.uncached = rows * vocab * width >= kUncached;
    return s;
}

// The gradient: lanes of a workgroup, vectors of each (32 bytes: 4096 x 65536 bf16: one vector 192 us, two 165, four 176;
// 2000 x 50001 f32: one 141, two 156, four 169), and whether it is stored past the caches.
constexpr int kGradLanes = 256;
struct GradientShape {
    unsigned chunk, chunks;      // vectors of a workgroup, workgroups of a row
    bool unkept;
};
inline GradientShape gradient_shape(size_t rows, size_t vocab, size_t width)
{
    const unsigned vecs = (unsigned)((vocab + kRowVec - 1) / kRowVec), chunk = (width == 4 ? 1u : 2u) * kGradLanes;
    return {chunk, (vecs + chunk - 1) / chunk, rows * vocab * width >= kUnkept};
}

}  // namespace
}  // namespace mics
