// What norm.hip and dropout.hip share besides the vectors of rows.h.
#pragma once

#include <algorithm>

#include "layer_internal.h"
#include "rows.h"

namespace mics {

// out_k[c] = the sum over the groups of rows of parts[k][group][c], rounded once; out_k may be NULL (dropout.hip).
int launch_column_sums(const float* parts, int sums, int groups, size_t cols, void* const* out, int kind, void* stream);

namespace {

constexpr size_t kUnits = 256;              // compute units of an MI355X

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

template <int KIND> __device__ __forceinline__ const char* row_at(const ConstRows& m, size_t row)
{
    return (const char*)m.data + row * m.stride * kWidth<KIND>;
}
template <int KIND> __device__ __forceinline__ char* row_at(const Rows& m, size_t row)
{
    return (char*)m.data + row * m.stride * kWidth<KIND>;
}

inline size_t vectors(size_t cols) { return (cols + kVec - 1) / kVec; }
inline int waves_of(size_t vecs, int per_lane) { return (int)((vecs + 64 * per_lane - 1) / (64 * per_lane)); }
// A grid of at most 2^20 workgroups: a launch's lanes have to stay below 2^32, the kernels stride over the rest.
inline unsigned grid_of(size_t blocks) { return (unsigned)std::min<size_t>(blocks, 1u << 20); }

}  // namespace
}  // namespace mics
