// Activations with their 8-bit checkpoints, forward and backward.
#include "rows.h"

#include <algorithm>

#include "activation.h"
#include "columns.h"
#include "linear_internal.h"

namespace mics {
namespace {

// Vectors in ascending order, one for each lane; every row takes whole blocks of lanes.
constexpr int kActLanes = 64;
struct ActivationArgs {
    ActivationPass a;
    size_t groups;                             // lanes of a row
};
template <int KIND>
__global__ __launch_bounds__(kActLanes) void activation_kernel(ActivationArgs p)
{
    const ActivationPass& a = p.a;
    const size_t lanes = a.rows * p.groups;
    const unsigned groups = (unsigned)p.groups;
    for (size_t base = (size_t)blockIdx.x * kActLanes; base < lanes; base += (size_t)gridDim.x * kActLanes) {
        if (base + threadIdx.x >= lanes) break;                                 // whole blocks of lanes
        const size_t row0 = base / p.groups;                                    // the same in all lanes
        const unsigned at = (unsigned)(base - row0 * p.groups) + threadIdx.x, up = at / groups, c = at - up * groups;
        const size_t row = row0 + up;
        const int valid = valid_at(c, a.cols);
        float v[kVec];
        unpack<KIND>(load_vec<KIND>(row_at<KIND>(a.x, row) + (size_t)c * (kVec * kWidth<KIND>), valid), v);
        finish<KIND>(a.e, row, c, a.cols, valid, v);
    }
}

struct ReadArgs {
    CheckpointRead a;
    size_t groups;
};
template <int KIND>
__global__ __launch_bounds__(kActLanes) void checkpoint_read_kernel(ReadArgs p)
{
    const CheckpointRead& a = p.a;
    const size_t lanes = a.rows * p.groups;
    const unsigned groups = (unsigned)p.groups;
    for (size_t base = (size_t)blockIdx.x * kActLanes; base < lanes; base += (size_t)gridDim.x * kActLanes) {
        if (base + threadIdx.x >= lanes) break;
        const size_t row0 = base / p.groups;
        const unsigned at = (unsigned)(base - row0 * p.groups) + threadIdx.x, up = at / groups, c = at - up * groups;
        const size_t row = row0 + up;
        const int valid = valid_at(c, a.cols);
        float v[kVec];
        load_codes((const char*)a.codes.data + row * a.codes.stride + (size_t)c * kVec, valid,
                   a.scales[row * (groups / kBlockLanes) + c / kBlockLanes], v);
        with_act(a.act, [&](auto A) {
            #pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = act_of<decltype(A)::value>(v[i]);
        });
        store_vec<KIND>(row_at<KIND>(a.y, row) + (size_t)c * (kVec * kWidth<KIND>), pack<KIND>(v), valid);
    }
}

// dx and, with dbias, the sums of a stripe of 64 vectors over the rows of a workgroup: every gridDim.x * kBackWaves-th one.
constexpr int kBackWaves = 4, kBackRows = 2, kBackBlocks = 4;
struct BackwardArgs {
    ActivationBackward a;
    unsigned blocks;
    void* dbias;                               // where a stripe has one workgroup, it stores the sums themselves
    int grad;
};
template <int KIND, bool CODES>
__global__ __launch_bounds__(64 * kBackWaves) void activation_backward_kernel(BackwardArgs p)
{
    const ActivationBackward& a = p.a;
    __shared__ float lds[kBackWaves - 1][kVec][64];
    const int wave = wave_index();
    const unsigned lane = threadIdx.x & 63u, c = blockIdx.y * 64 + lane;
    const int valid = valid_at(c, a.cols);
    const size_t at = (size_t)c * (kVec * kWidth<KIND>), step = (size_t)gridDim.x * kBackWaves;
    float acc[kVec] = {};
    for (size_t row0 = (size_t)blockIdx.x * kBackWaves + wave; row0 < a.rows; row0 += kBackRows * step) {
        Raw<KIND> dy[kBackRows];
        float z[kBackRows][kVec];
        #pragma unroll
        for (int u = 0; u < kBackRows; ++u) {
            const size_t row = min(row0 + u * step, a.rows - 1);
            dy[u] = load_vec<KIND>(row_at<KIND>(a.dy, row) + at, valid);
            if constexpr (CODES)
                load_codes((const char*)a.codes.data + row * a.codes.stride + (size_t)c * kVec, valid,
                           a.scales[row * p.blocks + min(c / kBlockLanes, p.blocks - 1)], z[u]);
            else unpack<KIND>(load_vec<KIND>(row_at<KIND>(a.z, row) + at, valid), z[u]);
        }
        #pragma unroll
        for (int u = 0; u < kBackRows; ++u) {
            const size_t row = row0 + u * step;
            if (row >= a.rows) break;
            float v[kVec];
            unpack<KIND>(dy[u], v);
            with_act(a.act, [&](auto A) {
                #pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] *= slope_of<decltype(A)::value>(z[u][i]);
            });
            #pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] += v[i];
            if (a.dx.data) store_vec<KIND>(row_at<KIND>(a.dx, row) + at, pack<KIND>(v), valid);
        }
    }
    if (!p.dbias) return;
    if (wave > 0) {
        #pragma unroll
        for (int i = 0; i < kVec; ++i) lds[wave - 1][i][lane] = acc[i];
    }
    __syncthreads();
    if (wave == 0) {
        for (int w = 0; w < kBackWaves - 1; ++w) {
            #pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] += lds[w][i][lane];
        }
        if (gridDim.x > 1) store_vec<kF32>((char*)(a.parts + (size_t)blockIdx.x * a.cols + (size_t)c * kVec), pack<kF32>(acc), valid);
        else store_any((char*)p.dbias, p.grad, c, valid, acc);
    }
}

inline size_t row_lanes(size_t cols) { return (cols + kBlockCols - 1) / kBlockCols * kBlockLanes; }

}  // namespace

int launch_activation(const ActivationPass& a, int kind, void* stream)
{
    const ActivationArgs p{a, row_lanes(a.cols)};
    const dim3 grid(grid_of((a.rows * p.groups + kActLanes - 1) / kActLanes));
    return dispatch_kind(kind, [&](auto K) {
        return launch_args(activation_kernel<decltype(K)::value>, grid, dim3(kActLanes), 0, stream, p);
    });
}

int launch_checkpoint_read(const CheckpointRead& a, int kind, void* stream)
{
    const ReadArgs p{a, row_lanes(a.cols)};
    return dispatch_kind(kind, [&](auto K) {
        return launch_args(checkpoint_read_kernel<decltype(K)::value>, dim3(grid_of((a.rows * p.groups + kActLanes - 1) / kActLanes)),
                           dim3(kActLanes), 0, stream, p);
    });
}

int launch_activation_backward(const ActivationBackward& a, int kind, void* dbias, int grad, void* stream)
{
    const BackwardArgs p{a, (a.cols + kBlockCols - 1) / kBlockCols, dbias, grad};
    const size_t stripes = (vectors(a.cols) + 63) / 64;
    const size_t want = std::max<size_t>(1, kBackBlocks * kUnits / stripes);
    const bool one = a.rows > 0 && (a.rows <= 4 * kBackWaves * kBackRows || want == 1);
    const size_t workgroups = (a.rows + kBackWaves - 1) / kBackWaves;
    const int groups = one && dbias ? 1 : (int)std::min({want, 2 * kMostParts, workgroups});
    const int err = a.rows == 0 ? 0 : dispatch_kind(kind, [&](auto K) { return dispatch_flag(a.codes.data != nullptr, [&](auto C) {
        return launch_args(activation_backward_kernel<decltype(K)::value, decltype(C)::value>, dim3((unsigned)groups, (unsigned)stripes),
                           dim3(64 * kBackWaves), 0, stream, p);
    }); });
    return err || one || !dbias ? err : launch_column_sums(a.parts, 1, groups, a.cols, &dbias, grad, stream);
}

}  // namespace mics
