// Dropout with bias and residual, forward and backward, and the sums over groups of rows that backward passes leave.
#include "rows.h"

#include <algorithm>

#include "columns.h"
#include "layer_internal.h"

namespace mics {
namespace {

// out_k[c], k = blockIdx.y, for the 64 columns of a workgroup: 16 lanes take four columns each, the 16 rows of lanes every
// 16th group of rows in ascending order, eight loads in flight; then their 16 sums, in ascending order.
struct ColumnSumsArgs {
    const float* parts;
    void* out[3];
    unsigned cols;
    int groups, kind;
};
constexpr int kSumLanes = 256, kSumRows = 16, kSumFlight = 8;
__global__ __launch_bounds__(kSumLanes) void column_sums_kernel(ColumnSumsArgs p)
{
    __shared__ float lds[kSumRows][64];
    void* const out = p.out[blockIdx.y];
    if (!out) return;
    const unsigned row = threadIdx.x / 16, c = blockIdx.x * 64 + threadIdx.x % 16 * 4;
    const float* const from = p.parts + (size_t)blockIdx.y * p.groups * p.cols;
    float s[4] = {};
    if (c + 4 <= p.cols) {
        for (int g = row; g < p.groups; g += kSumRows * kSumFlight) {
            f32x4 v[kSumFlight];
            #pragma unroll
            for (int u = 0; u < kSumFlight; ++u)
                v[u] = *(const f32x4_a4*)(from + (size_t)min(g + u * kSumRows, p.groups - 1) * p.cols + c);
            #pragma unroll
            for (int u = 0; u < kSumFlight; ++u) {
                #pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += g + u * kSumRows < p.groups ? v[u][i] : 0.f;
            }
        }
    } else {
        for (int g = row; g < p.groups; g += kSumRows)
            for (unsigned i = 0; c + i < p.cols; ++i) s[i & 3] += from[(size_t)g * p.cols + c + i];
    }
    #pragma unroll
    for (int i = 0; i < 4; ++i) lds[row][threadIdx.x % 16 * 4 + i] = s[i];
    __syncthreads();
    const unsigned column = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x < 64 && column < p.cols) {
        float sum = 0.f;
        #pragma unroll
        for (int r = 0; r < kSumRows; ++r) sum += lds[r][threadIdx.x];
        if (p.kind == kBf16) store_one<kBf16>((uint16_t*)out + column, sum);
        else if (p.kind == kF16) store_one<kF16>((uint16_t*)out + column, sum);
        else store_one<kF32>((float*)out + column, sum);
    }
}

// ---------------------------------------------------------------------------
// Dropout.  Vectors of eight in ascending order, one for each lane; backward is the same with nothing added.  A vector takes one
// block of the generator: 16-bit numbers instead of 32-bit ones halve its cost, which is hidden almost whole behind memory
// (4096 x 8192 bf16, bias and residual: 42.4 us = 4.75 TB/s, 38.1 without dropout).  Caps on the wavefronts of a compute unit,
// which help kernels with less arithmetic, only cost here (12 a unit 54.2 us).
// ---------------------------------------------------------------------------
struct DropoutArgs {
    DropoutPass a;
    size_t groups;        // vectors, and generator blocks, of a row
    void* dbias;          // where a stripe has one workgroup, it stores the sums themselves
    int grad;
};
// Single wavefronts (us, 64 / 256 / 512 lanes: 4096 x 8192 bf16 42.1 / 42.9 / 43.2, 4096 x 2560 13.1 / 13.6 / 14.1).
constexpr int kDropLanes = 64;

template <int KIND, int TAIL>
__global__ __launch_bounds__(kDropLanes) void dropout_kernel(DropoutArgs p)
{
    const DropoutPass& a = p.a;
    const size_t vecs = a.rows * p.groups;
    const unsigned groups = (unsigned)p.groups;
    for (size_t base = (size_t)blockIdx.x * kDropLanes; base < vecs; base += (size_t)gridDim.x * kDropLanes) {
        if (base + threadIdx.x >= vecs) break;
        const size_t row0 = base / p.groups;                                    // the same in all lanes
        const unsigned at = (unsigned)(base - row0 * p.groups) + threadIdx.x, up = at / groups, c = at - up * groups;
        const size_t row = row0 + up;
        Raw<KIND> x = load_col<KIND, TAIL>(row_at<KIND>(a.x, row), c, a.cols), r{};
        if (a.residual.data) r = load_col<KIND, TAIL>(row_at<KIND>(a.residual, row), c, a.cols);
        float v[kVec], t[kVec];
        settle<KIND, TAIL>(x, c, a.cols);
        unpack<KIND>(x, v);
        if (a.bias) {
            load_param<TAIL>(a.bias, a.param, c, a.cols, 0.f, t);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += t[i];
        }
        if (a.drop.threshold) drop_vec(v, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
        if (a.residual.data) {
            settle<KIND, TAIL>(r, c, a.cols);
            unpack<KIND>(r, t);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += t[i];
        }
        store_col<KIND, TAIL>(row_at<KIND>(a.out, row), c, a.cols, pack<KIND>(v));
    }
}

// Backward with the bias's gradient: a workgroup's wavefronts take every gridDim.x * kStripeWaves-th row of a stripe of 64
// vectors, kStripeRows of them in flight.
// us, two rows / four / eight: 2047 x 5121 binary16 13.8 / 14.5 / 18.0; workgroups on a compute unit 4 / 8 / 16: 8192 x 2560
// bf16 20.1 / 22.6 / 22.3.
constexpr int kStripeWaves = 4, kStripeRows = 2, kStripeBlocks = 4;
template <int KIND, int TAIL>
__global__ __launch_bounds__(64 * kStripeWaves) void dropout_backward_kernel(DropoutArgs p)
{
    const DropoutPass& a = p.a;
    __shared__ float lds[kStripeWaves - 1][kVec][64];
    const int wave = wave_index();
    const unsigned lane = threadIdx.x & 63u, c = blockIdx.y * 64 + lane;
    const size_t step = (size_t)gridDim.x * kStripeWaves;
    float acc[kVec] = {};
    for (size_t row0 = (size_t)blockIdx.x * kStripeWaves + wave; row0 < a.rows; row0 += kStripeRows * step) {
        Raw<KIND> x[kStripeRows];
        #pragma unroll
        for (int u = 0; u < kStripeRows; ++u)
            x[u] = load_col<KIND, TAIL>(row_at<KIND>(a.x, min(row0 + u * step, a.rows - 1)), c, a.cols);
        #pragma unroll
        for (int u = 0; u < kStripeRows; ++u) {
            const size_t row = row0 + u * step;
            if (row >= a.rows) break;
            float v[kVec];
            settle<KIND, TAIL>(x[u], c, a.cols);
            unpack<KIND>(x[u], v);
            if (a.drop.threshold) drop_vec(v, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] += v[i];
            store_col<KIND, TAIL>(row_at<KIND>(a.out, row), c, a.cols, pack<KIND>(v));
        }
    }
    if (wave > 0) {
        #pragma unroll
        for (int i = 0; i < kVec; ++i) lds[wave - 1][i][lane] = acc[i];
    }
    __syncthreads();
    if (wave == 0) {
        for (int w = 0; w < kStripeWaves - 1; ++w) {
            #pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] += lds[w][i][lane];
        }
        if (gridDim.x > 1) store_col<kF32, TAIL>((char*)(a.parts + (size_t)blockIdx.x * a.cols), c, a.cols, pack<kF32>(acc));
        else if (p.grad == kBf16) store_col<kBf16, TAIL>((char*)p.dbias, c, a.cols, pack<kBf16>(acc));
        else if (p.grad == kF16) store_col<kF16, TAIL>((char*)p.dbias, c, a.cols, pack<kF16>(acc));
        else store_col<kF32, TAIL>((char*)p.dbias, c, a.cols, pack<kF32>(acc));
    }
}

}  // namespace

int launch_column_sums(const float* parts, int sums, int groups, size_t cols, void* const* out, int kind, void* stream)
{
    ColumnSumsArgs p{parts, {}, (unsigned)cols, groups, kind};
    for (int k = 0; k < sums; ++k) p.out[k] = out[k];
    return launch_args(column_sums_kernel, dim3((unsigned)((cols + 63) / 64), (unsigned)sums), dim3(kSumLanes), 0, stream, p);
}

int launch_dropout(const DropoutPass& a, int kind, void* stream)
{
    const DropoutArgs p{a, vectors(a.cols), nullptr, 0};
    return dispatch_kind(kind, [&](auto K) { return dispatch_tail(a.cols, [&](auto T) {
        return launch_args(dropout_kernel<decltype(K)::value, decltype(T)::value>,
                           dim3(grid_of((a.rows * p.groups + kDropLanes - 1) / kDropLanes)), dim3(kDropLanes), 0, stream, p);
    }); });
}

int launch_dropout_backward(const DropoutPass& a, int kind, void* dbias, int grad, void* stream)
{
    const DropoutArgs p{a, vectors(a.cols), dbias, grad};
    const size_t stripes = (p.groups + 63) / 64;
    const size_t want = std::max<size_t>(1, kStripeBlocks * kUnits / stripes);
    // few rows: one workgroup for each stripe, and no second launch (us, two / one: 4 x 4096 7.5 / 4.7, 32 x 4096 7.4 / 5.0,
    // 64 x 4096 7.3 / 7.9)
    const bool one = a.rows > 0 && (a.rows <= 4 * kStripeWaves * kStripeRows || want == 1);
    const int groups = one ? 1 : (int)std::min({want, 2 * kMostParts, (a.rows + kStripeWaves - 1) / kStripeWaves});
    const int err = a.rows == 0 ? 0 : dispatch_kind(kind, [&](auto K) { return dispatch_tail(a.cols, [&](auto T) {
        return launch_args(dropout_backward_kernel<decltype(K)::value, decltype(T)::value>,
                           dim3((unsigned)groups, (unsigned)stripes), dim3(64 * kStripeWaves), 0, stream, p);
    }); });
    return err || one ? err : launch_column_sums(a.parts, 1, groups, a.cols, &dbias, grad, stream);
}

}  // namespace mics
