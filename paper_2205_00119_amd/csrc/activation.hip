// Activations with their 8-bit checkpoints, forward and backward.
#include "rows.h"

#include <algorithm>

#include "activation.h"
#include "columns.h"
#include "linear_internal.h"

namespace mics {
namespace {

// A wavefront takes a stripe of 64 vectors of a row, or 64 >> shift narrow rows, and goes down the rows, FLIGHT of them at a time:
// places come from shifts alone and the bias is loaded once.  Workgroups that follow one another take a row's
// stripes, not rows: memory is slower where they take rows (us, 4096 x 10240 bf16 tanh 40.3 / 46.8), and where wavefronts go down many
// rows (4096 x 32768 115 / 128).
constexpr size_t kMostDown = 65535;            // workgroups above one another
template <int FLIGHT> struct Down {
    static constexpr int kLanes = FLIGHT == 1 ? 256 : 64;
    size_t rows;
    unsigned cols, shift;                      // shift: log2 of the lanes of a row
    struct Place {
        unsigned c;
        int valid;
        size_t row, step;
    };
    __device__ __forceinline__ Place place() const
    {
        const unsigned lane = threadIdx.x & 63u, c = blockIdx.x * 64 + (lane & ((1u << shift) - 1)), rows_at_once = (64u >> shift) * FLIGHT;
        constexpr size_t waves = kLanes / 64;
        return {c, valid_at(c, cols), ((size_t)blockIdx.y * waves + wave_index()) * rows_at_once + (lane >> shift),
                (size_t)gridDim.y * waves * rows_at_once};
    }
    __device__ __forceinline__ unsigned across() const { return 64u >> shift; }
};
// Memory bounds it where operations do not: an element has some 30 of them for the 5.06 bytes that it moves in 16 bits (4096 x 32768
// bf16 tanh 121 us, 5.6 TB/s; gelu, whose polynomial takes ten more, 148 to 151; runs of calls on two sets of matrices in turn, from
// event to event: a kernel trace has medians a fifth above that and the same minima).
template <int FLIGHT> struct ActivationArgs {
    ActivationPass a;
    Down<FLIGHT> down;
};
template <int KIND, int FLIGHT> __global__ __launch_bounds__(Down<FLIGHT>::kLanes) void activation_kernel(ActivationArgs<FLIGHT> p)
{
    const ActivationPass& a = p.a;
    const auto at = p.down.place();
    const size_t from = (size_t)at.c * (kVec * kWidth<KIND>);
    Epilogue e = a.e;
    float bias[kVec] = {};
    if (e.bias) load_any((const char*)e.bias, e.param, at.c, at.valid, bias);
    e.bias = nullptr;
    for (size_t row0 = at.row; row0 < a.rows; row0 += at.step) {
        Raw<KIND> x[FLIGHT];
        #pragma unroll
        for (int u = 0; u < FLIGHT; ++u)
            x[u] = load_vec<KIND>(row_at<KIND>(a.x, min(row0 + u * p.down.across(), a.rows - 1)) + from, at.valid);
        #pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const size_t row = row0 + u * p.down.across();
            if (row >= a.rows) break;                       // whole blocks of lanes
            float v[kVec];
            unpack<KIND>(x[u], v);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += bias[i];
            finish<KIND>(e, row, at.c, a.cols, at.valid, v);
        }
    }
}

// 3.06 bytes for some 18 operations with an activation (4096 x 32768 bf16 tanh 81 us, 5.1 TB/s, gelu 103, measured as above).
template <int FLIGHT> struct ReadArgs {
    CheckpointRead a;
    Down<FLIGHT> down;
    unsigned blocks;
};
template <int KIND, int FLIGHT> __global__ __launch_bounds__(Down<FLIGHT>::kLanes) void checkpoint_read_kernel(ReadArgs<FLIGHT> p)
{
    const CheckpointRead& a = p.a;
    const auto at = p.down.place();
    const unsigned block = min(at.c / kBlockLanes, p.blocks - 1);
    for (size_t row0 = at.row; row0 < a.rows; row0 += at.step) {
        u32x2 q[FLIGHT];
        float scale[FLIGHT];
        #pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const size_t row = min(row0 + u * p.down.across(), a.rows - 1);
            q[u] = load_codes((const char*)a.codes.data + row * a.codes.stride + (size_t)at.c * kVec, at.valid);
            scale[u] = a.scales[row * p.blocks + block];
        }
        #pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const size_t row = row0 + u * p.down.across();
            if (row >= a.rows) break;
            float v[kVec];
            restored(q[u].x, scale[u], v);
            restored(q[u].y, scale[u], v + 4);
            with_act(a.act, [&](auto A) {
                #pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] = act_of<decltype(A)::value>(v[i]);
            });
            store_vec<KIND>(row_at<KIND>(a.y, row) + (size_t)at.c * (kVec * kWidth<KIND>), pack<KIND>(v), at.valid);
        }
    }
}

// dx and, with dbias, column sums over the rows of a workgroup: a wavefront takes a stripe of 64 vectors, or 64 >> shift narrow
// rows, and every gridDim.y * kBackWaves-th set of rows, ROWS of them in flight.  Bound by memory (4096 x 32768 bf16 tanh 137 us,
// 4.95 TB/s; without sums 119 to 125, 5.4 to 5.7) and, in small calls, by the second launch, which joins the sums.
constexpr int kBackWaves = 4;
struct BackwardArgs {
    ActivationBackward a;
    unsigned blocks, shift;
    void* dbias;                               // where a stripe has one workgroup, it stores the sums themselves
    int grad;
};
template <int KIND, bool CODES, int ROWS>
__global__ __launch_bounds__(64 * kBackWaves) void activation_backward_kernel(BackwardArgs p)
{
    const ActivationBackward& a = p.a;
    __shared__ float lds[kBackWaves][kVec][64];
    const int wave = wave_index();
    const unsigned lane = threadIdx.x & 63u, c = blockIdx.x * 64 + (lane & ((1u << p.shift) - 1)), across = 64u >> p.shift;
    const int valid = valid_at(c, a.cols);
    const unsigned block = min(c / kBlockLanes, p.blocks - 1);
    const size_t at = (size_t)c * (kVec * kWidth<KIND>), step = (size_t)gridDim.y * kBackWaves * across;
    float acc[kVec] = {};
    for (size_t row0 = ((size_t)blockIdx.y * kBackWaves + wave) * across + (lane >> p.shift); row0 < a.rows; row0 += ROWS * step) {
        Raw<KIND> dy[ROWS];
        Raw<KIND> z[ROWS];
        u32x2 q[ROWS];
        float scale[ROWS];
        #pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const size_t row = min(row0 + u * step, a.rows - 1);
            dy[u] = load_vec<KIND>(row_at<KIND>(a.dy, row) + at, valid);
            if constexpr (CODES) {
                q[u] = load_codes((const char*)a.codes.data + row * a.codes.stride + (size_t)c * kVec, valid);
                scale[u] = a.scales[row * p.blocks + block];
            } else z[u] = load_vec<KIND>(row_at<KIND>(a.z, row) + at, valid);
        }
        #pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const size_t row = row0 + u * step;
            if (row >= a.rows) break;
            float v[kVec], t[kVec];
            unpack<KIND>(dy[u], v);
            if constexpr (CODES) {
                restored(q[u].x, scale[u], t);
                restored(q[u].y, scale[u], t + 4);
            } else unpack<KIND>(z[u], t);
            with_act(a.act, [&](auto A) {
                #pragma unroll
                for (int i = 0; i < kVec; ++i) v[i] *= slope_of<decltype(A)::value>(t[i]);
            });
            #pragma unroll
            for (int i = 0; i < kVec; ++i) acc[i] += v[i];
            if (a.dx.data) store_vec<KIND>(row_at<KIND>(a.dx, row) + at, pack<KIND>(v), valid);
        }
    }
    if (!p.dbias) return;
    #pragma unroll
    for (int i = 0; i < kVec; ++i) lds[wave][i][lane] = acc[i];
    __syncthreads();
    if (threadIdx.x >> p.shift == 0) {                          // the first row's lanes: wavefronts, then their rows, in ascending order
        #pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] = 0.f;
        for (int w = 0; w < kBackWaves; ++w)
            for (unsigned r = lane; r < 64; r += 1u << p.shift) {
                #pragma unroll
                for (int i = 0; i < kVec; ++i) acc[i] += lds[w][i][r];
            }
        if (gridDim.y > 1) store_vec<kF32>((char*)(a.parts + (size_t)blockIdx.y * a.cols + (size_t)c * kVec), pack<kF32>(acc), valid);
        else store_any((char*)p.dbias, p.grad, c, valid, acc);
    }
}

// log2 of the lanes of a row
inline unsigned shift_of(unsigned cols)
{
    unsigned shift = 3;
    while (shift < 6 && (cols + kBlockCols - 1) / kBlockCols * kBlockLanes > (1u << shift)) ++shift;
    return shift;
}
inline size_t stripes_of(unsigned cols) { return ((size_t)((cols + kBlockCols - 1) / kBlockCols) * kBlockLanes + 63) / 64; }
// Calls f(std::integral_constant<int, FLIGHT>, grid).  us, one row at a time by workgroups of 256 lanes / two by 64 / two by 256:
// 4096 x 32768 bf16 tanh 159 / 116 / 117, read 97 / 79 / 81, 8192 x 2560 20.4 / 18.8 / 18.6; 300 x 4099 4.4 / 5.3 / 5.1,
// 1003 x 5125 f32 10.6 / 11.1 / 11.6, 4096 x 16384 f32 read 71 / 79 / 75, 20000 x 100 5.3 / 6.3 / 6.1.
template <typename F> int down_rows(size_t rows, unsigned cols, int kind, F&& f)
{
    const size_t stripes = stripes_of(cols);
    auto go = [&](auto FLIGHT) {
        const size_t at_once = (size_t{64} >> shift_of(cols)) * decltype(FLIGHT)::value * (Down<decltype(FLIGHT)::value>::kLanes / 64);
        return f(FLIGHT, dim3((unsigned)stripes, (unsigned)std::min((rows + at_once - 1) / at_once, kMostDown)));
    };
    const bool two = kind != kF32 && rows >= ((size_t{1} << 21) + stripes * 64 - 1) / (stripes * 64);
    return two ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 1>{});
}

}  // namespace

int launch_activation(const ActivationPass& a, int kind, void* stream)
{
    return dispatch_kind(kind, [&](auto K) { return down_rows(a.rows, a.cols, kind, [&](auto F, dim3 grid) {
        constexpr int FLIGHT = decltype(F)::value;
        const ActivationArgs<FLIGHT> p{a, {a.rows, a.cols, shift_of(a.cols)}};
        return launch_args(activation_kernel<decltype(K)::value, FLIGHT>, grid, dim3(Down<FLIGHT>::kLanes), 0, stream, p);
    }); });
}

int launch_checkpoint_read(const CheckpointRead& a, int kind, void* stream)
{
    return dispatch_kind(kind, [&](auto K) { return down_rows(a.rows, a.cols, kind, [&](auto F, dim3 grid) {
        constexpr int FLIGHT = decltype(F)::value;
        const ReadArgs<FLIGHT> p{a, {a.rows, a.cols, shift_of(a.cols)}, (a.cols + kBlockCols - 1) / kBlockCols};
        return launch_args(checkpoint_read_kernel<decltype(K)::value, FLIGHT>, grid, dim3(Down<FLIGHT>::kLanes), 0, stream, p);
    }); });
}

int launch_activation_backward(const ActivationBackward& a, int kind, void* dbias, int grad, void* stream)
{
    const unsigned shift = shift_of(a.cols);
    const BackwardArgs p{a, (a.cols + kBlockCols - 1) / kBlockCols, shift, dbias, grad};
    const size_t stripes = stripes_of(a.cols), across = size_t{64} >> shift;
    // us, two rows and four workgroups for each compute unit / one and eight: 4096 x 32768 bf16 137 / 145, 8192 x 2560 25.2 / 24.4,
    // 2047 x 5121 binary16 18.1 / 17.5, 300 x 4099 9.3 / 8.3; without sums, as many workgroups as there are rows for, 125 / 116, 21.3 / 19.4
    const bool two = dbias && a.rows >= ((size_t{1} << 23) + stripes * 64 - 1) / (stripes * 64);
    const size_t want = std::max<size_t>(1, (two ? 4 : 8) * kUnits / stripes);
    const bool one = dbias && a.rows > 0 && (a.rows <= 8 * kBackWaves * across || want == 1);
    const size_t workgroups = ceil_div(a.rows, kBackWaves * across);
    const int groups = (int)(one ? 1 : std::min(workgroups, dbias ? std::min(want, 2 * kMostParts) : kMostDown));
    const int err = a.rows == 0 ? 0 : dispatch_kind(kind, [&](auto K) { return dispatch_flag(a.codes.data != nullptr, [&](auto C) {
        return dispatch_flag(two, [&](auto T) {
            return launch_args(activation_backward_kernel<decltype(K)::value, decltype(C)::value, decltype(T)::value ? 2 : 1>,
                               dim3((unsigned)stripes, (unsigned)groups), dim3(64 * kBackWaves), 0, stream, p);
        });
    }); });
    return err || one || !dbias ? err : launch_column_sums(a.parts, 1, groups, a.cols, &dbias, grad, stream);
}

}  // namespace mics
