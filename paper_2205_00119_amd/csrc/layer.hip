// Layer norm, dropout with bias and residual, and both in one pass, forward and backward.
//
// Every byte is read once and written once: a row stays in the registers of the lanes that read it, in binary32, from
// the load to the last store.  All are bound by HBM bandwidth at large sizes and by launches and reductions at small ones.
#include "rows.h"

#include <algorithm>
#include <type_traits>

#include "layer_internal.h"

namespace mics {
namespace {

constexpr int kMostWaves = 16;

// Sums of one row's lanes over the `waves` wavefronts that share it.  Every call of a workgroup takes the slot that
// its previous one did not, so that one barrier is enough.
struct RowSums {
    float2 slot[2][kMostWaves];
};
__device__ __forceinline__ float2 row_sum(RowSums& lds, int turn, int wave, int first, int waves, float a, float b)
{
    float2 s = {wave_sum(a), wave_sum(b)};
    if (waves == 1) return s;
    float2* const slot = lds.slot[turn & 1];
    if ((threadIdx.x & 63u) == 0) slot[wave] = s;
    __syncthreads();
    s = slot[first];
    for (int w = 1; w < waves; ++w) {
        s.x += slot[first + w].x;
        s.y += slot[first + w].y;
    }
    return s;
}
__device__ __forceinline__ float row_sum(RowSums& lds, int turn, int wave, int first, int waves, float a)
{
    return row_sum(lds, turn, wave, first, waves, a, 0.f).x;
}

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

template <int KIND> __device__ __forceinline__ const char* row_at(const ConstRows& m, size_t row)
{
    return (const char*)m.data + row * m.stride * kWidth<KIND>;
}
template <int KIND> __device__ __forceinline__ char* row_at(const Rows& m, size_t row)
{
    return (char*)m.data + row * m.stride * kWidth<KIND>;
}

// ---------------------------------------------------------------------------
// Forward.  A row is held by `waves` wavefronts, V vectors of eight columns in each lane; the variance is the mean
// square distance from the mean, from registers, so nothing cancels.
// FUSED: what is normalised is residual + D(x + bias) before it is rounded; the rounded sum is stored as well.
// ---------------------------------------------------------------------------
struct NormForwardArgs {
    NormForward a;
    size_t groups;        // generator blocks of a row
    int waves;            // of a row
};

template <int KIND, bool FUSED, bool RAGGED>
__device__ __forceinline__ void norm_input(const NormForwardArgs& p, size_t row, unsigned c, const Raw<KIND>& x,
                                           const Raw<KIND>& residual, float (&s)[kVec])
{
    const NormForward& a = p.a;
    unpack<KIND>(x, s);
    if constexpr (FUSED) {
        float t[kVec];
        if (a.bias) {
            load_param<RAGGED>(a.bias, a.param, c, a.cols, 0.f, t);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) s[i] += t[i];
        }
        if (a.drop.threshold) drop_vec(s, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
        if (a.residual.data) {
            unpack<KIND>(residual, t);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) s[i] += t[i];
        }
    }
}

template <int KIND, bool RAGGED>
__device__ __forceinline__ void norm_output(const NormForward& a, size_t row, unsigned c, float mean, float rstd,
                                            const float (&s)[kVec])
{
    float w[kVec], b[kVec], y[kVec];
    load_param<RAGGED>(a.weight, a.param, c, a.cols, 1.f, w);
    load_param<RAGGED>(a.norm_bias, a.param, c, a.cols, 0.f, b);
    #pragma unroll
    for (int i = 0; i < kVec; ++i) y[i] = __builtin_fmaf((s[i] - mean) * rstd, w[i], b[i]);
    store_col<KIND, RAGGED>(row_at<KIND>(a.y, row), c, a.cols, pack<KIND>(y));
}

template <int KIND, int V, bool FUSED, bool RAGGED, int LANES>
__global__ __launch_bounds__(LANES) void norm_kernel(NormForwardArgs p)
{
    const NormForward& a = p.a;
    __shared__ RowSums lds;
    const int wave = wave_index(), group = wave / p.waves, first = group * p.waves;
    const unsigned lanes = 64u * p.waves, lane = threadIdx.x - 64u * first;
    const unsigned per_block = blockDim.x / lanes;
    const float n = (float)a.cols;
    // rows of one wavefront need no barrier: those of a workgroup may differ in their number
    for (size_t row = (size_t)blockIdx.x * per_block + group; row < a.rows; row += (size_t)gridDim.x * per_block) {
        Raw<KIND> x[V], r[V];
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = load_col<KIND, RAGGED>(row_at<KIND>(a.x, row), lane + v * lanes, a.cols);
            if (FUSED && a.residual.data) r[v] = load_col<KIND, RAGGED>(row_at<KIND>(a.residual, row), lane + v * lanes, a.cols);
        }
        float s[V][kVec], total = 0.f;
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            const unsigned c = lane + v * lanes;
            const int valid = valid_at(c, a.cols);
            norm_input<KIND, FUSED, RAGGED>(p, row, c, x[v], r[v], s[v]);
            if (FUSED && a.sum.data) store_col<KIND, RAGGED>(row_at<KIND>(a.sum, row), c, a.cols, pack<KIND>(s[v]));
            float part = 0.f;
            #pragma unroll
            for (int i = 0; i < kVec; ++i) part += summand<RAGGED>(s[v][i], i, valid);
            total += vector_sum<RAGGED>(part, valid);
        }
        const float mean = row_sum(lds, 0, wave, first, p.waves, total) / n;
        float square = 0.f;
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            const int valid = valid_at(lane + v * lanes, a.cols);
            float part = 0.f;
            #pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float d = summand<RAGGED>(s[v][i] - mean, i, valid);
                part = __builtin_fmaf(d, d, part);
            }
            square += vector_sum<RAGGED>(part, valid);
        }
        const float rstd = 1.f / __builtin_sqrtf(row_sum(lds, 1, wave, first, p.waves, square) / n + a.eps);
        #pragma unroll
        for (int v = 0; v < V; ++v) norm_output<KIND, RAGGED>(a, row, lane + v * lanes, mean, rstd, s[v]);
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows that no workgroup's registers hold: three passes over them, the second and third from the caches.
template <int KIND, bool FUSED>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormForwardArgs p)
{
    const NormForward& a = p.a;
    __shared__ RowSums lds;
    const int wave = wave_index();
    const unsigned vecs = (unsigned)p.groups;
    const float n = (float)a.cols;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float mean = 0.f, rstd = 0.f;
        for (int pass = 0; pass < 3; ++pass) {
            float total = 0.f;
            for (unsigned c = threadIdx.x; c < vecs; c += 1024) {
                const Raw<KIND> x = load_col<KIND, true>(row_at<KIND>(a.x, row), c, a.cols);
                Raw<KIND> r{};
                if (FUSED && a.residual.data) r = load_col<KIND, true>(row_at<KIND>(a.residual, row), c, a.cols);
                float s[kVec];
                norm_input<KIND, FUSED, true>(p, row, c, x, r, s);
                if (pass == 2) {       // the last use of x and residual, which sum or y may replace
                    if (FUSED && a.sum.data) store_col<KIND, true>(row_at<KIND>(a.sum, row), c, a.cols, pack<KIND>(s));
                    norm_output<KIND, true>(a, row, c, mean, rstd, s);
                }
                const int valid = valid_at(c, a.cols);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float d = summand<true>(s[i] - mean, i, valid);      // mean is 0 in the first pass
                    total = pass == 0 ? total + d : __builtin_fmaf(d, d, total);
                }
            }
            if (pass == 0) mean = row_sum(lds, 0, wave, 0, kMostWaves, total) / n;
            if (pass == 1) rstd = 1.f / __builtin_sqrtf(row_sum(lds, 1, wave, 0, kMostWaves, total) / n + a.eps);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// ---------------------------------------------------------------------------
// Backward.  A workgroup takes every gridDim.x-th batch of `batch` rows, each held by `waves` wavefronts, and sums
// dy * hat, dy (and the gradient behind dropout) of its own columns in registers over all its rows; the sums of its
// batch rows are joined through the LDS and left in `parts`, one row for each workgroup, for column_sums_kernel.
// The next rows' loads are in flight while the present ones are reduced.
// ---------------------------------------------------------------------------
struct NormBackwardArgs {
    NormBackward a;
    size_t groups;
    int waves, batch;
};

template <int KIND, int V, bool FUSED, bool RAGGED> struct BackwardRow {
    Raw<KIND> dy[V], x[V], dsum[FUSED ? V : 1];
    float mean, rstd;
    __device__ __forceinline__ void load(const NormBackward& a, size_t row, unsigned c0, unsigned lanes)
    {
        mean = a.mean[row];
        rstd = a.rstd[row];
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            const unsigned c = c0 + v * lanes;
            dy[v] = load_col<KIND, RAGGED>(row_at<KIND>(a.dy, row), c, a.cols);
            x[v] = load_col<KIND, RAGGED>(row_at<KIND>(a.x, row), c, a.cols);
            if constexpr (FUSED)
                if (a.dsum.data) dsum[v] = load_col<KIND, RAGGED>(row_at<KIND>(a.dsum, row), c, a.cols);
        }
    }
};

template <int KIND, int V, bool FUSED, bool RAGGED, int LANES>
__global__ __launch_bounds__(LANES) void norm_backward_kernel(NormBackwardArgs p)
{
    const NormBackward& a = p.a;
    extern __shared__ float joined[];
    __shared__ RowSums lds;
    constexpr int SUMS = FUSED ? 3 : 2;
    const int wave = wave_index(), group = wave / p.waves, first = group * p.waves;
    const unsigned lanes = 64u * p.waves, lane = threadIdx.x - 64u * first;
    const unsigned c0 = blockIdx.y * lanes * V + lane;      // blockIdx.y: the tile of a row that is cut into tiles
    const float n = (float)a.cols;
    float acc[SUMS][V][kVec] = {}, w[V][kVec];
    #pragma unroll
    for (int v = 0; v < V; ++v) load_param<RAGGED>(a.weight, a.param, c0 + v * lanes, a.cols, 1.f, w[v]);
    const size_t step = (size_t)gridDim.x * p.batch;
    size_t row = (size_t)blockIdx.x * p.batch + group;
    BackwardRow<KIND, V, FUSED, RAGGED> now, next;
    if (row < a.rows) now.load(a, row, c0, lanes);
    int turn = 0;
    // all of a workgroup's wavefronts pass the same number of barriers, those past the last row included
    for (size_t base = (size_t)blockIdx.x * p.batch; base < a.rows; base += step, row += step, ++turn) {
        if (row + step < a.rows) next.load(a, row + step, c0, lanes);
        const bool mine = row < a.rows;
        float s1 = 0.f, s2 = 0.f;
        if (mine) {
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                float dy[kVec], x[kVec], p1 = 0.f, p2 = 0.f;
                unpack<KIND>(now.dy[v], dy);
                unpack<KIND>(now.x[v], x);
                const int valid = valid_at(c0 + v * lanes, a.cols);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float hat = (x[i] - now.mean) * now.rstd, d = summand<RAGGED>(dy[i] * w[v][i], i, valid);
                    acc[0][v][i] = __builtin_fmaf(dy[i], hat, acc[0][v][i]);
                    acc[1][v][i] += dy[i];
                    p1 += d;
                    p2 = __builtin_fmaf(d, hat, p2);
                }
                s1 += vector_sum<RAGGED>(p1, valid);
                s2 += vector_sum<RAGGED>(p2, valid);
            }
        }
        float2 s;
        if (a.row_sums) s = mine ? ((const float2*)a.row_sums)[row] : float2{0.f, 0.f};
        else s = row_sum(lds, turn, wave, first, p.waves, s1, s2);
        if (mine) {
            const float c1 = s.x / n, c2 = s.y / n;
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                const unsigned c = c0 + v * lanes;
                float dy[kVec], x[kVec], ds[kVec];
                unpack<KIND>(now.dy[v], dy);
                unpack<KIND>(now.x[v], x);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float hat = (x[i] - now.mean) * now.rstd;
                    ds[i] = now.rstd * ((dy[i] * w[v][i] - c1) - hat * c2);
                }
                if constexpr (FUSED) {
                    if (a.dsum.data) {
                        float t[kVec];
                        unpack<KIND>(now.dsum[v], t);
                        #pragma unroll
                        for (int i = 0; i < kVec; ++i) ds[i] += t[i];
                    }
                    if (a.dresidual.data) store_col<KIND, RAGGED>(row_at<KIND>(a.dresidual, row), c, a.cols, pack<KIND>(ds));
                    if (a.drop.threshold)
                        drop_vec(ds, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) acc[SUMS - 1][v][i] += ds[i];
                }
                store_col<KIND, RAGGED>(row_at<KIND>(a.dx, row), c, a.cols, pack<KIND>(ds));
            }
        }
        now = next;
    }
    // the batch rows' sums in ascending order
    float* const mine = joined + (size_t)(group - 1) * lanes * V * kVec;
    #pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        if (p.batch > 1) {
            __syncthreads();
            if (group > 0) {
                #pragma unroll
                for (int j = 0; j < V * kVec; ++j) mine[j * lanes + lane] = acc[k][j / kVec][j % kVec];
            }
            __syncthreads();
            if (group == 0)
                for (int g = 1; g < p.batch; ++g) {
                    const float* other = joined + (size_t)(g - 1) * lanes * V * kVec;
                    #pragma unroll
                    for (int j = 0; j < V * kVec; ++j) acc[k][j / kVec][j % kVec] += other[j * lanes + lane];
                }
        }
        if (group == 0) {
            float* const part = a.parts + ((size_t)k * gridDim.x + blockIdx.x) * a.cols;
            #pragma unroll
            for (int v = 0; v < V; ++v) store_col<kF32, RAGGED>((char*)part, c0 + v * lanes, a.cols, pack<kF32>(acc[k][v]));
        }
    }
}

// s1 and s2 of rows that are cut into tiles.
template <int KIND>
__global__ __launch_bounds__(1024) void row_sums_kernel(NormBackwardArgs p)
{
    const NormBackward& a = p.a;
    __shared__ RowSums lds;
    const int wave = wave_index();
    const unsigned vecs = (unsigned)p.groups;
    int turn = 0;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++turn) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
        for (unsigned c = threadIdx.x; c < vecs; c += 1024) {
            const int valid = valid_at(c, a.cols);
            float dy[kVec], x[kVec], w[kVec];
            unpack<KIND>(load_col<KIND, true>(row_at<KIND>(a.dy, row), c, a.cols), dy);
            unpack<KIND>(load_col<KIND, true>(row_at<KIND>(a.x, row), c, a.cols), x);
            load_param<true>(a.weight, a.param, c, a.cols, 1.f, w);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float d = summand<true>(dy[i] * w[i], i, valid);
                s1 += d;
                s2 = __builtin_fmaf(d, (x[i] - mean) * rstd, s2);
            }
        }
        const float2 s = row_sum(lds, turn, wave, 0, kMostWaves, s1, s2);
        if (threadIdx.x == 0) ((float2*)a.row_sums)[row] = s;
    }
}

// out_k[c] = the sum over the groups of rows of parts[k][group][c], k = blockIdx.y, rounded once.  16 wavefronts take
// every 16th group, in ascending order; then their 16 sums, in ascending order.
struct ColumnSumsArgs {
    const float* parts;
    void* out[3];
    size_t cols;
    int groups, kind;
};
__global__ __launch_bounds__(1024) void column_sums_kernel(ColumnSumsArgs p)
{
    __shared__ float lds[16][64];
    const unsigned lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const size_t c = (size_t)blockIdx.x * 64 + lane;
    void* const out = p.out[blockIdx.y];
    if (!out) return;
    float s = 0.f;
    if (c < p.cols)
        for (int g = wave; g < p.groups; g += 16) s += p.parts[((size_t)blockIdx.y * p.groups + g) * p.cols + c];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < p.cols) {
        for (int w = 1; w < 16; ++w) s += lds[w][lane];
        if (p.kind == kBf16) store_one<kBf16>((uint16_t*)out + c, s);
        else if (p.kind == kF16) store_one<kF16>((uint16_t*)out + c, s);
        else store_one<kF32>((float*)out + c, s);
    }
}
int launch_column_sums(const float* parts, int sums, int groups, size_t cols, void* const* out, int kind, void* stream)
{
    ColumnSumsArgs p{parts, {}, cols, groups, kind};
    for (int k = 0; k < sums; ++k) p.out[k] = out[k];
    return launch_args(column_sums_kernel, dim3((unsigned)((cols + 63) / 64), (unsigned)sums), dim3(1024), 0, stream, p);
}

// ---------------------------------------------------------------------------
// Dropout.  Vectors of eight in ascending order, one for each lane; backward is the same with nothing added.
// ---------------------------------------------------------------------------
struct DropoutArgs {
    DropoutPass a;
    size_t groups;        // vectors, and generator blocks, of a row
};
constexpr int kDropLanes = 256;

template <int KIND, bool RAGGED>
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
        const Raw<KIND> x = load_col<KIND, RAGGED>(row_at<KIND>(a.x, row), c, a.cols);
        Raw<KIND> r{};
        if (a.residual.data) r = load_col<KIND, RAGGED>(row_at<KIND>(a.residual, row), c, a.cols);
        float v[kVec], t[kVec];
        unpack<KIND>(x, v);
        if (a.bias) {
            load_param<RAGGED>(a.bias, a.param, c, a.cols, 0.f, t);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += t[i];
        }
        if (a.drop.threshold) drop_vec(v, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
        if (a.residual.data) {
            unpack<KIND>(r, t);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += t[i];
        }
        store_col<KIND, RAGGED>(row_at<KIND>(a.out, row), c, a.cols, pack<KIND>(v));
    }
}

// Backward with the bias's gradient: a workgroup's four wavefronts take four rows of a stripe of 64 vectors at a time.
constexpr int kStripeWaves = 4;
template <int KIND, bool RAGGED>
__global__ __launch_bounds__(64 * kStripeWaves) void dropout_backward_kernel(DropoutArgs p)
{
    const DropoutPass& a = p.a;
    __shared__ float lds[kStripeWaves - 1][kVec][64];
    const int wave = wave_index();
    const unsigned lane = threadIdx.x & 63u, c = blockIdx.y * 64 + lane;
    float acc[kVec] = {};
    #pragma unroll 4
    for (size_t row = (size_t)blockIdx.x * kStripeWaves + wave; row < a.rows; row += (size_t)gridDim.x * kStripeWaves) {
        float v[kVec];
        unpack<KIND>(load_col<KIND, RAGGED>(row_at<KIND>(a.x, row), c, a.cols), v);
        if (a.drop.threshold) drop_vec(v, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
        #pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] += v[i];
        store_col<KIND, RAGGED>(row_at<KIND>(a.out, row), c, a.cols, pack<KIND>(v));
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
        store_col<kF32, RAGGED>((char*)(a.parts + (size_t)blockIdx.x * a.cols), c, a.cols, pack<kF32>(acc));
    }
}

size_t vectors(size_t cols) { return (cols + kVec - 1) / kVec; }
int waves_of(size_t vecs, int per_lane) { return (int)((vecs + 64 * per_lane - 1) / (64 * per_lane)); }
// A grid of at most 2^20 workgroups: a launch's lanes have to stay below 2^32, the kernels stride over the rest.
unsigned grid_of(size_t blocks) { return (unsigned)std::min<size_t>(blocks, 1u << 20); }

constexpr size_t kUnits = 256;              // compute units of an MI355X

}  // namespace

int launch_norm(const NormForward& a, int kind, bool fused, void* stream)
{
    const size_t vecs = vectors(a.cols);
    NormForwardArgs p{a, vecs, 1};
    return dispatch_kind(kind, [&](auto K) { return dispatch_flag(fused, [&](auto F) {
        constexpr int KIND = decltype(K)::value;
        constexpr bool FUSED = decltype(F)::value;
        auto with = [&](auto VV, auto LL) { return dispatch_flag(a.cols % kVec != 0, [&](auto R) {
            constexpr int V = decltype(VV)::value, LANES = decltype(LL)::value;
            p.waves = waves_of(vecs, V);
            const unsigned per_block = p.waves == 1 ? 4 : 1;
            return launch_args(norm_kernel<KIND, V, FUSED, decltype(R)::value, LANES>,
                               dim3(grid_of((a.rows + per_block - 1) / per_block)), dim3(64u * p.waves * per_block), 0, stream, p);
        }); };
        if (waves_of(vecs, 1) <= 4) return with(std::integral_constant<int, 1>{}, std::integral_constant<int, 256>{});
        if (waves_of(vecs, 2) <= 8) return with(std::integral_constant<int, 2>{}, std::integral_constant<int, 512>{});
        if (waves_of(vecs, 4) <= 8) return with(std::integral_constant<int, 4>{}, std::integral_constant<int, 512>{});
        return launch_args(norm_long_kernel<KIND, FUSED>, dim3(grid_of(a.rows)), dim3(1024), 0, stream, p);
    }); });
}

int launch_norm_backward(const NormBackward& a, int kind, bool fused, void* const* grads, int grad, void* stream)
{
    const size_t vecs = vectors(a.cols);
    NormBackwardArgs p{a, vecs, 1, 1};
    int groups = 0;
    // no row: the gradients of the parameters are zero
    const int err = a.rows == 0 ? 0 : dispatch_kind(kind, [&](auto K) { return dispatch_flag(fused, [&](auto F) {
        constexpr int KIND = decltype(K)::value;
        constexpr bool FUSED = decltype(F)::value;
        auto with = [&](auto VV, auto LL) { return dispatch_flag(a.cols % kVec != 0, [&](auto R) {
            constexpr int V = decltype(VV)::value, LANES = decltype(LL)::value;
            p.waves = waves_of(std::min<size_t>(vecs, (size_t)LANES * V), V);
            p.batch = LANES / 64 / p.waves;
            groups = (int)std::min<size_t>(kUnits, (a.rows + p.batch - 1) / p.batch);
            const size_t lds = (size_t)(p.batch - 1) * 64 * p.waves * V * kVec * 4;
            const size_t tile = (size_t)64 * p.waves * V;
            return launch_args(norm_backward_kernel<KIND, V, FUSED, decltype(R)::value, LANES>,
                               dim3((unsigned)groups, (unsigned)((vecs + tile - 1) / tile)), dim3(64u * p.waves * p.batch), lds,
                               stream, p);
        }); };
        if (a.cols > kTiledCols) {
            if (int e = launch_args(row_sums_kernel<KIND>, dim3(grid_of(a.rows)), dim3(1024), 0, stream, p)) return e;
        } else {
            p.a.row_sums = nullptr;
        }
        if (waves_of(vecs, 1) <= 16) return with(std::integral_constant<int, 1>{}, std::integral_constant<int, 1024>{});
        return with(std::integral_constant<int, 4>{}, std::integral_constant<int, 512>{});
    }); });
    return err ? err : launch_column_sums(a.parts, fused ? 3 : 2, groups, a.cols, grads, grad, stream);
}

int launch_dropout(const DropoutPass& a, int kind, void* stream)
{
    const DropoutArgs p{a, vectors(a.cols)};
    return dispatch_kind(kind, [&](auto K) { return dispatch_flag(a.cols % kVec != 0, [&](auto R) {
        return launch_args(dropout_kernel<decltype(K)::value, decltype(R)::value>,
                           dim3(grid_of((a.rows * p.groups + kDropLanes - 1) / kDropLanes)), dim3(kDropLanes), 0, stream, p);
    }); });
}

int launch_dropout_backward(const DropoutPass& a, int kind, void* dbias, int grad, void* stream)
{
    const DropoutArgs p{a, vectors(a.cols)};
    const size_t stripes = (p.groups + 63) / 64;
    const size_t want = std::max<size_t>(1, 8 * kUnits / stripes);
    const int groups = (int)std::min({want, kMostParts, (a.rows + kStripeWaves - 1) / kStripeWaves});
    const int err = a.rows == 0 ? 0 : dispatch_kind(kind, [&](auto K) { return dispatch_flag(a.cols % kVec != 0, [&](auto R) {
        return launch_args(dropout_backward_kernel<decltype(K)::value, decltype(R)::value>,
                           dim3((unsigned)groups, (unsigned)stripes), dim3(64 * kStripeWaves), 0, stream, p);
    }); });
    return err ? err : launch_column_sums(a.parts, 1, groups, a.cols, &dbias, grad, stream);
}

}  // namespace mics
