// Layer norm, alone and behind bias, dropout and residual in one pass, forward and backward.
//
// Rows that fit a workgroup's registers (forward up to 16384 columns, backward up to 8192) are read once and written once: a row stays
// with the lanes that read it, from the load to the last store.  Longer ones are read three times forward and twice backward,
// from the caches where these hold them.  Bound by HBM bandwidth at large sizes, by launches and reductions at small ones.
// Workgroups stay on their compute unit and go from row to row; the loads of the next row are in flight while one is worked on.
//
// Measured on one MI355X, bf16, three sets of buffers in turn: forward 8192 x 8192 49.2 us = 5.46 TB/s (HBM traffic equal to the
// algorithmic bytes), with bias, dropout and residual 4096 x 5120 36.1 us = 4.65 TB/s; backward 4096 x 4096 25.4 us, 20 of them in
// the first kernel (5.0 TB/s), with all there is 4096 x 8192 74.1 us = 4.5 TB/s, 67 in the first.  Longer rows: forward 2048 x 16400
// 43.8 us = 3.1 TB/s, backward with all there is 4096 x 12288 150 us = 3.4 TB/s of what has to be moved.  Results are left to the caches
// for whoever reads them next: stored past them the forward pass is up to 20 % shorter by itself (4096 x 5120 28.5 us), but
// with the kernels that read y and sum behind it 4 % longer (69.2 / 71.9; 4096 x 4096 55.7 / 59.9).
#include "rows.h"

#include <algorithm>

#include "columns.h"
#include "layer_internal.h"

namespace mics {
namespace {

constexpr int kMostWaves = 16;

// ---------------------------------------------------------------------------
// Forward.  A row is held by `waves` wavefronts, V vectors of eight columns in each lane.  Every wavefront forms the mean
// of its columns and their square distance from it; those of n1, n2, ... columns join as
//     mean = sum ni mi / n,    M = sum (Mi + ni (mi - mean)^2),
// so that one barrier is enough and nothing cancels.
// FUSED: what is normalised is residual + D(x + bias) before it is rounded; the rounded sum is stored as well.
// ---------------------------------------------------------------------------
struct NormForwardArgs {
    NormForward a;
    size_t groups;        // generator blocks of a row
    int waves;            // of a row
    bool add;             // the residual
};

// Loads and stores of the loop that a branch could skip would make every wait in it one for all loads in flight: rows past
// the last are loaded as the last one, lanes past the end of a row repeat its end (Place), and what is absent is replaced by
// the host (residual: x, not added; sum: y, stored over).
// STATS: mean and rstd are both asked for.  KEEP: the parameters of the lane's columns stay in registers.
template <int KIND, int V, bool FUSED, int TAIL, bool STATS, bool KEEP, int BUFFERS, int LANES>
__global__ __launch_bounds__(LANES) void norm_kernel(NormForwardArgs p)
{
    const NormForward& a = p.a;
    __shared__ float2 parts[2][kMostWaves];
    const int wave = wave_index(), group = wave / p.waves;
    const unsigned lanes = 64u * p.waves, lane = threadIdx.x - lanes * group, per_block = blockDim.x / lanes;
    const size_t step = (size_t)gridDim.x * per_block;
    size_t row = (size_t)blockIdx.x * per_block + group;
    if (row >= a.rows) return;                           // a row of several wavefronts is alone in its workgroup
    auto place = [&](int v) { return Place<TAIL>(lane + v * lanes, a.cols); };
    Raw<KIND> x[BUFFERS][V], residual[FUSED ? BUFFERS : 1][V];
    auto load = [&](int k, size_t r) {
        r = min(r, a.rows - 1);
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            x[k][v] = place(v).template load<KIND>(row_at<KIND>(a.x, r));
            if constexpr (FUSED) residual[k][v] = place(v).template load<KIND>(row_at<KIND>(a.residual, r));
        }
    };
    #pragma unroll
    for (int k = 0; k < BUFFERS - 1; ++k) load(k, row + k * step);

    const float n = (float)a.cols;
    float mine = 0.f, others = 0.f;      // columns of this wavefront; of wavefront `lane`
    #pragma unroll
    for (int v = 0; v < V; ++v) mine += place(v).columns();
    mine = wave_sum(mine);
    #pragma unroll
    for (int v = 0; v < V; ++v) {
        const int l = threadIdx.x & 63u, begin = (l + p.waves * v) * 64 * kVec;
        others += l < p.waves ? (float)min(max((int)a.cols - begin, 0), 64 * kVec) : 0.f;
    }
    const float over = 1.f / mine;
    float w[KEEP ? V : 1][kVec], b[KEEP ? V : 1][kVec], bias[KEEP && FUSED ? V : 1][kVec];
    if constexpr (KEEP) {
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            place(v).param(a.weight, a.param, 1.f, w[v]);
            place(v).param(a.norm_bias, a.param, 0.f, b[v]);
            if constexpr (FUSED) place(v).param(a.bias, a.param, 0.f, bias[v]);
        }
    }
    for (int turn = 0;;) {
        #pragma unroll
        for (int k = 0; k < BUFFERS; ++k) {
            load((k + BUFFERS - 1) % BUFFERS, row + (BUFFERS - 1) * step);
            float s[V][kVec], total = 0.f;
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                const Place<TAIL> at = place(v);
                unpack<KIND>(x[k][v], s[v]);
                if constexpr (FUSED) {
                    float t[kVec];
                    if constexpr (!KEEP) at.param(a.bias, a.param, 0.f, bias[0]);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) s[v][i] += bias[KEEP ? v : 0][i];
                    if (a.drop.threshold)
                        drop_at(s[v], at, a.drop.offset + row * p.groups, a.drop.seed, a.drop.threshold, a.drop.scale);
                    unpack<KIND>(residual[k][v], t);
                    if (p.add) {
                        #pragma unroll
                        for (int i = 0; i < kVec; ++i) s[v][i] += t[i];
                    }
                }
                float sum = 0.f;
                #pragma unroll
                for (int i = 0; i < kVec; ++i) sum += at.element(s[v][i], i);
                total += at.vector(sum);
            }
            float mean = wave_sum(total) * over, square = 0.f;
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                const Place<TAIL> at = place(v);
                float sum = 0.f;
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float d = at.element(s[v][i] - mean, i);
                    sum = __builtin_fmaf(d, d, sum);
                }
                square += at.vector(sum);
            }
            square = wave_sum(square);
            if (p.waves > 1) {
                const int l = threadIdx.x & 63u;
                if (l == 0) parts[turn][wave] = {mean, square};
                barrier_lds();
                const float2 part = l < p.waves ? parts[turn][l] : float2{0.f, 0.f};
                mean = sum_of_16(others * part.x) / n;
                const float d = part.x - mean;
                square = sum_of_16(__builtin_fmaf(others * d, d, part.y));
                turn ^= 1;
            }
            const float rstd = 1.f / __builtin_sqrtf(square / n + a.eps);
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                const Place<TAIL> at = place(v);
                if constexpr (!KEEP) {
                    at.param(a.weight, a.param, 1.f, w[0]);
                    at.param(a.norm_bias, a.param, 0.f, b[0]);
                }
                const float (&wv)[kVec] = w[KEEP ? v : 0], (&bv)[kVec] = b[KEEP ? v : 0];
                float y[kVec];
                #pragma unroll
                for (int i = 0; i < kVec; ++i) y[i] = __builtin_fmaf((s[v][i] - mean) * rstd, wv[i], bv[i]);
                if constexpr (FUSED) at.template store<KIND>(row_at<KIND>(a.sum, row), pack<KIND>(s[v]));
                at.template store<KIND>(row_at<KIND>(a.y, row), pack<KIND>(y));
            }
            if (STATS || a.mean) a.mean[row] = mean;       // the same from every lane
            if (STATS || a.rstd) a.rstd[row] = rstd;
            row += step;
            if (row >= a.rows) return;
        }
    }
}

// Sums of a row over `waves` wavefronts.  Every call of a workgroup takes the slot that its previous one did not, so that
// one barrier is enough.
struct RowSums {
    float2 slot[2][kMostWaves];
};
__device__ __forceinline__ float2 row_sum(RowSums& lds, int turn, int wave, int first, int waves, float a, float b)
{
    float2 s = {wave_sum(a), wave_sum(b)};
    if (waves == 1) return s;
    float2* const slot = lds.slot[turn];
    const int lane = threadIdx.x & 63u;
    if (lane == 0) slot[wave] = s;
    barrier_lds();
    s = lane < waves ? slot[first + lane] : float2{0.f, 0.f};
    return {sum_of_16(s.x), sum_of_16(s.y)};
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
                float s[kVec], t[kVec];
                read_col<KIND>(row_at<KIND>(a.x, row), c, a.cols, s);
                if constexpr (FUSED) {
                    load_param<kRagged>(a.bias, a.param, c, a.cols, 0.f, t);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) s[i] += t[i];
                    if (a.drop.threshold)
                        drop_vec(s, a.drop.offset + row * p.groups + c, a.drop.seed, a.drop.threshold, a.drop.scale);
                    if (p.add) {
                        read_col<KIND>(row_at<KIND>(a.residual, row), c, a.cols, t);
                        #pragma unroll
                        for (int i = 0; i < kVec; ++i) s[i] += t[i];
                    }
                }
                if (pass == 2) {       // the last use of x and residual, which sum or y may replace
                    float w[kVec], b[kVec], y[kVec];
                    load_param<kRagged>(a.weight, a.param, c, a.cols, 1.f, w);
                    load_param<kRagged>(a.norm_bias, a.param, c, a.cols, 0.f, b);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) y[i] = __builtin_fmaf((s[i] - mean) * rstd, w[i], b[i]);
                    if (FUSED) store_col<KIND, kRagged>(row_at<KIND>(a.sum, row), c, a.cols, pack<KIND>(s));
                    store_col<KIND, kRagged>(row_at<KIND>(a.y, row), c, a.cols, pack<KIND>(y));
                }
                const int valid = valid_at(c, a.cols);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float d = summand<kRagged>(s[i] - mean, i, valid);      // mean is 0 in the first pass
                    total = pass == 0 ? total + d : __builtin_fmaf(d, d, total);
                }
            }
            if (pass == 0) mean = row_sum(lds, 0, wave, 0, kMostWaves, total, 0.f).x / n;
            if (pass == 1) rstd = 1.f / __builtin_sqrtf(row_sum(lds, 1, wave, 0, kMostWaves, total, 0.f).x / n + a.eps);
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
// MODE: the norm alone; with what is in front of it; with a gradient that reaches the sum as well.
// ---------------------------------------------------------------------------
enum { kAlone = 0, kBlock = 1, kBlockSum = 2 };
struct NormBackwardArgs {
    NormBackward a;
    size_t groups;
    int waves, batch;
    void* grads[3];       // where one workgroup has all rows, it stores the sums themselves
    int grad;
};

// What the loop must not skip is as in the forward pass (dresidual: dx, stored over).  TILED: s1 and s2 come from
// row_sums_kernel, and since no barrier keeps a tile's wavefronts together, lanes past the end of a row store nothing.
template <int KIND, int V, int MODE, int TAIL, int BUFFERS, bool TILED, int LANES>
__global__ __launch_bounds__(LANES) void norm_backward_kernel(NormBackwardArgs p)
{
    const NormBackward& a = p.a;
    extern __shared__ float joined[];
    __shared__ RowSums lds;
    constexpr int SUMS = MODE == kAlone ? 2 : 3;
    const int wave = wave_index(), group = wave / p.waves, first = group * p.waves;
    const unsigned lanes = 64u * p.waves, lane = threadIdx.x - lanes * group;
    const unsigned c0 = blockIdx.y * lanes * V + lane;      // blockIdx.y: the tile of a row that is cut into tiles
    const float over = 1.f / (float)a.cols;
    const size_t step = (size_t)gridDim.x * p.batch;
    size_t base = (size_t)blockIdx.x * p.batch;
    auto place = [&](int v) { return Place<TAIL>(c0 + v * lanes, a.cols); };
    struct Row {
        Raw<KIND> dy[V], x[V], dsum[MODE == kBlockSum ? V : 1];
        float mean, rstd, s1, s2;
    };
    Row buffer[BUFFERS];
    auto load = [&](Row& to, size_t row) {
        row = min(row, a.rows - 1);
        to.mean = a.mean[row];
        to.rstd = a.rstd[row];
        if constexpr (TILED) {
            to.s1 = a.row_sums[2 * row];
            to.s2 = a.row_sums[2 * row + 1];
        }
        #pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (TILED && TAIL == kRagged) {
                to.dy[v] = load_col<KIND, TAIL>(row_at<KIND>(a.dy, row), c0 + v * lanes, a.cols);
                to.x[v] = load_col<KIND, TAIL>(row_at<KIND>(a.x, row), c0 + v * lanes, a.cols);
                if constexpr (MODE == kBlockSum) to.dsum[v] = load_col<KIND, TAIL>(row_at<KIND>(a.dsum, row), c0 + v * lanes, a.cols);
            } else {
                to.dy[v] = place(v).template load<KIND>(row_at<KIND>(a.dy, row));
                to.x[v] = place(v).template load<KIND>(row_at<KIND>(a.x, row));
                if constexpr (MODE == kBlockSum) to.dsum[v] = place(v).template load<KIND>(row_at<KIND>(a.dsum, row));
            }
        }
    };
    #pragma unroll
    for (int k = 0; k < BUFFERS - 1; ++k) load(buffer[k], base + group + k * step);
    float acc[SUMS][V][kVec] = {}, w[V][kVec];
    #pragma unroll
    for (int v = 0; v < V; ++v) {
        if constexpr (TILED) load_param<TAIL>(a.weight, a.param, c0 + v * lanes, a.cols, 1.f, w[v]);
        else place(v).param(a.weight, a.param, 1.f, w[v]);
    }
    auto store = [&](const Rows& to, size_t row, int v, const Raw<KIND>& r) {
        if constexpr (TILED) store_col<KIND, TAIL>(row_at<KIND>(to, row), c0 + v * lanes, a.cols, r);
        else place(v).template store<KIND>(row_at<KIND>(to, row), r);
    };
    int turn = 0;
    // PART: `mine` is false in wavefronts past the last row, which pass the barrier only
    auto work = [&](auto PART, Row& now, size_t row, bool mine) {
        constexpr bool ALL = !decltype(PART)::value;
        float s1 = 0.f, s2 = 0.f, hat[V][kVec], d[V][kVec];
        if (ALL || mine) {
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                const Place<TAIL> at = place(v);
                if constexpr (TILED) {
                    settle<KIND, TAIL>(now.dy[v], c0 + v * lanes, a.cols);
                    settle<KIND, TAIL>(now.x[v], c0 + v * lanes, a.cols);
                    if constexpr (MODE == kBlockSum) settle<KIND, TAIL>(now.dsum[v], c0 + v * lanes, a.cols);
                }
                float dy[kVec], x[kVec], p1 = 0.f, p2 = 0.f;
                unpack<KIND>(now.dy[v], dy);
                unpack<KIND>(now.x[v], x);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    hat[v][i] = (x[i] - now.mean) * now.rstd;
                    d[v][i] = dy[i] * w[v][i];
                    acc[0][v][i] = __builtin_fmaf(dy[i], hat[v][i], acc[0][v][i]);
                    acc[1][v][i] += dy[i];
                    if constexpr (!TILED) {
                        const float own = at.element(d[v][i], i);
                        p1 += own;
                        p2 = __builtin_fmaf(own, hat[v][i], p2);
                    }
                }
                s1 += at.vector(p1);
                s2 += at.vector(p2);
            }
        }
        float2 s = {now.s1, now.s2};
        if constexpr (!TILED) {
            // dresidual may replace dsum: what other lanes read of it has arrived before the barrier
            if constexpr (MODE == kBlockSum) {
                #pragma unroll
                for (int v = 0; v < V; ++v) arrived<KIND>(now.dsum[v]);
            }
            s = row_sum(lds, turn, wave, first, p.waves, s1, s2);
            turn ^= 1;
        }
        if (ALL || mine) {
            // rstd (d - c1 - hat c2)
            const float c1 = -(now.rstd * over) * s.x, c2 = -(now.rstd * over) * s.y;
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                float ds[kVec];
                #pragma unroll
                for (int i = 0; i < kVec; ++i) ds[i] = __builtin_fmaf(hat[v][i], c2, __builtin_fmaf(d[v][i], now.rstd, c1));
                if constexpr (MODE == kBlockSum) {
                    float t[kVec];
                    unpack<KIND>(now.dsum[v], t);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) ds[i] += t[i];
                }
                if constexpr (MODE != kAlone) {
                    const Raw<KIND> unchanged = pack<KIND>(ds);
                    if (a.drop.threshold) {
                        const uint64_t block = a.drop.offset + row * p.groups;
                        if constexpr (TILED) drop_vec(ds, block + c0 + v * lanes, a.drop.seed, a.drop.threshold, a.drop.scale);
                        else drop_at(ds, place(v), block, a.drop.seed, a.drop.threshold, a.drop.scale);
                    }
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) acc[SUMS - 1][v][i] += ds[i];
                    store(a.dresidual, row, v, unchanged);
                }
                store(a.dx, row, v, pack<KIND>(ds));
            }
        }
    };
    while (base + p.batch <= a.rows) {
        #pragma unroll
        for (int k = 0; k < BUFFERS; ++k) {
            load(buffer[(k + BUFFERS - 1) % BUFFERS], base + group + (BUFFERS - 1) * step);
            work(std::false_type{}, buffer[k], base + group, true);
            base += step;
            if (base + p.batch > a.rows) break;
        }
    }
    if (base < a.rows) {               // the last batch, in part
        load(buffer[0], base + group);
        work(std::true_type{}, buffer[0], base + group, base + group < a.rows);
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
        if (group == 0 && !TILED && gridDim.x == 1) {
            if (p.grads[k]) {
                #pragma unroll
                for (int v = 0; v < V; ++v) place(v).round(p.grads[k], p.grad, acc[k][v]);
            }
        } else if (group == 0) {
            float* const part = a.parts + ((size_t)k * gridDim.x + blockIdx.x) * a.cols;
            #pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (TILED) store_col<kF32, TAIL>((char*)part, c0 + v * lanes, a.cols, pack<kF32>(acc[k][v]));
                else place(v).template store<kF32>((char*)part, pack<kF32>(acc[k][v]));
            }
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
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
        for (unsigned c = threadIdx.x; c < vecs; c += 1024) {
            const int valid = valid_at(c, a.cols);
            float dy[kVec], x[kVec], w[kVec];
            read_col<KIND>(row_at<KIND>(a.dy, row), c, a.cols, dy);
            read_col<KIND>(row_at<KIND>(a.x, row), c, a.cols, x);
            load_param<kRagged>(a.weight, a.param, c, a.cols, 1.f, w);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const float d = summand<kRagged>(dy[i] * w[i], i, valid);
                s1 += d;
                s2 = __builtin_fmaf(d, (x[i] - mean) * rstd, s2);
            }
        }
        const float2 s = row_sum(lds, turn, wave, 0, kMostWaves, s1, s2);
        if (threadIdx.x == 0) ((float2*)a.row_sums)[row] = s;
    }
}

// Wavefronts of a compute unit that stay and go from row to row (us, 16 / 24 / 32: 4096 x 5120 bf16 19.2 / 16.2 / 17.9,
// 8192 x 8192 49.4 / 49.2 / 49.4; with dropout, 16 / 20 / 24: 4096 x 5120 38.3 / 36.1 / 36.1).
constexpr int kNormWaves = 24, kBlockWaves = 20;
template <int N> using Int = std::integral_constant<int, N>;

}  // namespace

int launch_norm(const NormForward& given, int kind, bool fused, void* stream)
{
    NormForward a = given;
    const size_t vecs = vectors(a.cols);
    const bool add = a.residual.data;
    if (!a.residual.data) a.residual = a.x;
    if (!a.sum.data) a.sum = a.y;
    NormForwardArgs p{a, vecs, 1, add};
    return dispatch_kind(kind, [&](auto K) { return dispatch_flag(fused, [&](auto F) {
        constexpr int KIND = decltype(K)::value;
        constexpr bool FUSED = decltype(F)::value;
        auto with = [&](auto VV, auto BB, auto LL, auto KK) {
            constexpr int V = decltype(VV)::value, BUFFERS = decltype(BB)::value, LANES = decltype(LL)::value;
            constexpr bool KEEP = decltype(KK)::value;
            return dispatch_tail<V == 1>(a.cols, [&](auto T) { return dispatch_flag(a.mean && a.rstd, [&](auto S) {
                p.waves = waves_of(vecs, V);
                const unsigned per_block = p.waves == 1 ? 4 : 1;
                const size_t blocks = std::min<size_t>((a.rows + per_block - 1) / per_block,
                                                       kUnits * std::max<size_t>(1, (FUSED ? kBlockWaves : kNormWaves) / (p.waves * per_block)));
                return launch_args(norm_kernel<KIND, V, FUSED, decltype(T)::value, decltype(S)::value, KEEP, BUFFERS, LANES>,
                                   dim3((unsigned)blocks), dim3(64u * p.waves * per_block), 0, stream, p);
            }); });
        };
        // One vector in each lane for a row of one wavefront, two for longer ones (8192 x 8192 bf16: one 54.1 us, two 49.4); with
        // dropout one, whose parameters and two rows fit the registers (4096 x 5120: one 36.1 us, two 68.1), up to 8192 columns.  Up to
        // 16384 two, whose parameters are read again for every row (4096 x 12288 98.9 us = 4.1 TB/s; 2048 x 12285 f32, whose rest spills
        // five registers, 101.5).
        if (waves_of(vecs, 1) <= 1) return with(Int<1>{}, Int<3>{}, Int<256>{}, std::true_type{});
        if constexpr (FUSED) {
            if (waves_of(vecs, 1) <= kMostWaves) return with(Int<1>{}, Int<2>{}, Int<1024>{}, std::true_type{});
            if (waves_of(vecs, 2) <= kMostWaves) return with(Int<2>{}, Int<2>{}, Int<1024>{}, std::false_type{});
        } else {
            if (waves_of(vecs, 2) <= kMostWaves) return with(Int<2>{}, Int<2>{}, Int<1024>{}, std::true_type{});
        }
        return launch_args(norm_long_kernel<KIND, FUSED>, dim3(grid_of(a.rows)), dim3(1024), 0, stream, p);
    }); });
}

int launch_norm_backward(const NormBackward& given, int kind, bool fused, void* const* grads, int grad, void* stream)
{
    NormBackward a = given;
    if (!a.dresidual.data) a.dresidual = a.dx;
    const size_t vecs = vectors(a.cols);
    NormBackwardArgs p{a, vecs, 1, 1, {grads[0], grads[1], fused ? grads[2] : nullptr}, grad};
    int groups = 0;
    bool sums = true;
    // no row: the gradients of the parameters are zero
    const int err = a.rows == 0 ? 0 : dispatch_kind(kind, [&](auto K) {
        constexpr int KIND = decltype(K)::value;
        auto mode = [&](auto M) {
            constexpr int MODE = decltype(M)::value;
            auto with = [&](auto VV, auto BB, auto TT) {
                constexpr int V = decltype(VV)::value, BUFFERS = decltype(BB)::value, LANES = 1024;
                return dispatch_tail<!decltype(TT)::value>(a.cols, [&](auto T) {
                    p.waves = waves_of(std::min<size_t>(vecs, (size_t)LANES * V), V);
                    p.batch = LANES / 64 / p.waves;
                    // few rows: one workgroup, and no second launch (us, two / one: 1 x 2560 8.2 / 4.9, 8 x 2560 in three batches 7.8 / 7.1,
                    // 4 x 8192 in four 7.7 / 7.7)
                    const bool one = !decltype(TT)::value && a.rows <= 2 * (size_t)p.batch;
                    sums = !one;
                    groups = one ? 1 : (int)std::min<size_t>(kMostParts, (a.rows + p.batch - 1) / p.batch);
                    const size_t lds = (size_t)(p.batch - 1) * 64 * p.waves * V * kVec * 4;
                    const size_t tile = (size_t)64 * p.waves * V;
                    return launch_args(norm_backward_kernel<KIND, V, MODE, decltype(T)::value, BUFFERS, decltype(TT)::value, LANES>,
                                       dim3((unsigned)groups, (unsigned)((vecs + tile - 1) / tile)), dim3(64u * p.waves * p.batch),
                                       lds, stream, p);
                });
            };
            // One vector in each lane, two rows in registers (4096 x 8192 bf16 with all there is: two 74 us, three 94, which
            // spill).  Two spill as well where there is most to hold: behind dropout with a rest 6 to 12 registers of 128 (f32 10
            // to 33), f32 with dsum 9 on whole vectors, tiles with dsum 2 to 22.  4096 x 5120 f32 without dsum 70.6 us and with it
            // 92.2, 4096 x 5121 133.3; bf16 4096 x 5121 without 49.5 and with 76.9.  Longer rows in tiles of 8192 columns: two vectors
            // in each lane are faster for the norm alone (4096 x 12288 bf16: tiles 105 us, so 93) and much slower with all there
            // is (150 / 273; 1024 x 12288 f32 59 / 70), and one way serves all.
            if (a.cols > kTiledCols) {
                if (int e = launch_args(row_sums_kernel<KIND>, dim3(grid_of(a.rows)), dim3(1024), 0, stream, p)) return e;
                return with(Int<1>{}, Int<2>{}, std::true_type{});
            }
            return with(Int<1>{}, Int<2>{}, std::false_type{});
        };
        if (!fused) return mode(Int<kAlone>{});
        if (!a.dsum.data) return mode(Int<kBlock>{});
        return mode(Int<kBlockSum>{});
    });
    return err || !sums ? err : launch_column_sums(a.parts, fused ? 3 : 2, groups, a.cols, grads, grad, stream);
}

}  // namespace mics
