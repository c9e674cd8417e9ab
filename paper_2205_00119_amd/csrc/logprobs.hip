// Log probabilities of given tokens with the row's log-sum-exp, entropy and best alternatives, and the gradient.
//
// With m the largest logit of a row, Z = sum e^(x-m) and T = sum (x-m) e^(x-m):
//     log p_j = x_j - m - log Z,    entropy = log Z - T / Z,
// so one pass that keeps (m, Z, T) and rescales them when m grows reads every logit once.  Z and T of two parts join as
//     Z = Z1 e^(m1-m) + Z2 e^(m2-m),    T = sum of e^(mi-m) (Ti + (mi-m) Zi).
// Bound by HBM bandwidth with many rows, by latency with few.
#include "rows.h"

#include <algorithm>

#include "layer_internal.h"

namespace mics {
namespace {

constexpr float kLowest = -3.402823466e38f, kLog2e = 1.4426950408889634f;
// e^-200 is 0 in binary32: the factor of such a term may stop there, which keeps 0 * inf out of the sums.
constexpr float kFar = -200.f;

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
__device__ __forceinline__ float infinity() { return __builtin_inff(); }

// m: the largest logit (NaN aside), -inf if there is none.  A NaN or +inf among the logits makes z and t NaN.
struct Stat {
    float m, z, t;
    __device__ __forceinline__ float base() const { return fmaxf(m, kLowest); }
    __device__ __forceinline__ void move_to(float base_to)
    {
        const float d = base() - base_to, e = exp_of(d);
        t = e * __builtin_fmaf(fmaxf(d, kFar), z, t);
        z *= e;
    }
};

// Lanes in the same fixed order as wave_sum; the result is in every lane.
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_max(float v)
{
    const int low = __builtin_bit_cast(int, -infinity());
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(low, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false)));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = dpp_max<0x111, 0xF>(v);
    v = dpp_max<0x112, 0xF>(v);
    v = dpp_max<0x114, 0xF>(v);
    v = dpp_max<0x118, 0xF>(v);
    v = dpp_max<0x142, 0xA>(v);
    v = dpp_max<0x143, 0xC>(v);
    return lane_value(v, 63);
}
// Largest of each aligned run of LANES lanes, in all of them.
template <int LANES> __device__ __forceinline__ float run_max(float v)
{
    v = dpp_max<0xB1, 0xF>(v);                                  // quad_perm 1,0,3,2
    v = dpp_max<0x4E, 0xF>(v);                                  // quad_perm 2,3,0,1
    if constexpr (LANES >= 8) v = dpp_max<0x141, 0xF>(v);       // row_half_mirror
    if constexpr (LANES >= 16) v = dpp_max<0x140, 0xF>(v);      // row_mirror
    return v;
}

// The order of alternatives: larger first, NaN before all, the lower index first among equals (-0 and +0 are equal).
// No element has key 0.
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float x, unsigned index)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.f ? 0.f : x);
    const uint32_t up = x != x ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (Key)up << 32 | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float value_of(Key k)
{
    const uint32_t up = (uint32_t)(k >> 32);
    if (up == 0xFFFFFFFFu) return __builtin_nanf("");
    return __builtin_bit_cast(float, up & 0x80000000u ? up ^ 0x80000000u : ~up);
}
__device__ __forceinline__ unsigned index_of(Key k) { return 0xFFFFFFFFu - (uint32_t)k; }

constexpr int kCandidates = 2048;

template <int LANES, bool TOP> struct LogProbsLds {
    Stat stat[LANES / 64];
};
template <int LANES> struct LogProbsLds<LANES, true> {
    Stat stat[LANES / 64];
    float run[64];
    float threshold;
    int count;
    Key best[kMostTop];
    Key wave_best[LANES / 64];
    Key candidate[kCandidates];
};

struct LogProbsArgs {
    LogProbs a;
    int splits;
    unsigned chunk;        // vectors of a split
};
// What a split leaves: a Stat padded to 16 bytes, then its best keys in order, 0 where it has fewer.

// Vectors [begin, end) of a row; the last one of the row may be short.
template <int KIND> struct Span {
    const char* row;
    unsigned begin, end, cols;
    // vectors with eight elements
    __device__ __forceinline__ unsigned whole() const { return min(end, cols / kVec); }
    __device__ __forceinline__ void vec(unsigned c, float (&x)[kVec]) const
    {
        const int valid = valid_at(c, cols);
        unpack<KIND>(load_vec<KIND>(row + (size_t)c * (kVec * kWidth<KIND>), valid), x);
        #pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = i < valid ? x[i] : -infinity();
    }
};

template <int N> __device__ __forceinline__ void add_logits(Stat& s, const float (&x)[N])
{
    float most = s.m;
    #pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, x[i]);
    const float base = fmaxf(most, kLowest);
    s.move_to(base);
    s.m = most;
    #pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = x[i] - base, e = exp_of(d);
        s.z += e;
        s.t = __builtin_fmaf(fmaxf(d, kFar), e, s.t);
    }
}

// A lane's part of the span: U vectors in flight.
template <int KIND, int LANES, int U> __device__ __forceinline__ Stat lane_stat(const Span<KIND>& span)
{
    Stat s = {-infinity(), 0.f, 0.f};
    const unsigned whole = span.whole();
    for (unsigned c = span.begin + threadIdx.x; c < whole; c += LANES * U) {
        Raw<KIND> r[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load_vec<KIND>(span.row + (size_t)min(c + u * LANES, whole - 1) * (kVec * kWidth<KIND>), kVec);
        #pragma unroll
        for (int u = 0; u < U; u += 2) {
            float x[2][kVec], both[2 * kVec];
            #pragma unroll
            for (int h = 0; h < 2; ++h) {
                unpack<KIND>(r[u + h], x[h]);
                const bool in = c + (u + h) * LANES < whole;
                #pragma unroll
                for (int i = 0; i < kVec; ++i) both[h * kVec + i] = in ? x[h][i] : -infinity();
            }
            add_logits(s, both);
        }
    }
    if (whole >= span.begin && whole < span.end && threadIdx.x == 0) {
        float x[kVec];
        span.vec(whole, x);
        add_logits(s, x);
    }
    return s;
}

// The workgroup's, in lane order within wavefronts, then by wavefront; in all lanes.
template <int LANES> __device__ __forceinline__ Stat block_stat(Stat (&lds)[LANES / 64], Stat s)
{
    const float most = wave_max(s.m);
    s.move_to(fmaxf(most, kLowest));
    s = {most, wave_sum(s.z), wave_sum(s.t)};
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63u) == 0) lds[wave] = s;
    __syncthreads();
    Stat all = lds[0];
    for (int w = 1; w < LANES / 64; ++w) all.m = fmaxf(all.m, lds[w].m);
    float z = 0.f, t = 0.f;
    for (int w = 0; w < LANES / 64; ++w) {
        Stat part = lds[w];
        part.move_to(all.base());
        z += part.z;
        t += part.t;
    }
    return {all.m, z, t};
}

// Calls f(x, index) for every element of the span, each by one lane.
template <int KIND, int LANES, typename F> __device__ __forceinline__ void each(const Span<KIND>& span, F&& f)
{
    for (unsigned c = span.begin + threadIdx.x; c < span.end; c += LANES) {
        float x[kVec];
        const int valid = valid_at(c, span.cols);
        if (valid >= kVec) unpack<KIND>(load_vec<KIND>(span.row + (size_t)c * (kVec * kWidth<KIND>), kVec), x);
        else span.vec(c, x);
        #pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < valid) f(x[i], c * kVec + i);
    }
}

template <int LANES> __device__ __forceinline__ void keep_candidate(LogProbsLds<LANES, true>& lds, float x, unsigned index)
{
    const int at = atomicAdd(&lds.count, 1);      // their order does not matter: they are ranked by key
    if (at < kCandidates) lds.candidate[at] = key_of(x, index);
}

// The `top` best of the span into lds.best in order, behind a barrier; 0 where the span has fewer.  most: the lane's
// largest logit.  The top-th largest of 64 runs' largest logits is at most the top-th largest logit, and few others
// reach it: those that do are ranked.  Where too many do (equal logits, a mask that leaves fewer than `top`), those above
// it, and as many of those equal to it, lowest index first; failing that, one after the other.
template <int KIND, int LANES> __device__ __forceinline__ void best_of(LogProbsLds<LANES, true>& lds, const Span<KIND>& span, int top, float most)
{
    constexpr int kRun = LANES / 64;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const float of_run = run_max<kRun>(most);
    if (tid % kRun == 0) lds.run[tid / kRun] = of_run;
    if (tid < kMostTop) lds.best[tid] = 0;
    if (tid == 0) lds.count = 0;
    __syncthreads();
    if (wave == 0) {
        const float mine = lds.run[lane];
        int rank = 0;
        for (int j = 0; j < 64; ++j) {
            const float other = lds.run[j];
            rank += other > mine || (other == mine && j < lane);
        }
        if (rank == top - 1) lds.threshold = mine;
    }
    __syncthreads();
    const float threshold = lds.threshold;
    // -inf: all elements reach it
    const bool all = threshold == -infinity();
    if (!all) {
        each<KIND, LANES>(span, [&](float x, unsigned i) { if (!(x < threshold)) keep_candidate(lds, x, i); });
        __syncthreads();
    }
    bool fill = false;
    if (all || lds.count > kCandidates) {
        __syncthreads();
        if (tid == 0) lds.count = 0;
        __syncthreads();
        each<KIND, LANES>(span, [&](float x, unsigned i) { if (!(x <= threshold)) keep_candidate(lds, x, i); });
        __syncthreads();
        fill = true;
    }
    const int n = lds.count;
    if (n <= kCandidates) {
        for (int i = tid; i < n; i += LANES) {
            const Key mine = lds.candidate[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += lds.candidate[j] > mine;
            if (rank < top) lds.best[rank] = mine;
        }
        if (fill && wave == 0) {
            int have = n;
            for (unsigned c = span.begin; c < span.end && have < top; c += 64) {
                float x[kVec];
                unsigned equal = 0;
                const int valid = c + lane < span.end ? valid_at(c + lane, span.cols) : 0;
                if (valid > 0) {
                    span.vec(c + lane, x);
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) equal |= (unsigned)(i < valid && x[i] == threshold) << i;
                }
                // elements before this lane's: bit by bit of the lanes' counts
                const int count = __popc(equal);
                int before = 0, total = 0;
                #pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const unsigned long long lanes = __ballot(count >> b & 1);
                    before += __popcll(lanes & ((1ull << lane) - 1)) << b;
                    total += __popcll(lanes) << b;
                }
                int at = have + before;
                #pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (equal >> i & 1) {
                        if (at < top) lds.best[at] = key_of(threshold, (c + lane) * kVec + i);
                        ++at;
                    }
                have += total;
            }
        }
    } else {
        Key last = ~(Key)0;
        for (int k = 0; k < top; ++k) {
            Key next = 0;
            each<KIND, LANES>(span, [&](float x, unsigned i) {
                const Key key = key_of(x, i);
                if ((key < last || (k == 0 && key == last)) && key > next) next = key;
            });
            #pragma unroll
            for (int step = 1; step < 64; step <<= 1) {
                const Key other = __shfl_xor(next, step);
                if (other > next) next = other;
            }
            if (lane == 0) lds.wave_best[wave] = next;
            __syncthreads();
            for (int w = 0; w < LANES / 64; ++w)
                if (lds.wave_best[w] > next) next = lds.wave_best[w];
            if (tid == 0) lds.best[k] = next;
            last = next;
            __syncthreads();
        }
    }
    __syncthreads();
}

// What a row's statistics give.  By one lane.
template <int KIND> __device__ __forceinline__ float finish_row(const LogProbs& a, size_t row, const Stat& s)
{
    // no logit but -inf: nothing can be drawn
    const float log_z = __builtin_logf(s.z);
    const float lse = s.z == 0.f ? -infinity() : s.m + log_z;
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = s.z == 0.f ? 0.f : log_z - s.t / s.z;
    const int64_t target = a.targets[row];
    float logprob = 0.f;
    if (target >= (int64_t)a.vocab) logprob = __builtin_nanf("");
    else if (target >= 0) {
        const char* const at = (const char*)a.logits.data + (row * a.logits.stride + (size_t)target) * kWidth<KIND>;
        const float x = KIND == kF32 ? *(const float*)at : widen<KIND>(*(const uint16_t*)at);
        logprob = s.z == 0.f ? -infinity() : x - s.m - log_z;
    }
    a.logprob[row] = logprob;
    return lse;
}
__device__ __forceinline__ void write_best(const LogProbs& a, size_t row, int k, Key key, const Stat& s)
{
    a.top_ids[row * a.top + k] = index_of(key);
    const float v = value_of(key);
    a.top_logprobs[row * a.top + k] = s.z == 0.f ? -infinity() : v - s.m - __builtin_logf(s.z);
}

template <int KIND, int LANES, int U, bool TOP>
__global__ __launch_bounds__(LANES) void logprobs_kernel(LogProbsArgs p)
{
    const LogProbs& a = p.a;
    __shared__ LogProbsLds<LANES, TOP> lds;
    const size_t units = a.rows * p.splits;
    const unsigned vecs = (a.vocab + kVec - 1) / kVec;
    for (size_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const size_t row = unit / p.splits;
        const unsigned split = (unsigned)(unit - row * p.splits);
        const Span<KIND> span = {(const char*)a.logits.data + row * a.logits.stride * kWidth<KIND>, split * p.chunk,
                                 min(vecs, (split + 1) * p.chunk), a.vocab};
        const Stat mine = lane_stat<KIND, LANES, U>(span);
        const Stat s = block_stat<LANES>(lds.stat, mine);
        if constexpr (TOP) best_of<KIND, LANES>(lds, span, a.top, mine.m);
        if (p.splits == 1) {
            if (threadIdx.x == 0) finish_row<KIND>(a, row, s);
            if constexpr (TOP)
                if ((int)threadIdx.x < a.top) write_best(a, row, threadIdx.x, lds.best[threadIdx.x], s);
        } else {
            char* const part = (char*)a.parts + unit * split_bytes(a.top);
            if (threadIdx.x == 0) *(Stat*)part = s;
            if constexpr (TOP)
                if ((int)threadIdx.x < a.top) ((Key*)(part + 16))[threadIdx.x] = lds.best[threadIdx.x];
        }
        __syncthreads();       // the LDS is free for the next row
    }
}

// Joins the splits of a row, one workgroup a row.  A key's rank is its place in its own list and what every other list
// has above it.
constexpr int kJoinLanes = 256;
template <int KIND>
__global__ __launch_bounds__(kJoinLanes) void join_kernel(LogProbsArgs p)
{
    const LogProbs& a = p.a;
    extern __shared__ Key lists[];
    const size_t bytes = split_bytes(a.top);
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const char* const parts = (const char*)a.parts + row * p.splits * bytes;
        Stat s = {-infinity(), 0.f, 0.f};
        for (int i = 0; i < p.splits; ++i) s.m = fmaxf(s.m, ((const Stat*)(parts + i * bytes))->m);
        for (int i = 0; i < p.splits; ++i) {
            Stat part = *(const Stat*)(parts + i * bytes);
            part.move_to(s.base());
            s.z += part.z;
            s.t += part.t;
        }
        if (threadIdx.x == 0) finish_row<KIND>(a, row, s);
        const int n = p.splits * a.top;
        for (int i = threadIdx.x; i < n; i += kJoinLanes)
            lists[i] = ((const Key*)(parts + (i / a.top) * bytes + 16))[i % a.top];
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kJoinLanes) {
            const Key mine = lists[i];
            int rank = i % a.top;
            for (int l = 0; l < p.splits && rank < a.top; ++l) {
                if (l == i / a.top) continue;
                int low = 0, high = a.top;                  // keys above mine: a prefix of the list
                while (low < high) {
                    const int mid = (low + high) / 2;
                    if (lists[l * a.top + mid] > mine) low = mid + 1;
                    else high = mid;
                }
                rank += low;
            }
            if (rank < a.top && mine != 0) write_best(a, row, rank, mine, s);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Gradient:  dlogits_j = g (1[j = target] - p_j) - h p_j (log p_j + entropy),  g and h those of the row's log
// probability and entropy.  Rows that neither reaches are zero and not read.
// ---------------------------------------------------------------------------
struct LogProbsBackwardArgs {
    LogProbsBackward a;
    unsigned chunk, chunks;      // vectors of a workgroup, workgroups of a row
};
constexpr int kGradLanes = 256;

template <int KIND, bool RAGGED>
__global__ __launch_bounds__(kGradLanes) void logprobs_backward_kernel(LogProbsBackwardArgs p)
{
    const LogProbsBackward& a = p.a;
    const size_t units = a.rows * p.chunks;
    const unsigned vecs = (a.vocab + kVec - 1) / kVec;
    for (size_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const size_t row = unit / p.chunks;
        const unsigned begin = (unsigned)(unit - row * p.chunks) * p.chunk, end = min(vecs, begin + p.chunk);
        const char* const x_row = (const char*)a.logits.data + row * a.logits.stride * kWidth<KIND>;
        char* const d_row = (char*)a.dlogits.data + row * a.dlogits.stride * kWidth<KIND>;
        const int64_t target = a.targets[row];
        const float lse = a.lse[row], h = a.dentropy ? a.dentropy[row] : 0.f, entropy = a.dentropy ? a.entropy[row] : 0.f;
        const float g = target < 0 ? 0.f : a.dlogprob[row];
        const bool bad = target >= (int64_t)a.vocab;
        const bool none = !bad && ((g == 0.f && h == 0.f) || lse == -infinity());
        for (unsigned c = begin + threadIdx.x; c < end; c += kGradLanes) {
            float d[kVec] = {};
            if (!none) {
                float x[kVec];
                unpack<KIND>(load_col<KIND, RAGGED>(x_row, c, a.vocab), x);
                const unsigned hit = (unsigned)((uint64_t)target - (uint64_t)c * kVec < kVec ? target - (int64_t)c * kVec : kVec);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float logp = x[i] - lse, prob = exp_of(logp);
                    d[i] = prob * __builtin_fmaf(-h, fmaxf(logp, kFar) + entropy, -g);
                    if (hit == (unsigned)i) d[i] += g;
                    if (bad) d[i] = __builtin_nanf("");
                }
            }
            store_col<KIND, RAGGED>(d_row, c, a.vocab, pack<KIND>(d));
        }
    }
}

unsigned grid_of(size_t blocks) { return (unsigned)std::min<size_t>(blocks, 1u << 20); }

constexpr size_t kUnits = 256;              // compute units of an MI355X

}  // namespace

// Enough workgroups for every compute unit, but none with less than 8192 logits.
int row_splits(size_t rows, size_t vocab)
{
    if (rows == 0 || rows >= kUnits) return 1;
    return (int)std::max<size_t>(1, std::min<size_t>({kUnits / rows, vocab / 8192, 64}));
}

int launch_logprobs(const LogProbs& a, int kind, void* stream)
{
    const unsigned vecs = (unsigned)(((size_t)a.vocab + kVec - 1) / kVec);
    LogProbsArgs p{a, row_splits(a.rows, a.vocab), 0};
    p.chunk = (vecs + p.splits - 1) / p.splits;
    return dispatch_kind(kind, [&](auto K) {
        constexpr int KIND = decltype(K)::value;
        const int err = dispatch_flag(a.top > 0, [&](auto T) {
            return launch_args(logprobs_kernel<KIND, 1024, 4, decltype(T)::value>, dim3(grid_of(a.rows * p.splits)), dim3(1024), 0,
                               stream, p);
        });
        if (err || p.splits == 1) return err;
        return launch_args(join_kernel<KIND>, dim3(grid_of(a.rows)), dim3(kJoinLanes), sizeof(Key) * p.splits * a.top, stream, p);
    });
}

int launch_logprobs_backward(const LogProbsBackward& a, int kind, void* stream)
{
    const unsigned vecs = (unsigned)(((size_t)a.vocab + kVec - 1) / kVec);
    LogProbsBackwardArgs p{a, 4 * kGradLanes, 0};
    p.chunks = (vecs + p.chunk - 1) / p.chunk;
    return dispatch_kind(kind, [&](auto K) { return dispatch_flag(a.vocab % kVec != 0, [&](auto R) {
        return launch_args(logprobs_backward_kernel<decltype(K)::value, decltype(R)::value>, dim3(grid_of(a.rows * p.chunks)),
                           dim3(kGradLanes), 0, stream, p);
    }); });
}

}  // namespace mics
