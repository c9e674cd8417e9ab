// Log probabilities of given tokens with the row's log-sum-exp, entropy and best alternatives, and the gradient.
//
// With m the largest logit of a row, Z = sum e^(x-m) and T = sum (x-m) e^(x-m):
//     log p_j = x_j - m - log Z,    entropy = log Z - T / Z,
// so one pass that keeps (m, Z, T) and rescales them when m grows reads every logit once.  Z and T of two parts join as
//     Z = Z1 e^(m1-m) + Z2 e^(m2-m),    T = sum of e^(mi-m) (Ti + (mi-m) Zi).
// Bound by HBM bandwidth with many rows, by latency with few.  Measured on one MI355X: 4096 x 65536 bf16 with entropy 83.3 us =
// 6.45 TB/s; 500 x 50001 f32 with 5 alternatives 22.3 us = 4.5 TB/s; 4 x 131072 bf16 with 8 12.4 us, two launches; the gradient of
// 4096 x 65536 165.8 us = 6.5 TB/s read and written.
#include "rows.h"

#include <algorithm>

#include "layer_internal.h"
#include "logprobs_rules.h"

namespace mics {
namespace {

constexpr float kLowest = -3.402823466e38f, kLog2e = 1.4426950408889634f;
// e^-200 is 0 in binary32: the factor of such a term may stop there, which keeps 0 * inf out of the sums.
constexpr float kFar = -200.f;

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
// With what the product v log2 e loses, and with subnormal results: 32-bit gradients of far logits show both (without, up to 64 units
// of 2^-24 of a gradient at v = -85).  16-bit gradients do not, and in the sums of a row such terms weigh nothing.  It costs
// nothing behind memory: 2000 x 50001 f32 with entropy 141.5 us without, 141.9 so.
__device__ __forceinline__ float exp_exactly(float v)
{
    constexpr float kRest = (float)(1.4426950408889634 - (double)kLog2e), kLn2 = 0.6931471805599453f;
    v = v < kFar ? kFar : v;          // a NaN stays
    const float h = v * kLog2e, l = __builtin_fmaf(v, kRest, __builtin_fmaf(v, kLog2e, -h)), e = __builtin_exp2f(h);
    return __builtin_fmaf(e, l * kLn2, e);
}
__device__ __forceinline__ float infinity() { return __builtin_inff(); }

// z = sum e^(x-base), t = sum (x-base) e^(x-base).  A NaN or +inf among the logits makes z NaN; logits of -inf alone, or
// none, leave z = 0.
struct Stat {
    float base, z, t;
    __device__ __forceinline__ void move_to(float to)
    {
        const float d = base - to, e = exp_of(d);
        t = e * __builtin_fmaf(fmaxf(d, kFar), z, t);
        z *= e;
        base = to;
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
    if constexpr (LANES >= 2) v = dpp_max<0xB1, 0xF>(v);        // quad_perm 1,0,3,2
    if constexpr (LANES >= 4) v = dpp_max<0x4E, 0xF>(v);        // quad_perm 2,3,0,1
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

template <int LANES, bool TOP> struct LogProbsLds {
    Stat stat[LANES / 64];
};
template <int LANES> struct LogProbsLds<LANES, true> {
    float run[64];
    Stat stat[LANES / 64];
    float threshold;
    int count;
    Key best[kMostTop];
    Key wave_best[LANES / 64];
    Key candidate[kCandidates + 4];
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

template <int N> __device__ __forceinline__ float largest(const float (&x)[N])
{
    float most = -infinity();
    #pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, x[i]);
    return most;
}
// The base is the largest logit so far.  A lower one would do for Z, but log Z, T / Z and logits less the base would then be as large
// as it is too low, and what they leave of each other -- the entropy, the log probability of what is almost certain -- would keep
// their rounding alone.
template <bool ENTROPY, int N> __device__ __forceinline__ void add_logits(Stat& s, const float (&x)[N], float most)
{
    if (__builtin_amdgcn_ballot_w64(most > s.base)) s.move_to(fmaxf(most, s.base));
    #pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = x[i] - s.base, e = exp_of(d);
        s.z += e;
        if constexpr (ENTROPY) s.t = __builtin_fmaf(fmaxf(d, kFar), e, s.t);
    }
}

// Joins the lanes of a wavefront, in a fixed order; the result is in every lane.
__device__ __forceinline__ Stat wave_stat(Stat s)
{
    s.move_to(wave_max(s.base));
    return {s.base, wave_sum(s.z), wave_sum(s.t)};
}
template <int LANES> __device__ __forceinline__ Stat block_stat(Stat (&lds)[LANES / 64], Stat s)
{
    s = wave_stat(s);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (lane == 0) lds[wave] = s;
    barrier_lds();
    return wave_stat(lane < LANES / 64 ? lds[lane] : Stat{kLowest, 0.f, 0.f});
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

// The top-th largest of the largest logits of 64 runs of lanes: at most the top-th largest logit of all, and few others
// reach it.  Also empties the list of candidates.
template <int LANES> __device__ __forceinline__ float reached_by(LogProbsLds<LANES, true>& lds, int top, float most)
{
    constexpr int kRun = LANES / 64;
    const int tid = threadIdx.x, lane = tid & 63;
    const float of_run = run_max<kRun>(most);
    if (tid % kRun == 0) lds.run[tid / kRun] = of_run;
    if (tid == 0) lds.count = 0;
    barrier_lds();
    if (tid < 64) {
        const float mine = lds.run[lane];
        int rank = 0;
        for (int j = 0; j < 64; ++j) {
            const float other = lane_value(mine, j);
            rank += other > mine || (other == mine && j < lane);
        }
        if (rank == top - 1) lds.threshold = mine;
    }
    barrier_lds();
    return lds.threshold;
}

// The first `top` of the n candidates in order into lds.best, n the same in all lanes.  Many candidates are thinned out
// first, by the threshold of their own runs (300 x 100000 bf16, half of them masked, 50 alternatives: some 1150 candidates, 259 us
// without, 47.7 so).
template <int LANES> __device__ __forceinline__ void rank_candidates(LogProbsLds<LANES, true>& lds, int n, int top)
{
    if (n > 3 * 64) {
        constexpr int kEach = kCandidates / LANES;
        Key mine[kEach];
        float most = -infinity();
        #pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = threadIdx.x + j * LANES;
            mine[j] = i < n ? lds.candidate[i] : 0;
            if (mine[j]) most = fmaxf(most, value_of(mine[j]));
        }
        const float threshold = reached_by<LANES>(lds, top, most);
        #pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (mine[j] && !(value_of(mine[j]) < threshold)) lds.candidate[atomicAdd(&lds.count, 1)] = mine[j];
        barrier_lds();
        n = lds.count;
    }
    // behind the n: no key, so that four can be compared at a time
    if (threadIdx.x < 4) lds.candidate[n + threadIdx.x] = 0;
    barrier_lds();
    for (int i = threadIdx.x; i < n; i += LANES) {
        const Key mine = lds.candidate[i];
        int rank = 0;
        for (int j = 0; j < n; j += 4) {
            #pragma unroll
            for (int u = 0; u < 4; ++u) rank += lds.candidate[j + u] > mine;
        }
        if (rank < top) lds.best[rank] = mine;
    }
}

// Fills lds.best from place `have` on with the first elements of the span that equal `value`.  By one wavefront.
template <int KIND, int LANES>
__device__ __forceinline__ void fill_equal(LogProbsLds<LANES, true>& lds, const Span<KIND>& span, int have, int top, float value)
{
    const int lane = threadIdx.x & 63;
    for (unsigned c = span.begin; c < span.end && have < top; c += 64) {
        float x[kVec];
        unsigned equal = 0;
        const int valid = c + lane < span.end ? valid_at(c + lane, span.cols) : 0;
        if (valid > 0) {
            span.vec(c + lane, x);
            #pragma unroll
            for (int i = 0; i < kVec; ++i) equal |= (unsigned)(i < valid && x[i] == value) << i;
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
                if (at < top) lds.best[at] = key_of(value, (c + lane) * kVec + i);
                ++at;
            }
        have += total;
    }
}

// The `top` best of a span that the candidates did not settle (too many of them, NaN):
// those that reach the threshold of the whole span; where these are too many still, those above it and as many of those
// equal to it, lowest index first; failing that, one after the other.
template <int KIND, int LANES> __device__ __forceinline__ void best_of_any(LogProbsLds<LANES, true>& lds, const Span<KIND>& span, int top)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    float most = -infinity();
    each<KIND, LANES>(span, [&](float x, unsigned) { most = fmaxf(most, x); });
    const float threshold = reached_by<LANES>(lds, top, most);
    // -inf: all elements reach it
    const bool all = threshold == -infinity();
    if (!all) {
        each<KIND, LANES>(span, [&](float x, unsigned i) { if (!(x < threshold)) keep_candidate(lds, x, i); });
        barrier_lds();
    }
    bool fill = false;
    if (all || lds.count > kCandidates) {
        barrier_lds();
        if (tid == 0) lds.count = 0;
        barrier_lds();
        each<KIND, LANES>(span, [&](float x, unsigned i) { if (!(x <= threshold)) keep_candidate(lds, x, i); });
        barrier_lds();
        fill = true;
    }
    const int n = lds.count;
    barrier_lds();       // and before it is set back
    if (n <= kCandidates) {
        rank_candidates<LANES>(lds, n, top);
        if (fill && wave == 0) fill_equal<KIND, LANES>(lds, span, n, top, threshold);
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
            barrier_lds();
            for (int w = 0; w < LANES / 64; ++w)
                if (lds.wave_best[w] > next) next = lds.wave_best[w];
            if (tid == 0) lds.best[k] = next;
            last = next;
            barrier_lds();
        }
    }
}

// A row's target and its logit, loaded before the pass over the row, which hides both.
struct Target {
    int64_t at;
    float logit;
};
template <int KIND> __device__ __forceinline__ Target target_of(const LogProbs& a, size_t row)
{
    const int64_t at = a.targets[row];
    const size_t column = at < 0 ? 0 : at >= (int64_t)a.vocab ? a.vocab - 1 : (size_t)at;
    const char* const p = (const char*)a.logits.data + (row * a.logits.stride + column) * kWidth<KIND>;
    return {at, KIND == kF32 ? *(const float*)p : widen<KIND>(*(const uint16_t*)p)};
}
// What a row's statistics give.  By one lane.
__device__ __forceinline__ void finish_row(const LogProbs& a, size_t row, const Stat& s, const Target& target)
{
    // no logit but -inf: nothing can be drawn
    const float log_z = __builtin_logf(s.z);
    if (a.lse) a.lse[row] = s.z == 0.f ? -infinity() : s.base + log_z;
    if (a.entropy) a.entropy[row] = s.z == 0.f ? 0.f : log_z - s.t / s.z;
    float logprob = s.z == 0.f ? -infinity() : target.logit - s.base - log_z;
    if (target.at < 0) logprob = 0.f;
    if (target.at >= (int64_t)a.vocab) logprob = __builtin_nanf("");
    a.logprob[row] = logprob;
}
__device__ __forceinline__ void write_best(const LogProbs& a, size_t row, int k, Key key, const Stat& s)
{
    a.top_ids[row * a.top + k] = index_of(key);
    const float v = value_of(key);
    a.top_logprobs[row * a.top + k] = s.z == 0.f ? -infinity() : v - s.base - __builtin_logf(s.z);
}

// One pass: U vectors of every lane are worked on while the next U are loaded.  TOP: the first U tell a threshold, and what
// reaches it is kept as a candidate on the way.
// Four wavefronts for each unit of a compute unit, which takes 128 registers, where that spills little: two registers of 16-bit logits
// (2048 x 32768 bf16, 5 alternatives: three wavefronts 42.3 us, four 38.8).  32-bit ones keep their 172 (500 x 50001, 5
// alternatives: 22.3 us, four 25.9).  1024 lanes leave no choice: two registers spill, of 32-bit logits 12 to 17 (1 x 32000 f32, 5
// alternatives, 10.9 us).
template <int KIND, int LANES, int U, bool TOP, bool ENTROPY, bool NT>
__global__ __launch_bounds__(LANES, LANES == 256 && U == 4 && TOP && KIND != kF32 ? 4 : 1) void logprobs_kernel(LogProbsArgs p)
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
        const unsigned whole = span.whole();
        const Target target = target_of<KIND>(a, row);
        Stat s = {kLowest, 0.f, 0.f};
        float threshold = -infinity();
        bool masked = true;                  // the first vectors hold too few logits but -inf: all but those are candidates
        auto load = [&](Raw<KIND> (&r)[U], unsigned from) {
            #pragma unroll
            for (int u = 0; u < U; ++u)
                r[u] = load_vec<KIND, NT>(span.row + (size_t)min(from + u * LANES, whole - 1) * (kVec * kWidth<KIND>), kVec);
        };
        // a lane's logits that reach the threshold, by index: one place in the list for each, all of them at once
        auto keep = [&](auto N, const float* x, unsigned c) {
            if constexpr (TOP) {
                constexpr int COUNT = decltype(N)::value * kVec;
                uint32_t reached = 0;
                #pragma unroll
                for (int i = 0; i < COUNT; ++i) reached |= x[i] < threshold ? 0u : 1u << i;
                if (!reached) return;
                int to = atomicAdd(&lds.count, __popc(reached));
                for (; reached; reached &= reached - 1, ++to) {
                    const unsigned i = __builtin_ctz(reached);
                    if (to < kCandidates) lds.candidate[to] = (c + i / kVec * LANES) * kVec + i % kVec;
                }
            }
        };
        auto read = [&](auto PART, const Raw<KIND> (&r)[U], unsigned c, float (&x)[U * kVec]) {
            #pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[kVec];
                unpack<KIND>(r[u], v);
                const bool in = !decltype(PART)::value || c + u * LANES < whole;
                #pragma unroll
                for (int i = 0; i < kVec; ++i) x[u * kVec + i] = in ? v[i] : -infinity();
            }
        };
        auto add = [&](const float (&x)[U * kVec], float most, unsigned c) {
            if (TOP && !(most < threshold)) keep(std::integral_constant<int, U>{}, x, c);
            add_logits<ENTROPY>(s, x, most);
        };
        if constexpr (TOP)
            if (threadIdx.x < kMostTop) lds.best[threadIdx.x] = 0;
        if (span.begin < whole) {
            constexpr unsigned kStep = LANES * U;
            Raw<KIND> r[2][U];
            unsigned at = span.begin + threadIdx.x;                  // the first lane's is below `whole`
            load(r[0], at);
            load(r[1], at + kStep);
            {
                float x[U * kVec];
                read(std::true_type{}, r[0], at, x);
                const float most = largest(x);
                if constexpr (TOP) {
                    threshold = reached_by<LANES>(lds, a.top, most);
                    masked = threshold == -infinity();
                    threshold = fmaxf(threshold, kLowest);
                }
                add(x, most, at);
            }
            for (unsigned from = span.begin + kStep; from < whole;) {
                #pragma unroll
                for (int k = 1; k >= 0; --k) {
                    if (from >= whole) break;
                    at = from + threadIdx.x;
                    load(r[1 - k], at + kStep);
                    float x[U * kVec];
                    if (from + kStep <= whole) read(std::false_type{}, r[k], at, x);
                    else read(std::true_type{}, r[k], at, x);
                    add(x, largest(x), at);
                    from += kStep;
                }
            }
        } else if constexpr (TOP) {
            threshold = fmaxf(reached_by<LANES>(lds, a.top, -infinity()), kLowest);
        }
        if (whole >= span.begin && whole < span.end && threadIdx.x == 0) {       // the last part of a vector
            float x[kVec];
            span.vec(whole, x);
            add_logits<ENTROPY>(s, x, largest(x));
            keep(std::integral_constant<int, 1>{}, x, whole);
        }
        s = block_stat<LANES>(lds.stat, s);
        if constexpr (TOP) {
            const int n = lds.count;      // behind block_stat's barrier
            barrier_lds();              // and before it is set back
            if (s.z == s.z && n <= kCandidates) {
                // a register cannot be chosen by a number, so their logits are read again
                for (int i = threadIdx.x; i < n; i += LANES) {
                    const unsigned index = (unsigned)lds.candidate[i];
                    const char* const from = span.row + (size_t)index * kWidth<KIND>;
                    lds.candidate[i] = key_of(KIND == kF32 ? *(const float*)from : widen<KIND>(*(const uint16_t*)from), index);
                }
                barrier_lds();
                rank_candidates<LANES>(lds, n, a.top);
                if (masked && n < a.top && threadIdx.x < 64) fill_equal<KIND, LANES>(lds, span, n, a.top, -infinity());
            } else {
                best_of_any<KIND, LANES>(lds, span, a.top);
            }
            barrier_lds();
        }
        if (p.splits == 1) {
            if (threadIdx.x == 0) finish_row(a, row, s, target);
            if constexpr (TOP)
                if ((int)threadIdx.x < a.top) write_best(a, row, threadIdx.x, lds.best[threadIdx.x], s);
        } else {
            char* const part = (char*)a.parts + unit * split_bytes(a.top);
            if (threadIdx.x == 0) *(Stat*)part = s;
            if constexpr (TOP)
                if ((int)threadIdx.x < a.top) ((Key*)(part + 16))[threadIdx.x] = lds.best[threadIdx.x];
        }
        barrier_lds();       // the LDS is free for the next row
    }
}

// Joins the splits of a row, one workgroup a row: at most 64 of them, with at most kCandidates keys.
constexpr int kJoinLanes = 256;
template <int KIND, bool TOP>
__global__ __launch_bounds__(kJoinLanes) void join_kernel(LogProbsArgs p)
{
    const LogProbs& a = p.a;
    __shared__ LogProbsLds<kJoinLanes, TOP> lds;
    const size_t bytes = split_bytes(a.top);
    const int lane = threadIdx.x & 63;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const char* const parts = (const char*)a.parts + row * p.splits * bytes;
        const Target target = target_of<KIND>(a, row);
        const Stat s = wave_stat(lane < p.splits ? *(const Stat*)(parts + lane * bytes) : Stat{kLowest, 0.f, 0.f});
        if (threadIdx.x == 0) finish_row(a, row, s, target);
        if constexpr (TOP) {
            const int n = p.splits * a.top;
            for (int i = threadIdx.x; i < n; i += kJoinLanes)
                lds.candidate[i] = ((const Key*)(parts + (i / a.top) * bytes + 16))[i % a.top];
            barrier_lds();
            rank_candidates<kJoinLanes>(lds, n, a.top);
            barrier_lds();
            if ((int)threadIdx.x < a.top) write_best(a, row, threadIdx.x, lds.best[threadIdx.x], s);
            barrier_lds();
        }
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

template <int KIND, int TAIL, bool ENTROPY, bool NT>
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
        const float lse = a.lse[row], h = ENTROPY ? a.dentropy[row] : 0.f, entropy = ENTROPY ? a.entropy[row] : 0.f;
        const float g = target < 0 ? 0.f : a.dlogprob[row];
        const bool bad = target >= (int64_t)a.vocab;
        const bool none = !bad && ((g == 0.f && h == 0.f) || lse == -infinity());
        for (unsigned c = begin + threadIdx.x; c < end; c += kGradLanes) {
            float d[kVec] = {};
            if (!none) {
                float x[kVec];
                Raw<KIND> r = load_col<KIND, TAIL>(x_row, c, a.vocab);
                settle<KIND, TAIL>(r, c, a.vocab);
                unpack<KIND>(r, x);
                const unsigned hit = (unsigned)((uint64_t)target - (uint64_t)c * kVec < kVec ? target - (int64_t)c * kVec : kVec);
                #pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float logp = x[i] - lse, prob = KIND == kF32 ? exp_exactly(logp) : exp_of(logp);
                    d[i] = prob * (ENTROPY ? __builtin_fmaf(-h, fmaxf(logp, kFar) + entropy, -g) : -g);
                }
                if (hit < kVec) {
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) d[i] += hit == (unsigned)i ? g : 0.f;
                }
                if (bad) {
                    #pragma unroll
                    for (int i = 0; i < kVec; ++i) d[i] = __builtin_nanf("");
                }
            }
            store_col<KIND, TAIL, NT>(d_row, c, a.vocab, pack<KIND>(d));
        }
    }
}

unsigned grid_of(size_t blocks) { return (unsigned)std::min<size_t>(blocks, 1u << 20); }

}  // namespace

int row_splits(size_t rows, size_t vocab, int top) { return splits_of(rows, vocab, top); }

int launch_logprobs(const LogProbs& a, int kind, void* stream)
{
    static_assert(kRowVec == kVec, "");
    const LogProbsShape shape = logprobs_shape(a.rows, a.vocab, a.top, kind == kF32 ? 4 : 2);
    const LogProbsArgs p{a, shape.splits, shape.chunk};
    return dispatch_kind(kind, [&](auto K) {
        constexpr int KIND = decltype(K)::value;
        auto run = [&](auto L, auto U, auto N) { return dispatch_flag(a.top > 0, [&](auto T) { return dispatch_flag(a.entropy, [&](auto E) {
            constexpr int LANES = decltype(L)::value;
            return launch_args(logprobs_kernel<KIND, LANES, decltype(U)::value, decltype(T)::value, decltype(E)::value, decltype(N)::value>,
                               dim3(grid_of(a.rows * p.splits)), dim3(LANES), 0, stream, p);
        }); }); };
        using std::integral_constant;
        const int err = shape.lanes == 1024 ? run(integral_constant<int, 1024>{}, integral_constant<int, 4>{}, std::false_type{})
                      : shape.flight == 2   ? run(integral_constant<int, 256>{}, integral_constant<int, 2>{}, std::false_type{})
                      : shape.uncached      ? run(integral_constant<int, 256>{}, integral_constant<int, 4>{}, std::true_type{})
                                            : run(integral_constant<int, 256>{}, integral_constant<int, 4>{}, std::false_type{});
        if (err || p.splits == 1) return err;
        return dispatch_flag(a.top > 0, [&](auto T) {
            return launch_args(join_kernel<KIND, decltype(T)::value>, dim3(grid_of(a.rows)), dim3(kJoinLanes), 0, stream, p);
        });
    });
}

int launch_logprobs_backward(const LogProbsBackward& a, int kind, void* stream)
{
    const GradientShape shape = gradient_shape(a.rows, a.vocab, kind == kF32 ? 4 : 2);
    const LogProbsBackwardArgs p{a, shape.chunk, shape.chunks};
    return dispatch_kind(kind, [&](auto K) { return dispatch_tail(a.vocab, [&](auto T) { return dispatch_flag(a.dentropy, [&](auto E) {
        return dispatch_flag(shape.unkept, [&](auto N) {
            return launch_args(logprobs_backward_kernel<decltype(K)::value, decltype(T)::value, decltype(E)::value, decltype(N)::value>,
                               dim3(grid_of(a.rows * p.chunks)), dim3(kGradLanes), 0, stream, p);
        });
    }); }); });
}

}  // namespace mics
