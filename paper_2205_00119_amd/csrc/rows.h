// Rows of bf16, binary16 or binary32 in vectors of eight elements: what the kernels of norm.hip, dropout.hip and
// logprobs.hip share.  A lane owns columns 8c to 8c + 7; the last vector of a row may hold fewer.  Rows may begin on any element:
// the accesses are 128 bits wide on under-aligned types, which gfx950 executes at full speed from 4 bytes on.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#pragma clang fp contract(off)

namespace mics {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
typedef u32x2 u32x2_a4 __attribute__((aligned(4)));
typedef uint32_t u32_a2 __attribute__((aligned(2)));

constexpr int kBf16 = 0, kF16 = 1, kF32 = 2;
constexpr int kVec = 8;

template <int KIND> constexpr size_t kWidth = KIND == kF32 ? 4 : 2;

// Eight elements as they lie in memory.
template <int KIND> struct Raw {
    u32x4 q[KIND == kF32 ? 2 : 1];
};

template <int KIND> __device__ __forceinline__ float widen(uint32_t bits)
{
    if constexpr (KIND == kBf16) return __builtin_bit_cast(float, bits << 16);
    else if constexpr (KIND == kF16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    else return __builtin_bit_cast(float, bits);
}
// Round to nearest even.
template <int KIND> __device__ __forceinline__ uint32_t narrow2(float a, float b)
{
    const f32x2 f = {a, b};
    if constexpr (KIND == kBf16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));
}
template <int KIND> __device__ __forceinline__ void store_one(void* p, float v)
{
    if constexpr (KIND == kF32) *(float*)p = v;
    else *(uint16_t*)p = (uint16_t)narrow2<KIND>(v, 0.f);
}

template <int KIND> __device__ __forceinline__ void unpack(const Raw<KIND>& r, float (&v)[kVec])
{
    #pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const uint32_t b = KIND == kF32 ? r.q[i / 4 * (KIND == kF32)][i % 4] : r.q[0][i / 2];
        if constexpr (KIND == kF32) v[i] = __builtin_bit_cast(float, b);
        else if constexpr (KIND == kBf16) v[i] = __builtin_bit_cast(float, i % 2 ? b & 0xFFFF0000u : b << 16);
        else v[i] = widen<kF16>(b >> (16 * (i % 2)) & 0xFFFFu);
    }
}
template <int KIND> __device__ __forceinline__ Raw<KIND> pack(const float (&v)[kVec])
{
    Raw<KIND> r;
    #pragma unroll
    for (int i = 0; i < kVec; i += 2) {
        if constexpr (KIND == kF32) {
            r.q[i / 4][i % 4] = __builtin_bit_cast(uint32_t, v[i]);
            r.q[i / 4][i % 4 + 1] = __builtin_bit_cast(uint32_t, v[i + 1]);
        } else {
            r.q[0][i / 2] = narrow2<KIND>(v[i], v[i + 1]);
        }
    }
    return r;
}

// NT: non-temporal, past the caches.
#define MICS_ROW_LD(NT, p) ((NT) ? __builtin_nontemporal_load(p) : *(p))
#define MICS_ROW_ST(NT, p, v) do { if (NT) __builtin_nontemporal_store(v, p); else *(p) = (v); } while (0)

// The vector at `p`, of which `valid` elements exist (8 and more: all); the others read as 0.  A part of a vector
// comes in pieces of four, two and one elements.
template <int KIND, bool NT = false> __device__ __forceinline__ Raw<KIND> load_vec(const char* p, int valid)
{
    Raw<KIND> r{};
    if (valid >= kVec) {
        if constexpr (KIND == kF32) {
            r.q[0] = MICS_ROW_LD(NT, (const u32x4_a4*)p);
            r.q[1] = MICS_ROW_LD(NT, (const u32x4_a4*)p + 1);
        } else {
            r.q[0] = MICS_ROW_LD(NT, (const u32x4_a2*)p);
        }
    } else if (valid > 0) {
        const bool four = valid & 4;
        const char* const q = p + (four ? 4 * kWidth<KIND> : 0);
        if constexpr (KIND == kF32) {
            u32x4 low{}, high{};
            if (four) low = *(const u32x4_a4*)p;
            if (valid & 2) {
                const u32x2 t = *(const u32x2_a4*)q;
                high.x = t.x;
                high.y = t.y;
            }
            if (valid & 1) {
                const uint32_t t = *(const uint32_t*)(q + (valid & 2) * 4);
                if (valid & 2) high.z = t; else high.x = t;
            }
            r.q[0] = four ? low : high;
            r.q[1] = four ? high : u32x4{};
        } else {
            u32x2 low{}, high{};
            if (four) low = *(const u32x2_a2*)p;
            if (valid & 2) high.x = *(const u32_a2*)q;
            if (valid & 1) {
                const uint32_t t = *(const uint16_t*)(q + (valid & 2) * 2);
                if (valid & 2) high.y = t; else high.x = t;
            }
            r.q[0] = four ? u32x4{low.x, low.y, high.x, high.y} : u32x4{high.x, high.y, 0, 0};
        }
    }
    return r;
}
template <int KIND, bool NT = false> __device__ __forceinline__ void store_vec(char* p, const Raw<KIND>& r, int valid)
{
    if (valid >= kVec) {
        if constexpr (KIND == kF32) {
            MICS_ROW_ST(NT, (u32x4_a4*)p, r.q[0]);
            MICS_ROW_ST(NT, (u32x4_a4*)p + 1, r.q[1]);
        } else {
            MICS_ROW_ST(NT, (u32x4_a2*)p, r.q[0]);
        }
    } else if (valid > 0) {
        const bool four = valid & 4;
        char* const q = p + (four ? 4 * kWidth<KIND> : 0);
        if constexpr (KIND == kF32) {
            const u32x4 rest = four ? r.q[1] : r.q[0];
            if (four) *(u32x4_a4*)p = r.q[0];
            if (valid & 2) *(u32x2_a4*)q = u32x2{rest.x, rest.y};
            if (valid & 1) *(uint32_t*)(q + (valid & 2) * 4) = valid & 2 ? rest.z : rest.x;
        } else {
            const u32x2 rest = four ? u32x2{r.q[0].z, r.q[0].w} : u32x2{r.q[0].x, r.q[0].y};
            if (four) *(u32x2_a2*)p = u32x2{r.q[0].x, r.q[0].y};
            if (valid & 2) *(u32_a2*)q = rest.x;
            if (valid & 1) *(uint16_t*)(q + (valid & 2) * 2) = (uint16_t)(valid & 2 ? rest.y : rest.x);
        }
    }
}

// Elements of a row of `cols` in the vector c: 8 and more but at the row's end, 0 and less behind it.
__device__ __forceinline__ int valid_at(unsigned c, unsigned cols) { return (int)(cols - c * kVec); }

// How rows end: with a whole vector; with a part of one; rows of fewer than eight elements.
enum { kWhole = 0, kRagged = 1, kTiny = 2 };
inline int tail_of(size_t cols) { return cols < kVec ? kTiny : cols % kVec ? kRagged : kWhole; }

// Vector c of a row, loaded without a branch.  Lanes behind the end of a row read its last eight elements, as does the
// lane of a part of a vector; settle() moves that lane's to their places once they are there.
template <int KIND, int TAIL> __device__ __forceinline__ Raw<KIND> load_col(const char* row, unsigned c, unsigned cols)
{
    if constexpr (TAIL == kTiny) return load_vec<KIND>(row, c ? 0 : (int)cols);
    else return load_vec<KIND>(row + (size_t)min(c * kVec, cols - kVec) * kWidth<KIND>, kVec);
}
// Elements behind the end of the row become 0, in a vector of which at least one is inside.
template <int KIND, int TAIL> __device__ __forceinline__ void settle(Raw<KIND>& r, unsigned c, unsigned cols)
{
    if constexpr (TAIL == kRagged) {
        const int by = (int)(c * kVec + kVec - cols);        // elements too many
        if (__builtin_amdgcn_ballot_w64(by > 0)) {           // the same in all lanes: one wavefront of a row
            constexpr int N = KIND == kF32 ? 8 : 4;
            uint32_t w[N];
            #pragma unroll
            for (int i = 0; i < N; ++i) w[i] = r.q[i / 4][i % 4];
            #pragma unroll
            for (int step = N / 2; step; step /= 2) {
                const bool go = by > 0 && by & (KIND == kF32 ? step : 2 * step);
                #pragma unroll
                for (int i = 0; i < N; ++i) w[i] = go ? i + step < N ? w[i + step] : 0 : w[i];
            }
            if constexpr (KIND != kF32) {
                #pragma unroll
                for (int i = 0; i < N; ++i)
                    w[i] = by > 0 && by & 1 ? w[i] >> 16 | (i + 1 < N ? w[i + 1] << 16 : 0) : w[i];
            }
            #pragma unroll
            for (int i = 0; i < N; ++i) r.q[i / 4][i % 4] = w[i];
        }
    }
}
template <int KIND, int TAIL, bool NT = false>
__device__ __forceinline__ void store_col(char* row, unsigned c, unsigned cols, const Raw<KIND>& r)
{
    char* const p = row + (size_t)c * (kVec * kWidth<KIND>);
    const int valid = valid_at(c, cols);
    if constexpr (TAIL == kWhole) { if (valid > 0) store_vec<KIND, NT>(p, r, kVec); }
    else store_vec<KIND, NT>(p, r, valid);
}
// Element i of a vector where it has one, else 0.
template <int TAIL> __device__ __forceinline__ float summand(float v, int i, int valid)
{
    return TAIL == kWhole || i < valid ? v : 0.f;
}

template <int KIND> __device__ __forceinline__ void read_col(const char* row, unsigned c, unsigned cols, float (&v)[kVec])
{
    Raw<KIND> r = load_col<KIND, kRagged>(row, c, cols);
    settle<KIND, kRagged>(r, c, cols);
    unpack<KIND>(r, v);
}

// Vector c of a parameter of a kind known at run time (the same in all lanes); NULL: `absent` everywhere.
template <int TAIL>
__device__ __forceinline__ void load_param(const void* p, int kind, unsigned c, unsigned cols, float absent, float (&v)[kVec])
{
    auto as = [&](auto K) {
        constexpr int KIND = decltype(K)::value;
        Raw<KIND> r = load_col<KIND, TAIL>((const char*)p, c, cols);
        settle<KIND, TAIL>(r, c, cols);
        unpack<KIND>(r, v);
    };
    if (!p) {
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = absent;
    }
    else if (kind == kBf16) as(std::integral_constant<int, kBf16>{});
    else if (kind == kF16) as(std::integral_constant<int, kF16>{});
    else as(std::integral_constant<int, kF32>{});
}

// The eight columns of a lane, where whole vectors are loaded and stored without a branch: from column `e` on, of which
// `out` are not the lane's to sum.  The lane of a part of a vector, and those behind the end of the row, take the row's last
// eight columns: they compute and store again what other lanes do, bit for bit.  So a row's loads have to be over before
// any of its results is stored in their place.  Rows of fewer than eight columns are lane 0's, in pieces.
template <int TAIL> struct Place {
    unsigned e;
    int out;
    __device__ __forceinline__ Place(unsigned c, unsigned cols)
    {
        if constexpr (TAIL == kTiny) {
            e = 0;
            out = c ? kVec : kVec - (int)cols;
        } else {
            e = min(c * kVec, cols - kVec);
            out = max((int)(c * kVec + kVec - cols), 0);
        }
    }
    // what element i adds to its vector's sum, and the vector to its lane's
    __device__ __forceinline__ float element(float v, int i) const
    {
        if constexpr (TAIL == kWhole) return v;
        else if constexpr (TAIL == kRagged) return i >= out ? v : 0.f;
        else return i < kVec - out ? v : 0.f;
    }
    __device__ __forceinline__ float vector(float s) const { return TAIL != kWhole || out == 0 ? s : 0.f; }
    __device__ __forceinline__ float columns() const { return (float)max(kVec - out, 0); }
    template <int KIND> __device__ __forceinline__ Raw<KIND> load(const char* row) const
    {
        return load_vec<KIND>(row + e * (unsigned)kWidth<KIND>, TAIL == kTiny ? kVec - out : kVec);
    }
    template <int KIND> __device__ __forceinline__ void store(char* row, const Raw<KIND>& r) const
    {
        store_vec<KIND>(row + e * (unsigned)kWidth<KIND>, r, TAIL == kTiny ? kVec - out : kVec);
    }
    // Stored in a kind known at run time (the same in all lanes).
    __device__ __forceinline__ void round(void* p, int kind, const float (&v)[kVec]) const
    {
        if (kind == kBf16) store<kBf16>((char*)p, pack<kBf16>(v));
        else if (kind == kF16) store<kF16>((char*)p, pack<kF16>(v));
        else store<kF32>((char*)p, pack<kF32>(v));
    }
    // A parameter of a kind known at run time (the same in all lanes); NULL: `absent` everywhere.
    __device__ __forceinline__ void param(const void* p, int kind, float absent, float (&v)[kVec]) const
    {
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = absent;
        if (!p) return;
        if (kind == kBf16) unpack<kBf16>(load<kBf16>((const char*)p), v);
        else if (kind == kF16) unpack<kF16>(load<kF16>((const char*)p), v);
        else unpack<kF32>(load<kF32>((const char*)p), v);
    }
};

// The loads of `r` are over here: the value is used, so the compiler waits for it.
template <int KIND> __device__ __forceinline__ void arrived(Raw<KIND>& r)
{
    #pragma unroll
    for (int i = 0; i < (KIND == kF32 ? 2 : 1); ++i) asm volatile("" : "+v"(r.q[i]));
}

// Waits for the LDS alone: loads from memory stay in flight across it.
__device__ __forceinline__ void barrier_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Orders LDS accesses of one wavefront's lanes before and after it.  They complete in program order, so this is no
// instruction: it tells the compiler, to whom the lanes' addresses do not alias, to keep that order.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Lanes are summed in a fixed order within rows of 16 by shifts, then across them; the result is in every lane.
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_zero(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp_zero<0x111, 0xF>(v);          // row_shr:1, 2, 4, 8
    v += dpp_zero<0x112, 0xF>(v);
    v += dpp_zero<0x114, 0xF>(v);
    v += dpp_zero<0x118, 0xF>(v);
    v += dpp_zero<0x142, 0xA>(v);          // row_bcast:15 into rows 1 and 3
    v += dpp_zero<0x143, 0xC>(v);          // row_bcast:31 into rows 2 and 3
    return lane_value(v, 63);
}

// The sum of the first 16 lanes, in all lanes.
__device__ __forceinline__ float sum_of_16(float v)
{
    v += dpp_zero<0x111, 0xF>(v);
    v += dpp_zero<0x112, 0xF>(v);
    v += dpp_zero<0x114, 0xF>(v);
    v += dpp_zero<0x118, 0xF>(v);
    return lane_value(v, 15);
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011) of the counter
// `block` under `key`: 128 bits, eight 16-bit numbers, the low half of word 0 first.
__device__ __forceinline__ u32x4 philox(uint64_t block, uint64_t key)
{
    uint32_t x0 = (uint32_t)block, x1 = (uint32_t)(block >> 32), x2 = 0, x3 = 0;
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
    #pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
        x0 = (uint32_t)(b >> 32) ^ x1 ^ k0;
        x1 = (uint32_t)b;
        x2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
        x3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{x0, x1, x2, x3};
}

// Drops elements of the vector that the generator's block `block` decides.  A dropped element becomes +0 whatever it held.
__device__ __forceinline__ void drop_vec(float (&v)[kVec], uint64_t block, uint64_t seed, uint32_t threshold, float scale)
{
    const u32x4 w = philox(block, seed);
    #pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const uint32_t u = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
        v[i] = u >= threshold ? v[i] * scale : 0.f;
    }
}

// As drop_vec for the columns of `at` in a row whose first block is `block`: those that begin inside a block take the rest
// from the next one.
template <int TAIL>
__device__ __forceinline__ void drop_at(float (&v)[kVec], const Place<TAIL>& at, uint64_t block, uint64_t seed, uint32_t threshold,
                                        float scale)
{
    const unsigned inside = at.e % kVec;
    if (TAIL != kRagged || !__builtin_amdgcn_ballot_w64(inside != 0)) {        // the same in all lanes
        drop_vec(v, block + at.e / kVec, seed, threshold, scale);
    } else {
        unsigned keep = 0;
        #pragma unroll
        for (int b = 0; b < 2; ++b) {
            const u32x4 w = philox(block + at.e / kVec + b, seed);
            #pragma unroll
            for (int i = 0; i < kVec; ++i)
                keep |= (unsigned)((i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu) >= threshold) << (b * kVec + i);
        }
        keep >>= inside;
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = keep >> i & 1 ? v[i] * scale : 0.f;
    }
}

// The launch call's own status: an earlier, unrelated error of the thread is neither reported nor cleared.
template <typename Args>
int launch_args(void (*kernel)(Args), dim3 grid, dim3 block, size_t lds, void* stream, Args args)
{
    void* ptrs[] = {(void*)&args};
    return (int)hipLaunchKernel((const void*)kernel, grid, block, ptrs, lds, (hipStream_t)stream);
}

// Calls f(std::integral_constant<int, KIND>).
template <typename F> int dispatch_kind(int kind, F&& f)
{
    switch (kind) {
        case kBf16: return f(std::integral_constant<int, kBf16>{});
        case kF16: return f(std::integral_constant<int, kF16>{});
        default: return f(std::integral_constant<int, kF32>{});
    }
}

// Calls f(std::integral_constant<int, TAIL>) for rows of `cols` elements; TINY: they may be fewer than eight.
template <bool TINY = true, typename F> int dispatch_tail(size_t cols, F&& f)
{
    if constexpr (TINY)
        if (tail_of(cols) == kTiny) return f(std::integral_constant<int, kTiny>{});
    return tail_of(cols) == kWhole ? f(std::integral_constant<int, kWhole>{}) : f(std::integral_constant<int, kRagged>{});
}
// Calls f(std::bool_constant<a>).
template <typename F> int dispatch_flag(bool a, F&& f) { return a ? f(std::true_type{}) : f(std::false_type{}); }

}  // namespace
}  // namespace mics
