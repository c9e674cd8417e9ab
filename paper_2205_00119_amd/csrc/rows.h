// Rows of bf16, binary16 or binary32 in vectors of eight elements: what the kernels of layer.hip and logprobs.hip
// share.  A lane owns columns 8c to 8c + 7; the last vector of a row may hold fewer.  Rows may begin on any element:
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

// The vector at `p`, of which `valid` elements exist (8 and more: all); the others read as 0.  A part of a vector
// comes in pieces of four, two and one elements.
template <int KIND> __device__ __forceinline__ Raw<KIND> load_vec(const char* p, int valid)
{
    Raw<KIND> r{};
    if (valid >= kVec) {
        if constexpr (KIND == kF32) {
            r.q[0] = ((const u32x4_a4*)p)[0];
            r.q[1] = ((const u32x4_a4*)p)[1];
        } else {
            r.q[0] = *(const u32x4_a2*)p;
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
template <int KIND> __device__ __forceinline__ void store_vec(char* p, const Raw<KIND>& r, int valid)
{
    if (valid >= kVec) {
        if constexpr (KIND == kF32) {
            ((u32x4_a4*)p)[0] = r.q[0];
            ((u32x4_a4*)p)[1] = r.q[1];
        } else {
            *(u32x4_a2*)p = r.q[0];
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

// Vector c of a row.  Whole rows (RAGGED false: the last vector has eight elements too) are loaded without a branch:
// lanes behind the end read the last vector, and what they make of it is neither summed nor stored.
template <int KIND, bool RAGGED> __device__ __forceinline__ Raw<KIND> load_col(const char* row, unsigned c, unsigned cols)
{
    if constexpr (RAGGED) return load_vec<KIND>(row + (size_t)c * (kVec * kWidth<KIND>), valid_at(c, cols));
    else return load_vec<KIND>(row + (size_t)min(c, cols / kVec - 1) * (kVec * kWidth<KIND>), kVec);
}
template <int KIND, bool RAGGED>
__device__ __forceinline__ void store_col(char* row, unsigned c, unsigned cols, const Raw<KIND>& r)
{
    char* const p = row + (size_t)c * (kVec * kWidth<KIND>);
    const int valid = valid_at(c, cols);
    if constexpr (RAGGED) store_vec<KIND>(p, r, valid);
    else if (valid > 0) store_vec<KIND>(p, r, kVec);
}
// What element i adds to its vector's sum, and the vector to its lane's.
template <bool RAGGED> __device__ __forceinline__ float summand(float v, int i, int valid)
{
    return !RAGGED || i < valid ? v : 0.f;
}
template <bool RAGGED> __device__ __forceinline__ float vector_sum(float s, int valid)
{
    return RAGGED || valid > 0 ? s : 0.f;
}

// Vector c of a parameter of a kind known at run time (the same in all lanes); NULL: `absent` everywhere.
template <bool RAGGED>
__device__ __forceinline__ void load_param(const void* p, int kind, unsigned c, unsigned cols, float absent, float (&v)[kVec])
{
    if (!p) {
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = absent;
    } else if (kind == kBf16) {
        unpack<kBf16>(load_col<kBf16, RAGGED>((const char*)p, c, cols), v);
    } else if (kind == kF16) {
        unpack<kF16>(load_col<kF16, RAGGED>((const char*)p, c, cols), v);
    } else {
        unpack<kF32>(load_col<kF32, RAGGED>((const char*)p, c, cols), v);
    }
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

// Calls f(std::bool_constant<a>).
template <typename F> int dispatch_flag(bool a, F&& f) { return a ? f(std::true_type{}) : f(std::false_type{}); }

}  // namespace
}  // namespace mics
