// Activations, their slopes, and the 8-bit checkpoint of a block: what activation.hip and linear.hip share.
#pragma once

#include "columns.h"
#include "linear_internal.h"
#include "rows.h"

namespace mics {
namespace {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

// The distribution function of the standard normal at -|z| is exp(-z^2/2) P(t) with t = 1/(1 + 0.23 |z|): P is a polynomial without
// a constant term, fitted to erfcx(|z|/sqrt 2)/2 by iterated reweighted least squares, relative error 3e-8 up to |z| = 2 and
// 1e-6 at 13; evaluated in binary32 it is within 4.1e-7 up to 4 and 1.3e-6 up to 13.
struct Normal {
    float below, bell, near;                   // the function at -|z|; exp(-z^2/2); |z|, at most 16, where both others are 0
};
__device__ __forceinline__ Normal normal_at(float z)
{
    const float a = __builtin_fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.23f, a, 1.f));      // keeps NaN, which `near` loses
    const float near = fminf(a, 16.f);
    const float bell = __builtin_amdgcn_exp2f(near * (near * -0.72134752f));   // log2 e / 2
    float s = __builtin_fmaf(-0.07516629248857498f, t, 0.27394965291023254f);
    s = __builtin_fmaf(s, t, -0.2431972622871399f);
    s = __builtin_fmaf(s, t, 0.26043280959129333f);
    s = __builtin_fmaf(s, t, -0.003819522215053439f);
    s = __builtin_fmaf(s, t, 0.10681562125682831f);
    s = __builtin_fmaf(s, t, 0.08907731622457504f);
    s = __builtin_fmaf(s, t, 0.09190764278173447f);
    return {bell * (s * t), bell, near};
}
// 1 / (1 + exp(-2 sqrt(2/pi) (z + 0.044715 z^3)))
__device__ __forceinline__ float tanh_share(float z)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * __builtin_fmaf(z * z, -0.10294324f, -2.3022082f)));
}
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }

// Factors that meet a 0 are kept finite: -inf gives 0.
template <int ACT> __device__ __forceinline__ float act_of(float z)
{
    const float high = fmaxf(z, -3.4028234664e38f);
    if constexpr (ACT == kActRelu) return z <= 0.f ? 0.f : z;
    else if constexpr (ACT == kActGelu) {
        const Normal n = normal_at(z);
        return __builtin_fmaf(-n.near, n.below, fmaxf(z, 0.f));
    }
    else if constexpr (ACT == kActGeluTanh) return high * tanh_share(z);
    else if constexpr (ACT == kActSilu) return high * logistic(z);
    else return z;
}
// Where the second factor of a product is 0 from some |z| on, the first stops growing there: no 0 * inf.
template <int ACT> __device__ __forceinline__ float slope_of(float z)
{
    const float c = __builtin_amdgcn_fmed3f(z, -16.f, 16.f);
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    else if constexpr (ACT == kActGelu) {
        const Normal n = normal_at(z);
        return __builtin_fmaf(c * 0.39894228f, n.bell, z < 0.f ? n.below : 1.f - n.below);
    } else if constexpr (ACT == kActGeluTanh) {
        const float s = tanh_share(z);         // 2 sqrt(2/pi) (1 + 3 * 0.044715 z^2)
        return __builtin_fmaf(c * s * (1.f - s), __builtin_fmaf(c * c, 0.21406538f, 1.5957691f), s);
    } else if constexpr (ACT == kActSilu) {
        const float s = logistic(z), far = __builtin_amdgcn_fmed3f(z, -200.f, 200.f);
        return s * __builtin_fmaf(far, 1.f - s, 1.f);
    } else return 1.f;
}

// Calls f(std::integral_constant<int, ACT>) for an activation known at run time, the same in all lanes.
template <typename F> __device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
        case kActRelu: f(std::integral_constant<int, kActRelu>{}); break;
        case kActGelu: f(std::integral_constant<int, kActGelu>{}); break;
        case kActGeluTanh: f(std::integral_constant<int, kActGeluTanh>{}); break;
        case kActSilu: f(std::integral_constant<int, kActSilu>{}); break;
        default: break;
    }
}

// The scale of a block and what its elements are multiplied by.  `top`: the largest magnitude's bits, so that infinities and
// NaN are larger than all numbers; such a block's codes are masked away.  Both quotients are correctly rounded: a product with the
// divisor's reciprocal, then its remainder, which is exact, times the reciprocal; for 127 / t the reciprocal is refined first, and
// where it would be subnormal the division is left to the compiler.
struct Coding {
    float scale, by;
    uint32_t keep;
};
__device__ __forceinline__ Coding coding_of(uint32_t top)
{
    if (top > 0x7F7FFFFFu) return {__builtin_nanf(""), 0.f, 0u};
    const float t = fmaxf(__builtin_bit_cast(float, top), 0x1p-100f);
    constexpr float r127 = 1.f / 127.f;
    const float q = t * r127, scale = __builtin_fmaf(__builtin_fmaf(-127.f, q, t), r127, q);
    if (t > 0x1p100f) return {scale, 127.f / t, ~0u};
    const float y = __builtin_amdgcn_rcpf(t), r = __builtin_fmaf(__builtin_fmaf(-t, y, 1.f), y, y), p = 127.f * r;
    return {scale, __builtin_fmaf(__builtin_fmaf(-t, p, 127.f), r, p), ~0u};
}
// rint(z * by) in the low 8 bits: of a number of at most 127 with 1.5 * 2^23 added the last bit counts ones.
__device__ __forceinline__ uint32_t code_of(float z, float by) { return __builtin_bit_cast(uint32_t, z * by + 12582912.f); }
__device__ __forceinline__ uint32_t codes_of(const float* z, const Coding& c)
{
    const uint32_t low = __builtin_amdgcn_perm(code_of(z[1], c.by), code_of(z[0], c.by), 0x0C0C0400u);
    const uint32_t high = __builtin_amdgcn_perm(code_of(z[3], c.by), code_of(z[2], c.by), 0x0C0C0400u);
    return __builtin_amdgcn_perm(high, low, 0x05040100u) & c.keep;
}
// What four codes stand for: code * scale, rounded once.  Signed bytes are converted where they lie (v_cvt_f32_i32 of a byte of its
// operand), two operations an element, and none gives more than the result: 128 scales of a block at the end of the range are infinite.
// us against a biased conversion whose 128 scales are taken away in a fused multiply: 4096 x 32768 bf16 read with tanh 80.9 / 83.4,
// with gelu 103 / 108, backward the same.
__device__ __forceinline__ void restored(uint32_t codes, float scale, float* v)
{
    #pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(codes >> (8 * i)) * scale;
}

typedef u32x2 u32x2_a1 __attribute__((aligned(1)));

// A block of 64 columns belongs to eight lanes of eight columns each; lanes behind the end of a row hold zeros.
constexpr unsigned kBlockLanes = kBlockCols / kVec;

// The largest of eight lanes, in all of them.
template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t max_of_8(uint32_t v)
{
    v = dpp_max<0xB1>(v);                      // quad_perm: lane ^ 1
    v = dpp_max<0x4E>(v);                      // quad_perm: lane ^ 2
    return dpp_max<0x141>(v);                  // row_half_mirror: the other four
}

// Eight elements from column 8c on of a vector or row of a kind known at run time.
__device__ __forceinline__ void load_any(const char* row, int kind, unsigned c, int valid, float (&v)[kVec])
{
    if (kind == kBf16) unpack<kBf16>(load_vec<kBf16>(row + (size_t)c * 16, valid), v);
    else if (kind == kF16) unpack<kF16>(load_vec<kF16>(row + (size_t)c * 16, valid), v);
    else unpack<kF32>(load_vec<kF32>(row + (size_t)c * 32, valid), v);
}
__device__ __forceinline__ void store_any(char* row, int kind, unsigned c, int valid, const float (&v)[kVec])
{
    if (kind == kBf16) store_vec<kBf16>(row + (size_t)c * 16, pack<kBf16>(v), valid);
    else if (kind == kF16) store_vec<kF16>(row + (size_t)c * 16, pack<kF16>(v), valid);
    else store_vec<kF32>(row + (size_t)c * 32, pack<kF32>(v), valid);
}
__device__ __forceinline__ u32x2 load_codes(const char* p, int valid)
{
    u32x2 q{};
    if (valid >= kVec) q = *(const u32x2_a1*)p;
    else
        for (int i = 0; i < valid; ++i) {
            const uint32_t b = (uint32_t)(uint8_t)p[i] << (i % 4 * 8);
            if (i < 4) q.x |= b; else q.y |= b;
        }
    return q;
}

// z = v + bias and everything after it, for vector c of a row of which `valid` elements exist; all lanes of a block come here.
template <int KIND>
__device__ __forceinline__ void finish(const Epilogue& e, size_t row, unsigned c, unsigned cols, int valid, float (&v)[kVec])
{
    float t[kVec];
    if (e.bias) {
        load_any((const char*)e.bias, e.param, c, valid, t);
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] += t[i];
    }
    Raw<KIND> residual;                        // loaded before anything is stored: pre may take its place
    if (e.residual.data) residual = load_vec<KIND>(row_at<KIND>(e.residual, row) + (size_t)c * (kVec * kWidth<KIND>), valid);
    if (e.pre.data) store_vec<KIND>(row_at<KIND>(e.pre, row) + (size_t)c * (kVec * kWidth<KIND>), pack<KIND>(v), valid);
    if (e.codes.data) {
        float most = 0.f;
        if (valid >= kVec) {
            #pragma unroll
            for (int i = 0; i < kVec; ++i) most = __builtin_elementwise_maximum(most, __builtin_fabsf(v[i]));
        } else {
            #pragma unroll
            for (int i = 0; i < kVec; ++i) most = i < valid ? __builtin_elementwise_maximum(most, __builtin_fabsf(v[i])) : most;
        }
        const Coding code = coding_of(max_of_8(__builtin_bit_cast(uint32_t, most) & 0x7FFFFFFFu));
        const u32x2 q = {codes_of(v, code), codes_of(v + 4, code)};
        char* const to = (char*)e.codes.data + row * e.codes.stride + (size_t)c * kVec;
        if (valid >= kVec) *(u32x2_a1*)to = q;
        else
            for (int i = 0; i < valid; ++i) to[i] = (char)((i < 4 ? q.x : q.y) >> (i % 4 * 8));
        if (c % kBlockLanes == 0 && valid > 0) e.scales[row * ((cols + kBlockCols - 1) / kBlockCols) + c / kBlockLanes] = code.scale;
    }
    if (!e.out.data) return;
    with_act(e.act, [&](auto A) {
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = act_of<decltype(A)::value>(v[i]);
    });
    if (e.residual.data) {
        unpack<KIND>(residual, t);
        #pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = t[i] + v[i];
    }
    store_any((char*)e.out.data + row * e.out.stride * (e.out_kind == kF32 ? 4 : 2), e.out_kind, c, valid, v);
}

}  // namespace
}  // namespace mics
