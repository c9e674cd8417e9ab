// Between the argument checks (linear_api.cpp) and the launchers (linear.hip, activation.hip) of the linear layer and of
// activations with 8-bit checkpoints.
#pragma once

#include "layer_internal.h"
#include "linear_rules.h"

namespace mics {

constexpr unsigned kBlockCols = 64;            // columns of a row that share a scale
constexpr int kActs = 5;

// What happens to a sum on its way out: z = sum + bias, out = residual + act(z), and z kept.  Kinds as in layer_internal.h.
struct Epilogue {
    Rows out, pre;                             // pre may be NULL
    Rows codes;                                // int8; may be NULL
    float* scales;
    const void* bias;                          // may be NULL
    ConstRows residual;                        // may be NULL
    int act, param, out_kind;                  // pre and residual are of the operands' kind
};

// out[m][n] = epilogue(sum over k of a(m, k) b(n, k)).  a(m, k) lies at a[m][k], or with a_turned at a[k][m]; b likewise.
struct Product {
    Epilogue e;
    ConstRows a, b;
    bool a_turned, b_turned;
    size_t m, n, k;
    float* parts;                              // [shared tile][split][row][column] of a plan with several splits; then copies
};
// Whether an operand's rows hold whole chunks of 16 bytes, and a tile's chunks lie within 31 bits of its first.
inline bool in_chunks(const ConstRows& m, bool turned, size_t rows, size_t k, size_t width)
{
    return (turned ? rows : k) * width >= 16 && m.stride < (size_t{1} << 31) / width / 256;
}
// Whether every chunk of an operand lies on 16 bytes.
inline bool on_16(const ConstRows& m, bool turned, size_t rows, size_t width)
{
    return (uintptr_t)m.data % 16 == 0 && m.stride * width % 16 == 0 && (!turned || rows * width % 16 == 0);
}
inline ProductPlan plan_of(const Product& p, size_t width)
{
    return plan_product({p.m, p.n, p.k, width, p.a_turned, p.b_turned, on_16(p.a, p.a_turned, p.m, width), on_16(p.b, p.b_turned, p.n, width),
                         in_chunks(p.a, p.a_turned, p.m, p.k, width) && in_chunks(p.b, p.b_turned, p.n, p.k, width), p.e.codes.data != nullptr});
}
// One launch, and one more each where the plan copies operands or has several splits.
int launch_product(const Product& p, const ProductPlan& plan, int kind, void* stream);

// z = x + bias
struct ActivationPass {
    Epilogue e;
    ConstRows x;
    size_t rows;
    unsigned cols;
};
int launch_activation(const ActivationPass& a, int kind, void* stream);

struct CheckpointRead {
    Rows y;
    ConstRows codes;
    const float* scales;
    size_t rows;
    unsigned cols;
    int act;
};
int launch_checkpoint_read(const CheckpointRead& a, int kind, void* stream);

struct ActivationBackward {
    Rows dx;                                   // may be NULL
    ConstRows dy, z, codes;                    // z or codes
    const float* scales;
    size_t rows;
    unsigned cols;
    int act;
    float* parts;
};
// As launch_dropout_backward; dbias may be NULL.
int launch_activation_backward(const ActivationBackward& a, int kind, void* dbias, int grad, void* stream);

}  // namespace mics
