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
    float* parts;                              // [split][m][n]
};
// One launch, and one more where linear_splits() > 1.
int launch_product(const Product& p, int kind, void* stream);

// z = x + bias, or the sum of `splits` parts of packed rows (x.data NULL) + bias.
struct ActivationPass {
    Epilogue e;
    ConstRows x;
    const float* parts;
    int splits;
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
