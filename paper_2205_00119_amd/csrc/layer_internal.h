// Between the argument checks (layer_api.cpp) and the launchers (norm.hip, dropout.hip, logprobs.hip) of the operators that a
// transformer layer's training step runs between the parameter gather and the gradient reduction.
#pragma once

#include <cstddef>
#include <cstdint>

namespace mics {

// Records a failure for mics_last_error and returns `code` (api.cpp).
int fail(int code, const char* fmt, ...);

// Dropout as the kernels apply it: an element stays where its 16-bit number is at least `threshold`, times `scale`.
// threshold 0: nothing is dropped and no number is made.
struct Dropout {
    uint64_t seed, offset;
    uint32_t threshold;
    float scale;
};

// A matrix of rows in device memory, `stride` elements from one row to the next; data NULL: not there.
struct Rows {
    void* data;
    size_t stride;
};
struct ConstRows {
    const void* data;
    size_t stride;
};

// Kinds: 0 bf16, 1 IEEE binary16, 2 binary32.  `kind` is that of the matrices, `param` that of the vectors.
struct NormForward {
    Rows y, sum;                          // sum may be NULL
    float *mean, *rstd;                   // may be NULL
    ConstRows x, residual;
    const void *bias, *weight, *norm_bias;   // may be NULL
    size_t rows;
    unsigned cols;
    Dropout drop;
    float eps;
    int param;
};
struct NormBackward {
    Rows dx, dresidual;                   // dresidual may be NULL
    ConstRows dy, dsum, x;                // dsum may be NULL; x: what was normalised
    const float *mean, *rstd;
    const void* weight;                   // may be NULL
    size_t rows;
    unsigned cols;
    Dropout drop;
    int param;
    float* row_sums;                      // 2 * rows, of rows longer than kTiledCols
    float* parts;                         // column sums by group of rows: [which][group][cols]
};
struct DropoutPass {
    Rows out;
    ConstRows x, residual;
    const void* bias;
    size_t rows;
    unsigned cols;
    Dropout drop;
    int param;
    float* parts;                         // backward with dbias
};

// Column sums are formed in groups of rows: of the norms' two or three sums at most so many groups, of the dropout's one twice as
// many.
constexpr size_t kMostParts = 256;
// Rows of more elements than this do not stay in a workgroup's registers in the backward pass.
constexpr size_t kTiledCols = 8192;
constexpr size_t row_sums_floats(size_t rows, size_t cols) { return cols > kTiledCols ? 2 * rows : 0; }
constexpr size_t parts_floats(size_t rows, size_t cols) { return (rows < kMostParts ? rows : kMostParts) * 3 * cols; }
constexpr size_t kMostCols = size_t{1} << 24;

// `fused`: bias, residual, dropout, sum; otherwise the norm alone.
int launch_norm(const NormForward& a, int kind, bool fused, void* stream);
// dx and the sums by group of rows, then the sums: two launches.  One where a workgroup takes all rows (few rows of at most
// kTiledCols) and without rows; rows longer than kTiledCols take one more, in front.  grads: dweight, dnorm_bias and, with
// `fused`, dbias, of kind `grad`, each may be NULL.
int launch_norm_backward(const NormBackward& a, int kind, bool fused, void* const* grads, int grad, void* stream);
int launch_dropout(const DropoutPass& a, int kind, void* stream);
// Two launches; one for few rows, for very long ones (one workgroup for each stripe of them) and without rows.
int launch_dropout_backward(const DropoutPass& a, int kind, void* dbias, int grad, void* stream);

struct LogProbs {
    float *logprob, *entropy, *lse;       // entropy and lse may be NULL
    int64_t* top_ids;
    float* top_logprobs;
    ConstRows logits;
    const int64_t* targets;
    size_t rows;
    unsigned vocab;
    int top;
    void* parts;                          // of row_splits() > 1
};
struct LogProbsBackward {
    Rows dlogits;
    ConstRows logits;
    const int64_t* targets;
    const float *lse, *entropy, *dlogprob, *dentropy;   // dentropy may be NULL
    size_t rows;
    unsigned vocab;
};
constexpr int kMostTop = 64;
// Workgroups that share a row, and the bytes that one of them leaves for the join.
int row_splits(size_t rows, size_t vocab, int top);
constexpr size_t split_bytes(int top) { return 16 + 8 * (size_t)top; }
int launch_logprobs(const LogProbs& a, int kind, void* stream);
int launch_logprobs_backward(const LogProbsBackward& a, int kind, void* stream);

}  // namespace mics
