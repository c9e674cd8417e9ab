// C ABI of the operators between the parameter gather and the gradient reduction: host-side argument validation and
// dispatch.  Every check runs before the first HIP call.
#include "../../include/mics.h"
#include "internal.h"
#include "layer_checks.h"
#include "layer_internal.h"

#include <cmath>

namespace {

using mics::addr;
using mics::Checked;
using mics::column_sizes;
using mics::fail;
using mics::hip_fail;
using mics::width;
using mics::workspace;

// Checks `drop` and fills `d`.
int dropout(const char* fn, float drop, uint64_t seed, uint64_t offset, mics::Dropout* d)
{
    if (!(drop >= 0.f && drop < 1.f)) return fail(MICS_ERR_INVALID_ARG, "%s: drop = %g must lie in [0, 1)", fn, (double)drop);
    const double t = std::nearbyint(65536.0 * (double)drop);
    d->threshold = t > 65535 ? 65535u : (uint32_t)t;
    d->scale = (float)(65536.0 / (65536.0 - d->threshold));
    d->seed = seed;
    d->offset = offset;
    return MICS_OK;
}

struct NormForwardCall {
    const char* fn;
    bool fused;
    void *y, *sum;
    float *mean, *rstd;
    const void *x, *bias, *residual, *weight, *norm_bias;
    const char* norm_bias_name;
};

int norm_forward(const NormForwardCall& c, size_t rows, size_t cols, const size_t* strides, float drop, uint64_t seed, uint64_t offset,
                 float eps, int dtype, int param_dtype, void* stream)
{
    Checked args(c.fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("param_dtype", param_dtype));
    MICS_TRY(args.sizes("cols"));
    if (!(eps >= 0.f)) return fail(MICS_ERR_INVALID_ARG, "%s: eps = %g must not be negative", c.fn, (double)eps);
    mics::NormForward a{};
    MICS_TRY(dropout(c.fn, drop, seed, offset, &a.drop));
    const size_t e = width(dtype), pe = width(param_dtype);
    int i = 0;
    a.y = {c.y, args.stride(strides, i++)};
    args.matrix("y", c.y, a.y.stride, e, true);
    if (c.fused) {
        a.sum = {c.sum, args.stride(strides, i++)};
        args.matrix("sum", c.sum, a.sum.stride, e, true, true);
    }
    a.x = {c.x, args.stride(strides, i++)};
    args.matrix("x", c.x, a.x.stride, e, false);
    if (c.fused) {
        a.residual = {c.residual, args.stride(strides, i++)};
        args.matrix("residual", c.residual, a.residual.stride, e, false, true);
        args.vector("bias", c.bias, cols, pe, false, true);
    }
    args.vector("mean", c.mean, rows, 4, true, true);
    args.vector("rstd", c.rstd, rows, 4, true, true);
    args.vector("weight", c.weight, cols, pe, false, true);
    args.vector(c.norm_bias_name, c.norm_bias, cols, pe, false, true);
    MICS_TRY(args.check());
    if (rows == 0) return MICS_OK;
    a.mean = c.mean; a.rstd = c.rstd;
    a.bias = c.bias; a.weight = c.weight; a.norm_bias = c.norm_bias;
    a.rows = rows; a.cols = (unsigned)cols; a.eps = eps; a.param = param_dtype;
    const int err = mics::launch_norm(a, dtype, c.fused, stream);
    return err ? hip_fail(c.fn, err) : MICS_OK;
}

struct NormBackwardCall {
    const char* fn;
    bool fused;
    void *dx, *dresidual, *dbias, *dweight, *dnorm_bias;
    const void *dy, *dsum, *x;
    const float *mean, *rstd;
    const void* weight;
    const char *dnorm_bias_name, *x_name;
};

int norm_backward(const NormBackwardCall& c, size_t rows, size_t cols, const size_t* strides, float drop, uint64_t seed,
                  uint64_t offset, int dtype, int param_dtype, int grad_dtype, void* work, size_t work_bytes, void* stream)
{
    Checked args(c.fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("param_dtype", param_dtype));
    MICS_TRY(args.dtype("grad_dtype", grad_dtype));
    MICS_TRY(args.sizes("cols"));
    mics::NormBackward a{};
    MICS_TRY(dropout(c.fn, drop, seed, offset, &a.drop));
    const size_t e = width(dtype), pe = width(param_dtype), ge = width(grad_dtype);
    const size_t needed = mics_column_workspace_bytes(rows, cols);
    int i = 0;
    a.dx = {c.dx, args.stride(strides, i++)};
    args.matrix("dx", c.dx, a.dx.stride, e, true);
    if (c.fused) {
        a.dresidual = {c.dresidual, args.stride(strides, i++)};
        args.matrix("dresidual", c.dresidual, a.dresidual.stride, e, true, true);
    }
    a.dy = {c.dy, args.stride(strides, i++)};
    args.matrix("dy", c.dy, a.dy.stride, e, false);
    if (c.fused) {
        a.dsum = {c.dsum, args.stride(strides, i++)};
        args.matrix("dsum", c.dsum, a.dsum.stride, e, false, true);
    }
    a.x = {c.x, args.stride(strides, i++)};
    args.matrix(c.x_name, c.x, a.x.stride, e, false);
    if (c.fused) args.vector("dbias", c.dbias, cols, ge, true, true);
    args.vector("dweight", c.dweight, cols, ge, true, true);
    args.vector(c.dnorm_bias_name, c.dnorm_bias, cols, ge, true, true);
    args.vector("mean", c.mean, rows, 4, false);
    args.vector("rstd", c.rstd, rows, 4, false);
    args.vector("weight", c.weight, cols, pe, false, true);
    args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(c.fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    a.mean = c.mean; a.rstd = c.rstd; a.weight = c.weight;
    a.rows = rows; a.cols = (unsigned)cols; a.param = param_dtype;
    a.row_sums = (float*)work;
    a.parts = a.row_sums + mics::row_sums_floats(rows, cols);
    void* const grads[3] = {c.dweight, c.dnorm_bias, c.dbias};
    const int err = mics::launch_norm_backward(a, dtype, c.fused, grads, grad_dtype, stream);
    return err ? hip_fail(c.fn, err) : MICS_OK;
}

}  // namespace

extern "C" {

uint64_t mics_dropout_counters(size_t rows, size_t cols) { return (uint64_t)rows * (cols / 8 + (cols % 8 ? 1 : 0)); }

size_t mics_column_workspace_bytes(size_t rows, size_t cols)
{
    if (!column_sizes(rows, cols)) return 0;
    return 4 * (mics::row_sums_floats(rows, cols) + mics::parts_floats(rows, cols));
}

int mics_layer_norm(void* y, float* mean, float* rstd, const void* x, const void* weight, const void* bias, size_t rows,
                    size_t cols, const size_t* strides, float eps, int dtype, int param_dtype, void* stream)
{
    return norm_forward({"mics_layer_norm", false, y, nullptr, mean, rstd, x, nullptr, nullptr, weight, bias, "bias"}, rows, cols,
                        strides, 0.f, 0, 0, eps, dtype, param_dtype, stream);
}

int mics_layer_norm_backward(void* dx, void* dweight, void* dbias, const void* dy, const void* x, const float* mean,
                             const float* rstd, const void* weight, size_t rows, size_t cols, const size_t* strides, int dtype,
                             int param_dtype, int grad_dtype, void* work, size_t work_bytes, void* stream)
{
    return norm_backward({"mics_layer_norm_backward", false, dx, nullptr, nullptr, dweight, dbias, dy, nullptr, x, mean, rstd,
                          weight, "dbias", "x"}, rows, cols, strides, 0.f, 0, 0, dtype, param_dtype, grad_dtype, work, work_bytes,
                         stream);
}

int mics_dropout_add_layer_norm(void* y, void* sum, float* mean, float* rstd, const void* x, const void* bias,
                                const void* residual, const void* weight, const void* norm_bias, size_t rows, size_t cols,
                                const size_t* strides, float drop, uint64_t seed, uint64_t offset, float eps, int dtype,
                                int param_dtype, void* stream)
{
    return norm_forward({"mics_dropout_add_layer_norm", true, y, sum, mean, rstd, x, bias, residual, weight, norm_bias,
                         "norm_bias"}, rows, cols, strides, drop, seed, offset, eps, dtype, param_dtype, stream);
}

int mics_dropout_add_layer_norm_backward(void* dx, void* dresidual, void* dbias, void* dweight, void* dnorm_bias, const void* dy,
                                         const void* dsum, const void* sum, const float* mean, const float* rstd,
                                         const void* weight, size_t rows, size_t cols, const size_t* strides, float drop,
                                         uint64_t seed, uint64_t offset, int dtype, int param_dtype, int grad_dtype, void* work,
                                         size_t work_bytes, void* stream)
{
    return norm_backward({"mics_dropout_add_layer_norm_backward", true, dx, dresidual, dbias, dweight, dnorm_bias, dy, dsum, sum,
                          mean, rstd, weight, "dnorm_bias", "sum"}, rows, cols, strides, drop, seed, offset, dtype, param_dtype,
                         grad_dtype, work, work_bytes, stream);
}

int mics_bias_dropout_add(void* out, const void* x, const void* bias, const void* residual, size_t rows, size_t cols,
                          const size_t* strides, float drop, uint64_t seed, uint64_t offset, int dtype, int param_dtype,
                          void* stream)
{
    const char* fn = "mics_bias_dropout_add";
    Checked args(fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("param_dtype", param_dtype));
    MICS_TRY(args.sizes("cols"));
    mics::DropoutPass a{};
    MICS_TRY(dropout(fn, drop, seed, offset, &a.drop));
    const size_t e = width(dtype);
    a.out = {out, args.stride(strides, 0)};
    a.x = {x, args.stride(strides, 1)};
    a.residual = {residual, args.stride(strides, 2)};
    args.matrix("out", out, a.out.stride, e, true);
    args.matrix("x", x, a.x.stride, e, false);
    args.matrix("residual", residual, a.residual.stride, e, false, true);
    args.vector("bias", bias, cols, width(param_dtype), false, true);
    MICS_TRY(args.check());
    if (rows == 0) return MICS_OK;
    a.bias = bias; a.rows = rows; a.cols = (unsigned)cols; a.param = param_dtype;
    const int err = mics::launch_dropout(a, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

int mics_bias_dropout_add_backward(void* dx, void* dbias, const void* dout, size_t rows, size_t cols, const size_t* strides,
                                   float drop, uint64_t seed, uint64_t offset, int dtype, int grad_dtype, void* work,
                                   size_t work_bytes, void* stream)
{
    const char* fn = "mics_bias_dropout_add_backward";
    Checked args(fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("grad_dtype", grad_dtype));
    MICS_TRY(args.sizes("cols"));
    mics::DropoutPass a{};
    MICS_TRY(dropout(fn, drop, seed, offset, &a.drop));
    const size_t e = width(dtype), needed = dbias ? mics_column_workspace_bytes(rows, cols) : 0;
    a.out = {dx, args.stride(strides, 0)};
    a.x = {dout, args.stride(strides, 1)};
    args.matrix("dx", dx, a.out.stride, e, true);
    args.matrix("dout", dout, a.x.stride, e, false);
    args.vector("dbias", dbias, cols, width(grad_dtype), true, true);
    if (needed) args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    a.rows = rows; a.cols = (unsigned)cols; a.parts = (float*)work;
    if (!dbias && rows == 0) return MICS_OK;
    const int err = dbias ? mics::launch_dropout_backward(a, dtype, dbias, grad_dtype, stream)
                          : mics::launch_dropout(a, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

size_t mics_token_logprobs_workspace_bytes(size_t rows, size_t vocab, int top_k)
{
    if (!column_sizes(rows, vocab) || top_k < 0 || top_k > MICS_MAX_TOP) return 0;
    const int splits = mics::row_splits(rows, vocab, top_k);
    return splits > 1 ? rows * (size_t)splits * mics::split_bytes(top_k) : 0;
}

int mics_token_logprobs(float* logprob, float* entropy, float* lse, int64_t* top_ids, float* top_logprobs, const void* logits,
                        const int64_t* targets, size_t rows, size_t vocab, size_t stride, int top_k, int dtype, void* work,
                        size_t work_bytes, void* stream)
{
    const char* fn = "mics_token_logprobs";
    static_assert(MICS_MAX_TOP == mics::kMostTop, "");
    Checked args(fn, rows, vocab);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.sizes("vocab"));
    if (top_k < 0 || top_k > MICS_MAX_TOP || (size_t)top_k > vocab)
        return fail(MICS_ERR_INVALID_ARG, "%s: top_k = %d not in [0, min(vocab, %d)]", fn, top_k, MICS_MAX_TOP);
    const size_t needed = mics_token_logprobs_workspace_bytes(rows, vocab, top_k);
    args.matrix("logits", logits, stride, width(dtype), false);
    args.vector("targets", targets, rows, 8, false);
    args.vector("logprob", logprob, rows, 4, true);
    args.vector("entropy", entropy, rows, 4, true, true);
    args.vector("lse", lse, rows, 4, true, true);
    args.vector("top_ids", top_k ? top_ids : nullptr, rows * top_k, 8, true);
    args.vector("top_logprobs", top_k ? top_logprobs : nullptr, rows * top_k, 4, true);
    if (needed) args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    if (rows == 0) return MICS_OK;
    const mics::LogProbs a{logprob, entropy, lse, top_ids, top_logprobs, {logits, stride}, targets, rows, (unsigned)vocab, top_k, work};
    const int err = mics::launch_logprobs(a, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

int mics_token_logprobs_backward(void* dlogits, const void* logits, const int64_t* targets, const float* lse,
                                 const float* entropy, const float* dlogprob, const float* dentropy, size_t rows, size_t vocab,
                                 const size_t* strides, int dtype, void* stream)
{
    const char* fn = "mics_token_logprobs_backward";
    Checked args(fn, rows, vocab);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.sizes("vocab"));
    const size_t e = width(dtype), d_stride = args.stride(strides, 0), x_stride = args.stride(strides, 1);
    args.matrix("dlogits", dlogits, d_stride, e, true);
    args.matrix("logits", logits, x_stride, e, false);
    args.vector("targets", targets, rows, 8, false);
    args.vector("lse", lse, rows, 4, false);
    args.vector("entropy", entropy, rows, 4, false, !dentropy);
    args.vector("dlogprob", dlogprob, rows, 4, false);
    args.vector("dentropy", dentropy, rows, 4, false, true);
    MICS_TRY(args.check());
    if (rows == 0) return MICS_OK;
    const mics::LogProbsBackward a{{dlogits, d_stride}, {logits, x_stride}, targets, lse, entropy, dlogprob, dentropy, rows,
                                   (unsigned)vocab};
    const int err = mics::launch_logprobs_backward(a, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

}  // extern "C"
