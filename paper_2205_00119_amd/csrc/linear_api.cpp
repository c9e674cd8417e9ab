// C ABI of the linear layer and of activations with 8-bit checkpoints: host-side argument validation and dispatch.  Every check
// runs before the first HIP call.
#include "../../include/mics.h"
#include "internal.h"
#include "layer_checks.h"
#include "linear_internal.h"

#include <algorithm>

namespace {

using mics::addr;
using mics::Checked;
using mics::column_sizes;
using mics::fail;
using mics::hip_fail;
using mics::width;
using mics::workspace;

static_assert(MICS_CHECKPOINT_BLOCK == mics::kBlockCols && MICS_ACT_SILU + 1 == mics::kActs
              && MICS_LINEAR_MOST_WORKSPACE == mics::kLinearWorkspace, "");

int activation(const char* fn, int act)
{
    return act >= 0 && act < mics::kActs ? MICS_OK : fail(MICS_ERR_UNSUPPORTED, "%s: act = %d is not one of MICS_ACT_*", fn, act);
}
int pair(const char* fn, const void* codes, const void* scales)
{
    return !codes == !scales ? MICS_OK : fail(MICS_ERR_INVALID_ARG, "%s: %s is NULL", fn, codes ? "scales" : "codes");
}
size_t blocks(size_t cols) { return mics::ceil_div(cols, mics::kBlockCols); }

// A plan's tiles are counted in 32 bits: more have no memory to lie in.
int countable(const char* fn, const mics::ProductPlan& p)
{
    return p.whole + p.shared * p.splits < (size_t{1} << 32) ? MICS_OK : fail(MICS_ERR_UNSUPPORTED, "%s: too many rows", fn);
}
// rows of in_features and of out_features
int features(const char* fn, size_t rows, size_t in, size_t out)
{
    MICS_TRY(Checked(fn, rows, in).sizes("in_features"));
    return Checked(fn, rows, out).sizes("out_features");
}
}  // namespace

extern "C" {

size_t mics_checkpoint_scales(size_t rows, size_t cols) { return column_sizes(rows, cols) ? rows * blocks(cols) : 0; }

int mics_activation(void* y, int8_t* codes, float* scales, const void* x, const void* bias, size_t rows, size_t cols,
                    const size_t* strides, int act, int dtype, int param_dtype, void* stream)
{
    const char* fn = "mics_activation";
    Checked args(fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("param_dtype", param_dtype));
    MICS_TRY(activation(fn, act));
    MICS_TRY(args.sizes("cols"));
    mics::ActivationPass a{};
    const size_t e = width(dtype);
    a.e.out = {y, args.stride(strides, 0)};
    a.e.codes = {codes, args.stride(strides, 1)};
    a.x = {x, args.stride(strides, 2)};
    MICS_TRY(pair(fn, codes, scales));
    if (!y && !codes && rows) return fail(MICS_ERR_INVALID_ARG, "%s: y and codes are NULL", fn);
    args.matrix("y", y, a.e.out.stride, e, true, true);
    args.matrix("codes", codes, a.e.codes.stride, 1, true, true);
    args.vector("scales", scales, mics_checkpoint_scales(rows, cols), 4, true, true);
    args.matrix("x", x, a.x.stride, e, false);
    args.vector("bias", bias, cols, width(param_dtype), false, true);
    MICS_TRY(args.check());
    if (rows == 0) return MICS_OK;
    a.e.scales = scales; a.e.bias = bias; a.e.act = act; a.e.param = param_dtype; a.e.out_kind = dtype;
    a.rows = rows; a.cols = (unsigned)cols;
    const int err = mics::launch_activation(a, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

int mics_checkpoint_read(void* y, const int8_t* codes, const float* scales, size_t rows, size_t cols, const size_t* strides, int act,
                         int dtype, void* stream)
{
    const char* fn = "mics_checkpoint_read";
    Checked args(fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(activation(fn, act));
    MICS_TRY(args.sizes("cols"));
    const mics::CheckpointRead a{{y, args.stride(strides, 0)}, {codes, args.stride(strides, 1)}, scales, rows, (unsigned)cols, act};
    args.matrix("y", y, a.y.stride, width(dtype), true);
    args.matrix("codes", codes, a.codes.stride, 1, false);
    args.vector("scales", scales, mics_checkpoint_scales(rows, cols), 4, false);
    MICS_TRY(args.check());
    if (rows == 0) return MICS_OK;
    const int err = mics::launch_checkpoint_read(a, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

int mics_activation_backward(void* dx, void* dbias, const void* dy, const void* z, const int8_t* codes, const float* scales, size_t rows,
                             size_t cols, const size_t* strides, int act, int dtype, int grad_dtype, void* work, size_t work_bytes,
                             void* stream)
{
    const char* fn = "mics_activation_backward";
    Checked args(fn, rows, cols);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("grad_dtype", grad_dtype));
    MICS_TRY(activation(fn, act));
    MICS_TRY(args.sizes("cols"));
    MICS_TRY(pair(fn, codes, scales));
    if (rows && !z && !codes) return fail(MICS_ERR_INVALID_ARG, "%s: z and codes are NULL", fn);
    if (z && codes) return fail(MICS_ERR_INVALID_ARG, "%s: z or codes has to be NULL", fn);
    if (rows && !dx && !dbias) return fail(MICS_ERR_INVALID_ARG, "%s: dx and dbias are NULL", fn);
    const size_t e = width(dtype), needed = dbias ? mics_column_workspace_bytes(rows, cols) : 0;
    mics::ActivationBackward a{};
    a.dx = {dx, args.stride(strides, 0)};
    a.dy = {dy, args.stride(strides, 1)};
    a.z = {z, args.stride(strides, 2)};
    a.codes = {codes, args.stride(strides, 3)};
    args.matrix("dx", dx, a.dx.stride, e, true, true);
    args.matrix("dy", dy, a.dy.stride, e, false);
    args.matrix("z", z, a.z.stride, e, false, true);
    args.matrix("codes", codes, a.codes.stride, 1, false, true);
    args.vector("scales", scales, mics_checkpoint_scales(rows, cols), 4, false, true);
    args.vector("dbias", dbias, cols, width(grad_dtype), true, true);
    if (needed) args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    if (!dbias && rows == 0) return MICS_OK;
    a.scales = scales; a.rows = rows; a.cols = (unsigned)cols; a.act = act; a.parts = (float*)work;
    const int err = mics::launch_activation_backward(a, dtype, dbias, grad_dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

size_t mics_linear_workspace_bytes(size_t rows, size_t in, size_t out)
{
    if (!column_sizes(rows, in) || !column_sizes(rows, out)) return 0;
    using mics::most_workspace;
    return std::max({most_workspace(rows, out, in, false, false), most_workspace(rows, in, out, false, true),
                     most_workspace(out, in, rows, true, true)});
}

int mics_linear(void* out, void* pre, int8_t* codes, float* scales, const void* x, const void* weight, const void* bias,
                const void* residual, size_t rows, size_t in, size_t outs, const size_t* strides, int act, int dtype, int param_dtype,
                void* work, size_t work_bytes, void* stream)
{
    const char* fn = "mics_linear";
    Checked args(fn, rows, outs);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("param_dtype", param_dtype));
    MICS_TRY(activation(fn, act));
    MICS_TRY(features(fn, rows, in, outs));
    MICS_TRY(pair(fn, codes, scales));
    const size_t e = width(dtype);
    mics::Product p{};
    p.m = rows; p.n = outs; p.k = in;
    p.e.out = {out, strides ? strides[0] : outs};
    p.e.pre = {pre, strides ? strides[1] : outs};
    p.e.codes = {codes, strides ? strides[2] : outs};
    p.a = {x, strides ? strides[3] : in};
    p.b = {weight, strides ? strides[4] : in};
    p.e.residual = {residual, strides ? strides[5] : outs};
    const mics::ProductPlan plan = mics::plan_of(p, e);
    const size_t needed = mics::workspace_of(plan);
    args.matrix("out", out, p.e.out.stride, e, true);
    args.matrix("pre", pre, p.e.pre.stride, e, true, true);
    args.matrix("codes", codes, p.e.codes.stride, 1, true, true);
    args.vector("scales", scales, mics_checkpoint_scales(rows, outs), 4, true, true);
    args.shaped("x", x, rows, in, p.a.stride, e, false, false, true);
    args.shaped("weight", weight, outs, in, p.b.stride, e, false, rows == 0, true);
    args.vector("bias", bias, outs, width(param_dtype), false, true);
    args.matrix("residual", residual, p.e.residual.stride, e, false, true);
    if (needed) args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    MICS_TRY(countable(fn, plan));
    if (rows == 0) return MICS_OK;
    p.e.scales = scales; p.e.bias = bias; p.e.act = act; p.e.param = param_dtype; p.e.out_kind = dtype;
    p.parts = (float*)work;
    const int err = mics::launch_product(p, plan, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

int mics_linear_backward_input(void* dx, const void* dz, const void* weight, const void* dsum, size_t rows, size_t in, size_t outs,
                               const size_t* strides, int dtype, void* work, size_t work_bytes, void* stream)
{
    const char* fn = "mics_linear_backward_input";
    Checked args(fn, rows, in);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(features(fn, rows, in, outs));
    const size_t e = width(dtype);
    mics::Product p{};
    p.m = rows; p.n = in; p.k = outs; p.b_turned = true;
    p.e.out = {dx, strides ? strides[0] : in};
    p.a = {dz, strides ? strides[1] : outs};
    p.b = {weight, strides ? strides[2] : in};
    p.e.residual = {dsum, strides ? strides[3] : in};
    const mics::ProductPlan plan = mics::plan_of(p, e);
    const size_t needed = mics::workspace_of(plan);
    args.matrix("dx", dx, p.e.out.stride, e, true);
    args.shaped("dz", dz, rows, outs, p.a.stride, e, false, false, true);
    args.shaped("weight", weight, outs, in, p.b.stride, e, false, rows == 0, true);
    args.matrix("dsum", dsum, p.e.residual.stride, e, false, true);
    if (needed) args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    MICS_TRY(countable(fn, plan));
    if (rows == 0) return MICS_OK;
    p.e.out_kind = dtype; p.parts = (float*)work;
    const int err = mics::launch_product(p, plan, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

int mics_linear_backward_weight(void* dweight, const void* dz, const void* x, size_t rows, size_t in, size_t outs, const size_t* strides,
                                int dtype, int grad_dtype, void* work, size_t work_bytes, void* stream)
{
    const char* fn = "mics_linear_backward_weight";
    Checked args(fn, outs, in);
    MICS_TRY(args.dtype("dtype", dtype));
    MICS_TRY(args.dtype("grad_dtype", grad_dtype));
    MICS_TRY(features(fn, rows, in, outs));
    const size_t e = width(dtype);
    mics::Product p{};
    p.m = outs; p.n = in; p.k = rows; p.a_turned = p.b_turned = true;
    p.e.out = {dweight, strides ? strides[0] : in};
    p.a = {dz, strides ? strides[1] : outs};
    p.b = {x, strides ? strides[2] : in};
    const mics::ProductPlan plan = mics::plan_of(p, e);
    const size_t needed = mics::workspace_of(plan);
    args.matrix("dweight", dweight, p.e.out.stride, width(grad_dtype), true);
    args.shaped("dz", dz, rows, outs, p.a.stride, e, false, false, true);
    args.shaped("x", x, rows, in, p.b.stride, e, false, false, true);
    if (needed) args.vector("workspace", work, needed, 1, true);
    MICS_TRY(workspace(fn, work, work_bytes, needed));
    MICS_TRY(args.check());
    p.e.out_kind = grad_dtype; p.parts = (float*)work;
    const int err = mics::launch_product(p, plan, dtype, stream);
    return err ? hip_fail(fn, err) : MICS_OK;
}

}  // extern "C"
