"""MI355X-native per-GPU data path of MiCS partitioned data parallelism.

Thin ctypes binding over ``libmics.so`` (see ``include/mics.h`` for the contract of each
call, ``include/mics_tuning.h`` for the three measurement knobs).  The functions here only marshal arguments -- device pointers, sizes and the
current HIP stream; every step of the path runs in the library's HIP kernels.  There is
no CPU fallback: if the library is missing, importing this package fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmics.so")

MICS_OK = 0
MICS_ERR_INVALID_ARG = -1
MICS_ERR_ALIGNMENT = -2
MICS_ERR_UNSUPPORTED = -3
MICS_ERR_HIP = -4
MICS_MAX_GROUP = 128

EXPORTS = (
    "mics_version", "mics_last_error", "mics_shard_elems", "mics_set_blocks_per_cu",
    "mics_set_stream_threshold_bytes", "mics_set_launch_shape",
    "mics_hier_gather_reorder", "mics_reduce_scatter_accum", "mics_replica_average",
    "mics_adam_shard", "mics_hier_gather_reorder_coalesced", "mics_reduce_scatter_accum_coalesced",
    "mics_replica_average_adam_shard", "mics_reduce_scatter_accum_typed",
    "mics_adam_shard_typed", "mics_replica_average_adam_shard_typed",
    "mics_reduce_scatter_accum_coalesced_typed",
    "mics_dropout_counters", "mics_column_workspace_bytes", "mics_token_logprobs_workspace_bytes",
    "mics_bias_dropout_add", "mics_bias_dropout_add_backward", "mics_layer_norm", "mics_layer_norm_backward",
    "mics_dropout_add_layer_norm", "mics_dropout_add_layer_norm_backward",
    "mics_token_logprobs", "mics_token_logprobs_backward",
    "mics_checkpoint_scales", "mics_linear_workspace_bytes", "mics_activation", "mics_checkpoint_read",
    "mics_activation_backward", "mics_linear", "mics_linear_backward_input", "mics_linear_backward_weight",
)
MICS_MAX_TOP = 64
MICS_CHECKPOINT_BLOCK = 64
MICS_LINEAR_MOST_WORKSPACE = 64 << 20
MICS_ACT_NONE, MICS_ACT_RELU, MICS_ACT_GELU, MICS_ACT_GELU_TANH, MICS_ACT_SILU = range(5)
MICS_DTYPE_BF16, MICS_DTYPE_F16, MICS_DTYPE_F32 = 0, 1, 2


class MicsError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libmics error {code}: {message}")
        self.code = code


MARSHAL_PATH = os.path.join(_HERE, "_marshal.so")
if not (os.path.exists(LIB_PATH) and os.path.exists(MARSHAL_PATH)):
    raise ImportError(
        f"{LIB_PATH} and {MARSHAL_PATH} are not both built. Run `python -c 'import __graft_entry__ as g; g.build()'` "
        "(or `python paper_2205_00119_amd/build.py`) first; there is no fallback path.")

# PyTorch ships its own HIP runtime (soname libamdhip64.so.7).  It must be in the process before
# libmics.so is opened, so that the library binds to that one runtime -- the one that owns the
# device memory and streams the caller passes in -- instead of loading a second copy.
import torch  # noqa: E402,F401
from . import _marshal  # noqa: E402

lib = ctypes.CDLL(LIB_PATH)

_vp, _sz, _i, _f = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
lib.mics_version.argtypes = []
lib.mics_version.restype = _i
lib.mics_last_error.argtypes = []
lib.mics_last_error.restype = ctypes.c_char_p
lib.mics_shard_elems.argtypes = [_sz, _i, _sz]
lib.mics_shard_elems.restype = _sz
lib.mics_set_blocks_per_cu.argtypes = [_i]
lib.mics_set_blocks_per_cu.restype = _i
lib.mics_set_stream_threshold_bytes.argtypes = [_sz]
lib.mics_set_stream_threshold_bytes.restype = _i
lib.mics_set_launch_shape.argtypes = [_i, _i, _i]
lib.mics_set_launch_shape.restype = _i
lib.mics_hier_gather_reorder.argtypes = [_vp, _vp, _sz, _sz, _i, _i, _i, _vp]
lib.mics_hier_gather_reorder.restype = _i
lib.mics_reduce_scatter_accum.argtypes = [_vp, _vp, _sz, _sz, _i, _i, _vp]
lib.mics_reduce_scatter_accum.restype = _i
lib.mics_replica_average.argtypes = [_vp, _vp, _sz, _i, _f, _vp]
lib.mics_replica_average.restype = _i
lib.mics_adam_shard.argtypes = [_vp, _vp, _vp, _vp, _vp, _sz, _f, _f, _f, _f, _f, _i, _vp]
lib.mics_adam_shard.restype = _i


class mics_segment(ctypes.Structure):
    """One separately sharded tensor of a coalesced call (offsets and sizes in elements)."""
    _fields_ = [("numel", ctypes.c_size_t), ("shard_elems", ctypes.c_size_t),
                ("src_offset", ctypes.c_size_t), ("dst_offset", ctypes.c_size_t)]


lib.mics_hier_gather_reorder_coalesced.argtypes = [_vp, _vp, ctypes.POINTER(mics_segment), _i, _i, _i,
                                                   _i, _vp]
lib.mics_hier_gather_reorder_coalesced.restype = _i
lib.mics_reduce_scatter_accum_coalesced.argtypes = [_vp, _vp, ctypes.POINTER(mics_segment), _i, _i, _i,
                                                    _vp]
lib.mics_reduce_scatter_accum_coalesced.restype = _i


lib.mics_replica_average_adam_shard.argtypes = [_vp, _vp, _vp, _vp, _vp, _sz, _i, _f, _f, _f, _f, _f, _f,
                                                _i, _vp]
lib.mics_replica_average_adam_shard.restype = _i


lib.mics_reduce_scatter_accum_coalesced_typed.argtypes = [_vp, _vp, ctypes.POINTER(mics_segment), _i, _i, _i, _i,
                                                          _vp]
lib.mics_reduce_scatter_accum_coalesced_typed.restype = _i
lib.mics_adam_shard_typed.argtypes = [_vp, _vp, _vp, _vp, _i, _vp, _sz, _f, _f, _f, _f, _f, _i, _vp]
lib.mics_adam_shard_typed.restype = _i
lib.mics_replica_average_adam_shard_typed.argtypes = [_vp, _vp, _vp, _vp, _i, _vp, _sz, _i, _f, _f, _f, _f, _f,
                                                      _f, _i, _vp]
lib.mics_replica_average_adam_shard_typed.restype = _i
lib.mics_reduce_scatter_accum_typed.argtypes = [_vp, _vp, _sz, _sz, _i, _i, _i, _vp]
lib.mics_reduce_scatter_accum_typed.restype = _i


_u64 = ctypes.c_uint64
lib.mics_dropout_counters.argtypes = [_sz, _sz]
lib.mics_dropout_counters.restype = _u64
lib.mics_column_workspace_bytes.argtypes = [_sz, _sz]
lib.mics_column_workspace_bytes.restype = _sz
lib.mics_token_logprobs_workspace_bytes.argtypes = [_sz, _sz, _i]
lib.mics_token_logprobs_workspace_bytes.restype = _sz
lib.mics_bias_dropout_add.argtypes = [_vp] * 4 + [_sz, _sz, _vp, _f, _u64, _u64, _i, _i, _vp]
lib.mics_bias_dropout_add_backward.argtypes = [_vp] * 3 + [_sz, _sz, _vp, _f, _u64, _u64, _i, _i, _vp, _sz, _vp]
lib.mics_layer_norm.argtypes = [_vp] * 6 + [_sz, _sz, _vp, _f, _i, _i, _vp]
lib.mics_layer_norm_backward.argtypes = [_vp] * 8 + [_sz, _sz, _vp, _i, _i, _i, _vp, _sz, _vp]
lib.mics_dropout_add_layer_norm.argtypes = [_vp] * 9 + [_sz, _sz, _vp, _f, _u64, _u64, _f, _i, _i, _vp]
lib.mics_dropout_add_layer_norm_backward.argtypes = [_vp] * 11 + [_sz, _sz, _vp, _f, _u64, _u64, _i, _i, _i, _vp, _sz, _vp]
lib.mics_token_logprobs.argtypes = [_vp] * 7 + [_sz, _sz, _sz, _i, _i, _vp, _sz, _vp]
lib.mics_token_logprobs_backward.argtypes = [_vp] * 7 + [_sz, _sz, _vp, _i, _vp]
_LAYER_CALLS = ("bias_dropout_add", "bias_dropout_add_backward", "layer_norm", "layer_norm_backward", "dropout_add_layer_norm",
                "dropout_add_layer_norm_backward", "token_logprobs", "token_logprobs_backward")
lib.mics_checkpoint_scales.argtypes = [_sz, _sz]
lib.mics_checkpoint_scales.restype = _sz
lib.mics_linear_workspace_bytes.argtypes = [_sz, _sz, _sz]
lib.mics_linear_workspace_bytes.restype = _sz
lib.mics_activation.argtypes = [_vp] * 5 + [_sz, _sz, _vp, _i, _i, _i, _vp]
lib.mics_checkpoint_read.argtypes = [_vp] * 3 + [_sz, _sz, _vp, _i, _i, _vp]
lib.mics_activation_backward.argtypes = [_vp] * 6 + [_sz, _sz, _vp, _i, _i, _i, _vp, _sz, _vp]
lib.mics_linear.argtypes = [_vp] * 8 + [_sz, _sz, _sz, _vp, _i, _i, _i, _vp, _sz, _vp]
lib.mics_linear_backward_input.argtypes = [_vp] * 4 + [_sz, _sz, _sz, _vp, _i, _vp, _sz, _vp]
lib.mics_linear_backward_weight.argtypes = [_vp] * 3 + [_sz, _sz, _sz, _vp, _i, _i, _vp, _sz, _vp]
_LINEAR_CALLS = ("activation", "checkpoint_read", "activation_backward", "linear", "linear_backward_input", "linear_backward_weight")
for _name in _LAYER_CALLS + _LINEAR_CALLS:
    getattr(lib, "mics_" + _name).restype = _i


def _segments(segs) -> ctypes.Array:
    """(numel, shard_elems, src_offset, dst_offset) tuples -> C array of mics_segment."""
    arr = (mics_segment * len(segs))()
    _marshal.segments(arr, segs)
    return arr


def _check(rc: int) -> None:
    if rc != MICS_OK:
        raise MicsError(rc, lib.mics_last_error().decode("utf-8", "replace"))


# Device address of a torch tensor (must be contiguous, else ValueError), or a raw integer address.
_dev_ptr = _marshal.address


def _table(items: Sequence) -> ctypes.Array:
    arr = (ctypes.c_void_p * len(items))()
    _marshal.addresses(arr, items)
    return arr


# The raw handle of torch's current stream, without the Stream object around it.
_raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device


def _stream(stream) -> Optional[int]:
    """hipStream_t handle: explicit integer, a torch stream, or torch's current stream."""
    if stream is None:
        return _raw_stream(_device()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


# Whole calls with plain arguments go past ctypes (csrc/marshal.cpp); what these functions answer with None, and the
# message of an error, goes through it.
_marshal.bind(tuple(ctypes.cast(getattr(lib, "mics_" + name), _vp).value for name in (
    "hier_gather_reorder", "hier_gather_reorder_coalesced", "reduce_scatter_accum", "reduce_scatter_accum_typed",
    "reduce_scatter_accum_coalesced", "reduce_scatter_accum_coalesced_typed", "replica_average", "adam_shard",
    "adam_shard_typed", "replica_average_adam_shard", "replica_average_adam_shard_typed")),
    _device, _raw_stream)
_marshal.bind_layer(tuple(ctypes.cast(getattr(lib, "mics_" + name), _vp).value for name in _LAYER_CALLS))
_marshal.bind_linear(tuple(ctypes.cast(getattr(lib, "mics_" + name), _vp).value for name in _LINEAR_CALLS))
_marshal.bind_segment(mics_segment)


def _done(rc) -> bool:
    """True after a call that went past ctypes; raises its error."""
    if rc is None:
        return False
    if rc:
        _check(rc)
    return True


def mics_version() -> int:
    return lib.mics_version()


def mics_last_error() -> str:
    return lib.mics_last_error().decode("utf-8", "replace")


def mics_shard_elems(n: int, p: int, align_elems: int = 8) -> int:
    return lib.mics_shard_elems(n, p, align_elems)


def mics_set_blocks_per_cu(blocks_per_cu: int) -> None:
    _check(lib.mics_set_blocks_per_cu(blocks_per_cu))


def mics_set_stream_threshold_bytes(nbytes: int) -> None:
    _check(lib.mics_set_stream_threshold_bytes(nbytes))


MICS_KERNELS_REORDER, MICS_KERNELS_REDUCE, MICS_KERNELS_AVERAGE, MICS_KERNELS_ADAM, MICS_KERNELS_FUSED = range(5)


def mics_set_launch_shape(kernel_family: int, lanes: int = 0, waves_per_cu: int = 0) -> None:
    _check(lib.mics_set_launch_shape(kernel_family, lanes, waves_per_cu))


def mics_hier_gather_reorder(dst_flat, stage1_bufs: Sequence, n_valid: int, shard_elems: int,
                             p: int, k: int, elem_bytes: int, stream=None) -> None:
    """Stage-1 buffers of the hierarchical all-gather -> contiguous flat parameter."""
    if _done(_marshal.gather(dst_flat, stage1_bufs, n_valid, shard_elems, p, k, elem_bytes, stream)):
        return
    if len(stage1_bufs) != k:
        raise ValueError(f"expected k = {k} stage-1 buffers, got {len(stage1_bufs)}")
    _check(lib.mics_hier_gather_reorder(_dev_ptr(dst_flat), _table(stage1_bufs), n_valid,
                                        shard_elems, p, k, elem_bytes, _stream(stream)))


def mics_reduce_scatter_accum(acc, grads_bf16: Sequence, elem_offset: int, count: int,
                              accumulate: bool, stream=None) -> None:
    """acc[0:count] (+)= sum over the p rank buffers of elements [elem_offset, +count)."""
    if _done(_marshal.reduce(acc, grads_bf16, elem_offset, count, accumulate, stream)):
        return
    _check(lib.mics_reduce_scatter_accum(_dev_ptr(acc), _table(grads_bf16), elem_offset, count,
                                         len(grads_bf16), int(bool(accumulate)), _stream(stream)))


def mics_replica_average(out, acc_copies: Sequence, count: int, scale: float, stream=None) -> None:
    """out = (sum over the r replica copies) * scale."""
    if _done(_marshal.average(out, acc_copies, count, scale, stream)):
        return
    _check(lib.mics_replica_average(_dev_ptr(out), _table(acc_copies), count, len(acc_copies),
                                    scale, _stream(stream)))


def mics_adam_shard(master, exp_avg, exp_avg_sq, param_bf16, grad, count: int, *, lr: float,
                    beta1: float, beta2: float, eps: float, weight_decay: float, step: int,
                    stream=None) -> None:
    """Mixed-precision Adam step in place on the fp32 shard; writes the bf16 parameter."""
    if _done(_marshal.adam(master, exp_avg, exp_avg_sq, param_bf16, grad, count, lr, beta1, beta2, eps, weight_decay, step, stream)):
        return
    _check(lib.mics_adam_shard(_dev_ptr(master), _dev_ptr(exp_avg), _dev_ptr(exp_avg_sq),
                               _dev_ptr(param_bf16), _dev_ptr(grad), count, lr, beta1, beta2, eps,
                               weight_decay, step, _stream(stream)))


def mics_hier_gather_reorder_coalesced(dst_flat, stage1_bufs: Sequence, segs, p: int, k: int,
                                       elem_bytes: int, stream=None) -> None:
    """The gather reorder for many separately sharded tensors in one call; ``segs`` holds
    (numel, shard_elems, src_offset, dst_offset) per tensor."""
    if _done(_marshal.gather_coalesced(dst_flat, stage1_bufs, segs, p, k, elem_bytes, stream)):
        return
    if len(stage1_bufs) != k:
        raise ValueError(f"expected k = {k} stage-1 buffers, got {len(stage1_bufs)}")
    arr = segs if isinstance(segs, ctypes.Array) else _segments(segs)
    _check(lib.mics_hier_gather_reorder_coalesced(_dev_ptr(dst_flat), _table(stage1_bufs), arr, len(arr),
                                                  p, k, elem_bytes, _stream(stream)))


def mics_reduce_scatter_accum_coalesced(acc, grads_bf16: Sequence, segs, accumulate: bool,
                                        stream=None) -> None:
    """Reduce-scatter-accumulate for many tensors in one call; ``segs`` holds
    (count, 0, src_offset, dst_offset) per tensor."""
    if _done(_marshal.reduce_coalesced(acc, grads_bf16, segs, accumulate, stream)):
        return
    arr = segs if isinstance(segs, ctypes.Array) else _segments(segs)
    _check(lib.mics_reduce_scatter_accum_coalesced(_dev_ptr(acc), _table(grads_bf16), arr, len(arr),
                                                   len(grads_bf16), int(bool(accumulate)),
                                                   _stream(stream)))


def mics_replica_average_adam_shard(master, exp_avg, exp_avg_sq, param_bf16, acc_copies: Sequence,
                                    count: int, scale: float, *, lr: float, beta1: float, beta2: float,
                                    eps: float, weight_decay: float, step: int, stream=None) -> None:
    """Replica average and Adam step in one pass; same results as the two separate calls."""
    if _done(_marshal.update(master, exp_avg, exp_avg_sq, param_bf16, acc_copies, count, scale, lr, beta1, beta2, eps, weight_decay,
                             step, stream)):
        return
    _check(lib.mics_replica_average_adam_shard(
        _dev_ptr(master), _dev_ptr(exp_avg), _dev_ptr(exp_avg_sq), _dev_ptr(param_bf16),
        _table(acc_copies), count, len(acc_copies), scale, lr, beta1, beta2, eps, weight_decay, step,
        _stream(stream)))


def mics_reduce_scatter_accum_coalesced_typed(acc, grads: Sequence, segs, accumulate: bool, grad_dtype: int,
                                              stream=None) -> None:
    """mics_reduce_scatter_accum_coalesced for bf16 / fp16 / fp32 gradient buffers (MICS_DTYPE_*)."""
    if _done(_marshal.reduce_coalesced_typed(acc, grads, segs, accumulate, grad_dtype, stream)):
        return
    arr = segs if isinstance(segs, ctypes.Array) else _segments(segs)
    _check(lib.mics_reduce_scatter_accum_coalesced_typed(_dev_ptr(acc), _table(grads), arr, len(arr), len(grads),
                                                         int(bool(accumulate)), grad_dtype, _stream(stream)))


def mics_adam_shard_typed(master, exp_avg, exp_avg_sq, param_out, param_dtype: int, grad, count: int, *,
                          lr: float, beta1: float, beta2: float, eps: float, weight_decay: float, step: int,
                          stream=None) -> None:
    """mics_adam_shard writing the 16-bit parameter as bf16 or binary16 (MICS_DTYPE_*)."""
    if _done(_marshal.adam_typed(master, exp_avg, exp_avg_sq, param_out, param_dtype, grad, count, lr, beta1, beta2, eps, weight_decay,
                                 step, stream)):
        return
    _check(lib.mics_adam_shard_typed(_dev_ptr(master), _dev_ptr(exp_avg), _dev_ptr(exp_avg_sq),
                                     _dev_ptr(param_out), param_dtype, _dev_ptr(grad), count, lr, beta1, beta2,
                                     eps, weight_decay, step, _stream(stream)))


def mics_replica_average_adam_shard_typed(master, exp_avg, exp_avg_sq, param_out, param_dtype: int,
                                          acc_copies: Sequence, count: int, scale: float, *, lr: float,
                                          beta1: float, beta2: float, eps: float, weight_decay: float,
                                          step: int, stream=None) -> None:
    """mics_replica_average_adam_shard writing the 16-bit parameter as bf16 or binary16."""
    if _done(_marshal.update_typed(master, exp_avg, exp_avg_sq, param_out, param_dtype, acc_copies, count, scale, lr, beta1, beta2, eps,
                                   weight_decay, step, stream)):
        return
    _check(lib.mics_replica_average_adam_shard_typed(
        _dev_ptr(master), _dev_ptr(exp_avg), _dev_ptr(exp_avg_sq), _dev_ptr(param_out), param_dtype,
        _table(acc_copies), count, len(acc_copies), scale, lr, beta1, beta2, eps, weight_decay, step,
        _stream(stream)))


def mics_reduce_scatter_accum_typed(acc, grads: Sequence, elem_offset: int, count: int,
                                    accumulate: bool, grad_dtype: int, stream=None) -> None:
    """mics_reduce_scatter_accum for bf16 / fp16 / fp32 gradient buffers (MICS_DTYPE_*)."""
    if _done(_marshal.reduce_typed(acc, grads, elem_offset, count, accumulate, grad_dtype, stream)):
        return
    _check(lib.mics_reduce_scatter_accum_typed(_dev_ptr(acc), _table(grads), elem_offset, count,
                                               len(grads), int(bool(accumulate)), grad_dtype,
                                               _stream(stream)))


# The operators between the parameter gather and the gradient reduction.  A matrix is a packed tensor, a tensor of two
# dimensions whose rows are as far apart as `strides` says, or an address; `strides` holds the row strides in elements of
# the matrices in the order in which the call takes them, None: all are packed.

def _strides(strides, n: int):
    if strides is None:
        return None
    if len(strides) != n:
        raise ValueError(f"expected {n} row strides, got {len(strides)}")
    return (ctypes.c_size_t * n)(*[int(x) for x in strides])


def _matrix(x, strides, k: int = 0):
    if strides is not None and isinstance(x, torch.Tensor) and x.dim() == 2 and x.stride(1) == 1 and x.stride(0) == strides[k]:
        return x.data_ptr()
    return _dev_ptr(x)


def mics_dropout_counters(rows: int, cols: int) -> int:
    """Counters that a dropout call uses: how far apart the offsets of calls with one seed have to be."""
    return lib.mics_dropout_counters(rows, cols)


def mics_column_workspace_bytes(rows: int, cols: int) -> int:
    """Workspace of the backward passes that sum over rows."""
    return lib.mics_column_workspace_bytes(rows, cols)


def mics_token_logprobs_workspace_bytes(rows: int, vocab: int, top_k: int = 0) -> int:
    return lib.mics_token_logprobs_workspace_bytes(rows, vocab, top_k)


def mics_bias_dropout_add(out, x, bias, residual, rows: int, cols: int, *, drop: float, seed: int, offset: int, dtype: int,
                          param_dtype: int, strides=None, stream=None) -> None:
    """out = residual + D(x + bias); strides: out, x, residual."""
    if _done(_marshal.bias_dropout_add(out, x, bias, residual, rows, cols, strides, drop, seed, offset, dtype, param_dtype, stream)):
        return
    st = _strides(strides, 3)
    _check(lib.mics_bias_dropout_add(_matrix(out, st, 0), _matrix(x, st, 1), _dev_ptr(bias), _matrix(residual, st, 2), rows, cols, st,
                                     drop, seed, offset, dtype, param_dtype, _stream(stream)))


def mics_bias_dropout_add_backward(dx, dbias, dout, rows: int, cols: int, *, drop: float, seed: int, offset: int, dtype: int,
                                   grad_dtype: int, workspace=None, workspace_bytes: int = 0, strides=None, stream=None) -> None:
    """dx = D(dout) and its column sums; strides: dx, dout."""
    if _done(_marshal.bias_dropout_add_backward(dx, dbias, dout, rows, cols, strides, drop, seed, offset, dtype, grad_dtype, workspace,
                                                workspace_bytes, stream)):
        return
    st = _strides(strides, 2)
    _check(lib.mics_bias_dropout_add_backward(_matrix(dx, st, 0), _dev_ptr(dbias), _matrix(dout, st, 1), rows, cols, st, drop, seed,
                                              offset, dtype, grad_dtype, _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def mics_layer_norm(y, mean, rstd, x, weight, bias, rows: int, cols: int, *, eps: float, dtype: int, param_dtype: int,
                    strides=None, stream=None) -> None:
    """Layer norm of every row; mean and rstd for the backward pass.  strides: y, x."""
    if _done(_marshal.layer_norm(y, mean, rstd, x, weight, bias, rows, cols, strides, eps, dtype, param_dtype, stream)):
        return
    st = _strides(strides, 2)
    _check(lib.mics_layer_norm(_matrix(y, st, 0), _dev_ptr(mean), _dev_ptr(rstd), _matrix(x, st, 1), _dev_ptr(weight), _dev_ptr(bias),
                               rows, cols, st, eps, dtype, param_dtype, _stream(stream)))


def mics_layer_norm_backward(dx, dweight, dbias, dy, x, mean, rstd, weight, rows: int, cols: int, *, dtype: int, param_dtype: int,
                             grad_dtype: int, workspace, workspace_bytes: int, strides=None, stream=None) -> None:
    """Gradients of rows, weight and bias; strides: dx, dy, x."""
    if _done(_marshal.layer_norm_backward(dx, dweight, dbias, dy, x, mean, rstd, weight, rows, cols, strides, dtype, param_dtype,
                                          grad_dtype, workspace, workspace_bytes, stream)):
        return
    st = _strides(strides, 3)
    _check(lib.mics_layer_norm_backward(_matrix(dx, st, 0), _dev_ptr(dweight), _dev_ptr(dbias), _matrix(dy, st, 1), _matrix(x, st, 2),
                                        _dev_ptr(mean), _dev_ptr(rstd), _dev_ptr(weight), rows, cols, st, dtype, param_dtype,
                                        grad_dtype, _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def mics_dropout_add_layer_norm(y, sum, mean, rstd, x, bias, residual, weight, norm_bias, rows: int, cols: int, *, drop: float,
                                seed: int, offset: int, eps: float, dtype: int, param_dtype: int, strides=None,
                                stream=None) -> None:
    """sum = residual + D(x + bias) and its layer norm in one pass; strides: y, sum, x, residual."""
    if _done(_marshal.dropout_add_layer_norm(y, sum, mean, rstd, x, bias, residual, weight, norm_bias, rows, cols, strides, drop, seed,
                                             offset, eps, dtype, param_dtype, stream)):
        return
    st = _strides(strides, 4)
    _check(lib.mics_dropout_add_layer_norm(
        _matrix(y, st, 0), _matrix(sum, st, 1), _dev_ptr(mean), _dev_ptr(rstd), _matrix(x, st, 2), _dev_ptr(bias),
        _matrix(residual, st, 3), _dev_ptr(weight), _dev_ptr(norm_bias), rows, cols, st, drop, seed, offset, eps, dtype, param_dtype,
        _stream(stream)))


def mics_dropout_add_layer_norm_backward(dx, dresidual, dbias, dweight, dnorm_bias, dy, dsum, sum, mean, rstd, weight, rows: int,
                                         cols: int, *, drop: float, seed: int, offset: int, dtype: int, param_dtype: int,
                                         grad_dtype: int, workspace, workspace_bytes: int, strides=None, stream=None) -> None:
    """Its gradients; strides: dx, dresidual, dy, dsum, sum."""
    if _done(_marshal.dropout_add_layer_norm_backward(
            dx, dresidual, dbias, dweight, dnorm_bias, dy, dsum, sum, mean, rstd, weight, rows, cols, strides, drop, seed, offset,
            dtype, param_dtype, grad_dtype, workspace, workspace_bytes, stream)):
        return
    st = _strides(strides, 5)
    _check(lib.mics_dropout_add_layer_norm_backward(
        _matrix(dx, st, 0), _matrix(dresidual, st, 1), _dev_ptr(dbias), _dev_ptr(dweight), _dev_ptr(dnorm_bias), _matrix(dy, st, 2),
        _matrix(dsum, st, 3), _matrix(sum, st, 4), _dev_ptr(mean), _dev_ptr(rstd), _dev_ptr(weight), rows, cols, st, drop, seed,
        offset, dtype, param_dtype, grad_dtype, _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def mics_token_logprobs(logprob, entropy, lse, top_ids, top_logprobs, logits, targets, rows: int, vocab: int, *, dtype: int,
                        top_k: int = 0, stride: Optional[int] = None, workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """Log probability of each row's target, entropy, log-sum-exp and the top_k best; stride: of the rows of logits."""
    if stride is None:
        stride = vocab
    if _done(_marshal.token_logprobs(logprob, entropy, lse, top_ids, top_logprobs, logits, targets, rows, vocab, stride, top_k, dtype,
                                     workspace, workspace_bytes, stream)):
        return
    _check(lib.mics_token_logprobs(_dev_ptr(logprob), _dev_ptr(entropy), _dev_ptr(lse), _dev_ptr(top_ids), _dev_ptr(top_logprobs),
                                   _matrix(logits, (stride,)), _dev_ptr(targets), rows, vocab, stride, top_k, dtype,
                                   _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def mics_token_logprobs_backward(dlogits, logits, targets, lse, entropy, dlogprob, dentropy, rows: int, vocab: int, *, dtype: int,
                                 strides=None, stream=None) -> None:
    """Gradient of the logits from those of logprob and entropy; strides: dlogits, logits."""
    if _done(_marshal.token_logprobs_backward(dlogits, logits, targets, lse, entropy, dlogprob, dentropy, rows, vocab, strides, dtype,
                                              stream)):
        return
    st = _strides(strides, 2)
    _check(lib.mics_token_logprobs_backward(_matrix(dlogits, st, 0), _matrix(logits, st, 1), _dev_ptr(targets), _dev_ptr(lse),
                                            _dev_ptr(entropy), _dev_ptr(dlogprob), _dev_ptr(dentropy), rows, vocab, st, dtype,
                                            _stream(stream)))


# The linear layer and activations with their 8-bit checkpoints; codes are int8 tensors, scales packed float32.

def mics_checkpoint_scales(rows: int, cols: int) -> int:
    """Scales of a checkpoint: one for every 64 columns of a row."""
    return lib.mics_checkpoint_scales(rows, cols)


def mics_linear_workspace_bytes(rows: int, in_features: int, out_features: int) -> int:
    """Workspace of the linear layer and of the gradients of its input and weight, at most 64 MiB."""
    return lib.mics_linear_workspace_bytes(rows, in_features, out_features)


def mics_activation(y, codes, scales, x, bias, rows: int, cols: int, *, act: int, dtype: int, param_dtype: int, strides=None,
                    stream=None) -> None:
    """y = act(x + bias) and the 8-bit checkpoint of x + bias; strides: y, codes, x."""
    if _done(_marshal.activation(y, codes, scales, x, bias, rows, cols, strides, act, dtype, param_dtype, stream)):
        return
    st = _strides(strides, 3)
    _check(lib.mics_activation(_matrix(y, st, 0), _matrix(codes, st, 1), _dev_ptr(scales), _matrix(x, st, 2), _dev_ptr(bias), rows, cols,
                               st, act, dtype, param_dtype, _stream(stream)))


def mics_checkpoint_read(y, codes, scales, rows: int, cols: int, *, act: int, dtype: int, strides=None, stream=None) -> None:
    """y = act(what the checkpoint stands for); strides: y, codes."""
    if _done(_marshal.checkpoint_read(y, codes, scales, rows, cols, strides, act, dtype, stream)):
        return
    st = _strides(strides, 2)
    _check(lib.mics_checkpoint_read(_matrix(y, st, 0), _matrix(codes, st, 1), _dev_ptr(scales), rows, cols, st, act, dtype,
                                    _stream(stream)))


def mics_activation_backward(dx, dbias, dy, z, codes, scales, rows: int, cols: int, *, act: int, dtype: int, grad_dtype: int,
                             workspace=None, workspace_bytes: int = 0, strides=None, stream=None) -> None:
    """dx = dy * act'(z) and its column sums, z a matrix or a checkpoint; strides: dx, dy, z, codes."""
    if _done(_marshal.activation_backward(dx, dbias, dy, z, codes, scales, rows, cols, strides, act, dtype, grad_dtype, workspace,
                                          workspace_bytes, stream)):
        return
    st = _strides(strides, 4)
    _check(lib.mics_activation_backward(_matrix(dx, st, 0), _dev_ptr(dbias), _matrix(dy, st, 1), _matrix(z, st, 2), _matrix(codes, st, 3),
                                        _dev_ptr(scales), rows, cols, st, act, dtype, grad_dtype, _dev_ptr(workspace), workspace_bytes,
                                        _stream(stream)))


def mics_linear(out, pre, codes, scales, x, weight, bias, residual, rows: int, in_features: int, out_features: int, *, act: int,
                dtype: int, param_dtype: int, workspace=None, workspace_bytes: int = 0, strides=None, stream=None) -> None:
    """out = residual + act(z), z = x weight^T + bias, and z as `pre` or as a checkpoint; strides: out, pre, codes, x, weight,
    residual."""
    if _done(_marshal.linear(out, pre, codes, scales, x, weight, bias, residual, rows, in_features, out_features, strides, act, dtype,
                             param_dtype, workspace, workspace_bytes, stream)):
        return
    st = _strides(strides, 6)
    _check(lib.mics_linear(_matrix(out, st, 0), _matrix(pre, st, 1), _matrix(codes, st, 2), _dev_ptr(scales), _matrix(x, st, 3),
                           _matrix(weight, st, 4), _dev_ptr(bias), _matrix(residual, st, 5), rows, in_features, out_features, st, act,
                           dtype, param_dtype, _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def mics_linear_backward_input(dx, dz, weight, dsum, rows: int, in_features: int, out_features: int, *, dtype: int, workspace=None,
                               workspace_bytes: int = 0, strides=None, stream=None) -> None:
    """dx = dz weight + dsum; strides: dx, dz, weight, dsum."""
    if _done(_marshal.linear_backward_input(dx, dz, weight, dsum, rows, in_features, out_features, strides, dtype, workspace,
                                            workspace_bytes, stream)):
        return
    st = _strides(strides, 4)
    _check(lib.mics_linear_backward_input(_matrix(dx, st, 0), _matrix(dz, st, 1), _matrix(weight, st, 2), _matrix(dsum, st, 3), rows,
                                          in_features, out_features, st, dtype, _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def mics_linear_backward_weight(dweight, dz, x, rows: int, in_features: int, out_features: int, *, dtype: int, grad_dtype: int,
                                workspace=None, workspace_bytes: int = 0, strides=None, stream=None) -> None:
    """dweight = dz^T x; strides: dweight, dz, x."""
    if _done(_marshal.linear_backward_weight(dweight, dz, x, rows, in_features, out_features, strides, dtype, grad_dtype, workspace,
                                             workspace_bytes, stream)):
        return
    st = _strides(strides, 3)
    _check(lib.mics_linear_backward_weight(_matrix(dweight, st, 0), _matrix(dz, st, 1), _matrix(x, st, 2), rows, in_features,
                                           out_features, st, dtype, grad_dtype, _dev_ptr(workspace), workspace_bytes, _stream(stream)))
