"""Calls with so many rows that every workgroup takes several of them, with a last batch that is one in part."""
import numpy as np
import pytest
import torch

import layer_ref as ref
from test_gpu_layer_ops import CODE, Matrix, get, intact, normal, scratch, vector

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
# rows, columns, padding, off the start, type: one wavefront a row (with three rows in registers), one with two vectors in each
# lane, several wavefronts, a whole workgroup, rows in tiles
SIZES = [(27001, 5, 0, 0, "f32"), (26003, 64, 3, 1, "bf16"), (20501, 509, 0, 0, "f16"), (20497, 512, 0, 0, "bf16"), (13007, 600, 0, 0, "bf16"),
         (12999, 1003, 5, 1, "f32"), (5003, 2100, 0, 0, "bf16"), (4999, 2101, 0, 1, "f16"), (1600, 5120, 8, 0, "bf16"), (600, 8187, 0, 0, "f32"),
         (700, 9001, 0, 1, "bf16"), (600, 16384, 0, 0, "bf16"), (530, 16380, 0, 0, "f16"), (30, 16401, 3, 0, "f32")]


def filled(rows, cols, pad, skew, fmt, seed, sigma=1.0, mean=0.0):
    return Matrix(rows, cols, fmt, pad, skew, normal(seed, rows, cols, sigma, mean))


@pytest.mark.parametrize("rows,cols,pad,skew,fmt", SIZES)
def test_layer_norm(rows, cols, pad, skew, fmt):
    st = (cols + pad,) * 3
    x, y = filled(rows, cols, pad, skew, fmt, 1, 2.0, 0.5), Matrix(rows, cols, fmt, pad, skew)
    w, b = vector(cols, "f32", normal(2, 1, cols, 0.2, 1.0)), vector(cols, "f32", normal(3, 1, cols, 0.2))
    mean, rstd = vector(rows, "f32"), vector(rows, "f32")
    mics.mics_layer_norm(y.t, mean.v, rstd.v, x.t, w.v, b.v, rows, cols, eps=1e-5, dtype=CODE[fmt], param_dtype=2, strides=st[:2])
    x64 = x.f64()
    (ry, sy), (rm, sm), (rr, sr) = ref.layer_norm(x64, np.abs(x64), get(w), get(b), 1e-5)
    assert ref.within(y.f64(), ry, sy, fmt) and ref.within(get(mean), rm, sm, "f32") and ref.within(get(rstd), rr, sr, "f32")
    assert intact(y, mean, rstd)
    dy, dx = filled(rows, cols, pad, skew, fmt, 4, 0.3), Matrix(rows, cols, fmt, pad, skew)
    dw, db = vector(cols, "f32"), vector(cols, "f32")
    ws, n = scratch(rows, cols)
    mics.mics_layer_norm_backward(dx.t, dw.v, db.v, dy.t, x.t, mean.v, rstd.v, w.v, rows, cols, dtype=CODE[fmt], param_dtype=2, grad_dtype=2,
                                  workspace=ws, workspace_bytes=n, strides=st)
    want = ref.layer_norm_backward(dy.f64(), x64, get(mean), get(rstd), get(w))
    assert ref.within(dx.f64(), *want[0], fmt) and ref.within(get(dw), *want[1], "f32") and ref.within(get(db), *want[2], "f32")
    assert intact(dx, dw, db) and bool((ws[n:] == 0x5A).all())


@pytest.mark.parametrize("rows,cols,pad,skew,fmt", SIZES)
@pytest.mark.parametrize("has_sum", [True, False])
def test_block(rows, cols, pad, skew, fmt, has_sum):
    mk = lambda *a: filled(rows, cols, pad, skew, fmt, *a)                             # noqa: E731
    out = lambda: Matrix(rows, cols, fmt, pad, skew)                                   # noqa: E731
    key, st, types = dict(drop=0.2, seed=77, offset=2 ** 40 - 5), (cols + pad,) * 5, dict(dtype=CODE[fmt], param_dtype=2)
    x, res, y, s, mean, rstd = mk(1), mk(2, 2.0, 0.2), out(), out(), vector(rows, "f32"), vector(rows, "f32")
    bias, w, b = (vector(cols, "f32", normal(k, 1, cols, 0.2, m)) for k, m in ((3, 0.0), (4, 1.0), (5, 0.0)))
    mics.mics_dropout_add_layer_norm(y.t, s.t, mean.v, rstd.v, x.t, bias.v, res.t, w.v, b.v, rows, cols, eps=1e-5, strides=st[:4], **key, **types)
    rs, ss = ref.bias_dropout_add(x.f64(), get(bias), res.f64(), *key.values())
    (ry, sy), (rm, sm), (rr, sr) = ref.layer_norm(rs, ss, get(w), get(b), 1e-5)
    assert ref.within(s.f64(), rs, ss, fmt) and ref.within(y.f64(), ry, sy, fmt)
    assert ref.within(get(mean), rm, sm, "f32") and ref.within(get(rstd), rr, sr, "f32") and intact(y, s, mean, rstd)
    dy, dsum, dx, dres = mk(6, 0.3), mk(7, 0.3) if has_sum else None, out(), out()
    grads = [vector(cols, "f32") for _ in range(3)]
    ws, n = scratch(rows, cols)
    mics.mics_dropout_add_layer_norm_backward(dx.t, dres.t, *[g.v for g in grads], dy.t, dsum.t if has_sum else None, s.t, mean.v, rstd.v, w.v,
                                              rows, cols, grad_dtype=2, workspace=ws, workspace_bytes=n, strides=st, **key, **types)
    want = ref.block_backward(dy.f64(), dsum.f64() if has_sum else None, s.f64(), get(mean), get(rstd), get(w), *key.values())
    assert ref.within(dx.f64(), *want[0], fmt) and ref.within(dres.f64(), *want[1], fmt)
    for g, v in zip(grads, want[2:]):
        assert ref.within(get(g), *v, "f32")
    assert intact(dx, dres, *grads) and bool((ws[n:] == 0x5A).all())


@pytest.mark.parametrize("rows,cols,pad,skew,fmt", SIZES)
def test_dropout_backward(rows, cols, pad, skew, fmt):
    key = dict(drop=0.3, seed=5, offset=2 ** 63)
    x, dx, db = filled(rows, cols, pad, skew, fmt, 1), Matrix(rows, cols, fmt, pad, skew), vector(cols, "f32")
    ws, n = scratch(rows, cols)
    mics.mics_bias_dropout_add_backward(dx.t, db.v, x.t, rows, cols, dtype=CODE[fmt], grad_dtype=2, workspace=ws, workspace_bytes=n,
                                        strides=(cols + pad,) * 2, **key)
    wdx, wdb = ref.bias_dropout_add_backward(x.f64(), *key.values())
    assert ref.within(dx.f64(), *wdx, fmt) and ref.within(get(db), *wdb, "f32") and intact(dx, db) and bool((ws[n:] == 0x5A).all())


@pytest.mark.parametrize("cols", [8, 20])
def test_dropout_of_more_vectors_than_a_grid_has_lanes(cols):
    """The largest grid is 2^20 wavefronts: parts of the rows, each from its own counter on, are the same."""
    groups = -(-cols // 8)
    rows = ((1 << 26) + 12345) // groups
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV).normal_()
    bias, whole, parts = torch.randn(cols, device=DEV), torch.empty_like(x), torch.empty_like(x)
    call = lambda out, x, n, at: mics.mics_bias_dropout_add(out, x, bias, None, n, cols, drop=0.4, seed=9, offset=at,      # noqa: E731
                                                            dtype=0, param_dtype=2)
    call(whole, x, rows, 11)
    for lo, hi in ((0, rows // 2), (rows // 2, rows)):
        call(parts[lo:hi], x[lo:hi], hi - lo, 11 + lo * groups)
    assert torch.equal(whole.view(torch.int16), parts.view(torch.int16))
    last = slice(rows - 1000, rows)
    want = ref.bias_dropout_add(x[last].double().cpu().numpy(), bias.double().cpu().numpy(), None, 0.4, 9, 11 + (rows - 1000) * groups)
    assert ref.within(whole[last].double().cpu().numpy(), *want, "bf16")


def test_log_probabilities_of_more_rows_than_a_grid_has_workgroups():
    rows, cols, top = (1 << 20) + 4321, 9, 3
    x = torch.empty(rows, cols, device=DEV).normal_()
    t = torch.randint(-1, cols, (rows,), device=DEV)
    lp, ent, lse, best = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, top, device=DEV)
    ids = torch.full((rows, top), -7, dtype=torch.int64, device=DEV)
    mics.mics_token_logprobs(lp, ent, lse, ids, best, x, t, rows, cols, dtype=2, top_k=top)
    for at in (slice(0, 3000), slice(rows - 6000, rows)):
        h = lambda v: v[at].double().cpu().numpy()                                     # noqa: E731
        want = ref.logprobs(h(x), t[at].cpu().numpy(), top)
        for got, name in ((lp, "logprob"), (ent, "entropy"), (lse, "lse"), (best, "top")):
            assert ref.within(h(got), *want[name], "f32"), name
        assert np.array_equal(ids[at].cpu().numpy(), want["ids"])
