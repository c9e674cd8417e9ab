"""Results in the place of inputs, and results that are not asked for, at sizes whose rows end inside a vector: there lanes
read what others store."""
import numpy as np
import pytest
import torch

from test_gpu_layer_ops import CODE, Matrix, intact, normal, scratch, vector

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

# one wavefront a row; two and more; one row a workgroup; tiles; with and without a rest
COLS = [3, 9, 61, 505, 512, 515, 1029, 2049, 4091, 4096, 8185, 8192, 8203, 12291, 16384, 17001]


def same(a, b):
    return torch.equal(a.t.contiguous().view(a.bits), b.t.contiguous().view(b.bits))


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("fmt,rows", [("bf16", 700), ("f32", 301), ("f16", 5)])
def test_in_place(fmt, rows, cols):
    t, key = dict(dtype=CODE[fmt], param_dtype=2), dict(drop=0.3, seed=6, offset=9)
    new = lambda seed: Matrix(rows, cols, fmt, 3, 1, normal(seed, rows, cols))     # noqa: E731
    out = lambda: Matrix(rows, cols, fmt, 3, 1)                                     # noqa: E731
    st = (cols + 3,) * 5
    w, b = vector(cols, "f32", normal(7, 1, cols)), vector(cols, "f32", normal(8, 1, cols))
    mean, rstd = vector(rows, "f32"), vector(rows, "f32")
    ws, n = scratch(rows, cols)
    back = dict(grad_dtype=2, workspace=ws, workspace_bytes=n)

    x, y = new(1), out()
    mics.mics_layer_norm(y.t, mean.v, rstd.v, x.t, w.v, b.v, rows, cols, eps=1e-5, strides=st[:2], **t)
    x2 = new(1)
    mics.mics_layer_norm(x2.t, None, None, x2.t, w.v, b.v, rows, cols, eps=1e-5, strides=st[:2], **t)
    assert same(y, x2) and intact(x2)

    dy, dx, g = new(2), out(), [vector(cols, "f32") for _ in range(5)]
    mics.mics_layer_norm_backward(dx.t, g[0].v, g[1].v, dy.t, x.t, mean.v, rstd.v, w.v, rows, cols, strides=st[:3], **t, **back)
    for in_dy in (True, False):
        dy2, x2 = new(2), new(1)
        at = dy2 if in_dy else x2
        mics.mics_layer_norm_backward(at.t, g[2].v, g[3].v, dy2.t, x2.t, mean.v, rstd.v, w.v, rows, cols, strides=st[:3], **t, **back)
        assert same(dx, at) and same(g[0], g[2]) and same(g[1], g[3]) and intact(at)

    res, s = new(3), out()
    block = dict(eps=1e-5, strides=st[:4], **key, **t)
    mics.mics_dropout_add_layer_norm(y.t, s.t, mean.v, rstd.v, x.t, b.v, res.t, w.v, b.v, rows, cols, **block)
    for first in (True, False):
        x2, res2 = new(1), new(3)
        ys, ss = (x2, res2) if first else (res2, x2)
        mics.mics_dropout_add_layer_norm(ys.t, ss.t, mean.v, rstd.v, x2.t, b.v, res2.t, w.v, b.v, rows, cols, **block)
        assert same(y, ys) and same(s, ss) and intact(ys, ss)

    dsum, dr = new(4), out()
    whole = dict(strides=st, **key, **t, **back)
    mics.mics_dropout_add_layer_norm_backward(dx.t, dr.t, g[0].v, g[1].v, None, dy.t, dsum.t, s.t, mean.v, rstd.v, w.v, rows, cols, **whole)
    for first in (True, False):
        dy2, dsum2 = new(2), new(4)
        a, c = (dy2, dsum2) if first else (dsum2, dy2)
        mics.mics_dropout_add_layer_norm_backward(a.t, c.t, g[2].v, g[3].v, None, dy2.t, dsum2.t, s.t, mean.v, rstd.v, w.v, rows, cols,
                                                  **whole)
        assert same(dx, a) and same(dr, c) and same(g[0], g[2]) and same(g[1], g[3]) and intact(a, c)

    o = out()
    mics.mics_bias_dropout_add(o.t, x.t, b.v, res.t, rows, cols, strides=st[:3], **key, **t)
    for first in (True, False):
        x2, res2 = new(1), new(3)
        at = x2 if first else res2
        mics.mics_bias_dropout_add(at.t, x2.t, b.v, res2.t, rows, cols, strides=st[:3], **key, **t)
        assert same(o, at) and intact(at)
    mics.mics_bias_dropout_add_backward(o.t, g[0].v, x.t, rows, cols, strides=st[:2], dtype=CODE[fmt], **key, **back)
    x2 = new(1)
    mics.mics_bias_dropout_add_backward(x2.t, g[2].v, x2.t, rows, cols, strides=st[:2], dtype=CODE[fmt], **key, **back)
    assert same(o, x2) and same(g[0], g[2]) and intact(x2)


@pytest.mark.parametrize("cols", COLS)
def test_results_that_are_not_asked_for(cols):
    """Leaving results out changes none of the others."""
    rows, t, key = 77, dict(dtype=0, param_dtype=0), dict(drop=0.2, seed=1, offset=2)
    new = lambda seed: Matrix(rows, cols, "bf16", data=normal(seed, rows, cols))   # noqa: E731
    x, res, dy = new(1), new(2), new(3)
    y, s, dx, dr = (Matrix(rows, cols, "bf16") for _ in range(4))
    mean, rstd, g = vector(rows, "f32"), vector(rows, "f32"), [vector(cols, "bf16") for _ in range(3)]
    ws, n = scratch(rows, cols)
    mics.mics_dropout_add_layer_norm(y.t, s.t, mean.v, rstd.v, x.t, None, res.t, None, None, rows, cols, eps=1e-5, **key, **t)
    for has in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 0, 0)):
        y2, s2, m2, r2 = Matrix(rows, cols, "bf16"), Matrix(rows, cols, "bf16"), vector(rows, "f32"), vector(rows, "f32")
        mics.mics_dropout_add_layer_norm(y2.t, s2.t if has[0] else None, m2.v if has[1] else None, r2.v if has[2] else None, x.t, None,
                                         res.t, None, None, rows, cols, eps=1e-5, **key, **t)
        assert same(y, y2) and (not has[0] or same(s, s2)) and (not has[1] or same(mean, m2)) and (not has[2] or same(rstd, r2))
    back = dict(grad_dtype=0, workspace=ws, workspace_bytes=n, **key, **t)
    mics.mics_dropout_add_layer_norm_backward(dx.t, dr.t, *[v.v for v in g], dy.t, None, s.t, mean.v, rstd.v, None, rows, cols, **back)
    for left_out in range(4):
        dx2, dr2, g2 = Matrix(rows, cols, "bf16"), Matrix(rows, cols, "bf16"), [vector(cols, "bf16") for _ in range(3)]
        give = [dr2.t, *[v.v for v in g2]]
        give[left_out] = None
        mics.mics_dropout_add_layer_norm_backward(dx2.t, *give, dy.t, None, s.t, mean.v, rstd.v, None, rows, cols, **back)
        assert same(dx, dx2) and (left_out == 0 or same(dr, dr2))
        assert all(same(p, q) for i, (p, q) in enumerate(zip(g, g2)) if i + 1 != left_out)


@pytest.mark.parametrize("rows", [1, 2, 3, 7, 16, 17, 31, 32, 33, 64, 65, 300])
@pytest.mark.parametrize("cols", [40, 515, 2560, 8192])
def test_column_sums_of_few_rows_and_of_many(rows, cols):
    """One launch for few rows, two for more: both against the sums in 64 bits."""
    import layer_ref as ref
    dy, x = Matrix(rows, cols, "f32", data=normal(rows, rows, cols)), Matrix(rows, cols, "f32", data=normal(cols, rows, cols))
    mean, rstd = vector(rows, "f32", normal(5, 1, rows) * 0.1), vector(rows, "f32", np.exp(normal(6, 1, rows) * 0.1))
    dx, g = Matrix(rows, cols, "f32"), [vector(cols, f) for f in ("f32", "bf16", "f16")]
    ws, n = scratch(rows, cols)
    want = ref.layer_norm_backward(dy.f64(), x.f64(), mean.t.double().cpu().numpy()[0], rstd.t.double().cpu().numpy()[0], None)
    for v, fmt in zip(g, ("f32", "bf16", "f16")):
        mics.mics_layer_norm_backward(dx.t, v.v, None, dy.t, x.t, mean.v, rstd.v, None, rows, cols, dtype=2, param_dtype=2,
                                      grad_dtype=CODE[fmt], workspace=ws, workspace_bytes=n)
        assert ref.within(v.t.double().cpu().numpy()[0], *want[1], fmt) and intact(v)
        mics.mics_bias_dropout_add_backward(dx.t, v.v, dy.t, rows, cols, drop=0.0, seed=0, offset=0, dtype=2, grad_dtype=CODE[fmt],
                                            workspace=ws, workspace_bytes=n)
        assert ref.within(v.t.double().cpu().numpy()[0], *want[2], fmt) and intact(v)
