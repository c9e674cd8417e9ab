"""Layer norm, dropout, their joined form and token log probabilities on the GPU against the 64-bit reference."""
import numpy as np
import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"bf16": mics.MICS_DTYPE_BF16, "f16": mics.MICS_DTYPE_F16, "f32": mics.MICS_DTYPE_F32}
CANARY = {2: 0x5A5A, 4: 0x5A5A5A5A}


class Matrix:
    """rows x cols with `pad` elements between rows, on an element `skew` off the allocation's start, canaries around."""

    def __init__(self, rows, cols, fmt, pad=0, skew=0, data=None):
        self.rows, self.cols, self.stride, self.fmt = rows, cols, cols + pad, fmt
        self.lead = 64 + skew
        dt = TORCH[fmt]
        self.bits = torch.int32 if fmt == "f32" else torch.int16
        self.whole = torch.empty(self.lead + max(rows, 1) * self.stride + 64, dtype=dt, device=DEV)
        self.whole.view(self.bits).fill_(CANARY[dt.itemsize])
        self.t = torch.as_strided(self.whole, (rows, cols), (self.stride, 1), self.lead)
        if data is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(data)))

    def f64(self):
        return self.t.double().cpu().numpy()

    def rest_intact(self):
        mask = torch.ones(self.whole.shape, dtype=torch.bool, device=DEV)
        torch.as_strided(mask, (self.rows, self.cols), (self.stride, 1), self.lead).fill_(False)
        return bool((self.whole.view(self.bits)[mask] == CANARY[self.whole.dtype.itemsize]).all())


def vector(n, fmt, data=None):
    m = Matrix(1, n, fmt, data=None if data is None else np.asarray(data).reshape(1, n))
    m.v = m.t[0]
    return m


def get(v):
    return None if v is None else v.t.double().cpu().numpy()[0]


def scratch(rows, cols):
    n = mics.mics_column_workspace_bytes(rows, cols)
    w = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device=DEV)
    return w, n


def intact(*ms):
    return all(m.rest_intact() for m in ms if m is not None)


def normal(seed, rows, cols, sigma=1.0, mean=0.0):
    return np.random.default_rng(seed).normal(mean, sigma, (rows, cols))


# rows, cols, pad, skew, matrices, parameters, gradients: lengths around a vector, a wavefront's and a workgroup's share of a
# row, rows that no workgroup holds, one row and many
SHAPES = [(1, 1, 0, 0, "f32", "f32", "f32"), (3, 7, 0, 0, "bf16", "bf16", "f32"), (5, 8, 0, 0, "f16", "f16", "f16"),
          (2, 9, 4, 1, "bf16", "f32", "bf16"), (70, 64, 0, 0, "bf16", "bf16", "bf16"), (33, 511, 0, 0, "f32", "f32", "f32"),
          (9, 512, 8, 0, "bf16", "bf16", "bf16"), (1030, 513, 3, 1, "bf16", "bf16", "bf16"), (4, 1000, 0, 3, "f32", "bf16", "f16"),
          (257, 2048, 0, 0, "bf16", "bf16", "bf16"), (6, 2049, 7, 0, "f16", "f32", "f32"), (40, 2560, 0, 0, "bf16", "bf16", "bf16"),
          (300, 4099, 0, 0, "f16", "f16", "f16"), (11, 5120, 8, 0, "bf16", "bf16", "f32"), (7, 8192, 0, 0, "f32", "f32", "f32"),
          (300, 8192, 0, 0, "bf16", "bf16", "bf16"), (5, 8195, 0, 1, "bf16", "bf16", "bf16"), (3, 16384, 0, 0, "bf16", "bf16", "bf16"),
          (2, 16377, 5, 0, "f32", "f32", "f32"), (3, 16392, 0, 0, "bf16", "bf16", "bf16"), (2, 40003, 1, 0, "f16", "f16", "f16"),
          (4000, 96, 0, 0, "bf16", "bf16", "bf16"), (1, 12288, 0, 0, "bf16", "bf16", "bf16")]


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,param,grad", SHAPES)
def test_layer_norm_forward_and_backward(rows, cols, pad, skew, fmt, param, grad):
    r = np.random.default_rng(rows * 1000 + cols)
    x = Matrix(rows, cols, fmt, pad, skew, r.normal(0.5, 2.0, (rows, cols)) * (1 + 20 * (r.random(cols) < 0.01)))
    y = Matrix(rows, cols, fmt, pad, skew)
    w, b = vector(cols, param, r.normal(1, 0.2, cols)), vector(cols, param, r.normal(0, 0.2, cols))
    mean, rstd = vector(rows, "f32"), vector(rows, "f32")
    st = (cols + pad,) * 2
    mics.mics_layer_norm(y.t, mean.v, rstd.v, x.t, w.v, b.v, rows, cols, eps=1e-5, dtype=CODE[fmt], param_dtype=CODE[param], strides=st)
    x64 = x.f64()
    (ry, sy), (rm, sm), (rr, sr) = ref.layer_norm(x64, np.abs(x64), get(w), get(b), 1e-5)
    assert ref.within(y.f64(), ry, sy, fmt)
    assert ref.within(get(mean), rm, sm, "f32") and ref.within(get(rstd), rr, sr, "f32")
    assert intact(y, mean, rstd)

    dy = Matrix(rows, cols, fmt, pad, skew, r.normal(0, 0.3, (rows, cols)))
    dx = Matrix(rows, cols, fmt, pad, skew)
    dw, db = vector(cols, grad), vector(cols, grad)
    ws, n = scratch(rows, cols)
    mics.mics_layer_norm_backward(dx.t, dw.v, db.v, dy.t, x.t, mean.v, rstd.v, w.v, rows, cols, dtype=CODE[fmt],
                                  param_dtype=CODE[param], grad_dtype=CODE[grad], workspace=ws, workspace_bytes=n,
                                  strides=(cols + pad,) * 3)
    want = ref.layer_norm_backward(dy.f64(), x64, get(mean), get(rstd), get(w))
    assert ref.within(dx.f64(), *want[0], fmt)
    assert ref.within(get(dw), *want[1], grad) and ref.within(get(db), *want[2], grad)
    assert intact(dx, dw, db) and bool((ws[n:] == 0x5A).all())


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,param,grad", SHAPES)
@pytest.mark.parametrize("drop", [0.1, 0.0])
def test_block_forward_and_backward(rows, cols, pad, skew, fmt, param, grad, drop):
    r = np.random.default_rng(rows * 1000 + cols + 1)
    key = dict(drop=drop, seed=2 ** 64 - 12345 - cols, offset=2 ** 64 - 7)        # the counter passes 2^64 on the way
    mk = lambda data=None: Matrix(rows, cols, fmt, pad, skew, data)               # noqa: E731
    x, res = mk(r.normal(0, 1, (rows, cols))), mk(r.normal(0.2, 2, (rows, cols)))
    bias, w, b = (vector(cols, param, r.normal(m, 0.2, cols)) for m in (0, 1, 0))
    y, s, mean, rstd = mk(), mk(), vector(rows, "f32"), vector(rows, "f32")
    types = dict(dtype=CODE[fmt], param_dtype=CODE[param])
    mics.mics_dropout_add_layer_norm(y.t, s.t, mean.v, rstd.v, x.t, bias.v, res.t, w.v, b.v, rows, cols, eps=1e-5,
                                     strides=(cols + pad,) * 4, **key, **types)
    rs, ss = ref.bias_dropout_add(x.f64(), get(bias), res.f64(), key["drop"], key["seed"], key["offset"])
    (ry, sy), (rm, sm), (rr, sr) = ref.layer_norm(rs, ss, get(w), get(b), 1e-5)
    assert ref.within(s.f64(), rs, ss, fmt) and ref.within(y.f64(), ry, sy, fmt)
    assert ref.within(get(mean), rm, sm, "f32") and ref.within(get(rstd), rr, sr, "f32")
    assert intact(y, s, mean, rstd)

    dy, dsum = mk(r.normal(0, 0.3, (rows, cols))), mk(r.normal(0, 0.3, (rows, cols)))
    for has_sum in (True, False):
        dx, dres = mk(), mk()
        grads = [vector(cols, grad) for _ in range(3)]
        ws, n = scratch(rows, cols)
        mics.mics_dropout_add_layer_norm_backward(
            dx.t, dres.t, *[g.v for g in grads], dy.t, dsum.t if has_sum else None, s.t, mean.v, rstd.v, w.v, rows, cols,
            grad_dtype=CODE[grad], workspace=ws, workspace_bytes=n, strides=(cols + pad,) * 5, **key, **types)
        want = ref.block_backward(dy.f64(), dsum.f64() if has_sum else None, s.f64(), get(mean), get(rstd), get(w), key["drop"],
                                  key["seed"], key["offset"])
        assert ref.within(dx.f64(), *want[0], fmt) and ref.within(dres.f64(), *want[1], fmt)
        for g, v in zip(grads, want[2:]):
            assert ref.within(get(g), *v, grad)
        assert intact(dx, dres, *grads) and bool((ws[n:] == 0x5A).all())


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,param,grad", SHAPES)
@pytest.mark.parametrize("drop,bias,residual", [(0.1, True, True), (0.0, True, False), (0.7, False, True), (0.99999, True, True)])
def test_dropout_forward_and_backward(rows, cols, pad, skew, fmt, param, grad, drop, bias, residual):
    r = np.random.default_rng(rows * 1000 + cols + 2)
    key = dict(drop=drop, seed=99 + cols, offset=2 ** 32 - 3)
    x = Matrix(rows, cols, fmt, pad, skew, r.normal(0, 1, (rows, cols)))
    res = Matrix(rows, cols, fmt, pad + 1, skew, r.normal(0, 2, (rows, cols))) if residual else None
    b = vector(cols, param, r.normal(0, 0.2, cols)) if bias else None
    out = Matrix(rows, cols, fmt, pad, skew)
    mics.mics_bias_dropout_add(out.t, x.t, b.v if b else None, res.t if res else None, rows, cols, dtype=CODE[fmt],
                               param_dtype=CODE[param], strides=(out.stride, x.stride, cols + pad + 1), **key)
    want = ref.bias_dropout_add(x.f64(), get(b), res.f64() if res else None, drop, key["seed"], key["offset"])
    assert ref.within(out.f64(), *want, fmt) and intact(out)

    dx, db = Matrix(rows, cols, fmt, pad, skew), vector(cols, grad)
    ws, n = scratch(rows, cols)
    mics.mics_bias_dropout_add_backward(dx.t, db.v, x.t, rows, cols, dtype=CODE[fmt], grad_dtype=CODE[grad], workspace=ws,
                                        workspace_bytes=n, strides=(dx.stride, x.stride), **key)
    wdx, wdb = ref.bias_dropout_add_backward(x.f64(), drop, key["seed"], key["offset"])
    assert ref.within(dx.f64(), *wdx, fmt) and ref.within(get(db), *wdb, grad)
    assert intact(dx, db) and bool((ws[n:] == 0x5A).all())
    again = Matrix(rows, cols, fmt, pad, skew)
    mics.mics_bias_dropout_add_backward(again.t, None, x.t, rows, cols, dtype=CODE[fmt], grad_dtype=CODE[grad],
                                        strides=(dx.stride, x.stride), **key)
    assert torch.equal(again.whole.view(again.bits), dx.whole.view(dx.bits))


def test_dropped_elements_are_zero_whatever_they_held():
    rows, cols = 4, 64
    key = dict(drop=0.5, seed=1, offset=0)
    for bad in (float("inf"), float("nan")):
        x = torch.full((rows, cols), bad, device=DEV)
        out = torch.empty_like(x)
        mics.mics_bias_dropout_add(out, x, None, None, rows, cols, dtype=CODE["f32"], param_dtype=CODE["f32"], **key)
        keep = ref.kept(rows, cols, 0.5, 1, 0)
        assert np.array_equal(out.cpu().numpy() == 0, ~keep)


def test_parameters_that_are_left_out():
    rows, cols = 5, 100
    x = Matrix(rows, cols, "f32", data=normal(1, rows, cols))
    y = Matrix(rows, cols, "f32")
    mics.mics_layer_norm(y.t, None, None, x.t, None, None, rows, cols, eps=0.0, dtype=CODE["f32"], param_dtype=CODE["f32"])
    (ry, sy), (m, _), (rs, _) = ref.layer_norm(x.f64(), np.abs(x.f64()), None, None, 0.0)
    assert ref.within(y.f64(), ry, sy, "f32")
    y2 = Matrix(rows, cols, "f32")
    mics.mics_dropout_add_layer_norm(y2.t, None, None, None, x.t, None, None, None, None, rows, cols, drop=0.0, seed=0, offset=0,
                                     eps=0.0, dtype=CODE["f32"], param_dtype=CODE["f32"])
    assert torch.equal(y.t, y2.t)
    mean, rstd = vector(rows, "f32", m), vector(rows, "f32", rs)
    dy = Matrix(rows, cols, "f32", data=normal(2, rows, cols))
    dx, dw = Matrix(rows, cols, "f32"), vector(cols, "f32")
    ws, n = scratch(rows, cols)
    mics.mics_layer_norm_backward(dx.t, dw.v, None, dy.t, x.t, mean.v, rstd.v, None, rows, cols, dtype=2, param_dtype=2, grad_dtype=2,
                                  workspace=ws, workspace_bytes=n)
    want = ref.layer_norm_backward(dy.f64(), x.f64(), get(mean), get(rstd), None)
    assert ref.within(dx.f64(), *want[0], "f32") and ref.within(get(dw), *want[1], "f32")
    dx2 = Matrix(rows, cols, "f32")
    mics.mics_dropout_add_layer_norm_backward(dx2.t, None, None, None, None, dy.t, None, x.t, mean.v, rstd.v, None, rows, cols,
                                              drop=0.0, seed=0, offset=0, dtype=2, param_dtype=2, grad_dtype=2, workspace=ws,
                                              workspace_bytes=n)
    assert torch.equal(dx.t, dx2.t)


def test_no_rows():
    cols = 1000
    ws, n = scratch(0, cols)
    g = [torch.full((cols,), 7.0, device=DEV) for _ in range(3)]
    e = torch.empty(0, device=DEV)
    t = dict(dtype=2, param_dtype=2)
    key = dict(drop=0.1, seed=0, offset=0)
    mics.mics_layer_norm(e, None, None, e, None, None, 0, cols, eps=1e-5, **t)
    mics.mics_bias_dropout_add(e, e, None, None, 0, cols, **key, **t)
    mics.mics_dropout_add_layer_norm(e, e, None, None, e, None, None, None, None, 0, cols, eps=1e-5, **key, **t)
    mics.mics_token_logprobs(e, e, e, None, None, e, e, 0, cols, dtype=2)
    mics.mics_token_logprobs_backward(e, e, e, e, None, e, None, 0, cols, dtype=2)
    mics.mics_layer_norm_backward(e, g[0], None, e, e, e, e, None, 0, cols, grad_dtype=2, workspace=ws, workspace_bytes=n, **t)
    mics.mics_bias_dropout_add_backward(e, g[1], e, 0, cols, dtype=2, grad_dtype=2, workspace=ws, workspace_bytes=n, **key)
    mics.mics_dropout_add_layer_norm_backward(e, e, None, None, g[2], e, None, e, e, e, None, 0, cols, grad_dtype=2, workspace=ws,
                                              workspace_bytes=n, **key, **t)
    for x in g:
        assert bool((x == 0).all())


@pytest.mark.parametrize("cols", [64, 1003, 8192, 20000])
def test_rows_of_extreme_values(cols):
    """Large means, constant rows, values near the largest: nothing cancels or overflows before the formula does."""
    big = Matrix(4, cols, "f32", data=np.stack([normal(5, 1, cols)[0] * 1e-2 + 3000.0, np.full(cols, -2.5),
                                                normal(6, 1, cols)[0] * 1e15, np.zeros(cols)]))
    y, mean, rstd = Matrix(4, cols, "f32"), vector(4, "f32"), vector(4, "f32")
    mics.mics_layer_norm(y.t, mean.v, rstd.v, big.t, None, None, 4, cols, eps=1e-5, dtype=2, param_dtype=2)
    (ry, sy), (rm, sm), (rr, sr) = ref.layer_norm(big.f64(), np.abs(big.f64()), None, None, 1e-5)
    assert ref.within(get(mean), rm, sm, "f32") and ref.within(get(rstd), rr, sr, "f32") and ref.within(y.f64(), ry, sy, "f32")


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [1000, 8192, 16400])
def test_results_in_the_place_of_inputs(fmt, cols):
    rows, key, t = 37, dict(drop=0.2, seed=3, offset=4), dict(dtype=CODE[fmt], param_dtype=2)
    new = lambda seed: Matrix(rows, cols, fmt, data=normal(seed, rows, cols))     # noqa: E731
    x, res, dy, dsum = new(1), new(2), new(3), new(4)
    y, s, dx, dr = (Matrix(rows, cols, fmt) for _ in range(4))
    mean, rstd = vector(rows, "f32"), vector(rows, "f32")
    g1, g2 = [vector(cols, "f32") for _ in range(3)], [vector(cols, "f32") for _ in range(3)]
    ws, n = scratch(rows, cols)
    back = dict(grad_dtype=2, workspace=ws, workspace_bytes=n, **key, **t)
    mics.mics_dropout_add_layer_norm(y.t, s.t, mean.v, rstd.v, x.t, None, res.t, None, None, rows, cols, eps=1e-5, **key, **t)
    mics.mics_dropout_add_layer_norm_backward(dx.t, dr.t, *[g.v for g in g1], dy.t, dsum.t, s.t, mean.v, rstd.v, None, rows, cols, **back)
    mics.mics_dropout_add_layer_norm(x.t, res.t, mean.v, rstd.v, x.t, None, res.t, None, None, rows, cols, eps=1e-5, **key, **t)
    assert torch.equal(x.t, y.t) and torch.equal(res.t, s.t)
    mics.mics_dropout_add_layer_norm_backward(dy.t, dsum.t, *[g.v for g in g2], dy.t, dsum.t, s.t, mean.v, rstd.v, None, rows, cols, **back)
    assert torch.equal(dx.t, dy.t) and torch.equal(dr.t, dsum.t)
    assert all(torch.equal(a.t, b.t) for a, b in zip(g1, g2))


def test_matrices_between_each_others_rows():
    rows, cols = 50, 520
    buf = torch.zeros(rows, 2 * cols, dtype=torch.bfloat16, device=DEV)
    x, y = buf[:, :cols], buf[:, cols:]
    x.copy_(torch.randn(rows, cols, device=DEV))
    want = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    t = dict(eps=1e-5, dtype=0, param_dtype=0)
    mics.mics_layer_norm(want, None, None, x.contiguous(), None, None, rows, cols, **t)
    mics.mics_layer_norm(y, None, None, x, None, None, rows, cols, strides=(2 * cols, 2 * cols), **t)
    assert torch.equal(y, want)


@pytest.mark.parametrize("rows,cols", [(3, 40), (130, 1000)])
def test_gradients_against_differences(rows, cols):
    """Directional derivatives of the kernels' own forward passes.  The sums are formed in 64 bits from binary32 outputs:
    a difference over 2h is off by h^2 (third derivatives) and by rounding / h."""
    r = np.random.default_rng(9)
    up = lambda a: torch.from_numpy(a).float().to(DEV)           # noqa: E731
    x, res, dy, dsum = (up(r.normal(size=(rows, cols))) for _ in range(4))
    bias, w, nb = (up(r.normal(size=cols)) for _ in range(3))
    key, t = dict(drop=0.25, seed=8, offset=1), dict(dtype=2, param_dtype=2)

    def forward(x, res, bias, w, nb):
        y, s, m, rs = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        mics.mics_dropout_add_layer_norm(y, s, m, rs, x, bias, res, w, nb, rows, cols, eps=1e-3, **key, **t)
        return y, s, m, rs

    args = [x, res, bias, w, nb]
    y, s, m, rs = forward(*args)
    dx, dr, db, dw, dnb = torch.empty_like(x), torch.empty_like(x), *(torch.empty(cols, device=DEV) for _ in range(3))
    ws, n = scratch(rows, cols)
    mics.mics_dropout_add_layer_norm_backward(dx, dr, db, dw, dnb, dy, dsum, s, m, rs, w, rows, cols, grad_dtype=2, workspace=ws,
                                              workspace_bytes=n, **key, **t)
    h = 2.0 ** -7
    for i, g in enumerate((dx, dr, db, dw, dnb)):
        v = up(r.normal(size=tuple(args[i].shape)))
        ends = []
        for sign in (1, -1):
            moved = list(args)
            moved[i] = args[i] + sign * h * v
            y, s, _, _ = forward(*moved)
            ends.append(float((y.double() * dy.double()).sum() + (s.double() * dsum.double()).sum()))
        got, want = float((g.double() * v.double()).sum()), (ends[0] - ends[1]) / (2 * h)
        size = float((g.double() * v.double()).square().sum().sqrt())
        # h^2 = 6e-5, times third derivatives of order 10 at most; 2^-24 / h = 8e-6 for each of the random roundings
        assert abs(got - want) < 2e-3 * size, (i, got, want, size)


# ---- log probabilities -------------------------------------------------------------------------

LOGITS = [(1, 1, 0, 0, "f32", 1), (3, 5, 0, 0, "bf16", 3), (2, 8, 3, 1, "f16", 8), (5, 9, 0, 0, "f32", 0), (9, 1000, 0, 0, "bf16", 5),
          (300, 1003, 7, 1, "bf16", 20), (2, 8192, 0, 0, "f32", 64), (1, 16384, 0, 0, "bf16", 1), (1, 50001, 0, 0, "bf16", 8),
          (4, 131072, 0, 0, "bf16", 50), (3, 100003, 5, 1, "f32", 64), (20, 40000, 0, 0, "f16", 5), (257, 32768, 0, 0, "bf16", 0),
          (400, 5001, 0, 1, "f32", 8), (64, 20000, 0, 0, "bf16", 0)]


def run_logprobs(x, targets, top, entropy=True):
    rows, cols = x.rows, x.cols
    out = [vector(max(rows, 1), "f32") for _ in range(3)]
    ids = torch.full((rows, top), -7, dtype=torch.int64, device=DEV)
    best = torch.full((rows, top), 7.0, device=DEV)
    n = mics.mics_token_logprobs_workspace_bytes(rows, cols, top)
    ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device=DEV)
    mics.mics_token_logprobs(out[0].v, out[1].v if entropy else None, out[2].v, ids, best, x.t, torch.from_numpy(targets).to(DEV), rows,
                             cols, dtype=CODE[x.fmt], top_k=top, stride=x.stride, workspace=ws, workspace_bytes=n)
    torch.cuda.synchronize()
    assert intact(*out) and bool((ws[n:] == 0x5A).all())
    return dict(logprob=get(out[0]), entropy=get(out[1]), lse=get(out[2]), ids=ids.cpu().numpy(), top=best.double().cpu().numpy())


def check_logprobs(x, targets, top):
    got, want = run_logprobs(x, targets, top), ref.logprobs(x.f64(), targets, top)
    for name in ("logprob", "entropy", "lse", "top"):
        assert ref.within(got[name], *want[name], "f32"), name
    assert np.array_equal(got["ids"], want["ids"])
    return got


def targets_of(r, rows, cols):
    t = r.integers(0, cols, rows)
    return np.where(r.random(rows) < 0.2, -1 - r.integers(0, 100, rows), t)


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,top", LOGITS)
@pytest.mark.parametrize("masked", [0.0, 0.5, 0.9995])
def test_log_probabilities(rows, cols, pad, skew, fmt, top, masked):
    r = np.random.default_rng(rows + cols)
    data = r.normal(0, 3, (rows, cols))
    data[r.random((rows, cols)) < masked] = -np.inf
    check_logprobs(Matrix(rows, cols, fmt, pad, skew, data), targets_of(r, rows, cols), top)


@pytest.mark.parametrize("rows,cols", [(3, 1000), (2, 70001), (300, 3001)])
@pytest.mark.parametrize("kind", ["equal", "zeros of both signs", "two values", "ascending", "descending", "lowest", "empty",
                                  "one left", "one run high"])
def test_alternatives_among_equals_and_in_order(rows, cols, kind):
    r = np.random.default_rng(5)
    lowest = float(np.finfo(np.float32).min)
    data = {"equal": np.full(cols, 1.5), "zeros of both signs": np.where(np.arange(cols) % 3 == 0, -0.0, 0.0),
            "two values": (r.random(cols) < 0.3) * 1.0, "ascending": np.arange(cols) / 512.0, "descending": -np.arange(cols) / 512.0,
            "lowest": np.where(np.arange(cols) % 97 == 5, 0.25, lowest), "empty": np.full(cols, -np.inf),
            "one left": np.where(np.arange(cols) == cols - 1, -4.0, -np.inf),
            # more high logits side by side than the runs' largest tell apart
            "one run high": np.where(np.arange(cols) // 8 % 128 == 3, 10.0 + r.random(cols), 0.0)}[kind]
    x = Matrix(rows, cols, "f32", data=np.tile(data, (rows, 1)))
    check_logprobs(x, targets_of(r, rows, cols), 50)
    check_logprobs(x, targets_of(r, rows, cols), 1)


@pytest.mark.parametrize("rows,cols", [(4, 1000), (4, 50000)])
def test_logits_that_are_not_numbers(rows, cols):
    r = np.random.default_rng(6)
    data = r.normal(size=(rows, cols))
    data[0, 17], data[1, [3, cols - 1]], data[2, cols // 2] = np.nan, np.inf, -np.nan
    data[3, 5] = 3e38
    check_logprobs(Matrix(rows, cols, "f32", data=data), np.array([2, 3, -1, 5]), 6)
    all_nan = Matrix(2, cols, "f32", data=np.full((2, cols), np.nan))
    check_logprobs(all_nan, np.array([0, -1]), 4)


@pytest.mark.parametrize("rows,cols,fmt", [(3, 1000, "f32"), (300, 3001, "bf16"), (2, 70001, "f16")])
@pytest.mark.parametrize("share", [0.3, 0.6])
def test_alternatives_among_many_that_are_not_numbers(rows, cols, fmt, share):
    r = np.random.default_rng(11)
    data = r.normal(size=(rows, cols))
    data[r.random((rows, cols)) < share] = np.nan
    check_logprobs(Matrix(rows, cols, fmt, data=data), targets_of(r, rows, cols), 20)


def test_targets_outside_the_vocabulary():
    x = Matrix(3, 100, "f32", data=normal(1, 3, 100))
    t = np.array([100, 2 ** 40, -2 ** 40])
    got = check_logprobs(x, t, 0)
    assert np.isnan(got["logprob"][:2]).all() and got["logprob"][2] == 0


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,top", LOGITS)
@pytest.mark.parametrize("with_entropy", [False, True])
def test_gradient_of_log_probabilities(rows, cols, pad, skew, fmt, top, with_entropy):
    r = np.random.default_rng(rows + cols + 7)
    data = r.normal(0, 3, (rows, cols))
    if rows > 2:
        data[1, r.random(cols) < 0.5] = -np.inf
        data[2] = -np.inf
    x = Matrix(rows, cols, fmt, pad, skew, data)
    t = targets_of(r, rows, cols)
    if rows > 4:
        t[4] = cols
    o = ref.logprobs(x.f64(), t, 0)
    lse, ent = vector(rows, "f32", o["lse"][0]), vector(rows, "f32", o["entropy"][0])
    g, h = vector(rows, "f32", r.normal(size=rows) * (r.random(rows) < 0.8)), vector(rows, "f32", r.normal(size=rows) * (r.random(rows) < 0.6))
    dx = Matrix(rows, cols, fmt, pad + 2, skew)
    args = (torch.from_numpy(t).to(DEV), lse.v, ent.v if with_entropy else None, g.v, h.v if with_entropy else None, rows, cols)
    mics.mics_token_logprobs_backward(dx.t, x.t, *args, dtype=CODE[fmt], strides=(dx.stride, x.stride))
    want, size = ref.logprobs_backward(x.f64(), t, get(lse), get(ent) if with_entropy else None, get(g), get(h) if with_entropy else None)
    assert ref.within(dx.f64(), want, size, fmt) and intact(dx)
    kept = dx.t.clone()
    mics.mics_token_logprobs_backward(x.t, x.t, *args, dtype=CODE[fmt], strides=(x.stride, x.stride))      # in place
    assert torch.equal(x.t.contiguous().view(x.bits), kept.contiguous().view(x.bits)) and intact(x)


def test_gradient_of_log_probabilities_against_differences():
    rows, cols, h = 6, 777, 2.0 ** -7
    r = np.random.default_rng(11)
    base, v = r.normal(size=(rows, cols)), r.normal(size=(rows, cols))
    t = np.array([0, 776, 5, -1, 9, 100])
    g, e = r.normal(size=rows), r.normal(size=rows)
    ends = []
    for sign in (1, -1):
        o = run_logprobs(Matrix(rows, cols, "f32", data=base + sign * h * v), t, 0)
        ends.append((o["logprob"] * g).sum() + (o["entropy"] * e).sum())
    x = Matrix(rows, cols, "f32", data=base)
    o = run_logprobs(x, t, 0)
    dx = Matrix(rows, cols, "f32")
    up = lambda a: torch.from_numpy(a).float().to(DEV)           # noqa: E731
    mics.mics_token_logprobs_backward(dx.t, x.t, torch.from_numpy(t).to(DEV), up(o["lse"]), up(o["entropy"]), up(g), up(e), rows, cols, dtype=2)
    got, want = (dx.f64() * v).sum(), (ends[0] - ends[1]) / (2 * h)
    # h^2 = 6e-5 times a third derivative of order 1; sums of six rows of size 7 at 2^-24 over h
    assert abs(got - want) < 1e-3 * (1 + abs(want))


# ---- streams, graphs, order --------------------------------------------------------------------

def step_buffers(rows=64, cols=1024, vocab=20000):
    r = np.random.default_rng(21)
    mk = lambda *s: torch.from_numpy(r.normal(size=s)).to(torch.bfloat16).to(DEV)      # noqa: E731
    f = lambda *s: torch.zeros(*s, device=DEV)                                          # noqa: E731
    b = dict(rows=rows, cols=cols, vocab=vocab, x=mk(rows, cols), res=mk(rows, cols), w=mk(cols), nb=mk(cols), bias=mk(cols), y=mk(rows, cols),
             s=mk(rows, cols), mean=f(rows), rstd=f(rows), dx=mk(rows, cols), dr=mk(rows, cols), g=[f(cols) for _ in range(3)],
             logits=mk(rows, vocab), t=torch.from_numpy(r.integers(0, vocab, rows)).to(DEV), lp=f(rows), ent=f(rows), lse=f(rows),
             ids=torch.zeros(rows, 5, dtype=torch.int64, device=DEV), best=f(rows, 5), dl=mk(rows, vocab), dlp=f(rows) - 1)
    b["ws"], b["n"] = scratch(rows, cols)
    b["ln"] = mics.mics_token_logprobs_workspace_bytes(rows, vocab, 5)
    b["lw"] = torch.zeros(b["ln"], dtype=torch.uint8, device=DEV)
    return b


def step(b, stream=None):
    n, c, v = b["rows"], b["cols"], b["vocab"]
    key, t = dict(drop=0.1, seed=5, offset=6), dict(dtype=0, param_dtype=0, stream=stream)
    mics.mics_dropout_add_layer_norm(b["y"], b["s"], b["mean"], b["rstd"], b["x"], b["bias"], b["res"], b["w"], b["nb"], n, c, eps=1e-5,
                                     **key, **t)
    mics.mics_dropout_add_layer_norm_backward(b["dx"], b["dr"], *b["g"], b["y"], None, b["s"], b["mean"], b["rstd"], b["w"], n, c,
                                              grad_dtype=2, workspace=b["ws"], workspace_bytes=b["n"], **key, **t)
    mics.mics_token_logprobs(b["lp"], b["ent"], b["lse"], b["ids"], b["best"], b["logits"], b["t"], n, v, dtype=0, top_k=5,
                             workspace=b["lw"], workspace_bytes=b["ln"], stream=stream)
    mics.mics_token_logprobs_backward(b["dl"], b["logits"], b["t"], b["lse"], b["ent"], b["dlp"], None, n, v, dtype=0, stream=stream)


def results(b):
    torch.cuda.synchronize()
    return [x.clone() for x in (b["y"], b["s"], b["dx"], b["dr"], *b["g"], b["lp"], b["ent"], b["lse"], b["ids"], b["best"], b["dl"])]


def test_graph_replays_give_what_eager_calls_give():
    b = step_buffers()
    step(b)
    results(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    for k in range(4):
        b["x"].mul_(1.0 + 0.1 * k)
        b["logits"].roll(1, 0)
        b["t"].add_(1).remainder_(b["vocab"])
        step(b)
        want = results(b)
        for x in (b["y"], b["dx"], b["dl"], b["lp"], b["best"], *b["g"]):
            x.zero_()
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(results(b), want)), k


def test_calls_are_ordered_by_the_stream_they_are_given():
    b = step_buffers()
    step(b)
    want = results(b)
    side = torch.cuda.Stream()
    for x in (b["y"], b["dx"], b["dl"]):
        x.zero_()
    torch.cuda.synchronize()
    big = torch.zeros(1 << 28, device=DEV)
    with torch.cuda.stream(side):
        held = b["x"].clone()
        b["x"].zero_()
        big.add_(1.0)                                       # keeps the stream busy
        b["x"].copy_(held)
        step(b)                                             # torch's current stream
    assert all(torch.equal(p, q) for p, q in zip(results(b), want))
    b["y"].zero_()
    torch.cuda.synchronize()
    step(b, stream=side)
    assert all(torch.equal(p, q) for p, q in zip(results(b), want))


def test_repeated_calls_give_the_same_bits():
    b = step_buffers(rows=700, cols=2560, vocab=9000)
    step(b)
    want = results(b)
    for _ in range(3):
        step(b)
        assert all(torch.equal(p, q) for p, q in zip(results(b), want))


def test_offsets_past_32_bits():
    """Rows whose byte offset passes 2^32: the last of a matrix of wide row stride."""
    cols, stride, rows = 1000, 1 << 21, 1100
    x = torch.zeros(rows * stride, dtype=torch.bfloat16, device=DEV)
    m = torch.as_strided(x, (rows, cols), (stride, 1))
    m[-1].copy_(torch.randn(cols, device=DEV))
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    mics.mics_layer_norm(y, None, None, m, None, None, rows, cols, eps=1e-5, dtype=0, param_dtype=0, strides=(cols, stride))
    row = m[-1].double().cpu().numpy()[None]
    (ry, sy), _, _ = ref.layer_norm(row, np.abs(row), None, None, 1e-5)
    assert ref.within(y[-1:].double().cpu().numpy(), ry, sy, "bf16")
    lp, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    t = torch.zeros(rows, dtype=torch.int64, device=DEV)
    mics.mics_token_logprobs(lp, None, lse, None, None, m, t, rows, cols, dtype=0, stride=stride)
    want = ref.logprobs(row, np.array([0]), 0)
    assert ref.within(lp[-1:].double().cpu().numpy(), *want["logprob"], "f32")
