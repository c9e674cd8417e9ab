"""The linear layer, the gradients of its input and weight, activations and their 8-bit checkpoints on the GPU against the 64-bit
reference."""
import numpy as np
import pytest
import torch

import layer_ref
import linear_ref as ref
from linear_shapes import SHAPES

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8}
BITS = {1: torch.int8, 2: torch.int16, 4: torch.int32}
CANARY = {1: 0x5A, 2: 0x5A5A, 4: 0x5A5A5A5A}
CODE = {"bf16": mics.MICS_DTYPE_BF16, "f16": mics.MICS_DTYPE_F16, "f32": mics.MICS_DTYPE_F32}
ACT = {n: i for i, n in enumerate(ref.ACTS)}


class Matrix:
    """rows x cols with `pad` elements between rows, on an element `skew` off the allocation's start, canaries around."""

    def __init__(self, rows, cols, fmt, pad=0, skew=0, data=None):
        self.shape, self.stride, self.fmt = (rows, cols), cols + pad, fmt
        self.lead = 64 + skew
        self.whole = torch.empty(self.lead + max(rows, 1) * self.stride + 64, dtype=TORCH[fmt], device=DEV)
        self.size = self.whole.dtype.itemsize
        self.whole.view(BITS[self.size]).fill_(CANARY[self.size])
        self.t = torch.as_strided(self.whole, (rows, cols), (self.stride, 1), self.lead)
        if data is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(data)))

    def f64(self):
        return self.t.double().cpu().numpy()

    def intact(self):
        mask = torch.ones(self.whole.shape, dtype=torch.bool, device=DEV)
        torch.as_strided(mask, self.shape, (self.stride, 1), self.lead).fill_(False)
        return bool((self.whole.view(BITS[self.size])[mask] == CANARY[self.size]).all())


class Vector(Matrix):
    def __init__(self, n, fmt, data=None):
        super().__init__(1, n, fmt, data=None if data is None else np.asarray(data).reshape(1, n))
        self.v = self.t[0]

    def f64(self):
        return super().f64()[0]


def scratch(n):
    return torch.full((n + 64,), 0x5A, dtype=torch.uint8, device=DEV), n


def linear_scratch(rows, cin, cout):
    w, n = scratch(mics.mics_linear_workspace_bytes(rows, cin, cout))
    return w, dict(workspace=w, workspace_bytes=n)


def spared(w):
    return bool((w[-64:] == 0x5A).all())


def mm(a, b):
    """The product of float64 matrices, large ones on the GPU."""
    if a.shape[0] * a.shape[1] * b.shape[1] < 1 << 30:
        return a @ b
    on = [torch.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in (a, b)]
    return torch.mm(*on).cpu().numpy()


def nearest(x, fmt):
    """float64 to the format and back."""
    with np.errstate(over="ignore"):
        return torch.from_numpy(np.asarray(x, np.float32)).to(TORCH[fmt]).double().numpy()




def whole_numbers(r, rows, cols, most):
    return r.integers(-most, most + 1, (rows, cols)).astype(np.float64)


@pytest.mark.parametrize("rows,cin,cout,pad,skew,fmt", SHAPES)
def test_products_of_whole_numbers_are_exact(rows, cin, cout, pad, skew, fmt):
    """Sums below 2^24 are exact in binary32 in any order: every result is the nearest of its format."""
    r = np.random.default_rng(rows + 7 * cin + 13 * cout)
    mk = lambda n, m, data=None, f=fmt: Matrix(n, m, f, pad, skew, data)               # noqa: E731
    x, w = mk(rows, cin, whole_numbers(r, rows, cin, 8)), mk(cout, cin, whole_numbers(r, cout, cin, 8))
    b, res = Vector(cout, "f32", r.integers(-64, 65, cout)), mk(rows, cout, whole_numbers(r, rows, cout, 64))
    out, pre = mk(rows, cout), mk(rows, cout)
    ws, work = linear_scratch(rows, cin, cout)
    si, so = cin + pad, cout + pad
    mics.mics_linear(out.t, pre.t, None, None, x.t, w.t, b.v, res.t, rows, cin, cout, act=mics.MICS_ACT_RELU, dtype=CODE[fmt],
                     param_dtype=CODE["f32"], strides=(so, so, so, si, si, so), **work)
    z = mm(x.f64(), w.f64().T) + b.f64()
    assert np.array_equal(pre.f64(), nearest(z, fmt)) and np.array_equal(out.f64(), nearest(np.maximum(z, 0) + res.f64(), fmt))
    dz, dsum, dx = mk(rows, cout, whole_numbers(r, rows, cout, 4)), mk(rows, cin, whole_numbers(r, rows, cin, 64)), mk(rows, cin)
    mics.mics_linear_backward_input(dx.t, dz.t, w.t, dsum.t, rows, cin, cout, dtype=CODE[fmt], strides=(si, so, si, si), **work)
    assert np.array_equal(dx.f64(), nearest(mm(dz.f64(), w.f64()) + dsum.f64(), fmt))
    for grad in ("f32", fmt):
        dw = mk(cout, cin, f=grad)
        mics.mics_linear_backward_weight(dw.t, dz.t, x.t, rows, cin, cout, dtype=CODE[fmt], grad_dtype=CODE[grad], strides=(si, so, si),
                                         **work)
        assert np.array_equal(dw.f64(), nearest(mm(dz.f64().T, x.f64()), grad)), grad
        assert dw.intact()
    assert all(m.intact() for m in (out, pre, dx)) and spared(ws)


@pytest.mark.parametrize("rows,cin,cout,pad,skew,fmt", [s for s in SHAPES[2::2] if s[0] * s[1] * s[2] < 1 << 32])
@pytest.mark.parametrize("act,keep,residual,param", [("gelu", "8", False, None), ("gelu_tanh", "full", True, "f32"), ("silu", "8", True, "bf16"),
                                                     ("none", "no", True, "f16"), ("relu", "both", False, "f32")])
def test_linear(rows, cin, cout, pad, skew, fmt, act, keep, residual, param):
    r = np.random.default_rng(rows + cin)
    mk = lambda n, m, data=None, f=fmt: Matrix(n, m, f, pad, skew, data)               # noqa: E731
    x, w = mk(rows, cin, r.normal(0, 1, (rows, cin))), mk(cout, cin, r.normal(0, cin ** -0.5, (cout, cin)))
    b = Vector(cout, param, r.normal(0, 0.5, cout)) if param else None
    res = mk(rows, cout, r.normal(0, 1, (rows, cout))) if residual else None
    out, pre = mk(rows, cout), mk(rows, cout) if keep in ("full", "both") else None
    eight = keep in ("8", "both")
    codes = mk(rows, cout, f="i8") if eight else None
    scales = Vector(mics.mics_checkpoint_scales(rows, cout), "f32") if eight else None
    ws, work = linear_scratch(rows, cin, cout)
    si, so = cin + pad, cout + pad
    mics.mics_linear(out.t, pre and pre.t, codes and codes.t, scales and scales.v, x.t, w.t, b and b.v, res and res.t, rows, cin, cout,
                     act=ACT[act], dtype=CODE[fmt], param_dtype=CODE[param or "f32"], strides=(so, so, so, si, si, so), **work)
    z, z_size = mm(x.f64(), w.f64().T), ref.scaled(mm(np.abs(x.f64()), np.abs(w.f64()).T), cin)
    if b:
        z, z_size = z + b.f64(), z_size + np.abs(b.f64())
    (y, y_size), (_, steep) = ref.act(z, act), ref.slope(z, act)
    y_size = y_size + z_size * np.maximum(steep, 0.25)           # slopes change by at most 1 where z changes by 1: z is off by far less
    if res:
        y, y_size = y + res.f64(), y_size + np.abs(res.f64())
    assert layer_ref.within(out.f64(), y, y_size, fmt)
    if pre:
        assert layer_ref.within(pre.f64(), z, z_size, fmt)
    if eight:
        back, s = ref.restored(codes.t.cpu().numpy(), scales.v.cpu().numpy().reshape(rows, -1)).astype(np.float64), scales.f64()
        step = np.repeat(s.reshape(rows, -1), 64, axis=1)[:, :cout]
        off = layer_ref.STEPS * layer_ref.U32 * z_size
        assert np.all(np.abs(back - z) <= 0.5 * step + off + 2.0 ** -20 * np.abs(z) + 2.0 ** -100)
        tops = np.zeros((rows, len(s) // rows * 64), np.int32)
        tops[:, :cout] = np.abs(codes.t.cpu().numpy().astype(np.int32))
        assert (tops.reshape(-1, 64).max(1) == 127).all()
        y8 = mk(rows, cout)
        mics.mics_checkpoint_read(y8.t, codes.t, scales.v, rows, cout, act=mics.MICS_ACT_NONE, dtype=CODE[fmt], strides=(so, so))
        assert np.array_equal(y8.f64(), nearest(back, fmt))
        assert codes.intact() and scales.intact() and y8.intact()
    assert out.intact() and (pre is None or pre.intact()) and spared(ws)


@pytest.mark.parametrize("rows,cin,cout,pad,skew,fmt", [s for s in SHAPES[3::2] if s[0] * s[1] * s[2] < 1 << 33])
def test_gradients(rows, cin, cout, pad, skew, fmt):
    r = np.random.default_rng(rows + cin + 1)
    mk = lambda n, m, data=None, f=fmt: Matrix(n, m, f, pad, skew, data)               # noqa: E731
    x, w, dz = mk(rows, cin, r.normal(0, 1, (rows, cin))), mk(cout, cin, r.normal(0, 0.1, (cout, cin))), mk(rows, cout, r.normal(0, 0.3, (rows, cout)))
    ws, work = linear_scratch(rows, cin, cout)
    si, so = cin + pad, cout + pad
    dx, dw = mk(rows, cin), mk(cout, cin)
    mics.mics_linear_backward_input(dx.t, dz.t, w.t, None, rows, cin, cout, dtype=CODE[fmt], strides=(si, so, si, si), **work)
    mics.mics_linear_backward_weight(dw.t, dz.t, x.t, rows, cin, cout, dtype=CODE[fmt], grad_dtype=CODE[fmt], strides=(si, so, si), **work)
    a, b, c = dz.f64(), w.f64(), x.f64()
    assert layer_ref.within(dx.f64(), mm(a, b), ref.scaled(mm(np.abs(a), np.abs(b)), cout), fmt)
    assert layer_ref.within(dw.f64(), mm(a.T, c), ref.scaled(mm(np.abs(a).T, np.abs(c)), rows), fmt)
    assert dx.intact() and dw.intact() and spared(ws)


# rows, cols, pad, skew, format, parameters and gradients
ROWS = [(1, 1, 0, 0, "f32", "f32"), (3, 7, 0, 0, "bf16", "f32"), (2, 9, 4, 1, "bf16", "f32"), (5, 63, 0, 0, "f16", "f16"), (70, 64, 0, 0, "bf16", "bf16"),
        (9, 65, 7, 1, "f16", "f32"), (33, 511, 0, 0, "f32", "f32"), (1030, 513, 3, 1, "bf16", "bf16"), (257, 2048, 0, 0, "bf16", "bf16"),
        (8, 10240, 0, 0, "bf16", "f32"), (300, 4099, 0, 0, "f16", "f16"), (5, 8195, 0, 1, "bf16", "bf16"), (2, 40003, 1, 0, "f32", "f32"),
        (4000, 96, 0, 0, "bf16", "bf16"), (1200, 8, 0, 0, "f32", "bf16"), (64, 32768, 0, 0, "bf16", "bf16")]


def spread(r, rows, cols):
    """Values of every size that an activation treats differently, zeros and a column that is far larger among them."""
    z = r.normal(0, 2, (rows, cols)) * 10.0 ** r.integers(-3, 2, (rows, cols)) * (1 + 30 * (r.random(cols) < 0.02))
    z[r.random((rows, cols)) < 0.05] = 0.0
    return np.clip(z, -3e4, 3e4)


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,param", ROWS)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("bias", [True, False])
def test_activation_and_its_checkpoint(rows, cols, pad, skew, fmt, param, act, bias):
    r = np.random.default_rng(rows + cols)
    mk = lambda data=None, f=fmt: Matrix(rows, cols, f, pad, skew, data)               # noqa: E731
    x, b = mk(spread(r, rows, cols)), Vector(cols, param, r.normal(0, 0.5, cols)) if bias else None
    y, codes, scales = mk(), mk(f="i8"), Vector(mics.mics_checkpoint_scales(rows, cols), "f32")
    s = cols + pad
    mics.mics_activation(y.t, codes.t, scales.v, x.t, b and b.v, rows, cols, act=ACT[act], dtype=CODE[fmt], param_dtype=CODE[param],
                         strides=(s, s, s))
    z = x.f64().astype(np.float32)
    if b:
        z = z + b.f64().astype(np.float32)
    want, steps = ref.checkpoint(z)
    assert np.array_equal(codes.t.cpu().numpy(), want) and np.array_equal(scales.v.cpu().numpy(), steps.ravel())
    assert layer_ref.within(y.f64(), *ref.act(z, act), fmt)
    assert y.intact() and codes.intact() and scales.intact()

    back = ref.restored(want, steps)
    again = mk()
    mics.mics_checkpoint_read(again.t, codes.t, scales.v, rows, cols, act=ACT[act], dtype=CODE[fmt], strides=(s, s))
    assert layer_ref.within(again.f64(), *ref.act(back, act), fmt) and again.intact()

    dy, dx, db = mk(r.normal(0, 0.3, (rows, cols))), mk(), Vector(cols, param)
    n = mics.mics_column_workspace_bytes(rows, cols)
    for z8 in (True, False):
        ws, n = scratch(n)
        mics.mics_activation_backward(dx.t, db.v, dy.t, None if z8 else x.t, codes.t if z8 else None, scales.v if z8 else None, rows, cols,
                                      act=ACT[act], dtype=CODE[fmt], grad_dtype=CODE[param], strides=(s, s, s, s), workspace=ws,
                                      workspace_bytes=n)
        d, size = ref.slope(back if z8 else x.f64(), act)
        d, size = d * dy.f64(), size * np.abs(dy.f64())
        assert layer_ref.within(dx.f64(), d, size, fmt)
        assert layer_ref.within(db.f64(), d.sum(0), size.sum(0), param)
        assert dx.intact() and db.intact() and spared(ws)


def test_parts_of_calls():
    """The checkpoint alone, the activation alone, the bias's gradient alone, the gradient alone, results in the place of inputs."""
    rows, cols = 37, 200
    r = np.random.default_rng(5)
    data = r.normal(0, 2, (rows, cols))
    x, y, codes, scales = Matrix(rows, cols, "bf16", data=data), Matrix(rows, cols, "bf16"), Matrix(rows, cols, "i8"), Vector(rows * 4, "f32")
    key = dict(act=ACT["gelu"], dtype=CODE["bf16"], param_dtype=CODE["bf16"])
    mics.mics_activation(y.t, codes.t, scales.v, x.t, None, rows, cols, **key)
    c2, s2, y2 = Matrix(rows, cols, "i8"), Vector(rows * 4, "f32"), Matrix(rows, cols, "bf16")
    mics.mics_activation(None, c2.t, s2.v, x.t, None, rows, cols, **key)
    mics.mics_activation(y2.t, None, None, x.t, None, rows, cols, **key)
    assert torch.equal(codes.t, c2.t) and torch.equal(scales.v, s2.v) and torch.equal(y.t, y2.t)
    mics.mics_activation(x.t, c2.t, s2.v, x.t, None, rows, cols, **key)                    # in place
    assert torch.equal(x.t, y.t) and torch.equal(codes.t, c2.t)

    n = mics.mics_column_workspace_bytes(rows, cols)
    ws, _ = scratch(n)
    back = dict(act=ACT["gelu"], dtype=CODE["bf16"], grad_dtype=CODE["f32"])
    dy, dx, db = Matrix(rows, cols, "bf16", data=r.normal(0, 1, (rows, cols))), Matrix(rows, cols, "bf16"), Vector(cols, "f32")
    mics.mics_activation_backward(dx.t, db.v, dy.t, None, codes.t, scales.v, rows, cols, workspace=ws, workspace_bytes=n, **back)
    dx2, db2 = Matrix(rows, cols, "bf16"), Vector(cols, "f32")
    mics.mics_activation_backward(None, db2.v, dy.t, None, codes.t, scales.v, rows, cols, workspace=ws, workspace_bytes=n, **back)
    mics.mics_activation_backward(dx2.t, None, dy.t, None, codes.t, scales.v, rows, cols, **back)
    assert torch.equal(dx.t, dx2.t) and torch.equal(db.v, db2.v)
    mics.mics_activation_backward(dy.t, db2.v, dy.t, None, codes.t, scales.v, rows, cols, workspace=ws, workspace_bytes=n, **back)
    assert torch.equal(dx.t, dy.t) and torch.equal(db.v, db2.v)

    w, res = Matrix(cols, cols, "bf16", data=r.normal(0, 0.1, (cols, cols))), Matrix(rows, cols, "bf16", data=data)
    ws, work = linear_scratch(rows, cols, cols)
    out = Matrix(rows, cols, "bf16")
    mics.mics_linear(out.t, None, None, None, y.t, w.t, None, res.t, rows, cols, cols, **key, **work)
    mics.mics_linear(res.t, None, None, None, y.t, w.t, None, res.t, rows, cols, cols, **key, **work)
    assert torch.equal(out.t, res.t)
    d1, d2 = Matrix(rows, cols, "bf16"), Matrix(rows, cols, "bf16", data=data)
    mics.mics_linear_backward_input(d1.t, y.t, w.t, d2.t, rows, cols, cols, dtype=CODE["bf16"], **work)
    mics.mics_linear_backward_input(d2.t, y.t, w.t, d2.t, rows, cols, cols, dtype=CODE["bf16"], **work)
    assert torch.equal(d1.t, d2.t)


def test_no_rows():
    dw, db = Matrix(5, 7, "bf16"), Vector(7, "f32")
    ws, work = linear_scratch(0, 7, 5)
    mics.mics_linear_backward_weight(dw.t, None, None, 0, 7, 5, dtype=CODE["bf16"], grad_dtype=CODE["bf16"], **work)
    mics.mics_activation_backward(None, db.v, None, None, None, None, 0, 7, act=ACT["gelu"], dtype=CODE["bf16"], grad_dtype=CODE["f32"])
    assert not dw.f64().any() and not db.f64().any() and dw.intact() and db.intact()
    mics.mics_linear(None, None, None, None, None, None, None, None, 0, 7, 5, act=0, dtype=0, param_dtype=0)
    mics.mics_linear_backward_input(None, None, None, None, 0, 7, 5, dtype=0)
    mics.mics_activation(None, None, None, None, None, 0, 7, act=1, dtype=0, param_dtype=0)
    mics.mics_checkpoint_read(None, None, None, 0, 7, act=1, dtype=0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["bf16", "f16", "f32"])
def test_infinities_and_nan(fmt):
    """A block that holds one stands for NaN, its neighbours for what they held; a product's row has its own alone."""
    rows, cols = 6, 200
    r = np.random.default_rng(3)
    data = r.normal(0, 1, (rows, cols))
    data[1, 3], data[2, 70], data[3, 199], data[4, 64:128] = np.inf, -np.inf, np.nan, 0.0
    x, y, codes, scales = Matrix(rows, cols, fmt, data=data), Matrix(rows, cols, fmt), Matrix(rows, cols, "i8"), Vector(rows * 4, "f32")
    for act in ref.ACTS:
        mics.mics_activation(y.t, codes.t, scales.v, x.t, None, rows, cols, act=ACT[act], dtype=CODE[fmt], param_dtype=0)
        want, steps = ref.checkpoint(x.f64().astype(np.float32))
        assert np.array_equal(codes.t.cpu().numpy(), want) and np.array_equal(scales.v.cpu().numpy(), steps.ravel(), equal_nan=True)
        got = y.f64()
        assert np.isnan(got[3, 199]) and got[1, 3] == np.inf
        assert got[2, 70] == (-np.inf if act == "none" else 0)
        got[1, 3] = got[2, 70] = got[3, 199] = 0
        assert np.isfinite(got).all()
        dy, dx = Matrix(rows, cols, fmt, data=np.ones((rows, cols))), Matrix(rows, cols, fmt)
        mics.mics_activation_backward(dx.t, None, dy.t, None, codes.t, scales.v, rows, cols, act=ACT[act], dtype=CODE[fmt], grad_dtype=0)
        back = ref.restored(want, steps)
        bad = np.isnan(back)
        assert bad.sum() == 64 + 64 + 8
        if act != "none":
            assert np.array_equal(np.isnan(dx.f64()), bad)
        mics.mics_activation_backward(dx.t, None, dy.t, x.t, None, None, rows, cols, act=ACT[act], dtype=CODE[fmt], grad_dtype=0)
        got = dx.f64()
        assert got[1, 3] == 1 and got[2, 70] == (1 if act == "none" else 0) and np.isnan(got[3, 199]) == (act != "none")
    w, out = Matrix(96, cols, fmt, data=r.normal(0, 1, (96, cols))), Matrix(rows, 96, fmt)
    ws, work = linear_scratch(rows, cols, 96)
    mics.mics_linear(out.t, None, None, None, x.t, w.t, None, None, rows, cols, 96, act=0, dtype=CODE[fmt], param_dtype=0, **work)
    got = out.f64()
    assert not np.isfinite(got[1:4]).any() and np.isfinite(got[[0, 4, 5]]).all()


def test_far_values_of_activations():
    """Where exponentials overflow and underflow: the limits, and slopes of 0 and 1."""
    z = np.array([[-3e38, -1e30, -1e12, -1e4, -200, -89, -20, -13.2, -1e-30, 0, 1e-30, 13.2, 20, 89, 200, 1e4, 1e12, 1e30, 3e38]])
    x, y, dx = (Matrix(1, z.size, "f32", data=z) for _ in range(3))
    dy = Matrix(1, z.size, "f32", data=np.ones_like(z))
    for act in ref.ACTS:
        key = dict(act=ACT[act], dtype=CODE["f32"])
        mics.mics_activation(y.t, None, None, x.t, None, 1, z.size, param_dtype=0, **key)
        mics.mics_activation_backward(dx.t, None, dy.t, x.t, None, None, 1, z.size, grad_dtype=0, **key)
        with np.errstate(all="ignore"):
            z32 = x.f64()
            v, size = ref.act(z32, act)
            assert layer_ref.within(y.f64(), v, np.where(np.isfinite(size), size, np.abs(v)), "f32"), act
            far = np.abs(z32) > 100
            s = np.where(far & (act != "none"), (z32 > 0).astype(float), ref.slope(np.where(far, 0, z32), act)[0])
        assert np.abs(dx.f64() - s).max() < 2e-6, act


@pytest.mark.parametrize("rows,cin,cout", [(8, 2048, 640), (300, 1100, 650), (64, 4096, 512), (1, 4000, 24)])
def test_results_in_the_place_of_what_is_added(rows, cin, cout):
    """Also where a second launch joins parts."""
    r = np.random.default_rng(rows)
    x, w = Matrix(rows, cin, "bf16", data=r.normal(0, 1, (rows, cin))), Matrix(cout, cin, "bf16", data=r.normal(0, cin ** -0.5, (cout, cin)))
    ws, work = linear_scratch(rows, cin, cout)
    data = r.normal(0, 1, (rows, cout))
    out, res = Matrix(rows, cout, "bf16"), Matrix(rows, cout, "bf16", data=data)
    key = dict(act=ACT["gelu"], dtype=CODE["bf16"], param_dtype=CODE["bf16"])
    mics.mics_linear(out.t, None, None, None, x.t, w.t, None, res.t, rows, cin, cout, **key, **work)
    mics.mics_linear(res.t, None, None, None, x.t, w.t, None, res.t, rows, cin, cout, **key, **work)
    assert torch.equal(out.t, res.t)
    dz, d1, d2 = Matrix(rows, cout, "bf16", data=data), Matrix(rows, cin, "bf16"), Matrix(rows, cin, "bf16", data=r.normal(0, 1, (rows, cin)))
    mics.mics_linear_backward_input(d1.t, dz.t, w.t, d2.t, rows, cin, cout, dtype=CODE["bf16"], **work)
    mics.mics_linear_backward_input(d2.t, dz.t, w.t, d2.t, rows, cin, cout, dtype=CODE["bf16"], **work)
    assert torch.equal(d1.t, d2.t)


@pytest.mark.parametrize("rows,cin,cout", [(8, 2048, 640), (300, 1100, 650), (1, 4000, 24), (129, 64, 131)])
@pytest.mark.parametrize("fmt", ["bf16", "f32"])
def test_what_is_kept_in_the_place_of_the_residual(rows, cin, cout, fmt):
    r = np.random.default_rng(rows)
    x, w = Matrix(rows, cin, fmt, data=r.normal(0, 1, (rows, cin))), Matrix(cout, cin, fmt, data=r.normal(0, cin ** -0.5, (cout, cin)))
    ws, work = linear_scratch(rows, cin, cout)
    out, pre, again = (Matrix(rows, cout, fmt) for _ in range(3))
    res = Matrix(rows, cout, fmt, data=r.normal(0, 1, (rows, cout)))
    key = dict(act=ACT["gelu"], dtype=CODE[fmt], param_dtype=0)
    mics.mics_linear(out.t, pre.t, None, None, x.t, w.t, None, res.t, rows, cin, cout, **key, **work)
    mics.mics_linear(again.t, res.t, None, None, x.t, w.t, None, res.t, rows, cin, cout, **key, **work)
    assert torch.equal(out.t, again.t) and torch.equal(pre.t, res.t)


@pytest.mark.parametrize("fmt,far", [("bf16", 1 << 22), ("f32", 1 << 21)])
def test_rows_too_far_apart_for_32_bit_offsets(fmt, far):
    rows, cin, cout = 3, 40, 24
    r = np.random.default_rng(1)
    x, w, dz = (Matrix(n, m, fmt, far, 0, whole_numbers(r, n, m, 8)) for n, m in ((rows, cin), (cout, cin), (rows, cout)))
    ws, work = linear_scratch(rows, cin, cout)
    out, dx, dw = Matrix(rows, cout, fmt), Matrix(rows, cin, fmt), Matrix(cout, cin, "f32")
    mics.mics_linear(out.t, None, None, None, x.t, w.t, None, None, rows, cin, cout, act=0, dtype=CODE[fmt], param_dtype=0,
                     strides=(cout, cout, cout, x.stride, w.stride, cout), **work)
    mics.mics_linear_backward_input(dx.t, dz.t, w.t, None, rows, cin, cout, dtype=CODE[fmt], strides=(cin, dz.stride, w.stride, cin), **work)
    mics.mics_linear_backward_weight(dw.t, dz.t, x.t, rows, cin, cout, dtype=CODE[fmt], grad_dtype=CODE["f32"],
                                     strides=(cin, dz.stride, x.stride), **work)
    assert np.array_equal(out.f64(), nearest(x.f64() @ w.f64().T, fmt)) and np.array_equal(dx.f64(), nearest(dz.f64() @ w.f64(), fmt))
    assert np.array_equal(dw.f64(), dz.f64().T @ x.f64())


@pytest.mark.parametrize("fmt,small,large", [("f16", 2.0 ** -20, 2.0 ** 10), ("bf16", 2.0 ** -130, 2.0 ** 100)])
@pytest.mark.parametrize("rows", [3, 200])
def test_subnormal_elements_count(fmt, small, large, rows):
    x, w = Matrix(rows, 64, fmt, data=np.full((rows, 64), small)), Matrix(40, 64, fmt, data=np.full((40, 64), large))
    out = Matrix(rows, 40, "bf16" if fmt == "bf16" else "f16")
    ws, work = linear_scratch(rows, 64, 40)
    assert (x.f64() == small).all()
    mics.mics_linear(out.t, None, None, None, x.t, w.t, None, None, rows, 64, 40, act=0, dtype=CODE[fmt], param_dtype=0, **work)
    assert (out.f64() == 64 * small * large).all()


def test_nan_behind_the_ends_of_rows_is_not_read_into_sums():
    """What lies between rows, and rows that belong to others, hold NaN."""
    for fmt in ("bf16", "f32"):
        for rows, cin, cout, pad in ((5, 70, 33, 10), (150, 201, 130, 7), (300, 1001, 260, 3)):
            r = np.random.default_rng(cin)
            x, w, dz = (Matrix(n, m, fmt, pad, 1, whole_numbers(r, n, m, 4)) for n, m in ((rows, cin), (cout, cin), (rows, cout)))
            for m in (x, w, dz):
                keep = m.t.clone()
                m.whole.fill_(float("nan"))
                m.t.copy_(keep)
            ws, work = linear_scratch(rows, cin, cout)
            out, dx, dw = Matrix(rows, cout, fmt), Matrix(rows, cin, fmt), Matrix(cout, cin, "f32")
            codes, scales = Matrix(rows, cout, "i8"), Vector(mics.mics_checkpoint_scales(rows, cout), "f32")
            work["workspace"].fill_(0xFF)
            mics.mics_linear(out.t, None, codes.t, scales.v, x.t, w.t, None, None, rows, cin, cout, act=0, dtype=CODE[fmt], param_dtype=0,
                             strides=(cout, cout, cout, x.stride, w.stride, cout), **work)
            work["workspace"].fill_(0xFF)
            mics.mics_linear_backward_input(dx.t, dz.t, w.t, None, rows, cin, cout, dtype=CODE[fmt], strides=(cin, dz.stride, w.stride, cin),
                                            **work)
            work["workspace"].fill_(0xFF)
            mics.mics_linear_backward_weight(dw.t, dz.t, x.t, rows, cin, cout, dtype=CODE[fmt], grad_dtype=CODE["f32"],
                                             strides=(cin, dz.stride, x.stride), **work)
            z = x.f64() @ w.f64().T
            assert np.array_equal(out.f64(), nearest(z, fmt)) and np.array_equal(dw.f64(), dz.f64().T @ x.f64())
            assert np.array_equal(dx.f64(), nearest(dz.f64() @ w.f64(), fmt))
            want, steps = ref.checkpoint(z.astype(np.float32))
            assert np.array_equal(codes.t.cpu().numpy(), want) and np.array_equal(scales.f64(), steps.ravel().astype(np.float64))
