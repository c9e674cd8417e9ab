"""Checkpoints of blocks whose largest magnitude lies at the end of the range: finite elements stand for code * scale as all others do,
in reads and in the activation's gradient.  Codes and scales are compared bit by bit with linear_ref.checkpoint, what they stand
for with linear_ref.restored.  127 times the scale of a block whose largest is the largest finite binary32 number rounds to
infinity: there alone a finite element stands for one."""
import numpy as np
import pytest
import torch

import layer_ref
import linear_ref as ref

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"bf16": mics.MICS_DTYPE_BF16, "f16": mics.MICS_DTYPE_F16, "f32": mics.MICS_DTYPE_F32}
ACT = {n: i for i, n in enumerate(ref.ACTS)}
F32_MOST = float(np.finfo(np.float32).max)
# the least of which 128 steps are no finite binary32 number lies between the first two
TOPS = {"bf16": [float.fromhex("0x1.fcp127"), float.fromhex("0x1.fep127"), 2.0 ** 120], "f16": [65504.0, 32768.0],
        "f32": [float.fromhex("0x1.fcp127"), float.fromhex("0x1.fc0002p127"), float.fromhex("0x1.fep127"), float.fromhex("0x1.fffffcp127"), F32_MOST]}


def on_gpu(data, fmt):
    return torch.from_numpy(np.ascontiguousarray(data, np.float64)).to(TORCH[fmt]).to(DEV)


def blocks(fmt, cols):
    """A row for each top and sign of it, in every block of the row: zeros, small numbers, parts of the top, the lowest value that a
    mask has."""
    r = np.random.default_rng(cols)
    rows = []
    for top in TOPS[fmt]:
        for sign in (1.0, -1.0):
            row = r.choice([0.0, 1.0, -3.0, top / 2, -top / 3, top / 127, -top / 200, top / 300], cols)
            row[::64] = sign * top
            rows.append(row)
    return np.stack(rows)


def f64(t):
    return t.double().cpu().numpy()


def within(*args):
    with np.errstate(invalid="ignore"):
        return layer_ref.within(*args)


def nearest(x, fmt):
    with np.errstate(over="ignore"):
        return torch.from_numpy(np.asarray(x, np.float32)).to(TORCH[fmt]).double().numpy()


@pytest.mark.parametrize("cols", [64, 77, 640, 3])
@pytest.mark.parametrize("fmt", list(TOPS))
def test_blocks_at_the_end_of_the_range(fmt, cols):
    x = on_gpu(blocks(fmt, cols), fmt)
    rows = x.shape[0]
    assert torch.isfinite(x).all()
    want, steps = ref.checkpoint(f64(x).astype(np.float32))
    assert np.isfinite(steps).all()
    with np.errstate(over="ignore"):
        back = ref.restored(want, steps)
    assert np.isfinite(back[np.abs(f64(x)).max(1) < F32_MOST]).all() and not np.isnan(back).any()
    codes, scales = torch.empty(rows, cols, dtype=torch.int8, device=DEV), torch.empty(mics.mics_checkpoint_scales(rows, cols), device=DEV)
    y, dx, dy = torch.empty_like(x), torch.empty_like(x), torch.ones_like(x)
    z = back.astype(np.float64)
    far = np.abs(z) > 100
    for act in ref.ACTS:
        key = dict(act=ACT[act], dtype=CODE[fmt])
        mics.mics_activation(y, codes, scales, x, None, rows, cols, param_dtype=0, **key)
        assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), steps.ravel())
        # far from zero an activation is z or 0, its slope 1 or 0; at zero, and near it, the formulas'
        mics.mics_checkpoint_read(y, codes, scales, rows, cols, **key)
        if act in ("none", "relu"):
            assert np.array_equal(f64(y), nearest(back if act == "none" else np.maximum(back, 0), fmt)), act
        else:
            near, size = ref.act(np.where(far, 0.0, z), act)
            v = np.where(far, np.maximum(z, 0.0), near)
            with np.errstate(over="ignore"):
                v = np.where(np.isinf(nearest(v, fmt)), np.inf, v)
            assert within(f64(y), v, np.where(far, np.where(np.isinf(v), 0.0, v), size), fmt), act
        mics.mics_activation_backward(dx, None, dy, None, codes, scales, rows, cols, grad_dtype=0, **key)
        s, size = ref.slope(np.where(far, 0.0, z), act)
        s = s if act == "none" else np.where(far, z > 0, s)
        assert within(f64(dx), s, np.where(far, 1.0, size), fmt), act


@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("fmt", ["bf16", "f32"])
def test_products_at_the_end_of_the_range(fmt, rows):
    """A product of one term, so that z is what one of its factors holds: the epilogue's checkpoint, read back."""
    cin, cout, top = 16, 130, TOPS[fmt][-3 if fmt == "f32" else 1]
    a, b = np.zeros((rows, cin)), np.zeros((cout, cin))
    a[:, 0] = 1.0
    b[:, 0] = np.random.default_rng(1).choice([0.0, 1.0, top / 2, -top / 3], cout)
    b[5, 0], b[70, 0], b[129, 0] = top, -top, top
    x, w = on_gpu(a, fmt), on_gpu(b, fmt)
    out, z = (torch.empty(rows, cout, dtype=TORCH[fmt], device=DEV) for _ in range(2))
    codes, scales = torch.empty(rows, cout, dtype=torch.int8, device=DEV), torch.empty(mics.mics_checkpoint_scales(rows, cout), device=DEV)
    n = mics.mics_linear_workspace_bytes(rows, cin, cout)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
    mics.mics_linear(out, None, codes, scales, x, w, None, None, rows, cin, cout, act=0, dtype=CODE[fmt], param_dtype=0, workspace=ws,
                     workspace_bytes=n)
    exact = np.broadcast_to(f64(w)[:, 0], (rows, cout))
    want, steps = ref.checkpoint(exact.astype(np.float32))
    assert np.array_equal(f64(out), exact)
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), steps.ravel())
    mics.mics_checkpoint_read(z, codes, scales, rows, cout, act=0, dtype=CODE[fmt])
    assert np.isfinite(f64(z)).all() and np.array_equal(f64(z), nearest(ref.restored(want, steps), fmt))
