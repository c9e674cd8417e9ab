"""Products that write a checkpoint, in every kernel that does (test_linear_codes_rules.py holds the sizes to that): sums of whole numbers
are exact, so codes and scales are compared bit by bit, with all else that the epilogue leaves."""
import numpy as np
import pytest

import linear_ref as ref
from linear_shapes import WITH_CODES

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

from test_gpu_linear import CODE, Matrix, Vector, linear_scratch, mm, nearest, spared, whole_numbers      # noqa: E402


@pytest.mark.parametrize("rows,cin,cout,pad,skew,fmt", WITH_CODES)
def test_checkpoints_of_whole_numbers_are_exact(rows, cin, cout, pad, skew, fmt):
    r = np.random.default_rng(rows + 3 * cin + 5 * cout)
    mk = lambda n, m, data=None, f=fmt: Matrix(n, m, f, pad, skew, data)               # noqa: E731
    x, w = mk(rows, cin, whole_numbers(r, rows, cin, 8)), mk(cout, cin, whole_numbers(r, cout, cin, 8))
    b, res = Vector(cout, "f32", r.integers(-64, 65, cout)), mk(rows, cout, whole_numbers(r, rows, cout, 64))
    out, pre, codes = mk(rows, cout), mk(rows, cout), mk(rows, cout, f="i8")
    scales = Vector(mics.mics_checkpoint_scales(rows, cout), "f32")
    ws, work = linear_scratch(rows, cin, cout)
    si, so = cin + pad, cout + pad
    z = mm(x.f64(), w.f64().T) + b.f64()                         # below 2^24: 64 * 13592 + 64
    want, steps = ref.checkpoint(z.astype(np.float32))
    key = dict(act=mics.MICS_ACT_RELU, dtype=CODE[fmt], param_dtype=CODE["f32"], strides=(so, so, so, si, si, so))
    mics.mics_linear(out.t, pre.t, codes.t, scales.v, x.t, w.t, b.v, res.t, rows, cin, cout, **key, **work)
    assert np.array_equal(codes.t.cpu().numpy(), want) and np.array_equal(scales.v.cpu().numpy(), steps.ravel())
    assert np.array_equal(pre.f64(), nearest(z, fmt)) and np.array_equal(out.f64(), nearest(np.maximum(z, 0) + res.f64(), fmt))
    # as a layer keeps it: the checkpoint alone beside the result
    out2, codes2, scales2 = mk(rows, cout), mk(rows, cout, f="i8"), Vector(len(scales.v), "f32")
    mics.mics_linear(out2.t, None, codes2.t, scales2.v, x.t, w.t, b.v, None, rows, cin, cout, **key, **work)
    assert np.array_equal(codes2.t.cpu().numpy(), want) and np.array_equal(scales2.v.cpu().numpy(), steps.ravel())
    assert np.array_equal(out2.f64(), nearest(np.maximum(z, 0), fmt))
    assert all(m.intact() for m in (out, pre, codes, scales, out2, codes2, scales2)) and spared(ws)
