"""Gradients of the linear layer and of activations against differences of the forward calls themselves."""
import numpy as np
import pytest
import torch

import layer_ref
import linear_ref as ref

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
F32 = mics.MICS_DTYPE_F32
ACT = {n: i for i, n in enumerate(ref.ACTS)}


@pytest.mark.parametrize("rows,cin,cout", [(3, 40, 24), (20, 64, 130), (70, 131, 66), (140, 96, 256)])
def test_products(rows, cin, cout):
    """The sum of dz * (x W^T + b) is linear in x and in W: with small whole numbers all of it is exact, differences too."""
    r = np.random.default_rng(cin)
    whole = lambda *s: torch.from_numpy(r.integers(-4, 5, s)).float().to(DEV)          # noqa: E731
    x, w, dz = whole(rows, cin), whole(cout, cin), whole(rows, cout)
    n = mics.mics_linear_workspace_bytes(rows, cin, cout)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
    work = dict(workspace=ws, workspace_bytes=n)
    dx, dw, out = torch.empty_like(x), torch.empty_like(w), torch.empty_like(dz)
    mics.mics_linear_backward_input(dx, dz, w, None, rows, cin, cout, dtype=F32, **work)
    mics.mics_linear_backward_weight(dw, dz, x, rows, cin, cout, dtype=F32, grad_dtype=F32, **work)

    def value():
        mics.mics_linear(out, None, None, None, x, w, None, None, rows, cin, cout, act=0, dtype=F32, param_dtype=F32, **work)
        return float((out.double() * dz.double()).sum())

    before = value()
    for m, grad in ((x, dx), (w, dw)):
        for i, j in [(0, 0), (m.shape[0] - 1, cin - 1)] + [(int(r.integers(m.shape[0])), int(r.integers(cin))) for _ in range(8)]:
            m[i, j] += 1
            assert value() - before == float(grad[i, j]), (i, j)
            m[i, j] -= 1


@pytest.mark.parametrize("act", ref.ACTS)
def test_activations(act):
    """(f(z + h) - f(z - h)) / 2h in binary32 at h = 2^-6: off by h^2 / 6 times the third derivative, which is below 1, and by what both
    values may be off (layer_ref.within) divided by 2h."""
    h = 2.0 ** -6
    z = np.arange(-384, 385) / 64.0                              # all three points are binary32 numbers
    if act == "relu":
        z = z[np.abs(z) > h]
    n = z.size
    points = torch.from_numpy(np.stack([z + h, z - h])).float().to(DEV)
    y, zt = torch.empty_like(points), torch.from_numpy(z.reshape(1, n)).float().to(DEV)
    mics.mics_activation(y, None, None, points, None, 2, n, act=ACT[act], dtype=F32, param_dtype=F32)
    dx = torch.empty_like(zt)
    mics.mics_activation_backward(dx, None, torch.ones_like(zt), zt, None, None, 1, n, act=ACT[act], dtype=F32, grad_dtype=F32)
    up, down = y.double().cpu().numpy()
    size = sum(layer_ref.STEPS * layer_ref.U32 * s + layer_ref.U32 * np.abs(v) for v, s in (ref.act(z + h, act), ref.act(z - h, act)))
    slope = layer_ref.STEPS * layer_ref.U32 * ref.slope(z, act)[1] + layer_ref.U32
    off = np.abs((up - down) / (2 * h) - dx.double().cpu().numpy()[0])
    assert np.all(off <= h * h / 6 + size / (2 * h) + slope)
