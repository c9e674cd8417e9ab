"""Every kernel of the log probabilities and of their gradient against the 64-bit reference, at sizes that reach it."""
import numpy as np
import pytest
import torch

import layer_ref as ref
from logprobs_shapes import GRADIENTS, SHAPES
from test_gpu_layer_ops import CODE, Matrix, get, intact, run_logprobs, vector

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
KINDS = 9


def fill(x, seed):
    """Row r is of kind r mod 9: plain; half of it masked; all but a few masked; integers, with many ties; NaN among them; an infinity;
    one value throughout; nothing but -inf; ascending, so that every part of it holds better ones than those before."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    for r0 in range(0, x.rows, 64):
        t = x.t[r0:r0 + 64]
        v = torch.empty(t.shape, device=DEV).normal_(0.0, 3.0, generator=gen)
        u = torch.rand(t.shape, device=DEV, generator=gen)
        kind = (torch.arange(r0, r0 + t.shape[0], device=DEV) % KINDS)[:, None]
        v = torch.where((kind == 1) & (u < 0.5) | (kind == 2) & (u < 0.9995) | (kind == 7), float("-inf"), v)
        v = torch.where(kind == 3, v.round(), v)
        v = torch.where((kind == 4) & (u < 8.0 / x.cols), float("nan"), v)
        v = torch.where((kind == 5) & (torch.arange(x.cols, device=DEV) == x.cols // 3), float("inf"), v)
        v = torch.where(kind == 6, 2.5, v)
        v = torch.where(kind == 8, torch.arange(x.cols, device=DEV) * (6.0 / x.cols), v)
        t.copy_(v)
    return x


def sample(rows):
    """One row of every kind, the first and the last."""
    return sorted({k for k in (*range(KINDS), rows // 2, rows - 1) if k < rows})


def targets_of(rows, cols):
    r = np.random.default_rng(rows)
    t = r.integers(0, cols, rows)
    return np.where(r.random(rows) < 0.1, -1, t)


def grown(size, serial):
    """Bounds for lanes that add up `serial` numbers one after the other, where the reference's allow for STEPS roundings in all: 60
    of them besides the lane's."""
    return size * max(1.0, (serial + 60) / ref.STEPS)


def numbers(x, rows):
    return x.t[torch.tensor(rows, device=DEV)].double().cpu().numpy()


def same_bits(a, b):
    return a.keys() == b.keys() and all(np.array_equal(a[k], b[k], equal_nan=a[k].dtype.kind == "f") for k in a)


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,top,runs", SHAPES)
def test_every_kernel(rows, cols, pad, skew, fmt, top, runs):
    lanes, _, uncached, splits = runs
    x, targets = fill(Matrix(rows, cols, fmt, pad, skew), rows + cols), targets_of(rows, cols)
    got, at = run_logprobs(x, targets, top), sample(rows)
    want, serial = ref.logprobs(numbers(x, at), targets[at], top), -(-cols // (splits * lanes)) + 8
    for name in ("logprob", "entropy", "lse", "top"):
        value, size = want[name]
        assert ref.within(got[name][at], value, grown(size, serial), "f32"), name
    assert np.array_equal(got["ids"][at], want["ids"])
    plain = run_logprobs(x, targets, top, entropy=False)
    for name in ("logprob", "lse", "ids", "top"):
        assert np.array_equal(got[name], plain[name], equal_nan=got[name].dtype.kind == "f"), name
    if uncached:           # the halves are small enough for the caches, and nothing else differs
        half = rows // 2
        for lo, hi in ((0, half), (half, rows)):
            part = Matrix.__new__(Matrix)
            part.__dict__.update(x.__dict__, rows=hi - lo, t=x.t[lo:hi])
            cached = run_logprobs(part, targets[lo:hi], top)
            assert same_bits(cached, {k: v[lo:hi] for k, v in got.items()})


@pytest.mark.parametrize("rows,cols,pad,skew,fmt,unkept", GRADIENTS)
@pytest.mark.parametrize("with_entropy", [False, True])
def test_every_kernel_of_the_gradient(rows, cols, pad, skew, fmt, unkept, with_entropy):
    x, t = Matrix(rows, cols, fmt, pad, skew), torch.from_numpy(targets_of(rows, cols)).to(DEV)
    if rows > 10 ** 5:
        x.t.normal_(0.0, 3.0)
    else:
        fill(x, rows + cols)
    lse, ent, g, h = (vector(rows, "f32") for _ in range(4))
    for r0 in range(0, rows, 1 << 16 if cols < 100 else 64):
        r1 = min(rows, r0 + (1 << 16 if cols < 100 else 64))
        wide = x.t[r0:r1].double()
        of = torch.logsumexp(wide, 1)
        of = torch.where(torch.isposinf(of), float("nan"), of)             # as the forward pass leaves it
        logp = wide - of[:, None]
        p = logp.exp()
        lse.v[r0:r1] = of.float()
        ent.v[r0:r1] = torch.where(torch.isneginf(of), 0.0, -torch.where(p == 0, 0.0, p * logp).sum(1)).float()
    g.v.normal_()
    h.v.normal_()
    g.v[3:7:2] = 0.0
    dx = Matrix(rows, cols, fmt, pad, skew)

    def call(to, lo=0, hi=rows):
        mics.mics_token_logprobs_backward(to.t[lo:hi], x.t[lo:hi], t[lo:hi], lse.v[lo:hi], ent.v[lo:hi] if with_entropy else None, g.v[lo:hi],
                                          h.v[lo:hi] if with_entropy else None, hi - lo, cols, dtype=CODE[fmt], strides=(x.stride,) * 2)

    call(dx)
    at = sample(rows)
    some = lambda v: get(v)[at]                                                        # noqa: E731
    want, size = ref.logprobs_backward(numbers(x, at), t.cpu().numpy()[at], some(lse), some(ent) if with_entropy else None, some(g),
                                       some(h) if with_entropy else None)
    assert ref.within(numbers(dx, at), want, size, fmt) and intact(dx)
    if unkept:             # parts that a cache keeps are the same
        other, parts = Matrix(rows, cols, fmt, pad, skew), 4
        for k in range(parts):
            call(other, rows * k // parts, rows * (k + 1) // parts)
        assert torch.equal(other.whole.view(other.bits), dx.whole.view(dx.bits))
