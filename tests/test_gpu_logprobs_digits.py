"""Digits of log probabilities that bounds on sums of order one cannot see: small entropies, gradients of far logits."""
import numpy as np
import pytest
import torch

from test_gpu_layer_ops import Matrix, run_logprobs

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

U = 2.0 ** -24

# rows, vocab, type, alternatives, columns of the lower and of the higher outcome: the same lane meets the lower one first, in a
# vector of an earlier pass of its loop (two vectors of 256 lanes, four of 256, four of 1024; the last two in splits)
PEAKED = [(300, 5000, "f32", 0, 16, 4112), (300, 5003, "bf16", 5, 16, 4112), (300, 40000, "bf16", 0, 24, 16408),
          (300, 40000, "f32", 5, 24, 16408), (300, 39997, "f16", 1, 27, 16411), (130, 70000, "f32", 0, 40, 32808),
          (130, 70001, "bf16", 5, 40, 32808), (100, 131072, "f32", 0, 40, 32808), (100, 131072, "bf16", 5, 65576, 98344),
          (3, 5, "f32", 2, 0, 4), (300, 5000, "f32", 2, 4112, 16), (300, 5000, "f32", 0, 9, 4999)]


@pytest.mark.parametrize("rows,cols,fmt,top,low,high", PEAKED)
def test_rows_with_two_outcomes(rows, cols, fmt, top, low, high):
    """Two outcomes g apart, e = exp(-g): Z = 1 + e, entropy = log Z + g e / Z, which is small beside either's magnitude at any
    other base than the larger logit.  Against that base, with U = 2^-24: the exponent g is rounded twice and multiplied by a rounded
    constant, and the exponential is within 2 U: e is off by (2.5 g + 4) U e at most; Z, in [1, 2), by U more, once (all other
    summands are 0); the logarithm and the product and quotient of the second term by a few U of themselves."""
    gap, m = np.linspace(0.5, 12.0, rows), 3.0
    data = np.full((rows, cols), -np.inf)
    data[:, low], data[:, high] = m - gap, m
    x = Matrix(rows, cols, fmt, data=data)
    targets = np.where(np.arange(rows) % 2, low, high)
    got = run_logprobs(x, targets, top)
    x64 = x.f64()
    g = x64[:, high] - x64[:, low]
    e = np.exp(-g)
    entropy, of_high = np.log1p(e) + g * e / (1 + e), -np.log1p(e)
    of_low = of_high - g
    near, far = U * (2 + (3 * g + 12) * e), U * (2 + (3 * g + 12) * e + 3 * g)
    worst = {"entropy": np.abs(got["entropy"] - entropy) / (U * (2 + (3 * g + 12) * (1 + g) * e)),
             "logprob": np.abs(got["logprob"] - np.where(np.arange(rows) % 2, of_low, of_high)) / np.where(np.arange(rows) % 2, far, near)}
    if top:
        assert np.array_equal(got["ids"][:, 0], np.full(rows, high))
        worst["first"] = np.abs(got["top"][:, 0] - of_high) / near
    if top > 1:
        assert np.array_equal(got["ids"][:, 1], np.full(rows, low))
        worst["second"] = np.abs(got["top"][:, 1] - of_low) / far
    worst = {k: float(v.max()) for k, v in worst.items()}
    assert max(worst.values()) <= 1, worst


@pytest.mark.parametrize("rows,cols", [(5, 7), (300, 5003), (40, 20000)])
@pytest.mark.parametrize("of_entropy", [False, True])
@pytest.mark.parametrize("moved", [False, True])
def test_gradient_of_far_logits_in_32_bits(rows, cols, of_entropy, moved):
    """Probabilities down to e^-85.  x - lse is exact where lse is 0, else within U |x - lse|; the exponential is within 2 U and a
    correction by U more, the factor (1, or x - lse with an entropy of 0) and the product are rounded once each."""
    r = np.random.default_rng(rows + cols)
    x = Matrix(rows, cols, "f32", data=-85.0 * r.random((rows, cols)))
    shift = r.normal(size=rows).astype(np.float32) if moved else np.zeros(rows, np.float32)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")              # noqa: E731
    ones, none = np.ones(rows, np.float32), np.zeros(rows, np.float32)
    # all targets in column 0, which is left out below
    g, h = (none, ones) if of_entropy else (ones, none)
    dx = Matrix(rows, cols, "f32")
    mics.mics_token_logprobs_backward(dx.t, x.t, up(np.zeros(rows, np.int64)), up(shift), up(none) if of_entropy else None, up(g),
                                      up(h) if of_entropy else None, rows, cols, dtype=mics.MICS_DTYPE_F32)
    logp = x.f64() - shift.astype(np.float64)[:, None]
    want = -np.exp(logp) * (logp if of_entropy else 1.0)
    bound = U * (8 + (2 if of_entropy else 1) * moved * np.abs(logp)) * np.abs(want)
    # a logarithm of a probability near 1 is itself the difference
    bound += U * moved * np.abs(x.f64()) * np.exp(logp) * of_entropy
    worst = float((np.abs(dx.f64() - want) / bound)[:, 1:].max())
    assert worst <= 1, worst
