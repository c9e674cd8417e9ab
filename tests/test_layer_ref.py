"""The 64-bit reference of the operators between gather and reduction: the generator against its published answers, the
gradients against differences."""
import numpy as np
import pytest

import layer_ref as ref


@pytest.mark.parametrize("counter,key,answer", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_gives_the_published_answers(counter, key, answer):
    got = ref.philox_words([np.array([c], np.uint64) for c in counter], key[0] | key[1] << 32)
    assert tuple(int(w) for w in got[0]) == answer


@pytest.mark.parametrize("drop", [0.1, 0.5, 0.9])
def test_share_and_mean_of_what_dropout_keeps(drop):
    rows, cols = 400, 1001
    k = ref.kept(rows, cols, drop, 12345, 1 << 40)
    share, n = 1 - ref.threshold(drop) / 65536, rows * cols
    assert abs(k.mean() - share) < 5 * np.sqrt(share * (1 - share) / n)
    # neighbours, rows and the halves of a word are not related
    centred = k - share
    for other in (np.roll(centred, 1, 1), np.roll(centred, 1, 0), np.roll(centred, 8, 1)):
        assert abs((centred * other).mean()) < 5 * share * (1 - share) / np.sqrt(n)


def numeric(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + eps
        up = f()
        x[i] = old - eps
        down = f()
        x[i] = old
        g[i] = (up - down) / (2 * eps)
    return g


@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_gradients_of_the_block_against_differences(drop):
    r = np.random.default_rng(3)
    rows, cols, key = 3, 11, (77, 5)
    x, res, dy, dsum = (r.normal(size=(rows, cols)) for _ in range(4))
    bias, weight, nb = (r.normal(size=cols) for _ in range(3))

    def forward():
        s, _ = ref.bias_dropout_add(x, bias, res, drop, *key)
        return s, ref.layer_norm(s, np.abs(s), weight, nb, 1e-3)

    def loss():
        s, out = forward()
        return (out[0][0] * dy).sum() + (s * dsum).sum()

    s, (_, (mean, _), (rstd, _)) = forward()
    got = ref.block_backward(dy, dsum, s, mean, rstd, weight, drop, *key)
    for (value, _), wrt in zip(got, (x, res, bias, weight, nb)):
        assert np.allclose(value, numeric(loss, wrt), rtol=1e-6, atol=1e-7)


def test_gradient_of_log_probabilities_against_differences():
    r = np.random.default_rng(4)
    x = r.normal(size=(4, 9)) * 2
    x[2, 5] = -np.inf
    t, g, h = np.array([3, -1, 0, 8]), r.normal(size=4), r.normal(size=4)

    def loss():
        o = ref.logprobs(x, t, 0)
        return (o["logprob"][0] * g).sum() + (o["entropy"][0] * h).sum()

    o = ref.logprobs(x, t, 0)
    got, _ = ref.logprobs_backward(x, t, o["lse"][0], o["entropy"][0], g, h)
    want = numeric(loss, x)
    fine = np.isfinite(x)
    assert np.allclose(got[fine], want[fine], rtol=1e-6, atol=1e-7) and got[2, 5] == 0


def test_log_probabilities_in_closed_form():
    o = ref.logprobs(np.array([[0.0, 0.0, -np.inf, 0.0], [-np.inf] * 4, [np.nan, 1.0, np.inf, 1.0]]), np.array([1, 2, 0]), 4)
    assert np.allclose(o["lse"][0][0], np.log(3)) and np.allclose(o["entropy"][0][0], np.log(3))
    assert np.isneginf(o["lse"][0][1]) and o["entropy"][0][1] == 0 and np.isneginf(o["logprob"][0][1])
    assert np.isnan(o["lse"][0][2])
    assert o["ids"].tolist() == [[0, 1, 3, 2], [0, 1, 2, 3], [0, 2, 1, 3]]
