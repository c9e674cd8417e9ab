"""The 64-bit reference of activations holds together: slopes are what differences of the activations say."""
import numpy as np
import pytest

import linear_ref as ref


def points():
    """Both sides of zero, near it and far, away from where RELU has no slope."""
    z = np.concatenate([np.linspace(-12, 12, 4801), [-40.0, 40.0, -1e-3, 1e-3]])
    return z[np.abs(z) > 5e-4]


@pytest.mark.parametrize("act", ref.ACTS)
def test_slopes_against_differences(act):
    """(8 (f(h) - f(-h)) - (f(2h) - f(-2h))) / 12h is off by h^4 / 30 times the fifth derivative, which is below 3 for all of them: 9.1e-14
    at h = 2^-10.  Values up to 40 are rounded to 2^-53 of themselves, some eight times each, which 18 / 12h of it multiplies:
    40 * 2^-53 * 8 * 1536 = 5.5e-11."""
    z, h = points(), 2.0 ** -10
    if act == "relu":
        z = z[np.abs(z) > 4 * h]
    f = lambda x: ref.act(x, act)[0]                             # noqa: E731
    d = (8 * (f(z + h) - f(z - h)) - (f(z + 2 * h) - f(z - 2 * h))) / (12 * h)
    assert np.abs(d - ref.slope(z, act)[0]).max() < 1e-10
