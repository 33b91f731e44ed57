"""Which polynomials cf_newton_schulz takes: those with which no singular value from 0 to 1
leaves the range of the products' factors on its way (no kernel is launched)."""
import os
import random

import numpy as np
import pytest

from paper_1808_04728_amd import binding as B

A = 0x7F0000000000  # fake, 16-byte aligned device addresses (never dereferenced)

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libcosmoflow_hip.so not built")


def taken(coef, steps):
    """Coefficients are looked at before the workspace, which is missing here."""
    with pytest.raises(B.CfError) as e:
        B.cf_newton_schulz(B.make_matrices([0], [64], [48]), "f32", B.make_ns_hparams(steps, coef), A, A + (1 << 30), None, 0, 0)
    assert e.value.status in (B.CF_ERR_UNSUPPORTED, B.CF_ERR_WORKSPACE)
    return e.value.status == B.CF_ERR_WORKSPACE


def largest(coef, steps, n=200000):
    """The largest value on the way of singular values from 0 to 1, each step's relative
    rounding of 2^-20 (a norm and products of a few units of 2^-23) in both directions."""
    a, b, c = coef
    x = np.concatenate([np.arange(n + 1) / n, 1 - 2.0 ** -np.arange(1.0, 40)])
    x = np.concatenate([x * (1 - 2.0 ** -20), x * (1 + 2.0 ** -20)])
    top = 1.0
    for _ in range(steps):
        h = np.minimum(x * x, 1e60)
        x = np.minimum(np.abs(x * (a + b * h + c * h * h)) * (1 + 2.0 ** -20), 1e30)
        top = max(top, float(x.max()))
    return top


# (a, b, c), steps: a narrow range of singular values leaves the factors' range, between
# values that do not
NARROW = [((3.2149347006642817, -8.490339039362288, 3.9845496399889178), 4),
          ((4.672865173660875, -13.35488059396478, 8.411673383392104), 5),
          ((2.803379971058804, -12.090328396595718, 8.909098254250761), 8),
          ((4.59416569169864, -14.260132866539616, 8.687910659579185), 7)]


@pytest.mark.parametrize("coef,steps", NARROW)
def test_narrow_ranges_that_grow_are_refused(coef, steps):
    assert not taken(coef, steps)


def test_growth_of_roundings_is_refused():
    """5 x - 20 x^3 + 16 x^5 maps [-1, 1] onto itself and steps away from 1 at 25 times the
    distance."""
    assert taken((5.0, -20.0, 16.0), 1)
    assert not taken((5.0, -20.0, 16.0), 12)


@pytest.mark.parametrize("coef", [B.NS_COEF, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (3.0, -16.0 / 5, 6.0 / 5), (15.0 / 8, -10.0 / 8, 3.0 / 8)])
def test_usual_polynomials_are_taken(coef):
    for steps in range(1, B.CF_NS_MAX_STEPS + 1):
        assert taken(coef, steps)


def test_taken_polynomials_stay_in_range():
    """Sampled densely, no polynomial that is taken leaves the range (32 for a singular value)."""
    rng, seen = random.Random(4), 0
    for k in range(4000):
        if k % 2:
            coef = (rng.uniform(2, 8), rng.uniform(-40, -2), rng.uniform(0, 60))
        else:
            coef = (3.4445 * rng.uniform(0.8, 1.8), -4.775 * rng.uniform(1, 3), 2.0315 * rng.uniform(0.5, 5))
        steps = rng.choice([4, 5, 6, 7, 8, 10, 12])
        if taken(coef, steps):
            seen += 1
            assert largest(coef, steps, 20000) < 33.0, (coef, steps)
    assert seen >= 50
