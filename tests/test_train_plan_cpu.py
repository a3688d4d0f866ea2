"""Which coefficients digest_orthogonalize accepts, before any device work: the
bounds that it follows through the steps, against the polynomials themselves.
Run on the CPU, every pointer a fake one that nothing reads."""
import ctypes

import numpy as np
import pytest

from paper_2206_00057_amd import digest as D

FAKE = ctypes.c_void_p(1 << 20)


def status(coeffs):
    """Status of one 8 x 8 matrix's call with these steps and no workspace:
    ENOMEM once the coefficients are accepted."""
    one = lambda v: (ctypes.c_void_p * 1)(v)
    eight = (ctypes.c_int32 * 1)(8)
    flat = [v for c in coeffs for v in c]
    return D._train_lib().digest_orthogonalize(
        1, eight, eight, D.F32, one(1 << 20), None, one(2 << 20), None, len(coeffs),
        (ctypes.c_float * len(flat))(*flat), FAKE, 0, None)


def bounds(coeffs):
    """The largest |x p(x^2)| and |p(x^2)| of each step on the bounds before, by a
    fine grid."""
    s, out = 1.0, []
    for a, b, c in np.float32(coeffs).astype(float):
        x = np.linspace(0, s, 200001)
        p = a + b * x ** 2 + c * x ** 4
        out.append((np.abs(x * p).max(), np.abs(p).max()))
        s = out[-1][0]
    return out


@pytest.mark.parametrize("c", [0.0, 1e-6, 1e-12, 1e-16, 1e-20, 1e-38, -1e-6, -1e-12, -1e-16,
                               -1e-20, -1e-38])
def test_a_vanishing_coefficient_keeps_the_extremum(c):
    """3 x - 3 x^3 ends at zero on [0, 1] and reaches 1.15 between: whatever is
    left of the fifth power, the step is accepted, alone and again."""
    assert status([(3.0, -3.0, c)]) == D.ENOMEM
    assert status([(3.0, -3.0, c)] * 3) == D.ENOMEM
    assert status([(-3.0, 3.0, c)]) == D.ENOMEM


def test_polynomials_without_a_middle_term():
    """Both signs of the ends, the extremum inside, outside and absent."""
    for a, c in ((1.0, -1.0), (-1.0, 1.0), (1.0, 1.0), (1.0, -0.1), (1.0, 0.0), (0.0, 1.0)):
        assert status([(a, 0.0, c)]) == D.ENOMEM, (a, c)


def test_bounds_decide():
    """Random polynomials, scaled so that the two bounds of the last step come out
    on both sides of the accepted range, 2^-20 .. 2^20."""
    rng = np.random.default_rng(0)
    limit, seen = 2.0 ** 20, set()
    for trial in range(400):
        c = rng.standard_normal(3) * (rng.random(3) < 0.8)
        c[2] *= 10.0 ** rng.integers(-30, 1)
        if not np.abs(c[:2]).max() > 1e-3:
            continue
        c *= 10.0 ** rng.uniform(-8, 8)
        p, q = bounds([c])[0]
        if min(abs(np.log2(v * k)) for v in (p, q) for k in (limit, 1 / limit)) < 1e-3:
            continue                      # (within the grid's error of a limit)
        ok = 1 / limit <= p <= limit and 1 / limit <= q <= limit
        assert status([c]) == (D.ENOMEM if ok else D.EINVAL), (list(c), p, q)
        seen.add(ok)
    assert seen == {True, False}
