"""digest_muon_average replaces weights and momenta: factors that would make
them NaN are refused before any device work.  Run on the CPU, every pointer a
fake one that nothing reads."""
import ctypes

import pytest

from paper_2206_00057_amd import digest as D

INF, NAN, BIG = float("inf"), float("nan"), 3e38


def status(lr=0.1, beta=0.9, decay=0.0, scales=None):
    """Status of a call on two matrices without a workspace: ENOMEM once the
    arguments are accepted."""
    ptrs = lambda *v: (ctypes.c_void_p * len(v))(*[x << 20 for x in v])
    rows, cols = (ctypes.c_int32 * 2)(4, 8), (ctypes.c_int32 * 2)(8, 4)
    return D._train_lib().digest_muon_average(
        2, rows, cols, ptrs(1, 2), ptrs(3, 4), ptrs(5, 6), 1, lr, beta, decay,
        None if scales is None else (ctypes.c_float * 2)(*scales), 1, 5, None,
        ctypes.c_void_p(7 << 20), 0, None)


@pytest.mark.parametrize("kw", [
    dict(lr=NAN), dict(lr=INF), dict(lr=-INF), dict(beta=NAN), dict(beta=INF), dict(decay=NAN),
    dict(decay=-INF), dict(lr=0.0, decay=INF), dict(lr=BIG, decay=10.0), dict(scales=(NAN, 1.0)),
    dict(scales=(1.0, INF)), dict(lr=0.0, scales=(1.0, INF)), dict(lr=10.0, scales=(1.0, BIG))])
def test_factors_that_are_not_finite(kw):
    assert status(**kw) == D.EINVAL
    assert b"not finite" in D.lib().digest_last_error()


@pytest.mark.parametrize("kw", [
    dict(), dict(lr=0.0), dict(lr=-0.1), dict(beta=0.0), dict(beta=1.0), dict(decay=0.5),
    dict(lr=2.0, decay=1.0), dict(scales=(0.0, -2.0)), dict(lr=1.0, scales=(BIG, 1e-40))])
def test_finite_factors(kw):
    assert status(**kw) == D.ENOMEM
