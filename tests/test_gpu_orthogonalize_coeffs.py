"""digest_orthogonalize with polynomials whose fifth power vanishes, against 64
bits: the scales of the planes follow the largest value on the singular values'
range, which lies between its ends.  Tolerances: test_gpu_orthogonalize."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_orthogonalize import D, _need_gpu, check, matrix, run  # noqa: E402,F401


@pytest.mark.parametrize("c", [0.0, 1e-12, 1e-20, -1e-20])
@pytest.mark.parametrize("shape", [(40, 70), (200, 150), (300, 900)])
def test_vanishing_fifth_power(D, shape, c):  # noqa: F811
    u = matrix(*shape, 11, "noise")
    for a, b in ((3.0, -2.9), (3.0, -3.0)):
        out = run(D, [u], steps=4, coeffs=(a, b, c))[0]
        assert bool(out.isfinite().all())
        check(out, u, steps=4, coeffs=(a, b, c))
