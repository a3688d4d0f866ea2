"""digest_orthogonalize and digest_muon_average where the large products run:
64-, 128- and 256-wide tiles, whole and split along k, in each place of a step
(X X^T, the polynomial, B X, the result in 32 and 16 bits, the weights), for
wide and tall matrices.  Against 64 bits, and equal bits from equal calls.
Tolerances: test_gpu_orthogonalize."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_orthogonalize import (  # noqa: E402,F401
    D, TYPES, U, _need_gpu, check, exact, matrix, muon_setup, run)


@pytest.mark.parametrize("shapes", [
    [(2048, 2176)],                              # X X^T on split 256-tiles, B X on 128 with rest
    [(2304, 2304)], [(2600, 2304)],              # B X on split 256-tiles; on 128-tiles, some split
    [(2048, 8192)], [(8192, 2048)],              # X X^T split, B X on whole 256-tiles
    [(4096, 4096)] * 2,                          # every product on 256-tiles, whole and split
    [(4096, 4096), (300, 200)],                  # split 256-tiles of two lengths
    [(1024, 1024), (4096, 1024), (1024, 4096)]])  # split 128-tiles of two lengths
def test_large_tiles(D, shapes):  # noqa: F811
    mats = [matrix(r, c, 5 + i) for i, (r, c) in enumerate(shapes)]
    outs = run(D, mats)
    for u, out in zip(mats, outs):
        check(out, u)
    again = run(D, mats)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("shapes", [
    [(1000, 1000)],                              # 64-tiles
    [(1024, 4096)], [(4096, 1024)],              # whole 128-tiles
    [(1030, 1100)], [(1100, 1030)],              # split 128-tiles
    [(2048, 8192)], [(8192, 2048)],              # whole 256-tiles
    [(2304, 2304)], [(2816, 2560)],              # split 256-tiles
    [(513, 1025)], [(2304, 2560)]])
def test_results_of_16_bits(D, shapes, t):  # noqa: F811
    mats = [matrix(r, c, 9 + i).to(TYPES[t]) for i, (r, c) in enumerate(shapes)]
    outs = run(D, mats)
    for u, out in zip(mats, outs):
        check(out, u)
    for _ in range(3):
        again = run(D, mats)
        assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.parametrize("shapes,M", [
    ([(1000, 1000), (700, 800)], 2),             # 64-tiles
    ([(1025, 513)], 1),
    ([(1024, 4096)], 1), ([(4096, 1024)], 3),    # whole 128-tiles
    ([(1030, 1100)], 2), ([(1100, 1030)], 1),    # split 128-tiles
    ([(1024, 1024), (4096, 1024), (1024, 4096)], 1),   # both
    ([(2048, 8192)], 1), ([(8192, 2048)], 1),    # whole 256-tiles
    ([(2304, 2304)], 2), ([(2816, 2560)], 1),    # split 256-tiles
    ([(2560, 2304), (30, 50)], 1)])              # whole and split 128-tiles
def test_muon_of_large_matrices(D, shapes, M):  # noqa: F811
    lr, beta, decay = 0.05, 0.9, 0.1
    scales = [1.0 + 0.5 * i for i in range(len(shapes))]
    w, mom, grads = muon_setup(shapes, M, 7)
    w0, m0 = [v.clone() for v in w], [v.clone() for v in mom]
    w1, m1 = [v.clone() for v in w], [v.clone() for v in mom]
    g0 = [[v.clone() for v in g] for g in grads]
    ws = torch.full((D.digest_orthogonalize_query(shapes),), 255, dtype=torch.uint8, device="cuda")
    D.digest_muon_average(w, mom, grads, ws, lr, beta, decay, scales)
    for i in range(len(shapes)):
        g = sum(v.double() for v in g0[i]) / M
        m = beta * m0[i].double() + g
        size = sum(v.double().abs() for v in g0[i]) / M + m0[i].double().abs()
        # M roundings of the sum, the mean's, the momentum's two
        assert bool(((mom[i].double() - m).abs() <= (M + 4) * U * size).all())
        u = g + beta * m
        start = (M + 8) * U * float(torch.linalg.vector_norm(2 * size) /
                                    torch.linalg.vector_norm(u))
        o, tol = exact(u, start=start)
        ref = (1 - lr * decay) * w0[i].double() - lr * scales[i] * o
        # the factor 1 - lr decay, its product, the step's and the difference
        room = 6 * U * float(torch.linalg.vector_norm(w0[i]) + torch.linalg.vector_norm(ref))
        err = w[i].double() - ref
        assert float(torch.linalg.vector_norm(err)) <= lr * scales[i] * tol + room, i
        # each weight by itself: no element of O is off by more than all of O, and
        # the weights' own roundings do not add up
        room = 6 * U * (w0[i].double().abs() + ref.abs())
        assert bool((err.abs() <= lr * scales[i] * tol + room).all()), i
        assert all(torch.equal(a, b) for a, b in zip(grads[i], g0[i]))
    D.digest_muon_average(w1, m1, grads, ws, lr, beta, decay, scales)
    assert all(torch.equal(a, b) for a, b in zip(w + mom, w1 + m1))
