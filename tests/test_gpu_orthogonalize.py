"""digest_orthogonalize and digest_muon_average against 64 bits, over sides from
1 to past the tiles, tall and wide, each element type, groups of matrices of
different sizes, strides, matrices that are zero or not finite.

Tolerances.  The error is followed through the steps in the Frobenius norm F.
A rounding of a stored value is rho = 2^-23 / sqrt(3) of it at most on
average; a product of two planes over K terms is off by eta = 2^-23 of a term
(both operands' roundings and the product of the low parts, which is left
out) and by 2^-25 of the sum for each of its 3 K / 16 roundings.  Roundings
are independent, so errors add as squares: an element of P Q^T is off by
eta |p_i| |q_j| / sqrt(K) off the diagonal and eta |p_i| |q_j| where the
terms have one sign, together at most sqrt(2) eta F_P F_Q / sqrt(r).  An
error already there grows by at most the largest divided difference of the
odd polynomial on the singular values' range (3.9 for the default one).  The
tests allow 4 times what this sums to."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
MUON = (3.4445, -4.7750, 2.0315)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def D():
    from paper_2206_00057_amd import digest
    return digest


def matrix(r, c, seed, kind="gradient"):
    g = torch.Generator().manual_seed(seed)
    u = torch.randn(r, c, generator=g)
    if kind == "gradient":   # strong directions over noise
        k = min(3, r, c)
        u = u * torch.exp(0.5 * torch.randn(r, 1, generator=g)) + torch.mm(
            torch.randn(r, k, generator=g), torch.randn(k, c, generator=g))
    return u.cuda()


def exact(u, steps=5, coeffs=MUON, start=0.0):
    """The result in 64 bits, and the allowed error in the Frobenius norm."""
    x = u.double()
    x = x / x.abs().max()
    x = x / torch.linalg.vector_norm(x)
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    r, c = x.shape
    rho, fro = 2.0 ** -23 / 3 ** 0.5, lambda v: float(torch.linalg.vector_norm(v))
    eta = lambda K: 2.0 ** -23 + (3 * K / 16) ** 0.5 * 2.0 ** -25
    table = coeffs if hasattr(coeffs[0], "__len__") else [coeffs] * steps
    err, s = start + rho, 1.0
    for a, b, k in table:
        y = torch.linspace(0, s, 4001, dtype=torch.float64)
        slope = float((a + 3 * b * y ** 2 + 5 * k * y ** 4).abs().max())
        q = float((a + b * y ** 2 + k * y ** 4).abs().max())
        A = torch.mm(x, x.t().contiguous())
        B = b * A + k * torch.mm(A, A) + a * torch.eye(r, dtype=torch.float64, device=x.device)
        dA = 2 ** 0.5 * eta(c) * fro(x) ** 2 / r ** 0.5 + rho * fro(A)
        dA2 = 2 * s * s * dA + 2 ** 0.5 * eta(r) * fro(A) ** 2 / r ** 0.5
        dB = abs(b) * dA + abs(k) * dA2 + rho * fro(B)
        dX = s * dB + q * rho * fro(x) + 2 ** 0.5 * eta(r) * fro(B) * fro(x) / r ** 0.5
        x = torch.mm(B, x)
        err = slope * err + dX + rho * fro(x)
        s = float((a * y + b * y ** 3 + k * y ** 5).abs().max())
    return (x.t().contiguous() if tall else x), 4 * err


def check(out, u, **kw):
    ref, tol = exact(u, **kw)
    t = torch.finfo(out.dtype)
    tol = tol + t.eps / 2 * float(torch.linalg.vector_norm(ref))
    if out.dtype == torch.float16:
        tol += 2.0 ** -25 * ref.numel() ** 0.5
    err = float(torch.linalg.vector_norm(out.double() - ref))
    assert err <= tol, (tuple(u.shape), err, tol)


def run(D, mats, outs=None, **kw):
    outs = [torch.full_like(m, float("nan")) for m in mats] if outs is None else outs
    ws = torch.full((D.digest_orthogonalize_query([m.shape for m in mats]),), 255,
                    dtype=torch.uint8, device="cuda")
    D.digest_orthogonalize(mats, outs, ws, **kw)
    return outs


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (5, 3), (16, 64), (33, 31), (64, 64), (65, 64), (47, 256),
          (256, 47), (100, 256), (128, 128), (127, 129), (130, 260), (255, 257), (257, 255),
          (64, 1000), (1000, 64), (300, 900), (602, 256), (700, 130), (513, 1025), (1, 5000),
          (1030, 1100)]


@pytest.mark.parametrize("r,c", SHAPES)
def test_shapes(D, r, c):
    for t in TYPES.values():
        u = matrix(r, c, r + c).to(t)
        out = run(D, [u])[0]
        check(out, u)
        assert torch.equal(out, run(D, [u])[0])


@pytest.mark.parametrize("r,c", SHAPES)
def test_layout_element_by_element(D, r, c):
    """(a, b, c) = (1, 0, 0) gives X_0: every element in its place, to the last bits."""
    u = matrix(r, c, 3 * r + c, "noise")
    ref = u.double() / torch.linalg.vector_norm(u.double())
    out = run(D, [u], steps=1, coeffs=(1.0, 0.0, 0.0))[0]
    # two roundings of X_0 (to fp32, then to the planes: 2^-23) and one product's
    # sum, one of whose terms is not zero (twice 3 roundings); subnormal low parts
    tol = ref.abs() * (2.0 ** -22 + 8 * U) + 2.0 ** -39
    assert bool(((out.double() - ref).abs() <= tol).all())


def test_singular_values(D):
    u = matrix(192, 320, 1, "noise")
    s = torch.linalg.svdvals(run(D, [u])[0].double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25


@pytest.mark.parametrize("coeffs,steps", [
    ((1.5, -0.5, 0.0), 3), ((1.875, -1.25, 0.375), 12),
    ([(4.0, -6.0, 3.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)], 3), (MUON, 1), (MUON, 2)])
def test_other_polynomials(D, coeffs, steps):
    for r, c in ((40, 70), (200, 150)):
        u = matrix(r, c, steps, "noise")
        check(run(D, [u], steps=steps, coeffs=coeffs)[0], u, steps=steps, coeffs=coeffs)


def test_groups(D):
    """More matrices than one launch takes, of all sizes: each as alone."""
    shapes = [SHAPES[i % len(SHAPES)] for i in range(0, 3 * len(SHAPES), 2)]
    mats = [matrix(r, c, 7 * i) for i, (r, c) in enumerate(shapes)]
    outs = run(D, mats)
    for u, out in zip(mats, outs):
        check(out, u)
    one = [run(D, [u])[0] for u in mats[:6]]
    assert all(float((a - b).abs().max()) <= 1e-4 for a, b in zip(one, outs))


@pytest.mark.parametrize("shapes", [
    [(1024, 1024), (300, 4096), (2500, 49), (1030, 1100)],   # long and short k side by side
    [(2048, 2048), (3, 5)], [(1500, 1500)], [(600, 4100), (4100, 600)],
    [(4096, 4096)], [(2300, 5000)], [(129, 9000), (4000, 257), (513, 513)]])
def test_large_groups(D, shapes):
    mats = [matrix(r, c, 3 + i) for i, (r, c) in enumerate(shapes)]
    outs = run(D, mats)
    for u, out in zip(mats, outs):
        check(out, u)
    again = run(D, mats)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


def test_offsets_past_32_bits(D):
    """Row strides that take the last rows past 2^31 elements."""
    ld, r, c = 1_200_000_000, 3, 70
    whole = torch.zeros(2 * ld + 1000, dtype=torch.bfloat16, device="cuda")
    u = whole.as_strided((r, c), (ld, 1), 11)
    out = whole.as_strided((r, c), (ld, 1), 311)
    u.copy_(matrix(r, c, 1, "noise"))
    run(D, [u], [out])
    check(out, u)
    assert int((whole != 0).sum()) <= 2 * r * c


def test_calls_in_turn_share_a_workspace(D):
    """Two captured updates over one workspace, replayed one after the other."""
    sets = [muon_setup(s, 2, 4) for s in ([(90, 200)], [(33, 40), (300, 70)])]
    mine = [[[v.clone() for v in w], [v.clone() for v in m]] for w, m, _ in sets]
    ws = torch.empty(max(D.digest_orthogonalize_query([v.shape for v in w]) for w, _, _ in sets),
                     dtype=torch.uint8, device="cuda")
    graphs = []
    for (w, m, g) in sets:
        D.digest_muon_average(w, m, g, ws, 0.0, 1.0)   # (lr 0: weights stay; momenta grow)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            D.digest_muon_average(w, m, g, ws, 0.1)
        graphs.append(graph)
    for (w, m), (_, _, g) in zip(mine, sets):
        D.digest_muon_average(w, m, g, ws, 0.0, 1.0)
    for i in range(3):
        for k, (w, m) in enumerate(mine):
            D.digest_muon_average(w, m, sets[k][2], ws, 0.1)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (w, m), (rw, rm, _) in zip(mine, sets):
            assert all(torch.equal(a, b) for a, b in zip(w + m, rw + rm)), i


def test_strides_and_in_place(D):
    for t in TYPES.values():
        # three column slices of one array, into slices of another
        whole = matrix(90, 400, 2).to(t)
        mats = [whole[:, 1:101], whole[:, 101:131], whole[:, 131:400]]
        dst = torch.full((90, 410), 7.0, dtype=t, device="cuda")
        outs = run(D, mats, [dst[:, 3:103], dst[:, 104:134], dst[:, 135:404]])
        for u, out in zip(mats, outs):
            check(out, u)
        for j in (0, 1, 2, 103, 134, 404, 409):
            assert bool((dst[:, j] == 7).all()), j
        tall = matrix(300, 31, 4).to(t)
        keep = tall.clone()
        run(D, [tall], [tall])
        check(tall, keep)


def test_scale_of_the_input_does_not_matter(D):
    u = matrix(70, 130, 5, "noise").half().float()   # few bits: exact at every scale
    ref = run(D, [u])[0]
    for e in (-120, -60, 60, 110):
        assert torch.equal(run(D, [u * 2.0 ** e])[0], ref), e
    tiny = torch.full((3, 5), 2.0 ** -149, device="cuda")       # the smallest number
    check(run(D, [tiny])[0], tiny)
    huge = torch.full((300, 500), torch.finfo(torch.float32).max, device="cuda")
    check(run(D, [huge])[0], huge)


def test_zero_and_not_finite_matrices_touch_no_other(D):
    mats = [matrix(60, 90, i) for i in range(5)]
    clean = run(D, mats)
    bad = [m.clone() for m in mats]
    bad[1].zero_()
    bad[2][7, 11] = float("nan")
    bad[4][59, 0] = float("-inf")
    outs = run(D, bad)
    assert not outs[1].any()
    assert bool(outs[2].isnan().all()) and bool(outs[4].isnan().all())
    assert torch.equal(outs[0], clean[0]) and torch.equal(outs[3], clean[3])


def test_rank_one_and_wide_spectrum(D):
    g = torch.Generator().manual_seed(1)
    one = (torch.randn(150, 1, generator=g) @ torch.randn(1, 170, generator=g)).cuda()
    check(run(D, [one])[0], one)
    # singular values over five decades
    q1, q2 = (torch.linalg.qr(torch.randn(120, 120, generator=g, dtype=torch.float64))[0]
              for _ in range(2))
    s = torch.logspace(0, -5, 120, dtype=torch.float64)
    u = (q1 * s @ q2).float().cuda()
    check(run(D, [u])[0], u)


def muon_setup(shapes, M, seed):
    w = [matrix(r, c, seed + 10 * i, "noise") for i, (r, c) in enumerate(shapes)]
    mom = [matrix(r, c, seed + 10 * i + 1) for i, (r, c) in enumerate(shapes)]
    g = [[matrix(r, c, seed + 1000 * i + 20 + m) for m in range(M)]
         for i, (r, c) in enumerate(shapes)]
    return w, mom, g


@pytest.mark.parametrize("shapes,M,nesterov", [
    ([(64, 64), (64, 16)], 4, True), ([(100, 256), (256, 256), (256, 47)], 8, False),
    ([(31, 7)] * 5, 64, True), ([(300, 200)], 1, True),
    ([(9 + i, 40 - i) for i in range(20)], 3, True)])
def test_muon_average(D, shapes, M, nesterov):
    w, mom, grads = muon_setup(shapes, M, 5)
    ws = torch.full((D.digest_orthogonalize_query(shapes),), 255, dtype=torch.uint8, device="cuda")
    lr, beta, decay = 0.05, 0.9, 0.1
    scales = [1.0 + 0.1 * i for i in range(len(shapes))]
    w0, m0 = [v.clone() for v in w], [v.clone() for v in mom]
    g0 = [[v.clone() for v in g] for g in grads]
    D.digest_muon_average(w, mom, grads, ws, lr, beta, decay, scales, nesterov)
    for i in range(len(shapes)):
        g = sum(v.double() for v in g0[i]) / M
        m = beta * m0[i].double() + g
        size = sum(v.double().abs() for v in g0[i]) / M + m0[i].double().abs()
        # M roundings of the sum, the mean's, the momentum's two
        assert bool(((mom[i].double() - m).abs() <= (M + 4) * U * size).all())
        u = g + beta * m if nesterov else m
        start = (M + 8) * U * float(torch.linalg.vector_norm(2 * size) /
                                    torch.linalg.vector_norm(u))
        o, tol = exact(u, start=start)
        ref = (1 - lr * decay) * w0[i].double() - lr * scales[i] * o
        # the factor 1 - lr decay, its product, the step's and the difference
        tol = lr * scales[i] * tol + 6 * U * float(torch.linalg.vector_norm(w0[i]) +
                                                   torch.linalg.vector_norm(ref))
        assert float(torch.linalg.vector_norm(w[i].double() - ref)) <= tol, i
        assert all(torch.equal(a, b) for a, b in zip(grads[i], g0[i]))


def test_muon_defaults_and_shared_gradients(D):
    shapes = [(50, 30)]
    w, mom, grads = muon_setup(shapes, 1, 9)
    ws = torch.empty(D.digest_orthogonalize_query(shapes), dtype=torch.uint8, device="cuda")
    w1, m1 = w[0].clone(), mom[0].clone()
    D.digest_muon_average(w, mom, grads, ws, 0.1)
    # the same gradient three times has itself as its mean (to a rounding or two)
    D.digest_muon_average([w1], [m1], [grads[0] * 3], ws, 0.1)
    assert float((w[0] - w1).abs().max()) <= 1e-5
    o = run(D, [grads[0][0] + 0.95 * mom[0]])[0]
    assert float((muon_setup(shapes, 1, 9)[0][0] - 0.1 * o - w[0]).abs().max()) <= 1e-5


def test_not_finite_gradient_stays_with_its_matrix(D):
    shapes = [(40, 40), (70, 20), (20, 90)]
    w, mom, grads = muon_setup(shapes, 2, 3)
    grads[1][0][3, 3] = float("nan")
    ws = torch.empty(D.digest_orthogonalize_query(shapes), dtype=torch.uint8, device="cuda")
    D.digest_muon_average(w, mom, grads, ws, 0.1)
    assert bool(w[1].isnan().all())
    assert bool(w[0].isfinite().all()) and bool(w[2].isfinite().all())
    assert int(mom[1].isnan().sum()) == 1


def test_streams_and_graph_replays(D):
    shapes = [(100, 256), (256, 47), (300, 300)]
    w, mom, grads = muon_setup(shapes, 3, 2)
    ew, em = [v.clone() for v in w], [v.clone() for v in mom]
    ws = torch.empty(D.digest_orthogonalize_query(shapes), dtype=torch.uint8, device="cuda")
    step = lambda a, b: D.digest_muon_average(a, b, grads, ws, 0.02, 0.95, 0.01)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(w, mom)
    torch.cuda.current_stream().wait_stream(side)
    step(ew, em)
    assert all(torch.equal(a, b) for a, b in zip(w + mom, ew + em))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(w, mom)
    for i in range(4):
        for g in grads:
            g[0].mul_(-1.5)
        step(ew, em)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(w + mom, ew + em)), i


def test_binding_refuses(D):
    u = torch.zeros(4, 8, device="cuda")
    ws = torch.zeros(D.digest_orthogonalize_query([(4, 8)]), dtype=torch.uint8, device="cuda")
    orth = lambda m=None, o=None, w=ws, **k: D.digest_orthogonalize(m or [u], o or [u.clone()], w,
                                                                    **k)
    for err, kw in [(TypeError, dict(m=[u.cpu()])), (TypeError, dict(m=[u.double()])),
                    (TypeError, dict(o=[u.half()])), (ValueError, dict(o=[u.t()])),
                    (ValueError, dict(m=[u.t()])), (ValueError, dict(m=[u[0]])),
                    (ValueError, dict(m=[u[:0]])), (ValueError, dict(o=[u, u])),
                    (TypeError, dict(m=[u, u.half()], o=[u, u])),
                    (ValueError, dict(coeffs=(1.0, 2.0))),
                    (ValueError, dict(coeffs=[(1.0, 0.0, 0.0)] * 4)),
                    (D.DigestError, dict(w=None)), (D.DigestError, dict(w=ws[:-1])),
                    (D.DigestError, dict(steps=0)), (D.DigestError, dict(steps=65)),
                    (D.DigestError, dict(coeffs=(float("nan"), 0.0, 0.0)))]:
        with pytest.raises(err):
            orth(**kw)
    orth()
    w, m, g = u.clone(), u.clone(), u.clone()
    muon = lambda a=None, b=None, c=None, **k: D.digest_muon_average(
        a or [w], b or [m], c or [[g]], ws, 0.1, **k)
    for err, kw in [(ValueError, dict(a=[w, w])), (ValueError, dict(c=[[]])),
                    (ValueError, dict(c=[[g[:, :7]]])), (TypeError, dict(a=[w.half()])),
                    (ValueError, dict(a=[torch.zeros(8, 4, device="cuda").t()])),
                    (D.DigestError, dict(b=[w])), (D.DigestError, dict(c=[[m]])),
                    (D.DigestError, dict(c=[[g] * 65])),
                    (ValueError, dict(scales=[1.0, 2.0]))]:
        with pytest.raises(err):
            muon(**kw)
    muon()
