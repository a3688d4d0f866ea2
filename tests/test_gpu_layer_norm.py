"""Layer norm (digest_layer_norm_forward / _backward) against the formulas in
64 bits, at widths on both sides of every row layout, row strides and starts
that are no multiple of a vector, each element type, and rows that are not
finite.

Tolerances count roundings.  u = 2^-24.  A row's sum adds at most 64 elements
in a lane, 6 times in a wave and 16 waves: fewer than 90 roundings, so that a
sum of terms t is off by at most 90 u sum |t|; rounding to the element type
adds eps / 2 of the value."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def D():
    from paper_2206_00057_amd import digest
    return digest


def half_step(t):
    return torch.finfo(t).eps / 2


def rows(n, d, t, seed, pad=0, start=0, scale=1.0, offset=0.3):
    """[n, d] rows of a wider array: row stride d + pad, first element `start`."""
    g = torch.Generator().manual_seed(seed)
    a = (torch.randn(n, d + pad + start, generator=g) * scale + offset).to(t).cuda()
    return a[:, start:start + d]


def params(d, seed):
    g = torch.Generator().manual_seed(seed)
    return ((1.0 + 0.2 * torch.randn(d, generator=g)).cuda(),
            (0.3 * torch.randn(d, generator=g)).cuda())


def forward64(x, gain, shift, relu):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
    xh = (x - mean) * rstd
    z = xh * (1.0 if gain is None else gain.double()) + (0.0 if shift is None else shift.double())
    return (z.clamp_min(0.0) if relu else z), mean, rstd, xh, z


def check_forward(y, stats, x, gain, shift, relu):
    ref, mean, rstd, xh, z = forward64(x, gain, shift, relu)
    g = 1.0 if gain is None else gain.double().abs()
    b = 0.0 if shift is None else shift.double().abs()
    level = x.double().abs().mean(1, keepdim=True)
    # mean: 90 roundings of a sum, carried into xh; rstd: 90 of the sum of squares, halved, and
    # the square root's, the division's and the last product's
    tol = U * (g * (95 * level * rstd + 60 * xh.abs()) + 2 * b + 2 * z.abs())
    tol = tol + half_step(y.dtype) * (z.abs() + tol)
    if y.dtype == torch.float16:
        tol = tol + 2.0 ** -25            # half a step of the subnormal numbers
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    if stats is not None:
        s = stats.double()
        assert bool(((s[:, :1] - mean).abs() <= 95 * U * level).all())
        assert bool(((s[:, 1:] - rstd).abs() <= U * rstd * (60 + 95 * level * rstd)).all())


def backward64(x, gain, y, dy, stats, relu):
    x, s = x.double(), stats.double()
    xh = (x - s[:, :1]) * s[:, 1:]
    D = dy.double() * ((y > 0).double() if relu else 1.0)
    e = D * (1.0 if gain is None else gain.double())
    dx = s[:, 1:] * (e - e.mean(1, keepdim=True) - xh * (e * xh).mean(1, keepdim=True))
    return dx, (D * xh).sum(0), D.sum(0), D, e, xh, s[:, 1:]


def check_backward(dx, dgain, dshift, x, gain, y, dy, stats, relu):
    rdx, rdg, rdb, D, e, xh, rstd = backward64(x, gain, y, dy, stats, relu)
    n = x.shape[0]
    if dx is not None:
        tol = U * rstd * (6 * e.abs() + 98 * e.abs().mean(1, keepdim=True) +
                          100 * xh.abs() * (e * xh).abs().mean(1, keepdim=True))
        tol = tol + half_step(dx.dtype) * (rdx.abs() + tol)
        if dx.dtype == torch.float16:
            tol = tol + 2.0 ** -25
        err = (dx.double() - rdx).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    # sums over n rows in any order: at most n roundings, and xh's and the product's
    if dgain is not None:
        assert bool(((dgain.double() - rdg).abs() <= (n + 4) * U * (D * xh).abs().sum(0)).all())
    if dshift is not None:
        assert bool(((dshift.double() - rdb).abs() <= n * U * D.abs().sum(0)).all())


def call_forward(D, x, gain, shift, relu, y=None, stats=True):
    y = torch.full_like(x, float("nan")) if y is None else y
    stats = torch.full((x.shape[0], 2), float("nan"), device="cuda") if stats else None
    D.digest_layer_norm_forward(x, gain, shift, y, stats, EPS,
                                D.ACT_RELU if relu else D.ACT_IDENTITY)
    return y, stats


def call_backward(D, x, gain, y, dy, stats, relu, dx=None):
    n, d = x.shape
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    dgain, dshift = (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
    ws = torch.full((D.digest_layer_norm_query(n, d),), 255, dtype=torch.uint8, device="cuda")
    D.digest_layer_norm_backward(x, gain, y, dy, stats, dx, dgain, dshift, ws,
                                 D.ACT_RELU if relu else D.ACT_IDENTITY)
    return dx, dgain, dshift


# both sides of each row layout: lanes of a row (2 .. 64), elements a lane,
# waves of a row, the widest with the sums beside it, the widest held
WIDTHS = [1, 2, 3, 7, 8, 9, 16, 17, 31, 47, 64, 65, 100, 128, 255, 256, 257, 500, 602, 1000, 1024,
          1025, 2048, 2051, 4096, 4099, 8192, 8193, 16384, 16385, 40001, 65536]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(D, d, t):
    n = 37 if d <= 4099 else 5
    relu = d % 2 == 0
    x, (gain, shift) = rows(n, d, TYPES[t], d), params(d, d + 1)
    y, stats = call_forward(D, x, gain, shift, relu)
    check_forward(y, stats, x, gain, shift, relu)
    dy = rows(n, d, TYPES[t], d + 2, offset=0.0)
    dx, dgain, dshift = call_backward(D, x, gain, y, dy, stats, relu)
    check_backward(dx, dgain, dshift, x, gain, y, dy, stats, relu)


@pytest.mark.parametrize("n,d,t", [(1, 256, "f32"), (2, 64, "bf16"), (5000, 64, "f32"),
                                   (4097, 41, "bf16"), (1031, 4096, "bf16"), (1030, 1024, "f16"),
                                   (20001, 7, "f32"), (1200, 3001, "f32"), (300, 9000, "bf16")])
def test_rows(D, n, d, t):
    x, (gain, shift) = rows(n, d, TYPES[t], n), params(d, 3)
    for relu in (False, True):
        y, stats = call_forward(D, x, gain, shift, relu)
        check_forward(y, stats, x, gain, shift, relu)
        dy = rows(n, d, TYPES[t], n + 1, offset=0.1)
        out = call_backward(D, x, gain, y, dy, stats, relu)
        check_backward(*out, x, gain, y, dy, stats, relu)
        again = call_backward(D, x, gain, y, dy, stats, relu)
        for a, b in zip(out, again):
            assert torch.equal(a, b)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("d,pad,start", [(64, 1, 0), (61, 3, 1), (256, 8, 5), (1030, 7, 3),
                                         (5001, 2, 1), (17000, 1, 1)])
def test_strides_leave_the_gaps_alone(D, d, pad, start, t):
    n, dt = 9, TYPES[t]
    x, (gain, shift) = rows(n, d, dt, 5, pad, start), params(d, 6)
    whole = torch.full((n, d + 7), 7.0, dtype=dt, device="cuda")
    y, stats = call_forward(D, x, gain, shift, True, y=whole[:, 3:3 + d])
    check_forward(y, stats, x, gain, shift, True)
    assert bool((whole[:, :3] == 7).all()) and bool((whole[:, 3 + d:] == 7).all())
    dy = rows(n, d, dt, 8, pad + 2, start + 1, offset=0.0)
    whole2 = torch.full((n, d + 5), 7.0, dtype=dt, device="cuda")
    out = call_backward(D, x, gain, y, dy, stats, True, dx=whole2[:, 1:1 + d])
    check_backward(*out, x, gain, y, dy, stats, True)
    assert bool((whole2[:, :1] == 7).all()) and bool((whole2[:, 1 + d:] == 7).all())


def test_in_place_and_absent_arrays(D):
    for d in (64, 1500, 9000, 20000):
        n = 11
        x = rows(n, d, torch.float32, 1)
        x0 = x.clone()
        y, stats = call_forward(D, x, None, None, False, y=x)
        check_forward(y, stats, x0, None, None, False)
        dy = rows(n, d, torch.float32, 2)
        dy0 = dy.clone()
        out = call_backward(D, x0, None, None, dy, stats, False, dx=dy)
        check_backward(*out, x0, None, None, dy0, stats, False)
        # one of the three at a time
        ws = torch.empty(D.digest_layer_norm_query(n, d), dtype=torch.uint8, device="cuda")
        only = torch.empty_like(dy0)
        D.digest_layer_norm_backward(x0, None, None, dy0, stats, only, None, None, None)
        assert torch.equal(only, dy)
        for k in (1, 2):
            v = torch.empty(d, device="cuda")
            D.digest_layer_norm_backward(x0, None, None, dy0, stats, None, v if k == 1 else None,
                                         v if k == 2 else None, ws)
            assert torch.equal(v, out[k])
        y2, none = call_forward(D, x0, None, None, False, stats=False)
        assert none is None and torch.equal(y2, y)


def test_offsets_past_32_bits(D):
    """Row strides that take the last rows past 2^31 elements."""
    ld, n, d = 1_200_000_000, 3, 133
    whole = torch.zeros(2 * ld + 2000, dtype=torch.bfloat16, device="cuda")
    part = lambda at: whole.as_strided((n, d), (ld, 1), at)
    x, y, dy, dx = part(3), part(303), part(601), part(901)
    x.copy_(rows(n, d, torch.bfloat16, 1))
    dy.copy_(rows(n, d, torch.bfloat16, 2))
    gain, shift = params(d, 3)
    _, stats = call_forward(D, x, gain, shift, True, y=y)
    check_forward(y, stats, x, gain, shift, True)
    out = call_backward(D, x, gain, y, dy, stats, True, dx=dx)
    check_backward(*out, x, gain, y, dy, stats, True)
    assert int((whole != 0).sum()) <= 4 * n * d


def test_no_rows(D):
    x = torch.empty(0, 70, device="cuda")
    y, stats = call_forward(D, x, None, None, True)
    dx, dgain, dshift = call_backward(D, x, None, y, x.clone(), stats, True)
    assert not dgain.any() and not dshift.any()


@pytest.mark.parametrize("d", [5, 64, 700, 3000, 17000])
def test_rows_that_are_not_finite_touch_no_other(D, d):
    n = 12
    x, (gain, shift) = rows(n, d, torch.float32, 4), params(d, 5)
    clean = call_forward(D, x, gain, shift, True)[0]
    bad = x.clone()
    bad[2, d // 2] = float("nan")
    bad[5, d - 1] = float("inf")
    bad[7, 0] = float("-inf")
    y, stats = call_forward(D, bad, gain, shift, True)
    keep = [i for i in range(n) if i not in (2, 5, 7)]
    assert torch.equal(y[keep], clean[keep])
    assert bool(y[[2, 5, 7]].isnan().all()) and bool(stats[[2, 5, 7], 1].isnan().all())
    # constant rows: eps keeps them finite
    x[3] = 2.5
    y, stats = call_forward(D, x, gain, shift, False)
    assert bool(((y[3] - shift).abs() <= 95 * U * 2.5 / EPS ** 0.5 * gain.abs()).all())


def test_far_offsets_keep_the_variance(D):
    # the deviations are 2^-10 of the offset: centred squares keep them
    d = 512
    g = torch.Generator().manual_seed(0)
    x = (1024.0 + torch.randint(-8, 9, (40, d), generator=g).float() / 8).cuda()   # exact in fp32
    y, stats = call_forward(D, x, None, None, False)
    check_forward(y, stats, x, None, None, False)


def test_gradient_against_differences(D):
    n, d, h = 3, 6, 1e-6
    x, (gain, shift), w = rows(n, d, torch.float32, 1), params(d, 2), rows(n, d, torch.float32, 3)
    for relu in (False, True):
        y, stats = call_forward(D, x, gain, shift, relu)
        dx, dgain, dshift = call_backward(D, x, gain, y, w, stats, relu)
        loss = lambda *a: float((forward64(*a, relu)[0] * w.double()).sum())
        for name, got, base in (("x", dx, x), ("gain", dgain, gain), ("shift", dshift, shift)):
            for i in range(got.numel()):
                out = []
                for s in (h, -h):
                    p = {"x": x.double(), "gain": gain.double(), "shift": shift.double()}
                    p[name] = p[name].clone()
                    p[name].view(-1)[i] += s
                    out.append(loss(p["x"], p["gain"], p["shift"]))
                diff = (out[0] - out[1]) / (2 * h)
                # differences: h^2 terms and 64-bit rounding over h; the kernel: fp32
                assert abs(diff - float(got.reshape(-1)[i])) <= 1e-4 * (1 + abs(diff)), (name, i)


def test_streams_and_graph_replays(D):
    n, d = 777, 602
    x, (gain, shift) = rows(n, d, torch.bfloat16, 1), params(d, 2)
    dy = rows(n, d, torch.bfloat16, 3)
    ref = call_forward(D, x, gain, shift, True)
    ref = ref + call_backward(D, x, gain, ref[0], dy, ref[1], True)
    y, stats, dx = torch.empty_like(x), torch.empty(n, 2, device="cuda"), torch.empty_like(x)
    dgain, dshift = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(D.digest_layer_norm_query(n, d), dtype=torch.uint8, device="cuda")

    def both():
        D.digest_layer_norm_forward(x, gain, shift, y, stats, EPS, D.ACT_RELU)
        D.digest_layer_norm_backward(x, gain, y, dy, stats, dx, dgain, dshift, ws, D.ACT_RELU)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((y, stats, dx, dgain, dshift), ref):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    keep = x.clone()
    for i in range(3):
        x.copy_(keep * (1 + i))
        eager = call_forward(D, x, gain, shift, True)
        eager = eager + call_backward(D, x, gain, eager[0], dy, eager[1], True)
        for v in (y, stats, dx, dgain, dshift):
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((y, stats, dx, dgain, dshift), eager):
            assert torch.equal(a, b)


def test_binding_refuses(D):
    x, y = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    ws = torch.zeros(D.digest_layer_norm_query(4, 8), dtype=torch.uint8, device="cuda")
    st, v = torch.zeros(4, 2, device="cuda"), torch.zeros(8, device="cuda")
    fwd = D.digest_layer_norm_forward
    bwd = lambda **k: D.digest_layer_norm_backward(
        k.get("x", x), k.get("gain"), k.get("y", y), k.get("dy", y), k.get("stats", st),
        k.get("dx"), k.get("dgain", v), None, k.get("ws", ws), D.ACT_RELU)
    with pytest.raises(TypeError):
        fwd(x.cpu(), None, None, y)
    with pytest.raises(TypeError):
        fwd(x.double(), None, None, y.double())
    with pytest.raises(TypeError):
        fwd(x, None, None, y.half())
    with pytest.raises(ValueError):
        fwd(x, None, None, y[:, :7])
    with pytest.raises(ValueError):
        fwd(x.t(), None, None, torch.zeros(8, 4, device="cuda"))
    with pytest.raises(ValueError):
        fwd(x[:1].expand(4, 8), None, None, y)
    with pytest.raises(ValueError):
        fwd(x, v[:7], None, y)
    with pytest.raises(D.DigestError):
        fwd(x, None, None, y, eps=0.0)
    with pytest.raises(ValueError):
        bwd(stats=None)
    with pytest.raises(ValueError):
        bwd(stats=st[:3])
    with pytest.raises(TypeError):
        bwd(y=None)
    with pytest.raises(D.DigestError):
        bwd(ws=None)
    with pytest.raises(D.DigestError):
        bwd(ws=ws[:-1])
    bwd()
