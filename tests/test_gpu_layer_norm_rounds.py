"""Layer norm over more rows than the workgroups take at once: a workgroup then
comes to several rounds of rows, some of its lanes to one fewer, and the sums
of dgain and dshift run over rounds, the workgroup's rows and the workgroups.

test_every_row_counts_once: with stats (0, 1) and no gain, x_hat is x, and
small integers make every product and sum of dgain and dshift an integer below
2^24: exact in fp32 in any order, so the two are compared for equality.
The other tolerances: test_gpu_layer_norm, with the depth of the sums in place
of the rows' number."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_layer_norm import (  # noqa: E402,F401
    D, TYPES, U, _need_gpu, backward64, call_backward, call_forward, check_backward,
    check_forward, params, rows)

# several rounds and a part of one (the backward runs at most 1,024 workgroups
# of up to 1,024 elements a row, 512 up to 4,096 and 256 beyond), whole
# vectors or not, lanes of a row from 2 to 64, waves from 1 to 16, the widths
# without room for the sums (9,000 on) and the widest, read again each pass
SIZES = [(9001, 256, "f32"), (70001, 64, "f32"), (140003, 47, "bf16"), (300001, 7, "f16"),
         (9001, 602, "bf16"), (5003, 1000, "f16"), (1601, 2051, "f32"), (1301, 4096, "bf16"),
         (700, 5000, "f32"), (700, 5003, "bf16"), (601, 9000, "f16"), (530, 16384, "f32"),
         (530, 17001, "bf16")]
# past the 16 rounds after which a lane's sums are set aside, whole runs and not
LONG = [(65536, 256, "f32"), (70001, 250, "f32"), (2300001, 5, "f32"), (1200001, 13, "bf16"),
        (18001, 1030, "f16"), (4500, 4100, "f32"), (70001, 600, "bf16"), (8500, 9000, "f16")]


def layout(n, d, t):
    """Rows of x that one lane adds up, rows of a workgroup at a time, workgroups."""
    vec = 4 if t == "f32" else 8
    lanes = 2
    while lanes < 64 and lanes * vec < d:
        lanes *= 2
    at_once = 256 // lanes if d <= 1024 else 1
    groups = min(-(-n // at_once), 1024 if d <= 1024 else 512 if d <= 4096 else 256)
    return -(-n // (groups * at_once)), at_once, groups


@pytest.mark.parametrize("n,d,t", SIZES + LONG)
def test_every_row_counts_once(D, n, d, t):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(n + d)
    ints = lambda k: torch.randint(-k, k + 1, (n, d), generator=g, device="cuda").to(TYPES[t])
    x, dy, y = ints(3), ints(2), ints(1)
    stats = torch.tensor([0.0, 1.0], device="cuda").repeat(n, 1)
    assert layout(n, d, t)[0] > 1
    for relu in (False, True):
        up = dy.float() * (y > 0) if relu else dy.float()
        want = (up * x.float()).sum(0, dtype=torch.float64), up.sum(0, dtype=torch.float64)
        assert float((up * x.float()).abs().sum(0).max()) < 2 ** 24
        _, dgain, dshift = call_backward(D, x, None, y, dy, stats, relu)
        assert torch.equal(dgain.double(), want[0])
        assert torch.equal(dshift.double(), want[1])


@pytest.mark.parametrize("n,d,t", SIZES)
def test_rounds_of_rows(D, n, d, t):  # noqa: F811
    x, (gain, shift) = rows(n, d, TYPES[t], n), params(d, 3)
    dy = rows(n, d, TYPES[t], n + 1, offset=0.1)
    for relu in (False, True):
        y, stats = call_forward(D, x, gain, shift, relu)
        check_forward(y, stats, x, gain, shift, relu)
        dx, dgain, dshift = call_backward(D, x, gain, y, dy, stats, relu)
        check_backward(dx, None, None, x, gain, y, dy, stats, relu)
        _, rdg, rdb, up, _, xh, _ = backward64(x, gain, y, dy, stats, relu)
        # x_hat is rounded twice, each row's product with the sum it joins; then the
        # sum over the workgroup's rows, and the result once
        own, at_once, _ = layout(n, d, t)
        depth = own + at_once + 1
        tol = (depth + 3) * U * (up * xh).abs().sum(0)
        assert bool(((dgain.double() - rdg).abs() <= tol).all())
        assert bool(((dshift.double() - rdb).abs() <= (depth + 1) * U * up.abs().sum(0)).all())
        again = call_backward(D, x, gain, y, dy, stats, relu)
        for a, b in zip(again, (dx, dgain, dshift)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n,d,t", [(9001, 256, "f32"), (70001, 64, "f32"), (4099, 13, "f32"),
                                   (1601, 2051, "f32"), (700, 5000, "f32"), (601, 9000, "f32")])
def test_sums_over_the_workgroups_are_rounded_once(D, n, d, t):  # noqa: F811
    """Integers again, a lane's sum and a workgroup's below 2^24, so exact in fp32,
    but not their total: it comes out as the nearest fp32 number."""
    own, at_once, _ = layout(n, d, t)
    most = 2 ** 23 // (own * at_once)
    g = torch.Generator(device="cuda").manual_seed(n)
    dy = torch.randint(most // 2, most, (n, d), generator=g, device="cuda").float()
    x = torch.randint(0, 2, (n, d), generator=g, device="cuda").float()
    stats = torch.tensor([0.0, 1.0], device="cuda").repeat(n, 1)
    _, dgain, dshift = call_backward(D, x, None, None, dy, stats, False)
    total = dy.double().sum(0)
    assert float(total.max()) > 2 ** 25
    assert torch.equal(dshift, total.float())
    assert torch.equal(dgain, (dy.double() * x.double()).sum(0).float())


@pytest.mark.parametrize("n,d,t", LONG)
def test_long_sums(D, n, d, t):  # noqa: F811
    """Equal rows, whose roundings do not cancel.  Of a lane's rows at most 16 are
    added one after another, then its runs, then as in test_rounds_of_rows; one wave
    with 16 elements a lane (513 to 1,024 wide) adds them in one sum."""
    own, at_once, _ = layout(n, d, t)
    g = torch.Generator().manual_seed(d)
    row = lambda: (1.0 + torch.rand(d, generator=g)).to(TYPES[t]).cuda().expand(n, d).contiguous()
    x, dy = row(), row()
    stats = torch.tensor([0.0, 1.0], device="cuda").repeat(n, 1)
    _, dgain, dshift = call_backward(D, x, None, None, dy, stats, False)
    depth = own if 512 < d <= 1024 else min(own, 16) + own // 16
    depth += at_once + 1
    for got, want in ((dgain, dy[0].double() * x[0].double() * n), (dshift, dy[0].double() * n)):
        assert bool(((got.double() - want).abs() <= (depth + 1) * U * want).all())
