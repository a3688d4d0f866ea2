"""Calls on rows held in 8 bits over more rows than two launches take (2^21 each):
every row is that row's, the ones around the launches' borders among them."""
import numpy as np
import pytest
import torch

from paper_2206_00057_amd import digest as D

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TURN = 2 ** 21
N = 3 * TURN + 77


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def random_codes(n, d, g):
    codes = torch.zeros(n, D.digest_q8_stride(d), dtype=torch.int8, device="cuda")
    codes[:, :d] = torch.randint(-127, 128, (n, d), generator=g, device="cuda", dtype=torch.int8)
    return codes, torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-2


def borders(n):
    """The rows next to a launch's first and last."""
    at = torch.arange(0, n, TURN, device="cuda")
    rows = torch.cat([at[:, None] + torch.arange(-100, 100, device="cuda"),
                      n - 1 - torch.arange(200, device="cuda")[None]]).reshape(-1)
    return rows[(rows >= 0) & (rows < n)].unique()


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
def test_product(t):
    g = gen(1)
    q, s = random_codes(N, 16, g)
    p, w = random_codes(5, 16, g)
    y = torch.empty(N, 5, dtype=t, device="cuda")
    D.digest_q8_product(q, s, p, w, y)
    want = torch.mm(q.double(), p.double().t().contiguous()) * s.double()[:, None] * w.double()
    h = 0.0 if t == torch.float32 else torch.finfo(t).eps / 2
    tiny = 2.0 ** -25 if t == torch.float16 else 0.0
    # an exact sum, rounded, times two scales, rounded to the type
    assert bool(((y.double() - want).abs() <= 1.001 * (3 * U + h) * want.abs() + tiny).all())


@pytest.mark.parametrize("k,m", [(256, 130), (800, 40)])
def test_product_by_tiles(k, m):
    """Through the other shapes of the product's kernels: rows next to the borders
    against 64 bits, all rows against the calls of a launch each."""
    g = gen(2)
    n = 2 * TURN + 77
    q, s = random_codes(n, k, g)
    p, w = random_codes(m, k, g)
    y = torch.empty(n, m, dtype=torch.bfloat16, device="cuda")
    D.digest_q8_product(q, s, p, w, y, D.ACT_RELU)
    rows = borders(n)
    want = torch.mm(q[rows].double(), p.double().t().contiguous())
    want = (want * s[rows].double()[:, None] * w.double()).clamp_min(0)
    assert bool(((y[rows].double() - want).abs() <= 1.001 * (3 * U + 2.0 ** -8) * want).all())
    for r in range(0, n, TURN):
        part = torch.empty_like(y[r:r + TURN])
        D.digest_q8_product(q[r:r + TURN], s[r:r + TURN], p, w, part, D.ACT_RELU)
        assert torch.equal(part, y[r:r + TURN]), r


@pytest.mark.parametrize("listed", [False, True])
def test_rows_into_codes_and_back(listed):
    g = gen(3)
    d = 13
    x = torch.randn(N, d, generator=g, device="cuda")
    idx = torch.randperm(N, generator=g, device="cuda") if listed else None
    codes = torch.full((N, 16), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((N,), 5.0, device="cuda")
    D.digest_quantize_rows(x, codes, scales, rows=idx)
    xs = x[idx] if listed else x
    s = (xs.abs().amax(1).double() / 127).float()
    assert torch.equal(scales, s)
    assert torch.equal(codes[:, :d], torch.round(xs.double() / s.double()[:, None]).to(torch.int8))
    assert not bool(codes[:, d:].any())
    want = codes[:, :d].float() * scales[:, None]
    if listed:
        want = want[idx]
    for ld in (d, d + 3):                             # whole rows in a run, rows apart
        y = torch.full((N, ld), 9.0, device="cuda")
        D.digest_dequantize_rows(codes, scales, y[:, :d], rows=idx)
        assert torch.equal(y[:, :d], want) and bool((y[:, d:] == 9).all())


def test_push_and_pull():
    """A partition of more owned and halo rows than two launches take."""
    n, n_halo, d = 2 * TURN + 77, 2 * TURN + 99, 9
    # row r reads halo nodes r and, the last ones, r + n
    rows = np.minimum(np.arange(n_halo), n - 1)
    indptr = np.searchsorted(rows, np.arange(n + 1))
    owned, halo = np.arange(n) * 2 + 1, np.arange(n_halo) * 2
    p = D.digest_partition_create(2 * n_halo + 1, indptr, halo, np.ones(n_halo, np.float32), owned,
                                  halo, [d, d, 2])
    D.digest_partition_set_pull_mode(p, D.PULL_ROWS)
    ws = torch.empty(p.workspace_bytes, dtype=torch.uint8, device="cuda")
    D.digest_partition_bind_workspace(p, ws)
    x = torch.randn(p.n_global, d, generator=gen(5), device="cuda")
    codes = torch.empty(p.n_global, 16, dtype=torch.int8, device="cuda")
    scales = torch.empty(p.n_global, device="cuda")
    D.digest_quantize_rows(x, codes, scales)
    to = torch.full_like(codes, 55), torch.full_like(scales, 3.0)
    mine = torch.from_numpy(owned).cuda()
    D.digest_push_q8(p, 1, x[mine], *to, D.PUSH_ALL_OWNED)
    assert torch.equal(to[0][mine], codes[mine]) and torch.equal(to[1][mine], scales[mine])
    rest = torch.ones(p.n_global, dtype=torch.bool, device="cuda")
    rest[mine] = False
    assert bool((to[0][rest] == 55).all()) and bool((to[1][rest] == 3).all())
    D.digest_pull_q8(p, 1, codes, scales)
    out = torch.empty(n_halo, d, device="cuda")
    D.digest_partition_read_halo(p, 1, out)
    theirs = torch.from_numpy(halo).cuda()
    assert torch.equal(out, codes[theirs, :d].float() * scales[theirs, None])
