"""A partition's calls on rows in 8 bits: stores, kept inputs, the forward with
the product in 8 bits, and the trainer that uses them together."""
import numpy as np
import pytest
import torch

from paper_2206_00057_amd import digest as D
from paper_2206_00057_amd import step, synth, train

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(n=700, n_halo=300, mean=9, widths=(40, 40, 33, 7), seed=0, keep=D.KEEP_F32,
         pull_mode=D.PULL_ROWS):
    """A random partition of n + n_halo + 50 nodes, and its dense matrix in 64 bits."""
    rng = np.random.default_rng(seed)
    deg = rng.integers(0, 2 * mean, n)
    if n > 200:
        deg[3], deg[5] = 0, 200                    # an empty row, a long one
    cols = [np.sort(rng.choice(n + n_halo, d, replace=False)) for d in deg]
    indptr = np.concatenate([[0], np.cumsum(deg)])
    indices = np.concatenate(cols).astype(np.int64)
    values = rng.uniform(0.1, 1.0, indices.size).astype(np.float32) / mean
    owned = np.arange(n) + 50
    halo = np.arange(n, n + n_halo) + 50
    p = D.digest_partition_create(n + n_halo + 50, indptr, indices + 50, values, owned, halo,
                                  list(widths))
    D.digest_partition_set_pull_mode(p, pull_mode)
    if keep:
        D.digest_partition_set_keep_mode(p, keep)
    bind(p)
    dense = np.zeros((n, n + n_halo))
    np.add.at(dense, (np.repeat(np.arange(n), deg), indices), values)
    return p, torch.from_numpy(dense)


def bind(p):
    ws = torch.full((p.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")
    D.digest_partition_bind_workspace(p, ws)


def rnd(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def held_rows(x):
    codes, scales = step.q8_rows(x.shape[0], x.shape[1])
    D.digest_quantize_rows(x, codes, scales)
    return codes, scales


def values_of(codes, scales, d):
    return codes[:, :d].double() * scales.double()[:, None]


@pytest.mark.parametrize("mode", [D.PUSH_BOUNDARY, D.PUSH_ALL_OWNED])
@pytest.mark.parametrize("d", [7, 40, 130])
def test_push(d, mode):
    p, _ = make(widths=(8, d, 4))
    h = rnd(p.n_own, d)
    codes, scales = step.q8_rows(p.n_global, d)
    codes.fill_(55), scales.fill_(3.0)
    D.digest_push_q8(p, 1, h, codes, scales, mode)
    bnd = D.digest_partition_export_maps(p)[2]
    rows = torch.arange(p.n_own, device="cuda") if mode == D.PUSH_ALL_OWNED else \
        torch.from_numpy(bnd.astype(np.int64)).cuda()
    want_q, want_s = step.q8_rows(p.n_global, d)
    want_q.fill_(55), want_s.fill_(3.0)
    q, s = held_rows(h)
    want_q[rows + 50], want_s[rows + 50] = q[rows], s[rows]
    assert torch.equal(codes, want_q) and torch.equal(scales, want_s)


@pytest.mark.parametrize("pull_mode", [D.PULL_ROWS, D.PULL_AGGREGATE])
@pytest.mark.parametrize("d", [7, 16, 40, 100, 130, 300])
def test_pull(d, pull_mode):
    """The halo rows, and a forward through their aggregate, against the sums in
    64 bits of the values that the store holds."""
    p, dense = make(widths=(d, d, 4), pull_mode=pull_mode)
    codes, scales = held_rows(rnd(p.n_global, d, seed=1))
    D.digest_pull_q8(p, 0, codes, scales)
    halo = values_of(codes, scales, d)[p.n_own + 50:]
    if pull_mode == D.PULL_ROWS:
        out = torch.empty(p.n_halo, d, device="cuda")
        D.digest_partition_read_halo(p, 0, out)
        assert torch.equal(out, halo.float())
    h = rnd(p.n_own, d, seed=2)
    eye = torch.eye(d, device="cuda")
    y = torch.empty(p.n_own, d, device="cuda")
    D.digest_layer_forward(p, 1, h, eye, y, D.ACT_RELU)
    src = torch.cat([h.double(), halo]).cpu()
    want, size = dense @ src, dense.abs() @ src.abs()
    # the sums of at most 200 terms in fp32, each rounded thrice at most, and the product
    err = (y.cpu().double() - want.clamp_min(0)).abs()
    assert bool((err <= 220 * U * size + 1e-30).all()), float((err / size.clamp_min(1e-30)).max())


@pytest.mark.parametrize("pull_mode", [D.PULL_ROWS, D.PULL_AGGREGATE])
@pytest.mark.parametrize("d", [3, 47, 64, 65, 256, 602, 1100])
def test_pull_of_long_rows(d, pull_mode):
    """Rows of up to 1,000 halo entries, repeated ones among them, and one without
    an entry; the same bits each time."""
    rng = np.random.default_rng(d)
    n, n_halo = 40, 500
    deg = np.array([0, 1, 2, 63, 64, 65, 66, 500, 511, 512, 513, 1000] + [5] * (n - 12))
    cols = n + rng.integers(0, n_halo, deg.sum())
    indptr = np.concatenate([[0], np.cumsum(deg)])
    values = rng.uniform(-1, 1, deg.sum()).astype(np.float32)
    p = D.digest_partition_create(n + n_halo, indptr, cols, values, np.arange(n),
                                  np.arange(n, n + n_halo), [d, 5])
    D.digest_partition_set_pull_mode(p, pull_mode)
    bind(p)
    codes, scales = held_rows(rnd(p.n_global, d, seed=1))
    dense = np.zeros((n, n_halo))
    np.add.at(dense, (np.repeat(np.arange(n), deg), cols - n), values)
    size = np.zeros((n, n_halo))
    np.add.at(size, (np.repeat(np.arange(n), deg), cols - n), np.abs(values))
    halo = values_of(codes, scales, d)[n:].cpu()
    want, size = torch.from_numpy(dense) @ halo, torch.from_numpy(size) @ halo.abs()
    w = rnd(d, 5, seed=2)
    h = torch.zeros(n, d, device="cuda")
    ys = []
    for _ in range(2):
        D.digest_pull_q8(p, 0, codes, scales)
        ys.append(torch.empty(n, 5, device="cuda"))
        D.digest_layer_forward(p, 1, h, w, ys[-1], D.ACT_IDENTITY)
    assert torch.equal(*ys)
    W = w.cpu().double()
    # terms rounded three times at most, 1,001 sums, then the product over d
    bound = (1010 + d) * U * (size @ W.abs())
    assert bool(((ys[0].cpu().double() - want @ W).abs() <= bound).all())


@pytest.mark.parametrize("pull_mode", [D.PULL_ROWS, D.PULL_AGGREGATE])
def test_pull_of_rows_that_are_nan(pull_mode):
    p, dense = make(widths=(12, 9, 4), pull_mode=pull_mode)
    x = rnd(p.n_global, 12)
    x[50 + p.n_own + 4, 3] = float("inf")
    D.digest_pull_q8(p, 0, *held_rows(x))
    y = torch.empty(p.n_own, 9, device="cuda")
    D.digest_layer_forward(p, 1, rnd(p.n_own, 12), rnd(12, 9), y, D.ACT_IDENTITY)
    touched = dense[:, p.n_own + 4] != 0
    assert torch.equal(torch.isnan(y).any(1).cpu(), touched)


def run_layer(p, layer, h, w, dy, forward, act=D.ACT_RELU, halo=False):
    y = torch.empty(p.n_own, p.widths[layer], device="cuda")
    dw = torch.empty_like(w)
    dh = torch.empty(p.n_own, p.widths[layer - 1], device="cuda")
    forward(y)
    if halo:
        dhalo = torch.empty(p.n_halo, p.widths[layer - 1], device="cuda")
        D.digest_layer_backward_halo(p, layer, h, y, dy, w, dw, dh, dhalo)
        return y, dw, dh, dhalo
    D.digest_layer_backward(p, layer, h, y, dy, w, dw, dh)
    return y, dw, dh


def aggregated(p, dense, h, store):
    src = torch.cat([h, store[p.n_own + 50:]]).cpu().double()
    return dense @ src


@pytest.mark.parametrize("n,layer,widths,act", [
    (700, 2, (16, 40, 33, 7), D.ACT_RELU), (700, 2, (16, 40, 33, 7), D.ACT_IDENTITY),
    (700, 3, (16, 40, 33, 7), D.ACT_IDENTITY), (17000, 2, (16, 100, 90, 7), D.ACT_RELU),
    (700, 2, (16, 33, 130, 7), D.ACT_RELU), (1, 2, (16, 33, 130, 7), D.ACT_RELU),
    (3000, 2, (8, 602, 256, 5), D.ACT_RELU)])
def test_kept_inputs(n, layer, widths, act):
    """dw is that of the AH held in 8 bits; everything else is as before."""
    d, m = widths[layer - 1], widths[layer]
    pair = [make(n=n, widths=widths, keep=k) if n < 4000 else sparse(n, widths, k)
            for k in (D.KEEP_F32, D.KEEP_Q8)]
    h, w, dy = rnd(n, d, seed=1), rnd(d, m, seed=2) / d ** 0.5, rnd(n, m, seed=3)
    outs = []
    for p, dense in pair:
        store = rnd(p.n_global, d, seed=4)
        D.digest_pull(p, layer - 1, store)
        outs.append(run_layer(p, layer, h, w, dy,
                              lambda y: D.digest_layer_forward(p, layer, h, w, y, act), act))
    (y0, dw0, dh0), (y1, dw1, dh1) = outs
    assert torch.equal(y0, y1) and torch.equal(dh0, dh1)
    if D.digest_partition_plan(pair[1][0], layer)["transform_first"] and act == D.ACT_IDENTITY:
        assert torch.equal(dw0, dw1)
        return
    # AH's values are off by half a scale each (and a little: AH itself is rounded)
    ah = (dense @ torch.cat([h, store[p.n_own + 50:]]).cpu().double()) if dense is not None else None
    mask = (y0 > 0).double().cpu() if act == D.ACT_RELU else 1.0
    D64 = (dy.cpu().double() * mask).abs()
    if ah is not None:
        s = ah.abs().amax(1) / 127
        bound = torch.mm((s[:, None] * 0.501).expand(-1, d).t(), D64)
        bound = bound + 2 * (n + 300) * U * torch.mm(ah.abs().t(), D64)
        want = torch.mm(ah.t(), dy.cpu().double() * mask)
        assert bool(((dw1.cpu().double() - want).abs() <= bound).all())
    rel = float((dw1 - dw0).norm() / dw0.norm())
    assert 0 < rel < 0.03, rel


def sparse(n, widths, keep):
    """A partition of the size where the fused passes run, its own chain of rows."""
    idx = (np.arange(n)[:, None] + np.array([0, 1, 7])) % n
    halo = n + np.arange(n) % 200
    indices = np.concatenate([idx, halo[:, None]], 1).reshape(-1)
    p = D.digest_partition_create(n + 200, np.arange(n + 1) * 4, indices,
                                  np.full(4 * n, 0.25, np.float32), np.arange(n),
                                  np.arange(n, n + 200), list(widths))
    if keep:
        D.digest_partition_set_keep_mode(p, keep)
    bind(p)
    return p, None


@pytest.mark.parametrize("n,d,act,halo", [(700, 40, D.ACT_RELU, False), (700, 40, D.ACT_IDENTITY, True),
                                          (300, 33, D.ACT_RELU, True), (1, 20, D.ACT_RELU, False),
                                          (900, 260, D.ACT_RELU, False)])
def test_forward_q8(n, d, act, halo):
    p, dense = make(n=n, widths=(8, d, d, 5), keep=D.KEEP_Q8)
    h, w, dy = rnd(n, d, seed=1), rnd(d, d, seed=2) / d ** 0.5, rnd(n, d, seed=3)
    store = rnd(p.n_global, d, seed=4)
    D.digest_pull(p, 1, store)
    # through the unit matrix (codes 127 at scale 1 / 127, a value of 1 to 2^-23) the
    # layer gives its AH held in 8 bits
    eye = held_rows(torch.eye(d, device="cuda"))
    a = torch.empty(n, d, device="cuda")
    D.digest_layer_forward_q8(p, 2, h, *eye, a, D.ACT_IDENTITY)
    A = a.double().cpu()
    ah = aggregated(p, dense, h, store)
    s = ah.abs().amax(1, keepdim=True) / 127
    assert bool(((A - ah).abs() <= 0.5001 * s + 300 * U * ah.abs().amax(1, keepdim=True)).all())
    wq = held_rows(w.t().contiguous())
    fwd = lambda y: D.digest_layer_forward_q8(p, 2, h, *wq, y, act)
    outs = run_layer(p, 2, h, w, dy, fwd, act, halo)
    y, dw, dh = outs[:3]
    W = values_of(*wq, d).cpu().t()
    want = torch.mm(A, W)
    size = torch.mm(A.abs(), W.abs())
    got = y.cpu().double()
    ref = want.clamp_min(0) if act == D.ACT_RELU else want
    # A's 2^-22 (two scales' and products' roundings) and three more roundings
    assert bool(((got - ref).abs() <= 10 * U * size).all())
    mask = (y > 0).cpu().double() if act == D.ACT_RELU else torch.ones_like(want)
    D64 = dy.cpu().double() * mask
    assert bool(((dw.cpu().double() - torch.mm(A.t(), D64)).abs() <=
                 2 * (n + 10) * U * torch.mm(A.abs().t(), D64.abs())).all())
    g = torch.mm(D64, w.cpu().double().t())
    back = dense.t() @ g
    size = dense.t().abs() @ torch.mm(D64.abs(), w.cpu().double().abs().t())
    both = torch.cat([dh] + list(outs[3:])).cpu().double()
    assert bool(((both - back[:both.shape[0]]).abs() <= 600 * U * size[:both.shape[0]]).all())


def test_states():
    p, _ = make(widths=(8, 20, 5))
    h, w = rnd(p.n_own, 8), held_rows(rnd(20, 8))
    y = torch.empty(p.n_own, 20, device="cuda")
    D.digest_pull(p, 0, rnd(p.n_global, 8))
    with pytest.raises(D.DigestError) as e:         # inputs are not kept in 8 bits
        D.digest_layer_forward_q8(p, 1, h, *w, y, D.ACT_RELU)
    assert e.value.status == D.ESTATE
    D.digest_partition_set_keep_mode(p, D.KEEP_F32)  # no change: still bound
    D.digest_layer_forward(p, 1, h, rnd(8, 20), y, D.ACT_RELU)
    D.digest_partition_set_keep_mode(p, D.KEEP_Q8)   # a change: unbound
    with pytest.raises(D.DigestError) as e:
        D.digest_layer_forward(p, 1, h, rnd(8, 20), y, D.ACT_RELU)
    assert e.value.status == D.ESTATE
    bind(p)
    with pytest.raises(D.DigestError) as e:          # not pulled since
        D.digest_layer_forward_q8(p, 1, h, *w, y, D.ACT_RELU)
    assert e.value.status == D.ESTATE
    D.digest_pull(p, 0, rnd(p.n_global, 8))
    with pytest.raises(D.DigestError) as e:          # no forward since
        D.digest_layer_backward(p, 1, h, y, y, rnd(8, 20), rnd(8, 20))
    assert e.value.status == D.ESTATE
    D.digest_layer_forward_q8(p, 1, h, *w, y, D.ACT_RELU)
    D.digest_layer_backward(p, 1, h, y, y, rnd(8, 20), rnd(8, 20))
    for level in (0, 2):
        with pytest.raises(D.DigestError):
            D.digest_push_q8(p, level, y, *step.q8_rows(p.n_global, 20))
    with pytest.raises(ValueError):
        D.digest_push_q8(p, 1, y, *step.q8_rows(p.n_global, 40))
    with pytest.raises(TypeError):
        D.digest_pull_q8(p, 0, rnd(p.n_global, 16), rnd(p.n_global))
    with pytest.raises(ValueError):
        step.GpuPartition(3, None, [4, 4], keep="f32", product="q8")
    with pytest.raises(ValueError):
        step.GpuPartition(3, None, [4, 4], model="gat", atts=[None], keep="q8")


def trainer(K=2, **kw):
    cfg = synth.CONFIGS["tiny"]
    g = synth.make_graph(cfg)
    parts = [synth.make_partition(cfg, g, m) for m in range(4)]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    norms = None
    if kw.pop("normed", False):
        norms = [(torch.ones(d, device="cuda"), torch.zeros(d, device="cuda"))
                 for d in cfg.widths[1:-1]]
    atts = None
    if kw.get("model") == "gat":
        atts = [rnd(d, 2, seed=5) * (2 / (d + 2)) ** 0.5 for d in cfg.widths[1:]]
    tr = train.DigestTrainer(g.n, parts, cfg.widths, dev(synth.features(cfg)),
                             dev(synth.labels(cfg)), [dev(w) for w in synth.weights(cfg)], 0.1, K,
                             norms=norms, atts=atts, **kw)
    tr.init_stores()
    return tr


FLAVOURS = [dict(store="q8"), dict(keep="q8"), dict(keep="q8", product="q8"),
            dict(store="q8", keep="q8", product="q8", grad_exchange="fresh"),
            dict(store="q8", keep="q8", product="q8", normed=True, optimizer="muon"),
            dict(store="q8", model="gat")]


@pytest.mark.parametrize("kw", FLAVOURS)
def test_trainer_near_float(kw):
    """The gradients of two rounds are those of the float32 trainer but for the
    roundings.  An element is held to a 254th of its row's largest, three or four
    times its typical size: off by up to 0.8% of that, with three roundings up to
    1.1% (e) in a layer's output and below 5% in a gradient's norm.  With products in 8
    bits a ReLU's input moves too: of two normal numbers at the angle e an e / pi part
    differ in sign, 0.35% of all, and each takes a whole element of D, of which half
    are not zero, out or in: sqrt(0.0035 / 0.5) = 8.4% of its norm more."""
    plain = {k: v for k, v in kw.items() if k in ("grad_exchange", "normed", "optimizer", "model")}
    a, b = trainer(**kw), trainer(**plain)
    for r in (1, 2):
        a.round(r), b.round(r)
    for x, y in zip(a.gps, b.gps):
        for l in range(1, a.L + 1):
            rel = float((x.dW[l] - y.dW[l]).norm() / y.dW[l].norm())
            assert rel < 0.05 + 0.084, (l, rel)
    assert abs(a.mean_loss() - b.mean_loss()) < 0.01 * b.mean_loss()


@pytest.mark.parametrize("kw", FLAVOURS)
def test_trainer_replays(kw):
    """Rounds replayed from graphs equal eager ones bit for bit."""
    a, b = trainer(**kw), trainer(**kw)
    state = lambda t: t.W + [v for s in t.stores[1:] for v in (s if isinstance(s, tuple) else (s,))]
    keep = [v.clone() for v in state(b)] + [m.clone() for m in getattr(b, "momenta", [])]
    more = [v for n in (b.norms or []) for v in n] + list(b.att or [])
    kept_more = [v.clone() for v in more]
    b.capture()
    for v, k in zip(state(b) + list(getattr(b, "momenta", [])) + more, keep + kept_more):
        v.copy_(k)
    for gp in b.gps:                                 # the stores as they were, pulled again
        for lev in range(1, b.L):
            step.pull(gp.p, lev, b.stores[lev])
    if b.grad_exchange != "none":
        for gs in b.gstores[1:]:
            gs.zero_()
    for r in range(1, 6):
        a.round(r)
        b.replay(r)
        torch.cuda.synchronize()
        for x, y in zip(state(a), state(b)):
            assert torch.equal(x, y), r


def test_single_partition_rounds():
    """step.GpuPartition with its store in 8 bits, in line and with pulls and pushes
    on a second stream."""
    cfg = synth.CONFIGS["tiny"]
    g = synth.make_graph(cfg)
    part = synth.make_partition(cfg, g, 0)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    X, Ws = dev(synth.features(cfg)), [dev(w) for w in synth.weights(cfg)]
    x_own, y = X[dev(part.owned)], dev(synth.labels(cfg)[part.owned])
    got = []
    for overlap in (False, True):
        stores = [X, held_rows(rnd(g.n, cfg.widths[1], seed=3).clamp_min(0))]
        gp = step.GpuPartition(g.n, part, cfg.widths, overlap_io=overlap, keep="q8", product="q8")
        gp.pull_all(stores)
        for r in range(1, 5):
            gp.round(r, 2, x_own, Ws, stores, y)
        torch.cuda.synchronize()
        got.append([gp.H[cfg.layers].clone(), *[w.clone() for w in gp.dW[1:]], *stores[1]])
    assert all(torch.equal(a, b) for a, b in zip(*got))
