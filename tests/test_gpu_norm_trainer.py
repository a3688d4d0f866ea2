"""The trainer with layer norms and the Muon update: whole rounds against the
same network in 64 bits (full graph, gradients by autograd), each update
against its formula on the gradients that the round left, graph replays, and
the plain settings left as they were."""
import numpy as np
import pytest

from paper_2206_00057_amd import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LR, EPS = 0.2, 1e-5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def setup(K=1, model="gcn", optimizer="muon", normed=True, exchange="fresh", seed=0):
    from paper_2206_00057_amd.train import DigestTrainer
    cfg = synth.scaled(synth.CONFIGS["tiny"], 2000, widths=(64, 48, 33, 16))
    g = synth.make_graph(cfg)
    parts = [synth.make_partition(cfg, g, m) for m in range(synth.num_partitions(cfg))]
    X, y, Ws = synth.features(cfg), synth.labels(cfg), synth.weights(cfg)
    rng = np.random.default_rng(seed)
    hidden = cfg.widths[1:-1]
    norms = [(dev((1 + 0.1 * rng.standard_normal(d)).astype(np.float32)),
              dev((0.1 * rng.standard_normal(d)).astype(np.float32))) for d in hidden]
    atts = [dev((0.3 * rng.standard_normal((d, 2))).astype(np.float32)) for d in cfg.widths[1:]]
    tr = DigestTrainer(g.n, parts, cfg.widths, dev(X), dev(y), [dev(w) for w in Ws], LR, K,
                       grad_exchange=exchange if model == "gcn" else "none", model=model,
                       atts=atts if model == "gat" else None, norms=norms if normed else None,
                       optimizer=optimizer, beta=0.9, decay=0.05)
    return cfg, g, parts, tr, X, y


def state(tr):
    out = list(tr.W) + list(tr.stores[1:])
    if tr.norms is not None:
        out += [v for n in tr.norms for v in n]
    if tr.optimizer == "muon":
        out += tr.momenta
    if tr.model == "gat":
        out += tr.att
    return out


def mean_grad(tr, name, l):
    return sum(getattr(gp, name)[l].double() for gp in tr.gps) / len(tr.gps)


def network64(g, parts, X, y, Ws, norms):
    """Mean over the subgraphs of their mean cross entropy, full graph, and its
    gradients: what K = 1 with the fresh gradient exchange computes."""
    P = torch.zeros(g.n, g.n, dtype=torch.float64)
    rows = np.repeat(np.arange(g.n), np.diff(g.indptr))
    P[torch.from_numpy(rows), torch.from_numpy(g.indices)] = torch.from_numpy(
        g.values.astype(np.float64))
    Ws = [w.double().cpu().requires_grad_() for w in Ws]
    norms = [[v.double().cpu().requires_grad_() for v in n] for n in norms]
    h = torch.from_numpy(X.astype(np.float64))
    for l, w in enumerate(Ws):
        h = P @ (h @ w)
        if l < len(Ws) - 1:
            if norms:
                mean = h.mean(1, keepdim=True)
                rstd = ((h - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
                h = (h - mean) * rstd * norms[l][0] + norms[l][1]
            h = h.clamp_min(0)
    logp = h.log_softmax(1)
    nll = -logp[torch.arange(g.n), torch.from_numpy(y.astype(np.int64))]
    loss = sum(nll[torch.from_numpy(p.owned)].mean() for p in parts) / len(parts)
    loss.backward()
    return (float(loss.detach()), h.detach(), [w.grad for w in Ws],
            [[v.grad for v in n] for n in norms])


def orth64(u):
    x = u / torch.linalg.vector_norm(u)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(5):
        A = x @ x.t()
        x = 3.4445 * x + (-4.7750 * A + 2.0315 * A @ A) @ x
    return x.t() if tall else x


def close(got, ref, name, tol=1e-4):
    """The library's parity bar: 1e-4 of the largest value."""
    err = float((got.double().cpu() - ref.cpu()).abs().max())
    assert err <= tol * float(ref.abs().max()) + 1e-7, (name, err)


@pytest.mark.parametrize("optimizer", ["sgd", "muon"])
def test_rounds_match_64_bits(optimizer):
    cfg, g, parts, tr, X, y = setup(optimizer=optimizer)
    tr.init_stores()
    for r in range(1, 4):
        W0 = [w.clone() for w in tr.W]
        n0 = [[v.clone() for v in n] for n in tr.norms]
        m0 = [m.clone() for m in tr.momenta] if optimizer == "muon" else None
        loss, logits, gW, gN = network64(g, parts, X, y, tr.W, tr.norms)
        tr.round(r)
        assert abs(tr.mean_loss() - loss) <= 1e-5 + 1e-4 * abs(loss)
        for m, p in enumerate(parts):
            close(tr.gps[m].H[cfg.layers], logits[torch.from_numpy(p.owned)], f"logits {r} {m}")
        for l in range(1, cfg.layers + 1):
            grad = mean_grad(tr, "dW", l)
            close(grad, gW[l - 1], f"dW{l} round {r}")
            if l < cfg.layers:
                close(mean_grad(tr, "dGain", l), gN[l - 1][0], f"dgain{l} round {r}")
                close(mean_grad(tr, "dShift", l), gN[l - 1][1], f"dshift{l} round {r}")
            # the update, from the gradients that the round left
            w = W0[l - 1].double()
            if optimizer == "sgd":
                assert float((tr.W[l - 1].double() - (w - LR * grad)).abs().max()) <= 1e-6
            else:
                mom = 0.9 * m0[l - 1].double() + grad
                close(tr.momenta[l - 1], mom, f"momentum {l}", 1e-6)
                scale = LR * max(1.0, w.shape[1] / w.shape[0]) ** 0.5
                ref = (1 - LR * 0.05) * w - scale * orth64(grad + 0.9 * mom)
                # the mean's and momentum's roundings, a few u of U, grow by at most
                # 3.9 a step (the largest difference quotient of the polynomial)
                tol = scale * 3.9 ** 5 * 16 * U + 6 * U * float(w.norm())
                assert float((tr.W[l - 1].double() - ref).norm()) <= 2 * tol, (l, r)
            if l < cfg.layers:
                for v, b, name in zip(tr.norms[l - 1], n0[l - 1], ("dGain", "dShift")):
                    ref = b.double() - LR * mean_grad(tr, name, l)
                    assert float((v.double() - ref).abs().max()) <= 1e-6


@pytest.mark.parametrize("model", ["gcn", "gat"])
@pytest.mark.parametrize("exchange", ["none", "stale"])
def test_graph_replay_matches_eager(model, exchange):
    cfg, g, parts, tr, X, y = setup(K=2, model=model, exchange=exchange)
    start = [t.clone() for t in state(tr)]

    def restart():
        for t, s in zip(state(tr), start):
            t.copy_(s)
        if tr.grad_exchange != "none":
            for gs in tr.gstores[1:]:
                gs.zero_()
        tr.init_stores()

    restart()
    eager = []
    for r in range(1, 5):
        tr.round(r)
        eager.append([t.clone() for t in state(tr)])
    restart()
    tr.capture()
    for again in range(2):
        restart()
        for r in range(1, 5):
            tr.replay(r)
            torch.cuda.synchronize()
            for a, b in zip(state(tr), eager[r - 1]):
                assert torch.equal(a, b), (again, r)


def test_gat_norm_gradients_by_differences():
    """One subgraph of a GAT network with norms: gain and shift gradients
    against differences of the loss, which is fp32: its roundings (a few 1e-7 of
    about 3) over the step of 2e-2 allow 1e-4, the third derivative as much.  The
    twentieth beside it is room for the rows whose ReLU changes side within the
    step (about one in a hundred), not a bound."""
    from paper_2206_00057_amd import digest as D
    cfg, g, parts, tr, X, y = setup(model="gat")
    gp = tr.gps[0]
    for lev in range(len(cfg.widths) - 1):
        store = dev(X) if lev == 0 else dev(synth.relu_normal((g.n, cfg.widths[lev]), seed=lev))
        D.digest_pull(gp.p, lev, store)
    x, lab = tr.x_own[0], tr.y_own[0]

    def loss():
        gp.forward(x, tr.W)
        D.digest_softmax_xent(gp.p, gp.H[gp.L], lab, gp.dH[gp.L], gp.loss)
        return float(gp.loss)

    loss()
    gp.backward(tr.W, lab)
    grads = {(l, k): (gp.dGain, gp.dShift)[k][l].clone() for l in (1, 2) for k in (0, 1)}
    for (l, k), gr in grads.items():
        for i in (0, 7, 31):
            v, h = tr.norms[l - 1][k], 1e-2
            keep = float(v[i])
            v[i] = keep + h
            up = loss()
            v[i] = keep - h
            down = loss()
            v[i] = keep
            diff = (up - down) / (2 * h)
            assert abs(diff - float(gr[i])) <= 2e-4 + 0.05 * abs(float(gr[i])), (l, k, i)


def test_io_overlap_gives_the_same_rows():
    from paper_2206_00057_amd import step
    cfg, g, parts, tr, X, y = setup()
    stores = [dev(X)] + [dev(synth.relu_normal((g.n, cfg.widths[l]), seed=l))
                         for l in range(1, cfg.layers)]
    out = []
    for overlap in (False, True):
        mine = [s.clone() for s in stores]
        gp = step.GpuPartition(g.n, parts[1], cfg.widths, overlap_io=overlap, norms=tr.norms)
        gp.pull_all(mine)
        gp.forward(dev(X[parts[1].owned]), tr.W, mine, True, True)
        torch.cuda.synchronize()
        out.append([gp.H[gp.L].clone()] + mine)
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_refusals():
    from paper_2206_00057_amd import step
    from paper_2206_00057_amd.train import DigestTrainer
    cfg, g, parts, tr, X, y = setup()
    with pytest.raises(ValueError):
        step.GpuPartition(g.n, parts[0], cfg.widths, norms=tr.norms[:1])
    with pytest.raises(ValueError):
        DigestTrainer(g.n, parts, cfg.widths, dev(X), dev(y), tr.W, LR, 1, optimizer="adam")
