"""The gradients of layers whose products run in 8 bits: those of the function that
ran, with its roundings as constants.  With Q(x) the values that x is held as,
  y = act(Q(AH) Q(W)),  AH = P_in h + P_out halo,  D = dy or dy 1[y > 0],
  dw = Q(AH)^T D,  dh = P_in^T D Q(W)^T,  dhalo = P_out^T D Q(W)^T.
"""
import numpy as np
import pytest
import torch

from paper_2206_00057_amd import digest as D
from paper_2206_00057_amd import step, synth, train

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def rnd(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def held(W):
    """(codes, scales) of W's columns, and the values that they stand for."""
    codes, scales = step.q8_rows(W.shape[1], W.shape[0])
    D.digest_quantize_columns(W, codes, scales)
    columns = torch.empty(W.shape[1], W.shape[0], device="cuda")
    D.digest_dequantize_rows(codes, scales, columns)
    return codes, scales, columns.t().contiguous()


def partition(n=300, n_halo=80, widths=(8, 20, 12, 5), seed=0):
    rng = np.random.default_rng(seed)
    deg = rng.integers(0, 9, n)
    cols = np.concatenate([np.sort(rng.choice(n + n_halo, d, replace=False)) for d in deg])
    values = rng.uniform(0.1, 1.0, cols.size).astype(np.float32) / 4
    p = D.digest_partition_create(n + n_halo, np.concatenate([[0], np.cumsum(deg)]), cols, values,
                                  np.arange(n), np.arange(n, n + n_halo), list(widths))
    D.digest_partition_set_keep_mode(p, D.KEEP_Q8)
    ws = torch.empty(p.workspace_bytes, dtype=torch.uint8, device="cuda")
    D.digest_partition_bind_workspace(p, ws)
    dense = np.zeros((n, n + n_halo))
    np.add.at(dense, (np.repeat(np.arange(n), deg), cols), values)
    return p, torch.from_numpy(dense), ws


@pytest.mark.parametrize("act", [D.ACT_RELU, D.ACT_IDENTITY])
@pytest.mark.parametrize("widths", [(8, 20, 12, 5), (8, 33, 130, 5)])
def test_backward_with_the_values_of_the_codes(widths, act):
    """Against the formulas, against differences of the function with its roundings
    held, and how far the gradients with the unrounded W are off."""
    p, dense, _ = partition(widths=widths)
    n, d, m = p.n_own, widths[1], widths[2]
    h, W, dy = rnd(n, d, seed=1), rnd(d, m, seed=2) / d ** 0.5, rnd(n, m, seed=3)
    store = rnd(p.n_global, d, seed=4)
    D.digest_pull(p, 1, store)
    codes, scales, value = held(W)
    y = torch.empty(n, m, device="cuda")
    D.digest_layer_forward_q8(p, 2, h, codes, scales, y, act)
    out = {}
    for name, w in (("value", value), ("whole", W)):
        dw, dh = torch.empty(d, m, device="cuda"), torch.empty(n, d, device="cuda")
        dhalo = torch.empty(p.n_halo, d, device="cuda")
        D.digest_layer_backward_halo(p, 2, h, y, dy, w, dw, dh, dhalo)
        out[name] = dw, torch.cat([dh, dhalo]).cpu().double()
    assert torch.equal(out["value"][0], out["whole"][0])
    mask = (y > 0).double().cpu() if act == D.ACT_RELU else torch.ones(n, m, dtype=torch.float64)
    D64, V = dy.cpu().double() * mask, value.cpu().double()
    want = dense.t() @ (D64 @ V.t())
    size = dense.t() @ (D64.abs() @ V.abs().t())
    # the two sums of at most m and n terms in fp32
    assert bool(((out["value"][1] - want).abs() <= (n + m + 10) * U * size).all())
    # the function with its roundings held, by differences in 64 bits
    src = torch.cat([h, store[n:]]).cpu().double()
    pre = (dense @ src) @ V
    live = mask

    def loss(x):
        return float((((dense @ x) @ V) * live * dy.cpu().double()).sum())
    step_of = 1e-3
    for r, c in ((0, 0), (n // 2, d - 1), (n + 3, 5)):
        e = torch.zeros_like(src)
        e[r, c] = step_of
        # (linear in x where the mask is held: no error but the sums')
        diff = (loss(src + e) - loss(src - e)) / (2 * step_of)
        total = float((pre.abs() * live * dy.cpu().double().abs()).sum())
        assert abs(diff - float(out["value"][1][r, c])) <= (
            (n + m + 10) * U * float(size[r, c]) + 1e-11 * total / step_of)
    # with the unrounded W: off by at most half a scale for each of D's elements
    half = dense.t() @ (D64.abs() @ (scales.cpu().double() / 2))[:, None].expand(-1, d)
    bound = half * (1 + 1e-5) + 2 * (n + m + 10) * U * size
    assert bool(((out["whole"][1] - want).abs() <= bound).all())
    assert bool(((out["whole"][1] - want).abs() > 2 * (n + m + 10) * U * size).any())


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def tiny():
    cfg = synth.CONFIGS["tiny"]
    return cfg, synth.make_graph(cfg)


def test_single_partition():
    """step.GpuPartition's backward takes the values that its forward multiplied by,
    also when the weights have changed since, eagerly and from a graph."""
    cfg, g = tiny()
    part = synth.make_partition(cfg, g, 0)
    X, Ws = dev(synth.features(cfg)), [dev(w) for w in synth.weights(cfg)]
    x_own, labels = X[dev(part.owned)], dev(synth.labels(cfg)[part.owned])
    gp = step.GpuPartition(g.n, part, cfg.widths, keep="q8", product="q8")
    stores = [X, step.q8_rows(g.n, cfg.widths[1])]
    gp.pull_all(stores)

    def check():
        for l in range(2, gp.L + 1):
            dw, dh = torch.empty_like(gp.dW[l]), torch.empty_like(gp.dH[l - 1])
            D.digest_layer_backward(gp.p, l, gp.H[l - 1], gp.H[l], gp.dH[l], values[l - 1], dw, dh)
            assert torch.equal(dw, gp.dW[l]) and torch.equal(dh, gp.dH[l - 1])
            assert bool(dh.any())
    values = [held(W)[2] for W in Ws]
    gp.forward(x_own, Ws)
    gp.backward(Ws, labels)
    check()
    gp.forward(x_own, Ws)
    for W in Ws:
        W.mul_(1.5)
    gp.backward(Ws, labels)
    check()
    gp.capture(2, x_own, Ws, stores, labels)
    for turn in range(3):
        for W in Ws:
            W.copy_(rnd(*W.shape, seed=turn) * 0.2)
        values = [held(W)[2] for W in Ws]
        gp.replay(1, 2)
        torch.cuda.synchronize()
        check()


@pytest.mark.parametrize("exchange", ["none", "fresh"])
def test_trainer(exchange):
    """A round's input and halo gradients are those of the weights' values."""
    cfg, g = tiny()
    parts = [synth.make_partition(cfg, g, m) for m in range(4)]
    tr = train.DigestTrainer(g.n, parts, cfg.widths, dev(synth.features(cfg)),
                             dev(synth.labels(cfg)), [dev(w) for w in synth.weights(cfg)], 0.1, 2,
                             store="q8", keep="q8", product="q8", grad_exchange=exchange)
    tr.init_stores()
    assert not any(wq for gp in tr.gps for wq in gp.Wq)   # (all take the trainer's)
    for r in (1, 2, 3):
        values = [held(W)[2] for W in tr.W]
        tr.round(r)
        for m, gp in enumerate(tr.gps):
            for l in range(2, tr.L + 1):
                dw, dh = torch.empty_like(gp.dW[l]), torch.empty_like(gp.dH[l - 1])
                if exchange == "none":
                    D.digest_layer_backward(gp.p, l, gp.H[l - 1], gp.H[l], gp.dH[l], values[l - 1],
                                            dw, dh)
                    assert torch.equal(dh, gp.dH[l - 1])
                else:                                 # (dH holds the others' parts too)
                    halo = torch.empty_like(tr.dh_halo[m][l - 1])
                    D.digest_layer_backward_halo(gp.p, l, gp.H[l - 1], gp.H[l], gp.dH[l],
                                                 values[l - 1], dw, dh, halo)
                    assert torch.equal(halo, tr.dh_halo[m][l - 1]) and bool(halo.any())
                assert torch.equal(dw, gp.dW[l])


def test_backward_before_a_forward():
    cfg, g = tiny()
    gp = step.GpuPartition(g.n, synth.make_partition(cfg, g, 0), cfg.widths, keep="q8",
                           product="q8")
    h, W = torch.zeros(gp.n_own, cfg.widths[1], device="cuda"), dev(synth.weights(cfg)[1])
    with pytest.raises(D.DigestError) as e:
        gp.layer_backward(2, h, W, gp.dH[1])
    assert e.value.status == D.ESTATE


def test_layer_on_another_stream():
    """A layer's calls on a stream given as an object or as a number."""
    cfg, g = tiny()
    part = synth.make_partition(cfg, g, 0)
    W, h = dev(synth.weights(cfg)[0]), dev(synth.features(cfg))[dev(part.owned)]
    got = []
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        gp = step.GpuPartition(g.n, part, cfg.widths, keep="q8", product="q8")
        D.digest_pull(gp.p, 0, dev(synth.features(cfg)))
        torch.cuda.synchronize()
        gp.layer_forward(1, h, W, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(gp.held[1].values, held(W)[2])
        got.append(gp.H[1].clone())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
