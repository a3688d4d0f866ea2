"""Performance cases of the operators on rows held in 8 bits: rows written into
a representation store and read back, the product of such rows by a weight
matrix in 8 bits, and the weight gradient from such rows kept as a checkpoint.

The format (row i of x, width d): a scale and d whole numbers,
  s_i = fl32(max_c |x_ic| / 127),  q_ic = x_ic / s_i rounded to the nearest
  (ties to even), value q_ic s_i;  s_i = 0 for a row of zeros.

  exchange     the rows sel of x go into the store, all of the store's rows
               come back in the reader's order idx: y_j = q_idx(j) s_idx(j)
  product      y_rj = act(s_r t_j sum_c q_rc p_jc), rows (q, s) with a scale
               each, the weight's output channels (p, t) with a scale each
  product of   the same from rows x and a weight W that are in hand as numbers:
  numbers      both are put into 8 bits first, W by its columns
  weight grad  D = dy (identity) or dy 1[y > 0] (ReLU),
               dw_cj = sum_r q_rc s_r D_rj

``own`` false: these in elementary torch operations; true: the calls of
``paper_2206_00057_amd.digest``.  The sizes are those of this repository's
workloads (``paper_2206_00057_amd/synth.py``: partitions of 500 to 306,250
rows, layers 64-64-16 to 602-256-41 and 100-256-256-47) and generic ones.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _exchange(name, rows, of, width, dtype):
    return dict(name=name, op="exchange", rows=rows, of=of, width=width, dtype=dtype)


def _product(name, rows, d_in, d_out, dtype, relu, numbers=False):
    return dict(name=name, op="product", rows=rows, d_in=d_in, d_out=d_out, dtype=dtype,
                relu=relu, numbers=numbers)


def _grad(name, rows, d_in, d_out, dtype, relu):
    return dict(name=name, op="grad", rows=rows, d_in=d_in, d_out=d_out, dtype=dtype, relu=relu)


def listed():
    return [
        # the boundary rows of a subgraph of a few hundred rows: launches are the cost
        _exchange("exchange_tiny", 334, 500, 64, "f32"),
        # the classes' level of the OGB-Products-sized partition: rows of an odd width
        _exchange("exchange_narrow", 304051, 306250, 47, "f32"),
        # the hidden level of the same partition
        _exchange("exchange_products", 304051, 306250, 256, "f32"),
        # wide 16-bit rows of an ordinary transformer-sized model
        _exchange("exchange_wide", 16384, 16384, 4096, "bf16"),
        # one token through a generic projection: the weight's codes are the cost
        _product("product_token", 1, 4096, 4096, "bf16", False),
        # the first layer of the Reddit-sized network on rows and weights in hand as numbers
        _product("product_dense", 29125, 602, 256, "f32", True, numbers=True),
        # a hidden layer of the OGB-Products-sized partition: the output's rows are the cost
        _product("product_products", 306250, 256, 256, "f32", True),
        # a generic projection over many tokens: the matrix instructions are the cost
        _product("product_large", 8192, 4096, 4096, "bf16", False),
        # the last layer of the smallest network
        _grad("grad_tiny", 500, 64, 16, "f32", False),
        # the first layer of the Reddit-sized network
        _grad("grad_dense", 29125, 602, 256, "f32", True),
        # a hidden layer of the OGB-Products-sized partition
        _grad("grad_products", 306250, 256, 256, "f32", True),
        # a generic projection's gradient from 16-bit rows
        _grad("grad_proj", 16384, 1024, 4096, "bf16", False),
    ]


def draw(rng):
    def log_uniform(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    def width(hi):
        return rng.choice([int(log_uniform(1, hi + 1)), rng.choice([47, 64, 100, 256, 602, 1024])])

    op = rng.choice(["exchange", "product", "grad"])
    dtype = rng.choice(list(TYPES))
    if op == "exchange":
        d = width(4096)
        of = max(1, int(min(log_uniform(1, 306251), 7.8e7 / d)))
        return dict(op=op, rows=max(1, int(of * rng.uniform(0.5, 1.0))), of=of, width=d,
                    dtype=dtype)
    d_in, d_out = width(4096), width(4096)
    # a draw costs no more than the largest case, in products and in elements
    most = min(6e10 / (d_in * d_out), 7.8e7 / max(d_in, d_out))
    rows = max(1, int(min(log_uniform(1, 306251), most)))
    case = dict(op=op, rows=rows, d_in=d_in, d_out=d_out, dtype=dtype, relu=rng.random() < 0.5)
    if op == "product":
        case["numbers"] = rng.random() < 0.3
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _padded(d):
    """Row stride of the codes of a row of d elements."""
    return (d + 15) // 16 * 16


def _activations(n, d, gen):
    """Rows of uneven scale with a few strong columns."""
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    return rnd(n, d) * torch.exp(0.5 * rnd(n, 1)) * torch.exp(0.5 * rnd(1, d))


def _codes(n, d, gen):
    """Rows as they are kept: whole numbers up to 127, zeros behind the width, scales."""
    q = (torch.randn(n, d, generator=gen, device=DEV) * 36.0).round().clamp(-127, 127)
    codes = torch.zeros(n, _padded(d), dtype=torch.int8, device=DEV)
    codes[:, :d] = q.to(torch.int8)
    return codes, torch.exp(0.5 * torch.randn(n, generator=gen, device=DEV)) * 2e-2


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    perm = lambda n: torch.randperm(n, generator=gen, device=DEV)
    t = TYPES[case["dtype"]]
    n = case["rows"]
    if case["op"] == "exchange":
        # boundary rows ascend, the reader has them in an order of its own
        sel = perm(case["of"])[:n].sort()[0]
        return dict(op="exchange", x=_activations(case["of"], case["width"], gen).to(t), sel=sel,
                    idx=perm(n))
    d_in, d_out = case["d_in"], case["d_out"]
    s = dict(op=case["op"], relu=case["relu"], d_in=d_in, type=t)
    if case["op"] == "product":
        if case["numbers"]:
            s["x"] = _activations(n, d_in, gen).to(t)
            s["w"] = (rnd(d_in, d_out) / math.sqrt(d_in)).to(t)
        else:
            s["codes"], s["scales"] = _codes(n, d_in, gen)
            s["w_codes"], s["w_scales"] = _codes(d_out, d_in, gen)
        return s
    s["codes"], s["scales"] = _codes(n, d_in, gen)
    s["dy"] = (1e-2 * rnd(n, d_out)).to(t)
    if case["relu"]:
        y = rnd(n, d_out).to(t)
        s["y"] = torch.where(y > 0, y, torch.zeros_like(y))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _quantised(x):
    """(whole numbers as float32, scales) of the rows of x; the quotients in 64
    bits, where values next to a border stay apart."""
    f = x.float()
    s = (f.abs().amax(1, keepdim=True).double() / 127.0).float()
    q = torch.where(s > 0, f.double() / s.double(), torch.zeros_like(f, dtype=torch.float64))
    return torch.round(q).float(), s[:, 0]


def _kept(state, key, make):
    """A buffer that a program allocates once and keeps."""
    if key not in state:
        state[key] = make()
    return state[key]


def run(state):
    if own:
        return _run_own(state)
    if state["op"] == "exchange":
        q, s = _quantised(state["x"].index_select(0, state["sel"]))
        codes = q.to(torch.int8)
        idx = state["idx"]
        back = codes.index_select(0, idx).float() * s.index_select(0, idx)[:, None]
        return back.to(state["x"].dtype), s
    if state["op"] == "product":
        if "x" in state:
            q, s = _quantised(state["x"])
            p, t = _quantised(state["w"].t())
        else:
            q, s = state["codes"].float(), state["scales"]
            p, t = state["w_codes"].float(), state["w_scales"]
        y = torch.mm(q, p.t()) * s[:, None] * t
        if state["relu"]:
            y = torch.where(y > 0, y, torch.zeros_like(y))
        return y.to(state["type"])
    D = state["dy"].float()
    if state["relu"]:
        D = torch.where(state["y"] > 0, D, torch.zeros_like(D))
    q = state["codes"][:, :state["d_in"]].float()
    return torch.mm(q.t(), D * state["scales"][:, None])


def _run_own(state):
    from paper_2206_00057_amd import digest as D

    if state["op"] == "exchange":
        x, sel, idx = state["x"], state["sel"], state["idx"]
        n, d = sel.numel(), x.shape[1]
        codes = _kept(state, "codes", lambda: torch.empty(
            n, D.digest_q8_stride(d), dtype=torch.int8, device=DEV))
        scales = _kept(state, "scales", lambda: torch.empty(n, device=DEV))
        back = _kept(state, "back", lambda: torch.empty(n, d, dtype=x.dtype, device=DEV))
        D.digest_quantize_rows(x, codes, scales, rows=sel)
        D.digest_dequantize_rows(codes, scales, back, rows=idx)
        return back, scales
    act = D.ACT_RELU if state["relu"] else D.ACT_IDENTITY
    if state["op"] == "product":
        if "x" in state:
            x, w = state["x"], state["w"]
            n, d_in, d_out = x.shape[0], x.shape[1], w.shape[1]
            ld = D.digest_q8_stride(d_in)
            for key, rows in (("codes", n), ("w_codes", d_out)):
                _kept(state, key, lambda: torch.empty(rows, ld, dtype=torch.int8, device=DEV))
            for key, rows in (("scales", n), ("w_scales", d_out)):
                _kept(state, key, lambda: torch.empty(rows, device=DEV))
            D.digest_quantize_rows(x, state["codes"], state["scales"])
            D.digest_quantize_columns(w, state["w_codes"], state["w_scales"])
        y = _kept(state, "out", lambda: torch.empty(
            state["codes"].shape[0], state["w_codes"].shape[0], dtype=state["type"], device=DEV))
        D.digest_q8_product(state["codes"], state["scales"], state["w_codes"], state["w_scales"],
                            y, act)
        return y
    n, d_out = state["dy"].shape
    dw = _kept(state, "dw", lambda: torch.empty(state["d_in"], d_out, device=DEV))
    ws = _kept(state, "workspace", lambda: torch.empty(
        D.digest_q8_weight_grad_query(n, state["d_in"], d_out), dtype=torch.uint8, device=DEV))
    D.digest_q8_weight_grad(state["codes"], state["scales"], state["dy"], dw, ws, act,
                            state.get("y"))
    return dw


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its values
# ---------------------------------------------------------------------------

def work(case):
    size = TYPES[case["dtype"]].itemsize
    n = case["rows"]
    if case["op"] == "exchange":
        # the rows and their indexes, the codes and scales written, the rows read back
        d = case["width"]
        return dict(bytes=2 * n * d * size + n * d + 4 * n + 16 * n, flops=6 * n * d)
    d_in, d_out = case["d_in"], case["d_out"]
    flops = 2 * n * d_in * d_out
    if case["op"] == "product":
        # a code of each element, or the number that it is made of; scales; the output
        each = size if case["numbers"] else 1
        return dict(bytes=(n + d_out) * (d_in * each + (0 if case["numbers"] else 4)) +
                    n * d_out * size, flops=flops)
    # the codes and scales, dy, with ReLU y, the gradient
    return dict(bytes=n * d_in + 4 * n + (2 if case["relu"] else 1) * n * d_out * size +
                4 * d_in * d_out, flops=flops)


def _exact_values(x):
    """The values that x's rows stand for once held in 8 bits, and the scales as
    they are held (float32), 64 bits: the nearest multiples of the scale, found
    from the whole number below and the distance to it."""
    v = x.double()
    s = torch.div(v.abs().max(dim=1).values, 127.0).to(torch.float32).double()
    safe = torch.where(s == 0, torch.ones_like(s), s)[:, None]
    low = torch.floor(v / safe)
    rest = v - low * safe            # exact: in [0, scale)
    up = (2 * rest > safe) | ((2 * rest == safe) & (low.remainder(2) == 1))
    return (low + up.double()) * s[:, None], s


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "exchange":
        v, scale = _exact_values(s["x"][s["sel"]])
        return v[s["idx"]], scale
    if case["op"] == "product":
        if case["numbers"]:
            a = _exact_values(s["x"])[0]
            b = _exact_values(s["w"].t())[0]
        else:
            k = case["d_in"]
            a = s["codes"][:, :k].double().mul_(s["scales"].double()[:, None])
            b = s["w_codes"][:, :k].double().mul_(s["w_scales"].double()[:, None])
        y = torch.mm(a, b.t().contiguous())
        return y.clamp_min(0) if case["relu"] else y
    a = s["codes"][:, :case["d_in"]].double().mul_(s["scales"].double()[:, None])
    D = s["dy"].double()
    if case["relu"]:
        D = D * (s["y"] > 0)
    return torch.mm(a.t().contiguous(), D)
