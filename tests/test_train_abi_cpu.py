"""What the operators of the normalised layers' training refuse, before any
device work: run on the CPU, every pointer a fake one that nothing reads."""
import ctypes

import pytest

from paper_2206_00057_amd import digest as D

FAKE = ctypes.c_void_p(1 << 20)
ODD = ctypes.c_void_p((1 << 20) + 2)


def test_layer_norm_refuses():
    L = D._train_lib()

    def fwd(n=4, d=8, t=D.F32, x=FAKE, ldx=8, gain=None, shift=None, eps=1e-5, act=0, y=FAKE,
            ldy=8, stats=None):
        return L.digest_layer_norm_forward(n, d, t, x, ldx, gain, shift, eps, act, y, ldy, stats,
                                           None)

    def bwd(n=4, d=8, t=D.F32, x=FAKE, ldx=8, gain=None, act=0, y=FAKE, ldy=8, dy=FAKE, lddy=8,
            stats=FAKE, dx=FAKE, lddx=8, dgain=FAKE, dshift=FAKE, ws=FAKE, nbytes=1 << 20):
        return L.digest_layer_norm_backward(n, d, t, x, ldx, gain, act, y, ldy, dy, lddy, stats,
                                            dx, lddx, dgain, dshift, ws, nbytes, None)

    bad = [dict(n=-1), dict(n=2 ** 31 - 1), dict(d=0), dict(d=65537), dict(t=3), dict(t=-1),
           dict(act=2), dict(x=None), dict(x=ODD), dict(ldx=7), dict(ldx=2 ** 31), dict(y=None),
           dict(ldy=7), dict(gain=ODD)]
    for kw in bad + [dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=1e-40),
                     dict(eps=float("inf")), dict(shift=ODD), dict(stats=ctypes.c_void_p(1028))]:
        assert fwd(**kw) == D.EINVAL, kw
    for kw in bad + [dict(dy=None), dict(lddy=7), dict(stats=None), dict(dx=ODD), dict(lddx=0),
                     dict(dgain=ODD), dict(dshift=ODD), dict(ws=None),
                     dict(ws=ctypes.c_void_p((1 << 20) + 128))]:
        assert bwd(**kw) == D.EINVAL, kw
    need = D.digest_layer_norm_query(4, 8)
    assert bwd(nbytes=need - 1) == D.ENOMEM
    assert b"workspace" in L.digest_last_error()
    assert fwd(n=0, x=None, y=None) == D.OK     # no rows: nothing to do


def test_layer_norm_query():
    q = D.digest_layer_norm_query
    for n, d in ((0, 1), (1, 65536), (500, 64), (306250, 256), (2 ** 31 - 2, 65536)):
        b = q(n, d)
        # the sums of gain and shift, and no more than 1,024 workgroups'
        assert b % 256 == 0 and 8 * d <= b <= 1024 * 8 * d + 256, (n, d, b)
    for n, d in ((-1, 8), (4, 0), (4, 65537), (2 ** 31 - 1, 8)):
        with pytest.raises(D.DigestError):
            q(n, d)


def _i32(*v):
    return (ctypes.c_int32 * len(v))(*v)


def _i64(*v):
    return (ctypes.c_int64 * len(v))(*v)


def _f32(*v):
    return (ctypes.c_float * len(v))(*v)


def _ptrs(*v):
    return (ctypes.c_void_p * len(v))(*v)


P = [(i + 1) << 20 for i in range(12)]   # fake addresses, a megabyte apart


def test_orthogonalize_refuses():
    L = D._train_lib()

    def call(n=2, rows=_i32(4, 8), cols=_i32(8, 4), t=D.F32, ins=_ptrs(P[0], P[1]), ldi=None,
             outs=_ptrs(P[2], P[3]), ldo=None, steps=5, coeffs=None, ws=FAKE, nbytes=1 << 30):
        return L.digest_orthogonalize(n, rows, cols, t, ins, ldi, outs, ldo, steps, coeffs, ws,
                                      nbytes, None)

    for kw in [dict(n=0), dict(n=-1), dict(n=257), dict(rows=None), dict(cols=None),
               dict(rows=_i32(0, 8)), dict(cols=_i32(8, 65537)), dict(t=3), dict(ins=None),
               dict(outs=None), dict(ins=_ptrs(P[0], None)), dict(ins=_ptrs(P[0] + 2, P[1])),
               dict(outs=_ptrs(P[2], P[3] + 1)), dict(ldi=_i64(7, 4)), dict(ldo=_i64(8, 3)),
               dict(ldi=_i64(8, 2 ** 31)), dict(outs=_ptrs(P[2], P[2])), dict(steps=0),
               dict(outs=_ptrs(P[1], P[3])),                      # the other's input
               dict(steps=65), dict(steps=1, coeffs=_f32(float("nan"), 0, 0)),
               dict(steps=1, coeffs=_f32(1, float("inf"), 0)),
               dict(steps=1, coeffs=_f32(0, 0, 0)),               # nothing is left
               dict(steps=2, coeffs=_f32(1e4, 0, 0, 1e4, 0, 0)),  # grows out of range
               dict(ws=None), dict(ws=ctypes.c_void_p((1 << 20) + 64))]:
        assert call(**kw) == D.EINVAL, kw
    need = D.digest_orthogonalize_query([(4, 8), (8, 4)])
    assert call(nbytes=need - 1) == D.ENOMEM
    assert call(outs=_ptrs(P[0], P[1]), nbytes=0) == D.ENOMEM     # in place is fine


def test_muon_refuses():
    L = D._train_lib()

    def call(n=2, rows=_i32(4, 8), cols=_i32(8, 4), w=_ptrs(P[0], P[1]), mom=_ptrs(P[2], P[3]),
             grads=_ptrs(P[4], P[5], P[6], P[7]), m=2, steps=5, coeffs=None, ws=FAKE,
             nbytes=1 << 30):
        return L.digest_muon_average(n, rows, cols, w, mom, grads, m, 0.1, 0.9, 0.0, None, 1,
                                     steps, coeffs, ws, nbytes, None)

    for kw in [dict(n=0), dict(n=257), dict(rows=None), dict(rows=_i32(4, 0)), dict(m=0),
               dict(m=65), dict(w=None), dict(mom=None), dict(grads=None),
               dict(w=_ptrs(P[0], None)), dict(mom=_ptrs(P[2], P[3] + 1)),
               dict(grads=_ptrs(P[4], P[5], None, P[7])), dict(steps=0),
               dict(w=_ptrs(P[0], P[0])),                         # one weight twice
               dict(w=_ptrs(P[0], P[0] + 124)),                   # overlapping by 4 bytes
               dict(mom=_ptrs(P[0], P[3])),                       # a momentum on a weight
               dict(grads=_ptrs(P[4], P[5], P[6], P[3] + 64)),    # a gradient on a momentum
               dict(grads=_ptrs(P[0] - 124, P[5], P[6], P[7])),   # its end on a weight
               dict(ws=None)]:
        assert call(**kw) == D.EINVAL, kw
    need = D.digest_orthogonalize_query([(4, 8), (8, 4)])
    assert call(nbytes=need - 1) == D.ENOMEM
    # side by side, and gradients shared, are fine: refused for the workspace alone
    assert call(w=_ptrs(P[0], P[0] + 128), mom=_ptrs(P[0] + 256, P[0] + 384),
                grads=_ptrs(*[P[0] + 512] * 4), nbytes=0) == D.ENOMEM


def test_orthogonalize_query():
    q = D.digest_orthogonalize_query
    # five planes of 4 bytes an element, padded: at most 128 x 128 more each side
    for shapes in ([(1, 1)], [(64, 16)], [(256, 602)], [(4096, 4096)], [(7, 9000), (40, 40)]):
        b = q(shapes)
        low = sum(4 * (3 * r * c + 2 * min(r, c) ** 2) for r, c in shapes)
        up = lambda v: v + 256
        high = sum(4 * (3 * up(r) * up(c) + 2 * up(min(r, c)) ** 2) + 8192 for r, c in shapes)
        assert b % 256 == 0 and low <= b <= high, (shapes, b)
        assert b < 2 ** 40
    # large ones: at most one part of a tile for each CU and split beside the planes
    for shapes in ([(65536, 65536)], [(1024, 4096)] * 16):
        low = sum(4 * (3 * r * c + 2 * min(r, c) ** 2) for r, c in shapes)
        assert low <= q(shapes) <= low + (16 * 8192 + (1 << 28)), shapes
    # groups of sixteen share their memory
    assert q([(100, 100)] * 40) == q([(100, 100)] * 16)
    with pytest.raises(D.DigestError):
        q([(0, 4)])
    with pytest.raises(ValueError):
        q([])


def test_layer_norm_refuses_shared_outputs():
    """y may be x and dx may be dy, with one stride; no other output lies where
    another array starts."""
    L = D._train_lib()

    def fwd(x, ldx, y, ldy):
        return L.digest_layer_norm_forward(4, 8, D.F32, x, ldx, None, None, 1e-5, 0, y, ldy, None,
                                           None)

    def bwd(x=P[0], y=P[1], dy=P[2], lddy=8, dx=P[3], lddx=8, dgain=P[4], dshift=P[5]):
        return L.digest_layer_norm_backward(4, 8, D.F32, x, 8, None, D.ACT_RELU, y, 8, dy, lddy,
                                            P[6], dx, lddx, dgain, dshift, P[7], 1 << 19, None)

    assert fwd(P[0], 8, P[0], 9) == D.EINVAL
    assert fwd(P[0], 9, P[0], 8) == D.EINVAL
    for kw in (dict(dx=P[2], lddx=9), dict(dx=P[0]), dict(dx=P[1]), dict(dgain=P[5])):
        assert bwd(**kw) == D.EINVAL, kw
