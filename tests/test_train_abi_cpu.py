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
