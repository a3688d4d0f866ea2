"""What the calls on rows held in 8 bits refuse, before any device work: run on
the CPU, every pointer a fake one that nothing reads."""
import ctypes

import pytest

from paper_2206_00057_amd import digest as D

P = [(i + 1) << 24 for i in range(8)]   # fake addresses, 16 MB apart


def refused(call, kws):
    for kw in kws:
        assert call(**kw) == D.EINVAL, kw


def test_quantize_rows_refuses():
    L = D._q8_lib()

    def call(n=4, d=20, t=D.F32, x=P[0], ldx=20, rows=None, n_x=4, codes=P[1], ldq=32, s=P[2]):
        return L.digest_quantize_rows(n, d, t, x, ldx, rows, n_x, codes, ldq, s, None)

    refused(call, [dict(n=-1), dict(n=2 ** 31 - 1), dict(d=0), dict(d=65537), dict(t=3),
                   dict(t=-1), dict(x=None), dict(x=P[0] + 2), dict(ldx=19), dict(ldx=2 ** 31),
                   dict(codes=None), dict(codes=P[1] + 8), dict(ldq=16), dict(ldq=40),
                   dict(ldq=2 ** 31), dict(s=None), dict(s=P[2] + 2), dict(rows=P[3] + 4),
                   dict(rows=P[3], n_x=-1), dict(rows=P[3], n_x=2 ** 31 - 1),
                   dict(codes=P[0]), dict(s=P[1] + 64), dict(s=P[0] + 316),
                   dict(rows=P[1] + 96),                        # the list in the codes' last row
                   dict(rows=P[3], n_x=1 << 20, codes=P[0] + (1 << 20))])
    assert call(n=0, x=None, codes=None, s=None) == D.OK        # no rows: nothing to do


def test_quantize_columns_refuses():
    L = D._q8_lib()

    def call(k=20, m=6, t=D.F32, w=P[0], ldw=6, codes=P[1], ldq=32, s=P[2]):
        return L.digest_quantize_columns(k, m, t, w, ldw, codes, ldq, s, None)

    refused(call, [dict(k=0), dict(k=65537), dict(m=0), dict(m=65537), dict(t=3), dict(w=None),
                   dict(w=P[0] + 1), dict(ldw=5), dict(codes=None), dict(codes=P[1] + 4),
                   dict(ldq=16), dict(ldq=24), dict(s=None), dict(s=P[2] + 1), dict(codes=P[0]),
                   dict(s=P[1] + 188)])


def test_dequantize_rows_refuses():
    L = D._q8_lib()

    def call(n=4, d=20, codes=P[1], ldq=32, s=P[2], rows=None, n_c=4, t=D.F32, y=P[0], ldy=20):
        return L.digest_dequantize_rows(n, d, codes, ldq, s, rows, n_c, t, y, ldy, None)

    refused(call, [dict(n=-1), dict(n=2 ** 31 - 1), dict(d=0), dict(d=65537), dict(t=3),
                   dict(codes=None), dict(codes=P[1] + 8), dict(ldq=16), dict(ldq=33),
                   dict(s=None), dict(s=P[2] + 2), dict(rows=P[3] + 4), dict(rows=P[3], n_c=-1),
                   dict(y=None), dict(y=P[0] + 2), dict(ldy=19), dict(ldy=2 ** 31),
                   dict(y=P[1]), dict(y=P[2] - 4), dict(rows=P[0] + 8)])
    assert call(n=0, codes=None, s=None, y=None) == D.OK


def test_product_refuses():
    L = D._q8_lib()

    def call(n=4, k=20, m=6, q=P[0], ldq=32, s=P[1], p=P[2], ldp=32, t=P[3], act=0, ty=D.F32,
             y=P[4], ldy=6):
        return L.digest_q8_product(n, k, m, q, ldq, s, p, ldp, t, act, ty, y, ldy, None)

    refused(call, [dict(n=-1), dict(n=2 ** 31 - 1), dict(k=0), dict(k=65537), dict(m=0),
                   dict(m=65537), dict(q=None), dict(q=P[0] + 8), dict(ldq=16), dict(ldq=40),
                   dict(s=None), dict(p=None), dict(p=P[2] + 1), dict(ldp=31), dict(t=None),
                   dict(t=P[3] + 2), dict(act=2), dict(ty=3), dict(y=None), dict(y=P[4] + 2),
                   dict(ldy=5), dict(y=P[0]), dict(y=P[2] + 176), dict(y=P[1] + 12),
                   dict(y=P[3] - 92)])
    assert call(n=0, q=None, s=None, y=None, p=None, t=None) == D.OK


def test_weight_grad_refuses():
    L = D._q8_lib()

    def call(n=4, k=20, m=6, q=P[0], ldq=32, s=P[1], ty=D.F32, dy=P[2], lddy=6, act=0, y=P[3],
             ldy=6, dw=P[4], ws=P[5], nbytes=1 << 20):
        return L.digest_q8_weight_grad(n, k, m, q, ldq, s, ty, dy, lddy, act, y, ldy, dw, ws,
                                       nbytes, None)

    refused(call, [dict(n=-1), dict(n=2 ** 31 - 1), dict(k=0), dict(k=65537), dict(m=0),
                   dict(m=65537), dict(q=None), dict(q=P[0] + 8), dict(ldq=16), dict(ldq=40),
                   dict(s=None), dict(ty=3), dict(dy=None), dict(dy=P[2] + 1), dict(lddy=5),
                   dict(act=2), dict(act=D.ACT_RELU, y=None), dict(act=D.ACT_RELU, ldy=5),
                   dict(dw=None), dict(dw=P[4] + 2), dict(ws=None), dict(ws=P[5] + 128),
                   dict(dw=P[2]), dict(dw=P[5]), dict(ws=P[2]),
                   dict(act=D.ACT_RELU, y=P[4] + 8)])
    need = D.digest_q8_weight_grad_query(4, 20, 6)
    assert call(nbytes=need - 1) == D.ENOMEM
    assert b"workspace" in L.digest_last_error()


def test_weight_grad_query():
    q = D.digest_q8_weight_grad_query
    for n, k, m in ((0, 1, 1), (1, 65536, 65536), (500, 64, 16), (306250, 256, 256),
                    (2 ** 31 - 2, 602, 41)):
        b = q(n, k, m)
        # partial sums of the rows' shares, 256 of them at most
        assert b % 256 == 0 and 256 <= b <= 256 * 4 * k * m + 256, (n, k, m, b)
    for n, k, m in ((-1, 8, 8), (4, 0, 8), (4, 65537, 8), (4, 8, 0), (2 ** 31 - 1, 8, 8)):
        with pytest.raises(D.DigestError):
            q(n, k, m)
    null = D._q8_lib().digest_q8_weight_grad_query(4, 8, 8, ctypes.c_void_p(0))
    assert null == D.EINVAL


def test_strides():
    assert [D.digest_q8_stride(d) for d in (1, 16, 17, 47, 64, 602)] == [16, 16, 32, 48, 64, 608]


def partition():
    """Three owned rows, two halo rows, 20 -> 24 -> 5."""
    import numpy as np
    return D.digest_partition_create(5, np.array([0, 2, 3, 5]), np.array([0, 3, 1, 2, 4]),
                                     np.ones(5, np.float32), np.arange(3), np.array([3, 4]),
                                     [20, 24, 5])


def test_partition_refuses():
    L, h = D._q8_lib(), partition()
    q = ctypes.c_void_p(P[0])
    for call in (lambda: L.digest_push_q8(h.handle, 1, q, q, q, 0, None),
                 lambda: L.digest_pull_q8(h.handle, 1, q, q, None),
                 lambda: L.digest_layer_forward_q8(h.handle, 1, q, q, q, q, 0, None)):
        assert call() == D.ESTATE                   # no workspace
    assert L.digest_push_q8(None, 1, q, q, q, 0, None) == D.EINVAL
    assert L.digest_pull_q8(None, 1, q, q, None) == D.EINVAL
    assert L.digest_partition_set_keep_mode(None, D.KEEP_Q8) == D.EINVAL
    for mode in (-1, 2):
        assert L.digest_partition_set_keep_mode(h.handle, mode) == D.EINVAL


def test_keep_mode_changes_the_workspace():
    import numpy as np
    n = 40000
    h = D.digest_partition_create(n, np.arange(n + 1), np.arange(n), np.ones(n, np.float32),
                                  np.arange(n), np.zeros(0, np.int64), [256, 256, 256, 256, 7])
    whole = h.workspace_bytes
    D.digest_partition_set_keep_mode(h, D.KEEP_Q8)
    # four AH of 4 bytes an element against one, codes of all and partial sums
    assert h.workspace_bytes < whole
    D.digest_partition_set_keep_mode(h, D.KEEP_Q8)
    D.digest_partition_set_keep_mode(h, D.KEEP_F32)
    assert h.workspace_bytes == whole
