"""Which rows each launch of the calls on rows held in 8 bits is handed, on the
CPU: the host half of the kernels' file over a runtime that records launches
(``recorded_launches.cpp``).  A call's rows go to the kernels in turns of 2^21;
every turn starts where the one before ended."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from conftest import ROOT
from paper_2206_00057_amd import build as B
from paper_2206_00057_amd import digest as D

TURN = 2 ** 21
# fake addresses, far apart and never read
X, Q, S, R, P, T, Y = [(i + 1) << 48 for i in range(7)]


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    obj, lib = str(d / "q8_kernels.o"), str(d / "libdigest_launches.so")
    tests = os.path.join(ROOT, "tests")
    subprocess.run([os.path.join(B.ROCM, "bin", "hipcc"), *B.HIPCC_FLAGS, "--offload-host-only",
                    "-fuse-cuid=none", "-w", "-O1", "-c", os.path.join(B.CSRC, "q8_kernels.hip"),
                    "-o", obj], check=True)
    subprocess.run(["g++", *B.CXX_FLAGS, "-fopenmp", "-shared", "-Wl,-Bsymbolic",
                    os.path.join(B.CSRC, "digest_host.cpp"), os.path.join(B.CSRC, "digest_q8.cpp"),
                    os.path.join(tests, "host_kernels.cpp"),
                    os.path.join(tests, "recorded_launches.cpp"), obj, "-o", lib], check=True)
    return lib


@pytest.fixture
def launches(library, monkeypatch):
    """The library, and what it has launched since the last call: rows, input,
    scales, output, list (or slices) of each."""
    monkeypatch.setattr(D, "LIB_PATH", library)
    monkeypatch.setattr(D, "_lib", None)
    L = D._q8_lib()

    def recorded():
        out = np.zeros((64, 5), np.int64)
        n = L.recorded_launches(out.ctypes.data_as(ctypes.c_void_p), 64)
        return out[:n].tolist()
    yield L, recorded
    monkeypatch.undo()
    D._q8 = None


def turns(n):
    return [(r, min(TURN, n - r)) for r in range(0, n, TURN)]


ROWS = [1, TURN, TURN + 1, 2 * TURN + 77, 3 * TURN + 77, 5 * TURN]


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("t", [D.F32, D.BF16])
# (weights in LDS; tiles of 64, 128 and 256 channels)
@pytest.mark.parametrize("k,m", [(16, 5), (256, 256), (700, 300), (1024, 40), (1024, 100),
                                 (1024, 600)])
def test_product(launches, n, k, m, t):
    L, recorded = launches
    ldp, ldy = D.digest_q8_stride(k), m + 3
    ldq = ldp + 16
    assert L.digest_q8_product(n, k, m, Q, ldq, S, P, ldp, T, D.ACT_RELU, t, Y, ldy, None) == D.OK
    size = 4 if t == D.F32 else 2
    assert recorded() == [[c, Q + r * ldq, S + 4 * r, Y + size * r * ldy, 0] for r, c in turns(n)]


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("t", [D.F32, D.F16])
@pytest.mark.parametrize("d", [20, 5000])
@pytest.mark.parametrize("listed", [False, True])
def test_rows_into_codes_and_back(launches, n, d, t, listed):
    L, recorded = launches
    ldx, ldq, size = d + 1, D.digest_q8_stride(d) + 16, 4 if t == D.F32 else 2
    rows, n_x = (R, 50) if listed else (None, 0)
    take = lambda a, step: a if listed else a + step
    lists = lambda r: R + 8 * r if listed else 0
    assert L.digest_quantize_rows(n, d, t, X, ldx, rows, n_x, Q, ldq, S, None) == D.OK
    assert recorded() == [[c, take(X, size * r * ldx), S + 4 * r, Q + r * ldq, lists(r)]
                          for r, c in turns(n)]
    for ldy in (d, d + 1):
        assert L.digest_dequantize_rows(n, d, Q, ldq, S, rows, n_x, t, Y, ldy, None) == D.OK
        assert recorded() == [[c, take(Q, r * ldq), take(S, 4 * r), Y + size * r * ldy, lists(r)]
                              for r, c in turns(n)]


def star(n, widths):
    """n owned rows of one entry each, their own."""
    return D.digest_partition_create(n, np.arange(n + 1), np.arange(n), np.ones(n, np.float32),
                                     np.arange(n), np.zeros(0, np.int64), widths)


@pytest.mark.parametrize("n,k,m", [(500, 64, 64), (513, 30, 64), (1000, 2, 3), (5000, 256, 256),
                                   (20000, 300, 300), (29125, 602, 602), (60000, 100, 128),
                                   (30, 4000, 4000)])
def test_planned_slices(launches, n, k, m):
    """digest_partition_plan's slices of a weight gradient from kept codes are the
    call's."""
    L, recorded = launches
    p = star(n, [k, m, m])
    D.digest_partition_set_keep_mode(p, D.KEEP_Q8)
    pl = D.digest_partition_plan(p, 1)
    assert pl["transform_first"] == 0
    need = D.digest_q8_weight_grad_query(n, k, m)
    assert L.digest_q8_weight_grad(n, k, m, Q, D.digest_q8_stride(k), S, D.F32, X, m, D.ACT_RELU, Y,
                                   m, P, T, need, None) == D.OK
    assert [r[4] for r in recorded()] == ([] if n <= 512 and k * m < 10 ** 6 else [pl["dw_slices"]])
    assert pl["dw_slices"] == 1 or n > 512


def test_modelled_costs():
    """The cost model under both keep modes: rows of 100, 256 and 250 floats, the
    last layer transform-first (no inputs kept)."""
    n, widths = 20000, [100, 256, 250, 256, 5]
    p = star(n, widths)
    plain = D.digest_profile_model(p)
    assert not any(key.startswith("quantize_rows") for key in plain)
    D.digest_partition_set_keep_mode(p, D.KEEP_Q8)
    kept = D.digest_profile_model(p)
    for l in range(1, 5):
        k, m = widths[l - 1:l + 1]
        dw, rows = f"gemm_dw_splitk.l{l}", f"quantize_rows.l{l}"
        if D.digest_partition_plan(p, l)["transform_first"]:
            assert rows not in kept and kept[dw] == plain[dw]
            assert kept[f"splitk_reduce_dw.l{l}"] == plain[f"splitk_reduce_dw.l{l}"]
            continue
        held = n * D.digest_q8_stride(k) + 4 * n
        assert kept[rows] == (4 * n * k + held, 0, 0)
        # the codes and scales in AH's place
        assert kept[dw] == (plain[dw][0] - 4 * n * k + held, 2 * n * k * m, 0)
        assert f"splitk_reduce_dw.l{l}" not in kept
    assert D.digest_partition_plan(p, 4)["transform_first"] == 1
    same = lambda d: {k: v for k, v in d.items()
                      if not k.startswith(("gemm_dw", "quantize", "splitk"))}
    assert same(plain) == same(kept)
    D.digest_partition_set_keep_mode(p, D.KEEP_F32)
    assert D.digest_profile_model(p) == plain


@pytest.mark.parametrize("first,then", [(D.KEEP_F32, D.KEEP_Q8), (D.KEEP_Q8, D.KEEP_F32)])
def test_keep_mode_without_host_memory(launches, first, then):
    """A change of the keep mode that finds no host memory changes nothing: the
    partition stays bound in its mode and can change later."""
    L, _ = launches
    p, other = star(100, [64, 64, 5]), star(100, [64, 64, 5])
    D.digest_partition_set_keep_mode(p, first)
    D.digest_partition_set_keep_mode(other, then)
    before = D.digest_partition_query(p)
    assert before != D.digest_partition_query(other)
    room = np.zeros(before["workspace_bytes"] + 256, np.uint8)
    ws = ctypes.c_void_p((room.ctypes.data + 255) // 256 * 256)
    assert L.digest_partition_bind_workspace(
        p.handle, ws, ctypes.c_size_t(before["workspace_bytes"]), None) == D.OK
    failed = 0
    for after in range(64):
        L.fail_allocation(ctypes.c_long(after))
        st = L.digest_partition_set_keep_mode(p.handle, then)
        L.fail_allocation(ctypes.c_long(-1))
        if st == D.OK:
            break
        failed += 1
        assert st == D.ENOMEM
        assert D.digest_partition_query(p) == before
        assert L.digest_partition_set_keep_mode(p.handle, first) == D.OK   # no change
        assert D.digest_partition_query(p) == before
        assert L.digest_pull_q8(p.handle, 0, None, None, None) == D.EINVAL  # (bound)
    assert failed > 0 and st == D.OK
    assert D.digest_partition_query(p) == D.digest_partition_query(other)
    assert L.digest_pull_q8(p.handle, 0, None, None, None) == D.ESTATE      # (unbound)
