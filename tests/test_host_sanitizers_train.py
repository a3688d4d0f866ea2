"""The host code of the training operators (argument checks, coefficient bounds,
workspace layout) under AddressSanitizer and UBSan, on the CPU: their ABI
tests and a seeded fuzz of matrix lists and norm sizes run in a child process
against the g++ sanitizer build.  Any report aborts the child.  No kernel is
launched."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT

TESTS = ("test_train_abi_cpu.py", "test_train_plan_cpu.py", "test_train_factors_cpu.py")

FUZZ = r'''
import ctypes
import sys
import numpy as np
sys.path.insert(0, sys.argv[1])
ctypes.CDLL(None)["__asan_init"]   # the preloaded AddressSanitizer runtime is live
from paper_2206_00057_amd import digest as D
assert D.LIB_PATH.endswith("libdigest_host_sanitized.so"), D.LIB_PATH
L = D._train_lib()
rng = np.random.default_rng(0)
size = lambda most: int(np.exp(rng.uniform(0, np.log(most))))
# every array is exactly as long as the call may read
i32 = lambda v: (ctypes.c_int32 * len(v))(*v)
ptrs = lambda v: (ctypes.c_void_p * len(v))(*v)
planned = short = refused = 0
for trial in range(300):
    n = size(300)
    rows, cols = [size(65536) for _ in range(n)], [size(65536) for _ in range(n)]
    if trial % 5 == 1:
        rows[int(rng.integers(n))] = int(rng.choice([0, -1, 65537]))
    need = ctypes.c_size_t(0)
    st = L.digest_orthogonalize_query(n, i32(rows), i32(cols), ctypes.byref(need))
    bad = n > 256 or min(rows) < 1 or max(rows) > 65536
    assert st == (D.EINVAL if bad else D.OK), (st, n)
    planned, refused = planned + (st == D.OK), refused + (st != D.OK)
    # the calls up to the workspace that is a byte too small; addresses apart by
    # more than the largest matrix, so that nothing overlaps
    steps, grads = int(rng.integers(1, 65)), int(rng.integers(1, 65))
    at = lambda k, i: (1 << 60) + ((k * n + i) << 36)
    ld = (ctypes.c_int64 * n)(*[max(1, c) + int(rng.integers(0, 9)) for c in cols])
    nbytes = need.value - 1 if st == D.OK else 0
    st1 = L.digest_orthogonalize(n, i32(rows), i32(cols), trial % 3,
                                 ptrs([at(0, i) for i in range(n)]), ld,
                                 ptrs([at(1, i) for i in range(n)]), ld, steps, None,
                                 ctypes.c_void_p(1 << 20), nbytes, None)
    st2 = L.digest_muon_average(n, i32(rows), i32(cols), ptrs([at(0, i) for i in range(n)]),
                                ptrs([at(1, i) for i in range(n)]),
                                ptrs([at(2 + m, i) for i in range(n) for m in range(grads)]),
                                grads, 0.1, 0.9, 0.01, (ctypes.c_float * n)(*[1.0] * n), 1, steps,
                                None, ctypes.c_void_p(1 << 20), nbytes, None)
    want = D.EINVAL if bad else D.ENOMEM
    assert st1 == want and st2 == want, (st1, st2, n)
    short += 2 * (want == D.ENOMEM)
    q = L.digest_layer_norm_query(int(rng.integers(0, 2 ** 31 - 1)), size(65536),
                                  ctypes.byref(need))
    assert q == D.OK
assert planned >= 150 and short >= 300 and refused >= 40, (planned, short, refused)
print("fuzz", planned, "planned", refused, "refused")
'''


@pytest.mark.timeout(600)
def test_training_host_code_clean_under_asan_and_ubsan(tmp_path):
    from paper_2206_00057_amd import build_sanitized
    lib = build_sanitized.build()
    env = dict(os.environ)
    env.update({
        "LD_PRELOAD": build_sanitized.runtime_preload(),
        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1:halt_on_error=1",
        "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1",
        "DIGEST_LIBRARY": lib,
    })
    script = tmp_path / "fuzz.py"
    script.write_text(FUZZ)
    for cmd in ([sys.executable, str(script), ROOT],
                [sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider"] +
                [os.path.join(ROOT, "tests", t) for t in TESTS]):
        res = subprocess.run(cmd, env=env, cwd=ROOT, stdout=subprocess.PIPE,
                             stderr=subprocess.STDOUT, text=True)
        assert res.returncode == 0, res.stdout[-4000:]
        assert "ERROR: AddressSanitizer" not in res.stdout and "runtime error" not in res.stdout
