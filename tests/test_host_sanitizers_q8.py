"""The host code of the calls on rows held in 8 bits (argument checks, overlaps,
workspace sizes, a partition's modes) under AddressSanitizer and UBSan, on the
CPU: their ABI tests and a seeded fuzz of sizes run in a child process against the
g++ sanitizer build.  Any report aborts the child.  No kernel is launched."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT

FUZZ = r'''
import ctypes
import sys
import numpy as np
sys.path.insert(0, sys.argv[1])
ctypes.CDLL(None)["__asan_init"]   # the preloaded AddressSanitizer runtime is live
from paper_2206_00057_amd import digest as D
assert D.LIB_PATH.endswith("libdigest_host_sanitized.so"), D.LIB_PATH
L = D._q8_lib()
rng = np.random.default_rng(0)
size = lambda most: int(np.exp(rng.uniform(0, np.log(most))))
at = lambda i: (1 << 40) + (i << 50)
refused = 0
for trial in range(2000):
    n, k, m = size(2 ** 31 - 2), size(65536), size(65536)
    need = D.digest_q8_weight_grad_query(n, k, m)
    assert need % 256 == 0 and need >= 256
    ldq, ld = D.digest_q8_stride(k) + 16 * int(rng.integers(0, 9)), m + int(rng.integers(0, 9))
    if trial % 4 == 0:
        ldq = min(ldq, 2 ** 31 - 16)
    t = int(rng.integers(0, 3))
    # a byte too small
    st = L.digest_q8_weight_grad(n, k, m, at(1), ldq, at(2), t, at(3), ld, 1, None, 0, at(4), at(5),
                                 need - 1, None)
    assert st == D.ENOMEM, st
    # outputs on inputs, at their last element
    last = ((n - 1) * ldq + D.digest_q8_stride(k) - 1) // 4 * 4
    st = L.digest_q8_weight_grad(n, k, m, at(1), ldq, at(2), t, at(3), ld, 1, None, 0,
                                 at(1) + last, at(5), need, None)
    assert st == D.EINVAL, st
    st = L.digest_q8_product(n, k, m, at(1), ldq, at(2), at(3), ldq, at(4), 1, t,
                             at(2) + 4 * (n - 1), ld, None)
    assert st == D.EINVAL, st
    st = L.digest_quantize_rows(n, k, t, at(1), 2 ** 31, None, 0, at(2), ldq, at(3), None)
    assert st == D.EINVAL, st
    refused += 4
for n in (1, 10, 300):
    h = D.digest_partition_create(n, np.arange(n + 1), np.arange(n), np.ones(n, np.float32),
                                  np.arange(n), np.zeros(0, np.int64),
                                  [size(700) for _ in range(1 + size(20))])
    first = h.workspace_bytes
    for mode in (1, 1, 0, 1, 0, 0):
        D.digest_partition_set_keep_mode(h, mode)
    assert h.workspace_bytes == first
print("fuzz", refused, "refused")
'''


@pytest.mark.timeout(600)
def test_host_code_of_8_bit_rows_clean_under_asan_and_ubsan(tmp_path):
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
                [sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                 os.path.join(ROOT, "tests", "test_q8_abi_cpu.py")]):
        res = subprocess.run(cmd, env=env, cwd=ROOT, stdout=subprocess.PIPE,
                             stderr=subprocess.STDOUT, text=True)
        assert res.returncode == 0, res.stdout[-4000:]
        assert "ERROR: AddressSanitizer" not in res.stdout and "runtime error" not in res.stdout
