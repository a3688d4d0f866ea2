"""The hash that a counter summary carries covers the kernels' sources whole."""
import os
import re

from paper_2206_00057_amd import pmc


def test_hash_covers_every_header_the_kernels_include():
    for name in pmc.KERNEL_SOURCES:
        with open(os.path.join(pmc.CSRC, name)) as f:
            for header in re.findall(r'#include "([^"]+)"', f.read()):
                if os.path.exists(os.path.join(pmc.CSRC, header)):
                    assert header in pmc.KERNEL_SOURCES, (name, header)


def test_hash_changes_with_each_source(tmp_path, monkeypatch):
    for name in pmc.KERNEL_SOURCES:
        with open(os.path.join(pmc.CSRC, name), "rb") as f:
            (tmp_path / name).write_bytes(f.read())
    monkeypatch.setattr(pmc, "CSRC", str(tmp_path))
    seen = {pmc.kernel_source_hash()}
    for name in pmc.KERNEL_SOURCES:
        with open(tmp_path / name, "ab") as f:
            f.write(b"\n")
        seen.add(pmc.kernel_source_hash())
    assert len(seen) == 1 + len(pmc.KERNEL_SOURCES)
