"""The kernel times of the rows held in 8 bits are of the code that is here."""
import os
import re

from conftest import ROOT
from paper_2206_00057_amd import pmc


def test_summary_names_the_present_code():
    with open(os.path.join(ROOT, "profiles", "q8_kernel_stats.txt")) as f:
        named = re.findall(r"^# code: ([0-9a-f]{16})$", f.read(), re.M)
    assert named == [pmc.code_hash(pmc.Q8_SOURCES)]


def test_hash_covers_every_header():
    for name in pmc.Q8_SOURCES:
        with open(os.path.join(pmc.CSRC, name)) as f:
            for header in re.findall(r'#include "([^"]+)"', f.read()):
                if os.path.exists(os.path.join(pmc.CSRC, header)):
                    assert header in pmc.Q8_SOURCES, (name, header)


def test_hash_is_of_the_code(tmp_path, monkeypatch):
    monkeypatch.setattr(pmc, "CSRC", str(tmp_path))

    def of(text):
        (tmp_path / "a.h").write_text(text)
        return pmc.code_hash(["a.h"])
    first = of('int a = 1; // one\nconst char *b = "//x";\n')
    assert first == of('/* a\n b */ int a =\n  1;\nconst char *b = "//x"; // "two\n')
    assert first != of('int a = 2; // one\nconst char *b = "//x";\n')
    assert first != of('int a = 1; // one\nconst char *b = "//y";\n')
