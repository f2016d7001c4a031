"""Kernels that may start before the kernel ahead of them has ended must not read memory through the read-only path, which
promises that nobody writes it while the kernel lives (a CPU test over the sources)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_06029_b200", "csrc")
SOURCES = {f: open(os.path.join(CSRC, f)).read() for f in sorted(os.listdir(CSRC)) if f.endswith((".cu", ".cuh"))}
DEPENDENT = [f for f, s in SOURCES.items() if re.search(r"\bdependency_wait\(\);|griddepcontrol\.wait", s)]


def test_there_are_some():
    assert "block_select.cu" in DEPENDENT and len(DEPENDENT) > 5


@pytest.mark.parametrize("name", DEPENDENT)
def test_no_read_only_loads(name):
    code = re.sub(r"//[^\n]*", "", SOURCES[name])
    assert not re.search(r"__ldg\b|ld\.global\.nc|__restrict__", code)
