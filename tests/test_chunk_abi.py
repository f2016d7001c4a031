"""Host side of lethe_chunk_attend and lethe_rotate without a GPU: the binding's structures have the layout that a C compiler
gives the header's, and the entry points refuse a missing context."""
import ctypes
import os
import subprocess

import pytest

from paper_2511_06029_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["lethe_score_mod", "lethe_rotary", "lethe_cache"])
def test_structure_layout_is_the_compilers(name, tmp_path):
    mirror = getattr(binding, name)
    fields = [f[0] for f in mirror._fields_]
    source = tmp_path / "layout.c"
    source.write_text(
        '#include <stddef.h>\n#include <stdio.h>\n#include "lethe.h"\nint main(void) {\n'
        + "".join(f'printf("%zu %zu\\n", offsetof({name}, {f}), sizeof((({name}*)0)->{f}));\n' for f in fields)
        + f'printf("%zu\\n", sizeof({name}));\nreturn 0;\n}}\n')
    program = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(program)], check=True)
    lines = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split("\n")
    for f, line in zip(fields, lines):
        assert (getattr(mirror, f).offset, getattr(mirror, f).size) == tuple(int(x) for x in line.split()), f
    assert ctypes.sizeof(mirror) == int(lines[len(fields)])


def test_no_context_is_refused():
    lib = binding.load()
    cache, rotary = binding.lethe_cache(), binding.lethe_rotary()
    assert lib.lethe_chunk_attend(None, ctypes.byref(cache), 0, 1, None, 1, 1, None, None, None, None, None, 1.0, None, None, None,
                                  None, None) == binding.ERR_INVALID_ARG
    assert lib.lethe_rotate(None, ctypes.byref(rotary), 1, 64, 1, 1, 1, 1, None, None, 0, None, None, None) == binding.ERR_INVALID_ARG
