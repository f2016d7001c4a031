"""Host side of the append and block-cache calls without a GPU: the binding's structure has the layout that a C compiler gives the
header's, the entry points refuse a missing context, and the plain statement of a block's codes keeps its bound."""
import ctypes
import os
import subprocess

import numpy as np

from block_reference import quantise
from paper_2511_06029_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_structure_layout_is_the_compilers(tmp_path):
    mirror, name = binding.lethe_block_cache, "lethe_block_cache"
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
    c, b = binding.lethe_cache(), binding.lethe_block_cache()
    INV = binding.ERR_INVALID_ARG
    assert lib.lethe_append(None, ctypes.byref(c), 0, 1, None, 1, 1, None, None, None, None, None, None, None) == INV
    assert lib.lethe_block_append(None, ctypes.byref(b), 0, 1, None, 1, 1, None, None, None, None, None, None) == INV
    assert lib.lethe_block_read(None, ctypes.byref(b), 0, 1, None, 1, None, None, None) == INV
    assert lib.lethe_block_select(None, ctypes.byref(b), 0, 1, None, 1, 0, 0, None, None) == INV
    assert lib.lethe_block_attend(None, ctypes.byref(b), 0, 1, None, None, None, 0, None, None, None) == INV


def test_codes_keep_their_bound():
    g = np.random.default_rng(0)
    x = (g.standard_normal((200, 16, 64)) * np.exp(8 * g.standard_normal((200, 1, 1)))).astype(np.float32)
    c, s = quantise(x)
    assert np.abs(c.astype(int)).max() == 127
    off = np.abs(x.astype(np.float64) - c * s.astype(np.float64)[:, None, None])
    assert (off <= s[:, None, None] * (0.5 + 2.0 ** -16)).all()
