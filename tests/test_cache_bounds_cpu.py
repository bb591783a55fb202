"""Arguments of the attention cache at the ends of their ranges, without a GPU."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1805_09863_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_the_slot_of_a_new_token_at_the_ends_of_int32():
    """The append's own function, evaluated by the compiler, for which an overflow is an error."""
    lo, hi = "(-2147483647 - 1)", "2147483647"
    want = [(n, cap, n_is) for cap in (1, 100, 1 << 24) for n, n_is in
            [(lo, -1), (f"{lo} + 1", -1), (-3, -1), (-1, -1), (0, -1), (1, 0), (cap, cap - 1), (cap + 1, -1), (hi, -1)]]
    src = '#include "cache_slot.hpp"\n' + "".join(
        f'static_assert(kb::new_slot({n}, {cap}) == {s}, "length {n} of {cap}");\n' for n, cap, s in want)
    r = subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-I", CSRC, "-x", "c++", "-"], input=src, text=True,
                       capture_output=True)
    assert r.returncode == 0, r.stderr


def test_the_append_takes_its_slot_from_there():
    with open(os.path.join(CSRC, "cache_append.hip")) as f:
        src = f.read()
    assert "new_slot(len, c.cap)" in src and "len - 1" not in src
