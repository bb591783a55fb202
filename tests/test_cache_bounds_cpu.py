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


# ---------------------------------------------------------------- sizes that C takes in 32 bits
torch = pytest.importorskip("torch")
kb = pytest.importorskip("paper_1805_09863_amd")
from paper_1805_09863_amd import binding  # noqa: E402


class Shaped:
    """A tensor on the GPU as far as its sizes go: nothing of it exists."""
    is_cuda, dtype, device = True, torch.float32, "cuda:0"

    def __init__(self, *shape, dtype=torch.float32):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def stride(self):
        s, n = [], 1
        for x in reversed(self.shape):
            s.append(n)
            n *= max(x, 1)
        return tuple(reversed(s))

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def element_size(self):
        return 4


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library, none of them made."""
    made = []

    def run(fn, dev, stream, *args):
        assert len(args) + 1 == len(fn.argtypes)
        made.append(args)
    monkeypatch.setattr(binding, "_run", run)
    monkeypatch.setattr(binding.torch, "Tensor", Shaped)
    return made


I32 = torch.int32


def cache(seqs=8, heads=2, dim=64, page=16, pages=100, cols=10):
    return Shaped(pages, heads, page, dim), Shaped(pages, heads, page, dim), Shaped(seqs, cols, dtype=I32)


def evict(keep, R=8, out_cols=10, **kw):
    k, v, t = cache()
    n = max(keep, 1) if keep <= 10 ** 6 else 32
    out = (Shaped(R, dtype=I32), Shaped(8, 2, 160), None, Shaped(R, 2, n, dtype=I32))
    more = {} if out_cols == 10 else dict(out_table=Shaped(R, out_cols, dtype=I32))
    return kb.cache_evict(k, v, t, Shaped(R, dtype=I32), keep, weight=Shaped(8, 2, 160), out=out, **more, **kw)


def attend(R=8, q_heads=4, max_len=160, c=None):
    k, v, t = c or cache()
    q = Shaped(R, q_heads, k.shape[3])
    return kb.cache_attend(q, k, v, t, Shaped(R, dtype=I32), max_len=max_len, out=q, ws=Shaped(1 << 40),
                           seq=Shaped(R, dtype=I32))


def append(R=8, q_heads=4, pairs=32, c=None):
    k, v, t = c or cache()
    x = Shaped(R, k.shape[1], k.shape[3])
    q = Shaped(R, q_heads, k.shape[3])
    return kb.cache_append(k, v, t, Shaped(R, dtype=I32), x, x, q=q, q_out=q, freq=Shaped(pairs, dtype=torch.float64),
                           pos=Shaped(R, dtype=I32), seq=Shaped(R, dtype=I32))


def test_sizes_within_32_bits_reach_the_library(calls):
    evict(32, first=1, recent=4)
    attend()
    append()
    attend(max_len=2 ** 40)                              # longer than the table: the table's slots
    assert len(calls) == 4 and calls[0][4:7] == (32, 1, 4) and calls[1][9] == calls[3][9] == 160


@pytest.mark.parametrize("call", [
    lambda: evict(2 ** 32 + 4), lambda: evict(-2 ** 32 + 5), lambda: evict(2 ** 31), lambda: evict(-2 ** 31 - 1),
    lambda: evict(32, first=2 ** 32), lambda: evict(32, first=-2 ** 32 + 1), lambda: evict(32, recent=2 ** 32 + 4),
    lambda: evict(32, recent=-2 ** 32), lambda: evict(32, R=2 ** 32 + 2), lambda: evict(32, out_cols=2 ** 32 + 10),
    lambda: attend(max_len=-2 ** 32 + 5), lambda: attend(R=2 ** 32 + 1), lambda: attend(q_heads=2 ** 32 + 4),
    lambda: attend(c=cache(heads=2 ** 32 + 2, pages=0), q_heads=2), lambda: attend(c=cache(dim=2 ** 32 + 64, pages=0)),
    lambda: attend(c=cache(page=2 ** 32 + 16, pages=0)),
    lambda: append(R=2 ** 32 + 1), lambda: append(q_heads=2 ** 32 + 4), lambda: append(pairs=2 ** 31 + 16),
    lambda: kb.cache_attend_workspace_bytes(*cache(), 2 ** 32 + 1, 4),
    lambda: kb.cache_attend_workspace_bytes(*cache(), 8, 2 ** 32 + 4),
    lambda: kb.cache_attend_workspace_bytes(*cache(), 8, 4, -2 ** 32 + 5),
    lambda: kb.cache_attend_workspace_bytes(*cache(), -2 ** 32 + 5, 4),
])
def test_sizes_past_32_bits_are_refused(calls, call):
    with pytest.raises(ValueError, match="32 bits"):
        call()
    assert not calls


# ---------------------------------------------------------------- rows that lie otherwise than the call takes them
def with_weights(name, *shape):
    """The call that takes the argument, with a tensor of this shape; the others as they should be.  8 sequences of
    2 heads and 160 slots, 4 query heads of 64 values, 40 slots kept, into pages of 48 slots a sequence."""
    k, v, t = cache()
    n, q, w, p = Shaped(8, dtype=I32), Shaped(8, 4, 64), Shaped(8, 2, 160), Shaped(8, 2, 160, dtype=I32)
    x = Shaped(*shape, dtype=I32 if name in ("position", "source", "out position") else torch.float32)
    if name in ("q_out", "append weight", "append position"):
        kw = dict(q_out=q, weight=w, position=p)
        kw[name.split()[-1]] = x if name != "append position" else Shaped(*shape, dtype=I32)
        return kb.cache_append(k, v, t, n, Shaped(8, 2, 64), Shaped(8, 2, 64), q=q, **kw)
    if name in ("out", "lse", "weight_in", "weight_out"):
        kw = dict(out=q, lse=Shaped(8, 4), weight_in=w, weight_out=w, ws=Shaped(1 << 30))
        kw[name] = x
        return kb.cache_attend(q, k, v, t, n, **kw)
    kw = dict(weight=w, position=p)
    out = {"length": n, "out weight": Shaped(8, 2, 48), "out position": Shaped(8, 2, 48, dtype=I32),
           "source": Shaped(8, 2, 40, dtype=I32)}
    (kw if name in kw else out)[name] = x
    return kb.cache_evict(k, v, t, n, 40, out_table=Shaped(8, 3, dtype=I32), out=tuple(out.values()), **kw)


ROWS = {"q_out": (4, 64), "out": (4, 64), "lse": (4,), "append weight": (2, 160), "append position": (2, 160),
        "weight_in": (2, 160), "weight_out": (2, 160), "weight": (2, 160), "position": (2, 160), "out weight": (2, 48),
        "out position": (2, 48), "source": (2, 40)}


@pytest.mark.parametrize("name", ROWS)
def test_rows_that_lie_as_the_call_takes_them(calls, name):
    *heads, last = ROWS[name]
    n = heads[0] if heads else 1
    shapes = [(8, *ROWS[name]), (9, *ROWS[name]), (8 * n * last,), (8 * n * last + 7,), (8, n * last), (8 * n, last),
              (3, 8, *ROWS[name])]
    if heads:
        shapes.append((8, n, last // 4, 4))
    for shape in shapes:
        with_weights(name, *shape)
    assert len(calls) == len(shapes)


@pytest.mark.parametrize("name", ROWS)
def test_rows_further_apart_are_refused(calls, name):
    *heads, last = ROWS[name]
    n = heads[0] if heads else 1
    shapes = [(8, *heads, last + 32), (8, *heads, 2 * last), (8, n * last + 8), (8 * n, last + 16)]
    if heads:
        shapes += [(8, n + 2, last), (8, 2 * n, last // 2), (8, n, last // 4, 8)]
    for shape in shapes:
        with pytest.raises(ValueError, match="rows of"):
            with_weights(name, *shape)
    for shape in ((7, *ROWS[name]), (8 * n * last - 1,)):
        with pytest.raises(ValueError, match="needed"):
            with_weights(name, *shape)
    assert not calls
