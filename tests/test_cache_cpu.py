"""The attention cache without a GPU: what its entry points refuse, the oracle against hand-worked
cases and second definitions, the frequencies of scaled positions.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co

kb = pytest.importorskip("paper_1805_09863_amd")
from paper_1805_09863_amd import binding  # noqa: E402

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F = 0x1000   # never dereferenced: every call here is refused or empty


def cache(**kw):
    d = dict(dtype=1, heads=2, dim=64, page_size=16, pages=100, seqs=8, max_pages=10, k=F, v=F, table=F)
    d.update(kw)
    return binding._Cache(*(d[n] for n, _ in binding._Cache._fields_))


def append(c=None, **kw):
    d = dict(R=4, n_dev=None, q_heads=4, q=F, q_stride=512, k=F, k_stride=512, v=F, v_stride=512, rot=64, pairs=0, pos=F,
             freq=F, amplitude=1.0, seq=None, length=F, q_out=F, position=None, weight=None, stream=None)
    d.update(kw)
    return binding.lib().kb_cache_append(c or cache(), *d.values())


def attend(c=None, **kw):
    d = dict(R=4, n_dev=None, q_heads=4, q=F, q_stride=512, scale=0.125, seq=None, length=F, max_len=160, out=F, lse=None,
             weight_in=None, weight_out=None, ws=F, ws_bytes=1 << 30, stream=None)
    d.update(kw)
    return binding.lib().kb_cache_attend(c or cache(), *d.values())


def evict(c=None, **kw):
    d = dict(R=4, n_dev=None, length=F, keep=32, first=1, recent=4, newest=F, weight=F, position=F, out_table=F,
             out_max_pages=10, out_length=F, out_weight=F, out_position=F, source=F, stream=None)
    d.update(kw)
    return binding.lib().kb_cache_evict(c or cache(), *d.values())


BAD_CACHES = [
    (dict(dtype=2), INVALID), (dict(heads=0), INVALID), (dict(dim=0), INVALID), (dict(dim=12), INVALID),
    (dict(dim=264), INVALID), (dict(page_size=0), INVALID), (dict(page_size=12), INVALID),
    (dict(page_size=2048), INVALID), (dict(page_size=-16), INVALID), (dict(pages=-1), INVALID),
    (dict(seqs=-1), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=1 << 21), UNSUPPORTED),
    (dict(pages=1 << 28), UNSUPPORTED), (dict(pages=2 ** 31 - 1, heads=2 ** 31 - 1), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID), (dict(k=F + 8), INVALID),
    (dict(v=F + 2), INVALID), (dict(table=F + 2), INVALID),
]


@pytest.mark.parametrize("call", [append, attend, evict])
@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_caches_refused(call, kw, status):
    c = cache(**kw)
    extra = dict(q_heads=c.heads) if call is attend and c.heads > 2 else {}
    assert call(c, **extra) == status
    assert binding.lib().kb_last_error()


@pytest.mark.parametrize("call", [append, attend, evict])
def test_no_rows_is_no_work(call):
    assert call(R=0) == OK
    assert call(R=-1) == INVALID


def test_null_cache_refused():
    L = binding.lib()
    assert L.kb_cache_append(None, 4, None, 0, None, 0, F, 512, F, 512, 0, 0, None, None, 1.0, None, F, None, None,
                             None, None) == INVALID
    assert L.kb_cache_attend(None, 4, None, 4, F, 512, 1.0, None, F, 160, F, None, None, None, None, 0, None) == INVALID
    assert L.kb_cache_evict(None, 4, None, F, 32, 0, 0, None, F, None, F, 10, F, F, None, F, None) == INVALID
    assert L.kb_cache_attend_workspace_bytes(None, 4, 4, 160, 1) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q_heads=-1), INVALID), (dict(rot=63), INVALID), (dict(rot=66), INVALID), (dict(rot=-2), INVALID),
    (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(q_out=F + 2), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=0, q=None), INVALID), (dict(q_stride=255), INVALID), (dict(k_stride=127), INVALID),
    (dict(v_stride=0), INVALID), (dict(k=None), INVALID), (dict(v=F + 1), INVALID), (dict(length=None), INVALID),
    (dict(pos=None), INVALID), (dict(freq=None), INVALID), (dict(freq=F + 4), INVALID),
    (dict(amplitude=math.nan), INVALID), (dict(R=9), INVALID), (dict(R=2 ** 31 - 1, seq=F), UNSUPPORTED),
    (dict(q_heads=2 ** 30), UNSUPPORTED),
])
def test_append_refused(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q_heads=0), INVALID), (dict(q_heads=3), INVALID), (dict(max_len=0), INVALID), (dict(scale=math.inf), INVALID),
    (dict(scale=-3e38), INVALID),
    (dict(q=None), INVALID), (dict(q=F + 1), INVALID), (dict(q_stride=100), INVALID), (dict(length=None), INVALID),
    (dict(out=None), INVALID), (dict(out=F + 4), INVALID), (dict(R=9), INVALID), (dict(weight_in=F), INVALID),
    (dict(weight_out=F, seq=F), UNSUPPORTED), (dict(weight_out=F, ws=None), WORKSPACE),
    (dict(weight_out=F, ws=F + 16), WORKSPACE), (dict(weight_out=F, ws_bytes=8), WORKSPACE),
    (dict(R=2 ** 31 - 1, seq=F), UNSUPPORTED), (dict(q_heads=2 ** 30), UNSUPPORTED),
])
def test_attend_refused(kw, status):
    assert attend(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(keep=0), INVALID), (dict(first=-1), INVALID), (dict(recent=-1), INVALID), (dict(first=30, recent=3), INVALID),
    (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID), (dict(out_max_pages=1), INVALID),
    (dict(out_max_pages=0), INVALID), (dict(out_max_pages=1 << 21), UNSUPPORTED), (dict(keep=2 ** 31 - 1), UNSUPPORTED),
    (dict(R=9), INVALID), (dict(length=None), INVALID), (dict(weight=None), INVALID), (dict(out_table=None), INVALID),
    (dict(out_length=None), INVALID), (dict(out_weight=None), INVALID), (dict(source=None), INVALID),
    (dict(out_position=None), INVALID), (dict(position=None), INVALID),
    (dict(position=None, out_position=None), INVALID), (dict(newest=None), INVALID),
    (dict(out_max_pages=9), INVALID), (dict(out_table=F + 64, out_max_pages=9), INVALID),
    (dict(out_table=F + 64, out_weight=F + 64, out_max_pages=9), INVALID),
])
def test_evict_refused(kw, status):
    assert evict(**kw) == status


def test_evict_refuses_longer_caches():
    big = dict(max_pages=(1 << 19) // 16 + 1)
    assert evict(cache(**big), out_max_pages=big["max_pages"]) == UNSUPPORTED
    assert attend(cache(**big), R=0) == OK


def test_attend_workspace_is_a_function_of_the_shape():
    need = binding.lib().kb_cache_attend_workspace_bytes
    assert need(cache(), 4, 4, 160, 1) == need(cache(), 4, 4, 160, 1) > 0
    assert need(cache(), 0, 4, 160, 1) == 0
    assert need(cache(dim=12), 4, 4, 160, 1) == need(cache(), 4, 3, 160, 1) == need(cache(), 4, 4, 0, 1) == 0


def test_attend_workspace_of_the_largest_call_serves_all():
    need = binding.lib().kb_cache_attend_workspace_bytes
    for weights in (0, 1):
        for dtype in (0, 1):
            c = cache(dtype=dtype, max_pages=600, seqs=5000)
            by_rows = [need(c, R, 4, 5000, weights) for R in (1, 7, 500, 1023, 1024, 1025, 1026, 5000)]
            by_len = [need(c, R, 4, n, weights) for R in (3, 2000)
                      for n in (1, 64, 65, 384, 385, 768, 769, 1024, 1025, 5000, 9600, 10 ** 6)]
            assert by_rows == sorted(by_rows) and by_len[:12] == sorted(by_len[:12]) and by_len[12:] == sorted(by_len[12:])
            assert by_rows[0] > 0 and by_rows[-1] < 2 ** 31


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("weights", [0, 1])
def test_attend_workspace_shrinks_neither_with_rows_nor_with_lengths(dtype, weights):
    need = binding.lib().kb_cache_attend_workspace_bytes
    c = cache(dtype=dtype, max_pages=600, seqs=5000)
    rows, lengths = (1, 63, 64, 128, 129, 1000, 1024, 1025, 1100, 3000), (1, 64, 65, 384, 385, 768, 769, 1024, 1025, 9600)
    for heads in (2, 34):
        got = [[need(c, R, heads, n, weights) for n in lengths] for R in rows]
        assert all(line == sorted(line) for line in got) and all(list(col) == sorted(col) for col in zip(*got))


def test_binding_refuses_host_tensors():
    k = torch.zeros((4, 2, 16, 64))
    t, n = torch.zeros((1, 2), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    q = torch.zeros((1, 2, 64))
    with pytest.raises(TypeError):
        kb.cache_attend(q, k, k, t, n)
    with pytest.raises(TypeError):
        kb.cache_append(k, k, t, n, q, q)
    with pytest.raises(TypeError):
        kb.cache_evict(k, k, t, n, 4, weight=torch.zeros(64))


def test_frequencies():
    w = kb.rotary_frequencies(64, device="cpu")
    assert w.dtype == torch.float64 and w[0] == 1 and abs(float(w[16]) - 0.01) < 1e-15
    assert torch.equal(kb.rotary_frequencies(64, factor=4.0, device="cpu"), w / 4)
    s = kb.rotary_frequencies(64, factor=4.0, trained_length=512, device="cpu")
    turns = 512 * w / (2 * math.pi)
    assert torch.equal(s[turns >= 32], w[turns >= 32])
    assert torch.allclose(s[turns <= 1], w[turns <= 1] / 4, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and torch.all((s[mid] < w[mid]) & (s[mid] > w[mid] / 4))
    for bad in (dict(rot_dim=63), dict(rot_dim=0), dict(rot_dim=64, factor=0.0), dict(rot_dim=64, base=-1.0),
                dict(rot_dim=64, slow=3.0, fast=3.0), dict(rot_dim=64, trained_length=0)):
        with pytest.raises(ValueError):
            kb.rotary_frequencies(bad.pop("rot_dim"), device="cpu", **bad)


# ---------------------------------------------------------------- the oracle
def test_oracle_rotation_is_the_complex_product():
    g = np.random.default_rng(0)
    x, freq = g.standard_normal(20), g.random(8)
    z = (x[0:16:2] + 1j * x[1:16:2]) * 1.5 * np.exp(1j * 77 * freq)
    y = co.rotate(x, 77, freq, True, 1.5)
    assert np.allclose(y[0:16:2], z.real) and np.allclose(y[1:16:2], z.imag) and np.array_equal(y[16:], x[16:])
    y = co.rotate(np.concatenate([x[0:16:2], x[1:16:2], x[16:]]), 77, freq, False, 1.5)
    assert np.allclose(y[:8], z.real) and np.allclose(y[8:16], z.imag) and np.array_equal(y[16:], x[16:])
    # scores of turned queries and keys depend on the distance of their positions alone
    a, b = g.standard_normal(16), g.standard_normal(16)
    dot = [co.rotate(a, p + 9, freq, False, 1.0) @ co.rotate(b, p, freq, False, 1.0) for p in (0, 5, 1000)]
    assert np.allclose(dot, dot[0])


def test_oracle_attention_by_hand():
    # one head, two slots in swapped pages of one slot, scores 0 and ln 3: probabilities 1/4 and 3/4
    k = np.zeros((3, 1, 1, 8))
    v = np.zeros((3, 1, 1, 8))
    k[0, 0, 0, 0] = math.log(3.0)
    v[1, 0, 0, :], v[0, 0, 0, :] = 4.0, 8.0
    table = np.array([[1, 0, -1], [-1, 0, 7]], np.int32)
    q = np.zeros((2, 1, 8))
    q[:, 0, 0] = 1.0
    out, lse, p, _, _ = co.attend(q, k, v, table, np.array([2, 3]), 1.0)
    assert np.allclose(p[0][0], [0.25, 0.75]) and np.allclose(out[0, 0], 7.0) and np.isclose(lse[0, 0], math.log(4.0))
    assert np.allclose(out[1, 0], 8.0) and np.isclose(lse[1, 0], math.log(3.0))   # holes around its one slot
    assert co.attended(table, np.array([9, -1]), 1, 3)[0][1] == [0, 1]


def test_oracle_eviction_by_hand():
    w = np.array([5.0, 1.0, 3.0, 3.0, 9.0, np.nan, 3.0], np.float32)
    # kept of 4: 0 (5), 4 (9), then the two lowest of the three 3s: 2, 3; slot 4 fills the dropped place 1
    assert co.kept_slots(w, None, 4, 0, 0, 0) == [0, 4, 2, 3]
    assert co.kept_slots(w, None, 7, 0, 0, 0) == list(range(7))
    pos = np.array([0, 1, 2, 3, 4, 5, 6])
    # the newest two (5, 6) and the first (0) are held, then 9
    assert co.kept_slots(w, pos, 4, 1, 2, 6) == [0, 4, 5, 6]
    assert co.kept_slots(w, pos, 2, 0, 1, 6) == [4, 6]


@pytest.mark.parametrize("seed", range(5))
def test_oracle_eviction_keeps_the_greatest(seed):
    g = np.random.default_rng(seed)
    L = int(g.integers(1, 60))
    w, keep = g.integers(0, 6, L).astype(np.float32), int(g.integers(1, 60))
    src = co.kept_slots(w, None, keep, 0, 0, 0)
    n = min(L, keep)
    assert len(set(src)) == len(src) == n
    assert sorted(w[src]) == sorted(w)[L - n:]
    moved = [t for i, t in enumerate(src) if t != i]
    assert all(t >= n for t in moved) and moved == sorted(moved)
