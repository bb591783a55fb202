"""The attention cache on the GPU against the fp64 oracle (oracle/cache_oracle.py).

Bounds, before any rounding of the output, from the operations' number (u = 2^-24, a float32
operation's half step):

* a turned pair: the reduced angle is right to 2^-26 quarter turns and to the three 64-bit roundings
  of pos * freq, here and in the oracle, its cosine and sine to 2^-22, the two products and their sum
  to 3 u each: within 2^-21 + 3 * 2^-53 |pos| of amplitude * (|x| + |y|);
* a score: dim products summed and two factors, (dim + 4) u of the largest scale * sum |q k|
  (``spread``), and what its own size costs in base 2, 2 u of it: d;
* a probability: e^(score - max) with both off by d, 2^-22 for the exponential, length u for the
  sum it is divided by: p (2 d + 2^-22 + length u), and one below 2^-126, the least normal float32,
  may become 0: 2^-126 more;
* an output: that, length u for its own sum, and 2^-16 where the probabilities are two bf16 pieces:
  all of sum p |v| (``size``);
* lse: d, length u and 2^-22 for the logarithm, and a rounding of its own.

A bf16 output is rounded once more: 2^-8 of its value.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


def f64(t):
    return t.detach().cpu().double().numpy()


def host(t):
    return t.detach().cpu().numpy()


def bits(t):
    return host(t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32))


def make_cache(g, dtype, seqs, heads, dim, page, cap, spare=3, dirty=True):
    """k, v, table: sequences of ``cap`` slots in scattered pages; with ``dirty`` every page holds NaN
    and infinities until fill() writes the referenced slots."""
    cols = -(-cap // page)
    pages = seqs * cols + spare
    table = torch.randperm(pages, generator=g)[:seqs * cols].to(torch.int32).view(seqs, cols)
    shape = (pages, heads, page, dim)
    k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
    if dirty:
        k = torch.full(shape, math.nan, dtype=dtype)
        v = torch.full(shape, math.inf, dtype=dtype)
    return k, v, table


def fill(g, k, v, table, length, seq=None, max_len=None):
    pages, heads, page, dim = k.shape
    for s, slots in co.attended(table.numpy(), length.numpy(), page, pages, seq, max_len):
        if slots:
            t = torch.tensor(slots)
            pg, pl = table[s][t // page].long(), t % page
            k[pg, :, pl] = torch.randn((len(slots), heads, dim), generator=g).to(k.dtype)
            v[pg, :, pl] = torch.randn((len(slots), heads, dim), generator=g).to(v.dtype)


def check_attend(kb, q, k, v, table, length, *, scale=None, seq=None, max_len=None, weight_in=None, weights=False,
                 ws=None):
    """One call on the GPU against the oracle; returns its outputs."""
    dim, dtype = q.shape[2], q.dtype
    sc = dim ** -0.5 if scale is None else scale
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    lse = torch.full(q.shape[:2], math.nan, device="cuda")
    R, Q = q.shape[:2]
    heads, page = k.shape[1:3]
    cap = table.shape[1] * page
    w_out = torch.full((table.shape[0], heads, cap), -7.0, device="cuda") if weights else None
    out = kb.cache_attend(dev(q), dev(k), dev(v), dev(table), dev(length), scale=scale, max_len=max_len, seq=dev(seq),
                          lse=lse, weight_in=dev(weight_in), weight_out=w_out, ws=ws)
    torch.cuda.synchronize()
    # the oracle never looks at a slot that is not attended to
    kk, vv = f64(k), f64(v)
    ref, ref_lse, probs, spread, size = co.attend(f64(q), kk, vv, table.numpy(), length.numpy(), sc,
                                                  seq=None if seq is None else seq.numpy(), max_len=max_len)
    rows = co.attended(table.numpy(), length.numpy(), page, k.shape[0], None if seq is None else seq.numpy(), max_len)
    n = np.array([len(s) for _, s in rows])[:, None]
    d = (dim + 6) * U * spread
    rel = 2 * d + 2.0 ** -22 + 2 * n * U + (2.0 ** -16 if dtype == torch.bfloat16 else 0)
    err = np.abs(f64(out) - ref)
    tol = rel[..., None] * size + ROUND[dtype] * np.abs(ref) + 1e-30
    assert np.all(err <= tol), f"out: worst {np.max(err / tol):.3g} of its bound"
    got = f64(lse)
    empty = np.broadcast_to(n == 0, got.shape)
    assert np.all(got[empty] == -np.inf) and np.all(f64(out)[empty] == 0)
    tol = (d + n * U + 2.0 ** -22 + 2 * U * np.abs(ref_lse))[~empty]
    err = np.abs(got[~empty] - ref_lse[~empty])
    assert np.all(err <= tol), f"lse: worst {np.max(err / tol):.3g} of its bound"
    if weights:
        want = np.full((table.shape[0], heads, cap), -7.0)
        bound = np.zeros_like(want)
        for r, (s, slots) in enumerate(rows):
            for h in range(heads):
                group = range(h * Q // heads, (h + 1) * Q // heads)
                for j, t in enumerate(slots):
                    p = sum(probs[r][x][j] for x in group)
                    want[r, h, t] = p + (0 if weight_in is None else float(weight_in[r, h, t]))
                    bound[r, h, t] = (p * (max(rel[r, x] for x in group) + len(group) * U) + len(group) * 2.0 ** -126
                                      + 2 * U * abs(want[r, h, t]))
        err = np.abs(f64(w_out) - want)
        assert np.all(err <= bound), f"weights: worst {np.max(err / np.maximum(bound, 1e-30)):.3g} of their bound"
    return out, lse, w_out


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 511, 700]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim,page", [
    (1, 1, 8, 1), (2, 2, 64, 16), (8, 2, 128, 32), (6, 2, 80, 4), (7, 1, 72, 64), (16, 1, 96, 128), (17, 1, 40, 2),
    (40, 2, 16, 8), (3, 3, 136, 256), (4, 2, 192, 16), (8, 1, 256, 1), (5, 5, 24, 1024), (64, 2, 64, 16),
])
def test_attend(kb, dtype, q_heads, heads, dim, page):
    g = torch.Generator().manual_seed(q_heads * 1000 + dim)
    length = torch.tensor(LENGTHS, dtype=torch.int32)
    k, v, table = make_cache(g, dtype, len(LENGTHS), heads, dim, page, max(LENGTHS))
    fill(g, k, v, table, length)
    q = torch.randn((len(LENGTHS), q_heads, dim), generator=g).to(dtype)
    w = torch.rand((len(LENGTHS), heads, table.shape[1] * page), generator=g)
    check_attend(kb, q, k, v, table, length, weights=True, weight_in=w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R,q_heads,heads,dim,page,length", [
    (1, 8, 2, 128, 64, 20011), (1, 1, 1, 64, 1, 5000), (2, 32, 8, 128, 16, 9000), (3, 4, 4, 256, 128, 6001),
    (1, 20, 1, 80, 8, 12000), (200, 4, 2, 64, 16, 300),
])
def test_attend_long(kb, dtype, R, q_heads, heads, dim, page, length):
    """Few rows and long caches, where the length is split and joined; and more rows than the card has units."""
    g = torch.Generator().manual_seed(length)
    n = torch.randint(1, length + 1, (R,), generator=g).to(torch.int32)
    n[0] = length
    k, v, table = make_cache(g, dtype, R, heads, dim, page, length)
    fill(g, k, v, table, n)
    q = torch.randn((R, q_heads, dim), generator=g).to(dtype)
    check_attend(kb, q, k, v, table, n, weights=R < 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R,q_heads,heads,dim,page,most,long", [
    (60, 40, 2, 64, 16, 2000, 8),      # cut rows and whole ones, empty ones among them, two tiles of query heads
    (300, 3, 3, 24, 1, 40, 1),         # one long row among short ones
    (1024, 2, 1, 16, 8, 30, 3),        # as many rows as shares take
    (1030, 2, 1, 16, 8, 30, 3),        # more: splits
    (520, 4, 2, 128, 4, 60, 0),        # many short rows: a wave each
    (520, 6, 2, 80, 1, 60, 0),
])
def test_attend_batches(kb, dtype, R, q_heads, heads, dim, page, most, long):
    """Batches of very different lengths, rows from the device's count on left alone."""
    g = torch.Generator().manual_seed(R + most)
    n = torch.randint(0, most + 1, (R,), generator=g).to(torch.int32)
    at = torch.randperm(R, generator=g)[:long]
    n[at] = torch.randint(900, 2500, (long,), generator=g).to(torch.int32)
    cap = int(n.max())
    k, v, table = make_cache(g, dtype, R, heads, dim, page, cap, spare=0, dirty=R < 100)
    if R < 100:
        fill(g, k, v, table, n)
    q = torch.randn((R, q_heads, dim), generator=g).to(dtype)
    out, lse, _ = check_attend(kb, q, k, v, table, n)
    part = torch.full_like(out, 5)
    part_lse = torch.full_like(lse, 5)
    count = R * 2 // 3
    kb.cache_attend(q.cuda(), k.cuda(), v.cuda(), table.cuda(), n.cuda(), out=part, lse=part_lse,
                    n_dev=torch.tensor([count], dtype=torch.int32, device="cuda"))
    assert torch.all(part[count:] == 5) and torch.all(part_lse[count:] == 5)
    # the count moves the shares' ends, and with them where a row's sums are joined
    near = 2 * (int(n.max()) * U + 2.0 ** -16) * float(v.float().abs().max()) + ROUND[dtype] * float(out.abs().max()) * 2
    assert float((part[:count].float() - out[:count].float()).abs().max()) <= near


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_attend_holes(kb, dtype, page):
    """Pages outside the pool at the start, in the middle, at the end and everywhere; lengths past the table."""
    g = torch.Generator().manual_seed(page)
    cap = 1000
    n = torch.tensor([1000, 1000, 1000, 1000, 5, 2 ** 31 - 1, -3, 640], dtype=torch.int32)
    k, v, table = make_cache(g, dtype, 8, 2, 64, page, cap)
    cols = table.shape[1]
    table[0, :cols // 2] = -1
    table[1, cols // 3:cols // 2 + 1] = 2 ** 31 - 1
    table[2, -(cols // 4):] = k.shape[0]
    table[3] = -2 ** 31
    table[4, 0] = -1
    table[7, ::2] = k.shape[0] + 5
    fill(g, k, v, table, n)
    q = torch.randn((8, 6, 64), generator=g).to(dtype)
    check_attend(kb, q, k, v, table, n, weights=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_attend_shared_sequences(kb, dtype):
    """Drafted tokens: rows of one sequence with lengths of their own, sequences out of range, a bound on the
    lengths; queries that are part of wider rows, at an odd element."""
    g = torch.Generator().manual_seed(5)
    seq = torch.tensor([2, 2, 2, 0, 0, 1, -1, 3, 2 ** 30], dtype=torch.int32)
    n = torch.tensor([70, 71, 72, 9, 10, 400, 5, 5, 5], dtype=torch.int32)
    k, v, table = make_cache(g, dtype, 3, 2, 48, 8, 400)
    fill(g, k, v, table, n, seq, 300)
    wide = torch.randn(9 * (6 * 48 + 37) + 1, generator=g).to(dtype)
    q = wide[1:].view(9, -1)[:, :6 * 48].unflatten(1, (6, 48))
    dev = wide.cuda()[1:].view(9, -1)[:, :6 * 48].unflatten(1, (6, 48))
    a, la, _ = check_attend(kb, q, k, v, table, n, seq=seq, max_len=300, scale=0.3)
    b = kb.cache_attend(dev, k.cuda(), v.cuda(), table.cuda(), n.cuda(), seq=seq.cuda(), max_len=300, scale=0.3)
    assert torch.equal(a, b)


def test_bounds_past_32_bits(kb):
    """A bound of the lengths above the table's slots is the table's slots, whatever its low 32 bits are; a
    budget that C cannot hold is refused."""
    g = torch.Generator().manual_seed(77)
    k, v, table = make_cache(g, torch.float32, 2, 1, 16, 4, 40)
    length = torch.tensor([40, 33], dtype=torch.int32)
    fill(g, k, v, table, length)
    q = torch.randn(2, 2, 16, generator=g).cuda()
    dk, dv, dt, dl = k.cuda(), v.cuda(), table.cuda(), length.cuda()
    want = kb.cache_attend(q, dk, dv, dt, dl)
    got = kb.cache_attend(q, dk, dv, dt, dl, max_len=2 ** 32 + 5)
    assert torch.equal(got, want)
    assert kb.cache_attend_workspace_bytes(dk, dv, dt, 2, 2, 2 ** 32 + 5, True) == kb.cache_attend_workspace_bytes(
        dk, dv, dt, 2, 2, weights=True)
    with pytest.raises(ValueError, match="32 bits"):
        kb.cache_evict(dk, dv, dt, dl, 2 ** 32 + 4, weight=torch.zeros(2, 1, 40, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_workspace_for_many_rows_serves_fewer(kb, dtype):
    """1,100 rows of up to 1,000 slots are a workgroup's each, 1,000 of the same lengths are shared out."""
    g = torch.Generator().manual_seed(78)
    k, v, table = make_cache(g, dtype, 1100, 1, 16, 8, 1000)
    length = torch.randint(0, 1001, (1100,), generator=g, dtype=torch.int32)
    length[0], length[1] = 1000, 0
    fill(g, k, v, table, length)
    q = torch.randn(1100, 1, 16, generator=g).to(dtype)
    ws = torch.empty(kb.cache_attend_workspace_bytes(k.cuda(), v.cuda(), table.cuda(), 1100, 1), dtype=torch.uint8,
                     device="cuda")
    check_attend(kb, q, k, v, table, length, ws=ws)
    check_attend(kb, q[:1000], k, v, table, length[:1000], ws=ws)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_attend_large_scores(kb, dtype):
    """Scores far apart and far from zero: one slot takes all the weight, at the first, a middle and the last place,
    rising and falling along the length; and a scale below zero."""
    g = torch.Generator().manual_seed(9)
    L, dim = 300, 64
    k, v, table = make_cache(g, dtype, 5, 1, dim, 16, L, dirty=False)
    q = torch.ones((5, 2, dim)).to(dtype)
    size = torch.tensor([[30.0 if t == (0, 150, L - 1)[r] else -30.0 for t in range(L)] for r in range(3)]
                        + [[t / 4.0 for t in range(L)], [-t / 4.0 for t in range(L)]])
    for r in range(5):
        for t in range(L):
            k[table[r, t // 16].long(), 0, t % 16] = (size[r, t] * torch.ones(dim)).to(dtype)
    n = torch.full((5,), L, dtype=torch.int32)
    check_attend(kb, q, k, v, table, n, weights=True)
    check_attend(kb, q, k, v, table, n, scale=-0.125)
    check_attend(kb, q, k, v, table, n, scale=0.0)


def test_attend_repeats_and_leaves_rows_alone(kb):
    """The same call twice gives the same bits; rows from the device's count on stay as they were; weights may be
    added in place; a stream and a workspace of the caller's, larger than needed and full of NaN."""
    g = torch.Generator().manual_seed(11)
    R, Q, heads, dim, page, L = 6, 8, 2, 128, 16, 900
    k, v, table = make_cache(g, torch.bfloat16, R, heads, dim, page, L)
    n = torch.tensor([900, 3, 400, 899, 64, 17], dtype=torch.int32)
    fill(g, k, v, table, n)
    q, k, v, table, n = (t.cuda() for t in (torch.randn((R, Q, dim), generator=g).bfloat16(), k, v, table, n))
    cap = table.shape[1] * page
    w = torch.rand((R, heads, cap), generator=g).cuda()
    lse = torch.zeros((R, Q), device="cuda")
    w2 = w.clone()
    whole = kb.cache_attend(q, k, v, table, n, lse=lse, weight_in=w, weight_out=w2)
    need = kb.cache_attend_workspace_bytes(k, v, table, R, Q, weights=True)
    ws = torch.full((need // 4 + 1000,), math.nan, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse2, w3 = torch.full_like(whole, 9), torch.full_like(lse, 9), w.clone()
    kb.cache_attend(q, k, v, table, n, out=out, lse=lse2, weight_in=w3, weight_out=w3, ws=ws, stream=side,
                    n_dev=torch.tensor([4], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(out[:4], whole[:4]) and torch.equal(lse2[:4], lse[:4]) and torch.equal(w3[:4], w2[:4])
    assert torch.all(out[4:] == 9) and torch.all(lse2[4:] == 9) and torch.equal(w3[4:], w[4:])


def test_results_lie_in_memory_of_the_calls_stream(kb):
    """Calls on a side stream that allocate for themselves take no memory that the current stream has freed but
    still reads."""
    g = torch.Generator().manual_seed(12)
    R, Q, heads, dim, page, L = 64, 8, 2, 128, 16, 1500
    k, v, table = make_cache(g, torch.float32, R, heads, dim, page, L, dirty=False)
    k, v, table = k.cuda(), v.cuda(), table.cuda()
    n = torch.full((R,), L, dtype=torch.int32, device="cuda")
    q = torch.randn((R, Q, dim), generator=g).cuda()
    w = torch.zeros((R, heads, table.shape[1] * page), device="cuda")
    sizes = [kb.cache_attend_workspace_bytes(k, v, table, R, Q, weights=True) // 4, R * Q * dim,
             R * heads * table.shape[1] * page, R * heads * 1000]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    read = [torch.ones(m, device="cuda") for m in sizes]
    copies = [torch.empty_like(x) for x in read]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)          # about 10 ms of the current stream
    for x, y in zip(read, copies):
        y.copy_(x)
    del read, x
    kb.cache_attend(q, k, v, table, n, weight_out=w, stream=side)
    kb.cache_append(k, v, table, n, q[:, :2], q[:, :2], q=q, stream=side)
    kb.cache_evict(k, v, table, n, 1000, weight=w, stream=side)
    torch.cuda.synchronize()
    assert all(bool((y == 1).all()) for y in copies)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim,rot,pairs,page,gap", [
    (4, 2, 128, 128, False, 16, 0), (4, 2, 128, 64, True, 1, 0), (3, 1, 72, 24, False, 8, 0),
    (2, 2, 64, 64, True, 32, 16), (5, 5, 40, 34, False, 4, 3), (1, 1, 8, 2, True, 1024, 0), (16, 4, 256, 256, False, 64, 1),
    (0, 3, 96, 96, True, 2, 0), (6, 3, 48, 0, False, 16, 8), (2, 1, 136, 130, True, 16, 0),
])
def test_append(kb, dtype, q_heads, heads, dim, rot, pairs, page, gap):
    g = torch.Generator().manual_seed(dim + rot)
    seqs, cap = 6, 100
    k_cache, v_cache, table = make_cache(g, dtype, seqs, heads, dim, page, cap, dirty=False)
    slots = table.shape[1] * page
    table[4, -1] = -5
    # two tokens of a prompt, a row without a token, one past the table, a hole, a sequence out of range
    seq = torch.tensor([0, 0, 1, 2, 3, 4, 5, 6, -1, 5], dtype=torch.int32)
    length = torch.tensor([1, 2, slots, 0, slots + 1, slots, 37, 3, 3, 38], dtype=torch.int32)
    R = len(seq)
    pos = torch.tensor([0, 1, 131071, 5, 1000003, 2 ** 31 - 1, -4, 77, 8, 123456], dtype=torch.int32)
    row = (q_heads + 2 * heads) * dim + gap
    qkv = torch.randn(R * row + gap, generator=g).to(dtype)
    split = lambda t: [x.unflatten(1, (-1, dim)) if x.shape[1] else None  # noqa: E731
                       for x in t[gap:].view(R, row)[:, :row - gap].split([q_heads * dim, heads * dim, heads * dim], 1)]
    freq = kb.rotary_frequencies(rot, factor=4.0, trained_length=512, device="cpu") if rot else None
    position = torch.full((seqs, heads, slots), -9, dtype=torch.int32)
    weight = torch.full((seqs, heads, slots), 5.0)
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    dk, dv, dp, dw = dev(k_cache), dev(v_cache), dev(position), dev(weight)
    q, k, v = split(qkv)
    dq, dkn, dvn = split(dev(qkv))
    amp = 1.25
    q_out = kb.cache_append(dk, dv, dev(table), dev(length), dkn, dvn, q=dq, pos=dev(pos), freq=dev(freq),
                            interleaved=pairs, amplitude=amp, seq=dev(seq), position=dp, weight=dw)
    torch.cuda.synchronize()
    ref = co.append(f64(k_cache), f64(v_cache), table.numpy(), length.numpy(), f64(k), f64(v),
                    q=None if q is None else f64(q), pos=pos.numpy(), freq=[] if freq is None else freq.numpy(),
                    interleaved=pairs, amplitude=amp, seq=seq.numpy(), position=position.numpy(), weight=weight.numpy())
    big = (2.0 ** -21 + 3 * 2.0 ** -53 * 2.0 ** 31) * amp * 2 * float(qkv.abs().max())

    def near(got, want):
        err = np.abs(f64(got) - want)
        assert np.all(err <= ROUND[dtype] * np.abs(want) + (big if rot else 0)), err.max()
    if q is not None:
        near(q_out, ref[0])
    near(dk, ref[1])
    changed = np.any(ref[1] != f64(k_cache), axis=-1)
    assert np.array_equal(bits(dk)[~changed], bits(k_cache)[~changed])
    assert np.array_equal(f64(dv), ref[2])
    assert np.array_equal(host(dp), ref[3]) and np.array_equal(host(dw), ref[4])
    if rot < dim and q is not None:
        assert np.array_equal(f64(q_out)[..., rot:], f64(q)[..., rot:])


def test_append_without_seq_and_past_the_count(kb):
    """Rows are their own sequences; rows from the device's count on are left alone; queries turned in place."""
    g = torch.Generator().manual_seed(3)
    k_cache, v_cache, table = make_cache(g, torch.float32, 5, 2, 64, 4, 20, dirty=False)
    length = torch.tensor([1, 20, 7, 3, 4], dtype=torch.int32)
    q, k, v = (torch.randn((5, h, 64), generator=g) for h in (4, 2, 2))
    pos = length - 1
    freq = kb.rotary_frequencies(64, device="cpu")
    dk, dv, dq = k_cache.cuda(), v_cache.cuda(), q.cuda()
    got = kb.cache_append(dk, dv, table.cuda(), length.cuda(), k.cuda(), v.cuda(), q=dq, pos=pos.cuda(), freq=freq.cuda(),
                          n_dev=torch.tensor([3], dtype=torch.int32, device="cuda"), q_out=dq)
    ref = co.append(f64(k_cache), f64(v_cache), table.numpy(), length.numpy(), f64(k), f64(v), q=f64(q),
                    pos=pos.numpy(), freq=freq.numpy(), n=3)
    assert got is dq
    assert np.abs(f64(dq)[:3] - ref[0][:3]).max() <= 2.0 ** -21 * 2 * float(q.abs().max()) + U * 8
    assert torch.equal(dq[3:].cpu(), q[3:])
    assert np.abs(f64(dk) - ref[1]).max() <= 2.0 ** -21 * 2 * float(k.abs().max()) + U * 8
    assert np.array_equal(f64(dv), ref[2])


def run_evict(kb, k, v, table, length, keep, weight, position=None, newest=None, first=0, recent=0, out_table=None,
              n=None, own=False):
    """The call on the GPU against the oracle, bit for bit.  ``own``: results over the inputs."""
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    R, heads, page = len(length), k.shape[1], k.shape[2]
    cols = (table if out_table is None else out_table).shape[1]
    shape = (R, heads, cols * page)
    ow = weight[:R].clone() if own else torch.full(shape, -3.0)
    op = None if position is None else position[:R].clone() if own else torch.full(shape, -3, dtype=torch.int32)
    dk, dv, dt, dl, dw, dp = (dev(x) for x in (k, v, table, length, weight, position))
    res = ((dl, dw, dp) if own else (torch.full((R,), -3, dtype=torch.int32, device="cuda"), dev(ow), dev(op)))
    res += (torch.full((R, heads, keep), -3, dtype=torch.int32, device="cuda"),)
    got = kb.cache_evict(dk, dv, dt, dl, keep, weight=dw, position=dp, newest=dev(newest), first=first, recent=recent,
                         out_table=dev(out_table), out=res,
                         n_dev=None if n is None else torch.tensor([n], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    rk, rv, rl, rw, rp, rs = co.evict(bits(k), bits(v), table.numpy(), length.numpy(), keep,
                                      weight=weight.numpy(), position=None if position is None else position.numpy(),
                                      newest=None if newest is None else newest.numpy(), first=first, recent=recent,
                                      out_table=None if out_table is None else out_table.numpy(), out_weight=ow.numpy(),
                                      out_position=None if op is None else op.numpy(), n=n)
    m = R if n is None else n
    assert np.array_equal(host(got[3])[:m], rs[:m]), "source"
    assert np.all(host(got[3])[m:] == -3)
    assert np.array_equal(host(got[0])[:m], rl[:m]), "length"
    assert np.array_equal(host(got[0])[m:], length.numpy()[m:] if own else np.full(R - m, -3))
    assert np.array_equal(host(got[1])[:R].view(np.int32), rw.view(np.int32)), "weight"
    if position is not None:
        assert np.array_equal(host(got[2])[:R], rp), "position"
    assert np.array_equal(bits(dk), rk) and np.array_equal(bits(dv), rv), "rows"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads,dim,page,cap,keep,first,recent", [
    (1, 8, 1, 40, 16, 0, 0), (2, 64, 16, 300, 256, 4, 64), (3, 72, 8, 1100, 500, 0, 100), (1, 128, 64, 2100, 1, 0, 1),
    (2, 256, 4, 70, 69, 69, 0), (1, 40, 1024, 5000, 1024, 3, 7), (2, 16, 2, 1500, 1400, 0, 0), (1, 8, 32, 20, 64, 1, 1),
    (2, 16, 1, 1101, 300, 1, 20), (3, 8, 1, 2503, 2400, 0, 5),
])
def test_evict(kb, dtype, heads, dim, page, cap, keep, first, recent):
    g = torch.Generator().manual_seed(cap + keep)
    lens = sorted({0, 1, min(keep, cap) - 1, min(keep, cap), min(keep + 1, cap), cap, cap - 1, (keep + cap) // 2})
    length = torch.tensor(lens, dtype=torch.int32)
    R = len(lens)
    k, v, table = make_cache(g, dtype, R + 1, heads, dim, page, cap, dirty=False)
    slots = table.shape[1] * page
    weight = torch.rand((R + 1, heads, slots), generator=g) ** 4
    position = torch.stack([torch.randperm(slots, generator=g) for _ in range((R + 1) * heads)])
    position = position.view(R + 1, heads, slots).to(torch.int32)
    newest = torch.full((R,), slots - 1, dtype=torch.int32)
    args = dict(position=position, newest=newest, first=first, recent=recent)
    run_evict(kb, k, v, table, length, keep, weight, **args)
    run_evict(kb, k, v, table, length, keep, weight, own=True, **args)
    run_evict(kb, k, v, table, length, keep, weight, n=R // 2, **args)
    run_evict(kb, k, v, table, length, keep, weight)
    # into pages of their own
    cols = -(-min(keep, slots) // page) + 1
    more = torch.randn((R * cols,) + tuple(k.shape[1:]), generator=g).to(dtype)
    out_table = (torch.randperm(R * cols, generator=g) + k.shape[0]).to(torch.int32).view(R, cols)
    out_table[0, -1] = -1
    k, v = torch.cat([k, more]), torch.cat([v, more])
    run_evict(kb, k, v, table, length, keep, weight, out_table=out_table, **args)


def test_evict_ties_and_special_values(kb):
    """Equal weights keep the lower slot; zeros of both signs are equal; NaN ranks below -inf; +inf above all
    numbers, below protected slots; a hole's slot is chosen as any other, its row not copied."""
    g = torch.Generator().manual_seed(1)
    L, keep = 3000, 1030
    k, v, table = make_cache(g, torch.bfloat16, 9, 1, 16, 8, L, dirty=False)
    length = torch.full((9,), L, dtype=torch.int32)
    w = torch.zeros((9, 1, table.shape[1] * 8))
    w[1] = math.nan
    w[2, :, ::2] = -0.0
    w[3] = torch.randint(0, 4, w[3].shape, generator=g).float()
    w[4] = torch.tensor([math.nan, -math.inf, math.inf, 1.0, -1.0])[torch.randint(0, 5, w[4].shape, generator=g)]
    w[5] = torch.arange(w.shape[2]).float()
    w[6] = -torch.arange(w.shape[2]).float()
    w[7, :, 2000:] = 1e-45
    w[8] = math.inf
    table[3, 10:20] = -1
    table[6, 200:] = 2 ** 30
    position = torch.arange(w.shape[2], dtype=torch.int32).expand(9, 1, -1).contiguous()
    newest = torch.full((9,), L - 1, dtype=torch.int32)
    run_evict(kb, k, v, table, length, keep, w)
    run_evict(kb, k, v, table, length, keep, w, position=position, newest=newest, first=2, recent=900)
    newest[:] = -2 ** 31  # newest - recent is below every int32: all slots are protected, the lowest stay
    run_evict(kb, k, v, table, length, keep, w, position=position, newest=newest, first=0, recent=5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R,heads,dim,page,cap,keeps", [
    (17, 8, 64, 16, 300, (1, 20, 63, 64, 65, 130, 256)),   # many heads: the selecting workgroups move the rows
    (43, 3, 16, 4, 2100, (100, 513, 1100)),                # the same, 16 waves each
    (2, 2, 256, 1, 2300, (500, 1150)),                     # few heads with much to move: a second launch does
    (127, 1, 72, 32, 700, (300,)),
    (1, 1, 256, 8, 200, (3, 64, 100)),                     # few with little
])
def test_evict_by_either_mover(kb, dtype, R, heads, dim, page, cap, keeps):
    """Rows moved by the workgroups that select them and by a launch of their own: in place, over the inputs,
    counted on the device, and elsewhere, with rows that are within the budget."""
    g = torch.Generator().manual_seed(R + cap)
    length = torch.randint(0, cap + 1, (R,), generator=g, dtype=torch.int32)
    length[0] = cap
    k, v, table = make_cache(g, dtype, R, heads, dim, page, cap, dirty=False)
    slots = table.shape[1] * page
    weight = torch.rand((R, heads, slots), generator=g).round(decimals=2)  # (with ties)
    position = torch.stack([torch.randperm(slots, generator=g) for _ in range(R * heads)])
    position = position.view(R, heads, slots).to(torch.int32)
    args = dict(position=position, newest=torch.full((R,), slots - 1, dtype=torch.int32))
    for keep in keeps:
        args.update(first=keep // 8, recent=keep // 4)
        run_evict(kb, k, v, table, length, keep, weight, own=True, **args)
        run_evict(kb, k, v, table, length, keep, weight, own=True, n=R - R // 3, **args)
        run_evict(kb, k, v, table, length, keep, weight, n=R // 2, **args)
        cols = -(-keep // page)
        more = torch.randn((R * cols,) + tuple(k.shape[1:]), generator=g).to(dtype)
        out_table = (torch.randperm(R * cols, generator=g) + k.shape[0]).to(torch.int32).view(R, cols)
        out_table[0, 0] = -7
        run_evict(kb, torch.cat([k, more]), torch.cat([v, more]), table, length, keep, weight, out_table=out_table,
                  **args)


@pytest.mark.parametrize("L,keeps", [(70000, (20000, 3, 69999)), (300001, (150000,)), (1 << 19, (1000,))])
def test_evict_long(kb, L, keeps):
    """Longer than what keys fit the chip, up to the longest; ties across wave and strip borders."""
    g = torch.Generator().manual_seed(L)
    k, v, table = make_cache(g, torch.bfloat16, 2, 1, 8, 128, L, dirty=False)
    length = torch.tensor([L, L // 2 - 1], dtype=torch.int32)
    w = (torch.rand((2, 1, table.shape[1] * 128), generator=g) * 5000).round()
    w[1] = 1
    for keep in keeps:
        run_evict(kb, k, v, table, length, keep, w)


@pytest.mark.parametrize("L,keep", [(16384, 5000), (20001, 20000), (30017, 2048), (32768, 31)])
def test_evict_of_many_slots_with_few_open(kb, L, keep):
    """After the first digit few slots are open, spread (row 0), side by side (row 1) or equal (row 2); all of
    them in row 3, and no more than a quarter short of none in row 4."""
    g = torch.Generator().manual_seed(L)
    k, v, table = make_cache(g, torch.bfloat16, 5, 1, 8, 128, L, dirty=False)
    slots = table.shape[1] * 128
    length = torch.full((5,), L, dtype=torch.int32)
    w = torch.rand((5, 1, slots), generator=g).clamp_min(1e-6) ** -0.7
    rank = torch.arange(slots, dtype=torch.float32)
    w[1, 0] = torch.where((rank - L + keep).abs() < L // 10, 1 + (rank % 500) / 4096, torch.where(rank < L - keep, 0.1, 9.0))
    w[2, 0] = torch.where((rank - L + keep).abs() < L // 10, 1.0, torch.where(rank < L - keep, 0.1, 9.0))
    w[3] = 1
    w[4] = torch.rand(slots, generator=g)
    for own in (False, True):
        run_evict(kb, k, v, table, length, keep, w, own=own)
    position = torch.stack([torch.randperm(slots, generator=g) for _ in range(5)]).view(5, 1, slots).to(torch.int32)
    newest = torch.full((5,), slots - 1, dtype=torch.int32)
    run_evict(kb, k, v, table, length, keep, w, position=position, newest=newest, first=4, recent=keep // 4)


@pytest.mark.parametrize("count", [0, -1, -2 ** 31])
def test_no_rows_on_the_device(kb, count):
    """A device count of none or less: every output stays as it was."""
    g = torch.Generator().manual_seed(6)
    for cap in (40, 2000):
        k, v, table = (x.cuda() for x in make_cache(g, torch.float32, 3, 2, 64, 8, cap, dirty=False))
        n = torch.full((3,), cap, dtype=torch.int32, device="cuda")
        nd = torch.tensor([count], dtype=torch.int32, device="cuda")
        x = torch.randn((3, 4, 64), generator=g).cuda()
        w = torch.ones((3, 2, table.shape[1] * 8), device="cuda")
        keep = [t.clone() for t in (k, v, w)]
        out, lse, q_out = torch.full_like(x, 7), torch.full((3, 4), 7.0, device="cuda"), torch.full_like(x, 7)
        res = (torch.full((3,), 7, dtype=torch.int32, device="cuda"), w, None,
               torch.full((3, 2, 9), 7, dtype=torch.int32, device="cuda"))
        kb.cache_append(k, v, table, n, x[:, :2], x[:, 2:], q=x, q_out=q_out, weight=w, n_dev=nd)
        kb.cache_attend(x, k, v, table, n, out=out, lse=lse, weight_out=w, n_dev=nd)
        kb.cache_evict(k, v, table, n, 9, weight=w, out=res, n_dev=nd)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((k, v, w), keep))
        for t in (out, lse, q_out, res[0], res[3]):
            assert bool((t == 7).all())


@pytest.mark.parametrize("pages,seqs,R", [(0, 4, 4), (3, 0, 4), (0, 0, 1100)])
def test_empty_pools_and_tables(kb, pages, seqs, R):
    """No pages or no sequences: nothing to attend to, nowhere to store, whatever the lengths say."""
    shape = (pages, 2, 16, 64)
    for cols in (1, 200):
        k, v = (torch.full(shape, math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        table = torch.zeros((seqs, cols), dtype=torch.int32, device="cuda")
        n = torch.full((R,), 10, dtype=torch.int32, device="cuda")
        seq = None if seqs else torch.zeros(R, dtype=torch.int32, device="cuda")
        q = torch.ones((R, 4, 64), dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros((R, 4), device="cuda")
        kb.cache_append(k, v, table, n, q[:, :2], q[:, 2:], q=q, seq=seq)
        out = kb.cache_attend(q, k, v, table, n, lse=lse, seq=seq)
        torch.cuda.synchronize()
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        assert pages == 0 or bool(torch.isnan(k).all())
    if seqs:
        w = torch.rand((seqs, 2, 3200), device="cuda")
        got = kb.cache_evict(k, v, table, n, 4, weight=w)
        assert got[0].tolist() == [4] * R
        assert torch.equal(got[1][:, :, :4].sort().values, w[:, :, :10].topk(4).values.sort().values)


def test_offsets_past_32_bits(kb):
    """The last pages of a pool of more than 2^32 bytes and 2^31 values give what the same pages of a small one do."""
    g = torch.Generator().manual_seed(16)
    R, Q, heads, dim, page, cap = 3, 8, 2, 256, 64, 1000
    k, v, table = make_cache(g, torch.bfloat16, R, heads, dim, page, cap, spare=0, dirty=False)
    pages = k.shape[0]
    big_pages = 2 ** 31 // (heads * page * dim) + 40000
    assert big_pages * heads * page * dim * 2 > 2 ** 32 and big_pages * heads * page < 2 ** 31
    k, v, table = k.cuda(), v.cuda(), table.cuda()
    bk, bv = (torch.empty((big_pages,) + tuple(k.shape[1:]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = torch.arange(big_pages - pages, big_pages, device="cuda")
    bk[at], bv[at] = k, v
    far = (table + big_pages - pages).to(torch.int32)
    n = torch.tensor([1000, 999, 64], dtype=torch.int32, device="cuda")
    x = torch.randn((R, Q + 2 * heads, dim), generator=g).bfloat16().cuda()
    pos, freq = n - 1, kb.rotary_frequencies(dim)
    res = []
    for kc, vc, t in ((k, v, table), (bk, bv, far)):
        w = torch.zeros((R, heads, t.shape[1] * page), device="cuda")
        q = kb.cache_append(kc, vc, t, n, x[:, Q:Q + heads], x[:, Q + heads:], q=x[:, :Q], pos=pos, freq=freq)
        lse = torch.zeros((R, Q), device="cuda")
        out = kb.cache_attend(q, kc, vc, t, n, lse=lse, weight_out=w)
        ev = kb.cache_evict(kc, vc, t, n, 300, weight=w)
        res.append((q, out, lse, w, ev[0], ev[1], ev[3]))
    torch.cuda.synchronize()
    for a, b in zip(*res):
        assert torch.equal(a, b)
    assert torch.equal(bk[at], k) and torch.equal(bv[at], v)


def test_attend_replayed_over_other_lengths(kb):
    """A graph of the shared-out attention, captured at some lengths, replayed at others and other tables: the work
    is shared out anew from what is on the device."""
    g = torch.Generator().manual_seed(14)
    R, Q, heads, dim, page, cap = 9, 6, 2, 64, 16, 2500
    k, v, table = make_cache(g, torch.bfloat16, R, heads, dim, page, cap, dirty=False)
    q = torch.randn((R, Q, dim), generator=g).bfloat16()
    dk, dv, dt, dq = k.cuda(), v.cuda(), table.cuda(), q.cuda()
    n = torch.full((R,), 100, dtype=torch.int32, device="cuda")
    w = torch.zeros((R, heads, dt.shape[1] * page), device="cuda")
    out, lse = torch.zeros_like(dq), torch.zeros((R, Q), device="cuda")
    ws = torch.empty(kb.cache_attend_workspace_bytes(dk, dv, dt, R, Q, weights=True), dtype=torch.uint8, device="cuda")
    call = lambda o, e, x: kb.cache_attend(dq, dk, dv, dt, n, out=o, lse=e, weight_out=x, ws=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, lse, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, w)
    for i in range(6):
        n.copy_(torch.randint(0, cap + 1, (R,), generator=g).to(torch.int32) if i != 3 else torch.zeros(R).int())
        dt.copy_(table[torch.randperm(R, generator=g)])
        graph.replay()
        a, b, c = torch.zeros_like(out), torch.zeros_like(lse), w.clone()
        torch.cuda.synchronize()
        call(a, b, c)
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, lse) and torch.equal(c, w), f"replay {i}"
    check_attend(kb, q, k, v, dt.cpu(), n.cpu(), weights=True)


def test_run_together_under_a_graph(kb):
    """Append, attend and evict as a decode loop calls them, captured once and replayed over changing inputs, with
    eager work and synchronizations between: every replay equals the eager calls on a copy of the state."""
    g = torch.Generator().manual_seed(4)
    S, Q, heads, dim, page, keep = 3, 4, 2, 64, 8, 40
    cap = 48
    k, v, table = make_cache(g, torch.bfloat16, S, heads, dim, page, cap, dirty=False)
    table = table.cuda()
    freq = kb.rotary_frequencies(dim)
    start = torch.tensor([30, 1, 39], dtype=torch.int32, device="cuda")

    def state():
        return dict(k=k.cuda(), v=v.cuda(), length=start.clone(), pos=start - 1,
                    position=torch.arange(cap, dtype=torch.int32, device="cuda").expand(S, heads, cap).contiguous(),
                    weight=torch.ones((S, heads, cap), device="cuda"),
                    source=torch.zeros((S, heads, keep), dtype=torch.int32, device="cuda"),
                    qkv=torch.zeros((S, Q + 2 * heads, dim), dtype=torch.bfloat16, device="cuda"),
                    out=torch.zeros((S, Q, dim), dtype=torch.bfloat16, device="cuda"),
                    q=torch.zeros((S, Q, dim), dtype=torch.bfloat16, device="cuda"))

    def step(s):
        s["length"] += 1
        s["pos"] += 1
        q, kn, vn = s["qkv"].split([Q, heads, heads], 1)
        kb.cache_append(s["k"], s["v"], table, s["length"], kn, vn, q=q, pos=s["pos"], freq=freq, q_out=s["q"],
                        position=s["position"], weight=s["weight"])
        kb.cache_attend(s["q"], s["k"], s["v"], table, s["length"], out=s["out"], weight_in=s["weight"],
                        weight_out=s["weight"])
        kb.cache_evict(s["k"], s["v"], table, s["length"], keep, weight=s["weight"], position=s["position"],
                       newest=s["pos"], first=1, recent=4,
                       out=(s["length"], s["weight"], s["position"], s["source"]))
    a, b = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = state()
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    for n in range(20):
        x = torch.randn((S, Q + 2 * heads, dim), generator=g).bfloat16().cuda()
        a["qkv"].copy_(x)
        b["qkv"].copy_(x)
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        for name in a:
            assert torch.equal(a[name], b[name]), f"replay {n}: {name}"
    assert a["length"].tolist() == [40, 21, 40]
    # the newest four tokens and the first are all still there
    for s in range(S):
        for h in range(heads):
            there = set(a["position"][s, h, :int(a["length"][s])].tolist())
            newest = int(a["pos"][s])
            assert {0, newest, newest - 1, newest - 2, newest - 3} <= there
