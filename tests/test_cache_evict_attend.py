"""Attention over what an eviction has kept is attention over the kept slots of the cache before it, where every slot
and every place has a page; with the oracle alone, and the operators one after the other on the GPU."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co

U = 2.0 ** -24


def problem(seed, R, Q, heads, dim, page, cap, keep, elsewhere):
    """Sequences over and within the budget, in scattered pages: float32 values, as host arrays."""
    g = np.random.default_rng(seed)
    cols, out_cols = -(-cap // page), -(-keep // page)
    pages = R * (cols + out_cols) + 3
    at = g.permutation(pages).astype(np.int32)
    table = at[:R * cols].reshape(R, cols)
    out_table = at[R * cols:R * (cols + out_cols)].reshape(R, out_cols) if elsewhere else None
    k, v = (g.standard_normal((pages, heads, page, dim)).astype(np.float32) for _ in range(2))
    slots = cols * page
    length = g.integers(1, cap + 1, R).astype(np.int32)
    length[0], length[-1] = cap, max(1, keep // 2)
    weight = g.random((R, heads, slots)).astype(np.float32) ** 4
    position = np.stack([g.permutation(slots) for _ in range(R * heads)]).reshape(R, heads, slots).astype(np.int32)
    newest = np.full(R, slots - 1, np.int32)
    q = g.standard_normal((R, Q, dim)).astype(np.float32)
    return dict(k=k, v=v, table=table, out_table=out_table, length=length, weight=weight, position=position,
                newest=newest, q=q, keep=keep, first=min(2, keep // 4), recent=keep // 4)


def kept_attention(p):
    """Attention of each row over the slots that stay, from the cache before: (out, spread, size, slots)."""
    R, Q, dim = p["q"].shape
    heads, page = p["k"].shape[1:3]
    out, size, spread = np.zeros((R, Q, dim)), np.zeros((R, Q, dim)), np.zeros((R, Q, 1))
    for r, L in enumerate(p["length"].tolist()):
        for h in range(Q):
            kv = h // (Q // heads)
            src = np.array(co.kept_slots(p["weight"][r, kv, :L], p["position"][r, kv, :L], p["keep"], p["first"],
                                         p["recent"], int(p["newest"][r])))
            pg, pl = p["table"][r][src // page], src % page
            K, V = p["k"][pg, kv, pl].astype(np.float64), p["v"][pg, kv, pl].astype(np.float64)
            x = K @ p["q"][r, h].astype(np.float64) * dim ** -0.5
            e = np.exp(x - x.max())
            e /= e.sum()
            out[r, h], size[r, h] = e @ V, e @ np.abs(V)
            spread[r, h] = (np.abs(K) @ np.abs(p["q"][r, h])).max() * dim ** -0.5
    return out, spread, size


CASES = [(0, 4, 4, 2, 16, 4, 60, 20, False), (1, 3, 6, 3, 24, 1, 41, 40, True), (2, 5, 2, 1, 8, 16, 100, 7, True),
         (3, 2, 2, 2, 16, 8, 30, 64, False)]


@pytest.mark.parametrize("case", CASES)
def test_oracle(case):
    p = problem(*case)
    to = p["table"] if p["out_table"] is None else p["out_table"]
    shape = p["k"].shape
    places = p["weight"].shape[:2] + (to.shape[1] * shape[2],)
    k, v, length, _, _, _ = co.evict(p["k"], p["v"], p["table"], p["length"], p["keep"], weight=p["weight"],
                                     position=p["position"], newest=p["newest"], first=p["first"], recent=p["recent"],
                                     out_table=p["out_table"], out_weight=np.zeros(places, np.float32),
                                     out_position=np.zeros(places, np.int32))
    got = co.attend(p["q"].astype(np.float64), k.astype(np.float64), v.astype(np.float64), to, length,
                    p["q"].shape[2] ** -0.5)[0]
    assert np.allclose(got, kept_attention(p)[0], rtol=1e-12, atol=1e-12)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES + [(4, 70, 8, 4, 64, 16, 700, 300, False), (5, 6, 8, 2, 128, 64, 3000, 1100, True),
                                          (6, 300, 2, 2, 32, 8, 90, 50, True)])
def test_on_the_gpu(case):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    p = problem(*case)
    d = {n: torch.from_numpy(x).cuda() for n, x in p.items() if isinstance(x, np.ndarray)}
    n, _, _, _ = kb.cache_evict(d["k"], d["v"], d["table"], d["length"], p["keep"], weight=d["weight"],
                                position=d["position"], newest=d["newest"], first=p["first"], recent=p["recent"],
                                out_table=d.get("out_table"))
    got = kb.cache_attend(d["q"], d["k"], d["v"], d.get("out_table", d["table"]), n)
    torch.cuda.synchronize()
    want, spread, size = kept_attention(p)
    # scores of dim products and a scale, their size in base 2, an exponential each and the sums over the slots, as
    # float32 operations of half a step; the output's own rounding
    dim, slots = p["q"].shape[2], min(p["keep"], int(p["length"].max()))
    tol = (2 * (dim + 6) * U * spread + 2.0 ** -22 + 2 * slots * U) * size + U * np.abs(want)
    assert np.all(np.abs(got.cpu().double().numpy() - want) <= tol)
