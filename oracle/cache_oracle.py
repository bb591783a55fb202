"""fp64 oracle of the attention cache, from the definitions: rotary positions, the append into
pages, attention of one token a row, eviction by accumulated weight.  Row by row and slot by
slot on the host; test infrastructure only.
"""
from __future__ import annotations

import math

import numpy as np


def slot_place(table_row, t, page_size, pages):
    """(page, place) of slot t, None for a hole."""
    p = int(table_row[t // page_size])
    return (p, t % page_size) if 0 <= p < pages else None


def rotate(x, pos, freq, interleaved, amplitude):
    """x: dim float64; the first 2 * len(freq) values turned."""
    y = x.copy()
    half = len(freq)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = math.cos(pos * f), math.sin(pos * f)
        y[a] = amplitude * (x[a] * c - x[b] * s)
        y[b] = amplitude * (x[a] * s + x[b] * c)
    return y


def append(k_cache, v_cache, table, length, k, v, *, q=None, pos=None, freq=(), interleaved=False, amplitude=1.0,
           seq=None, n=None, position=None, weight=None):
    """Float64 arrays in, new ones out: (q_out, k_cache, v_cache, position, weight); rows from n on are not worked on."""
    k_cache, v_cache = k_cache.copy(), v_cache.copy()
    position = None if position is None else position.copy()
    weight = None if weight is None else weight.copy()
    pages, heads, ps, _ = k_cache.shape
    seqs, cols = table.shape
    q_out = None if q is None else np.full(q.shape, np.nan)
    for r in range(len(length) if n is None else min(n, len(length))):
        p = None if pos is None else int(pos[r])
        if q is not None:
            for h in range(q.shape[1]):
                q_out[r, h] = rotate(q[r, h], p, freq, interleaved, amplitude)
        s, slot = (r if seq is None else int(seq[r])), int(length[r]) - 1
        if not 0 <= s < seqs or not 0 <= slot < cols * ps:
            continue
        at = slot_place(table[s], slot, ps, pages)
        if at is None:
            continue
        for h in range(heads):
            k_cache[at[0], h, at[1]] = rotate(k[r, h], p, freq, interleaved, amplitude)
            v_cache[at[0], h, at[1]] = v[r, h]
            if position is not None:
                position[s, h, slot] = slot if p is None else p
            if weight is not None:
                weight[s, h, slot] = 0.0
    return q_out, k_cache, v_cache, position, weight


def attended(table, length, page_size, pages, seq=None, max_len=None):
    """Per row, its sequence and the slots in [0, length) that have a page."""
    seqs, cols = table.shape
    rows = []
    for r in range(len(length)):
        s = r if seq is None else int(seq[r])
        n = min(int(length[r]), cols * page_size, cols * page_size if max_len is None else max_len)
        if not 0 <= s < seqs:
            rows.append((None, []))
        else:
            rows.append((s, [t for t in range(max(n, 0)) if slot_place(table[s], t, page_size, pages)]))
    return rows


def attend(q, k_cache, v_cache, table, length, scale, *, seq=None, max_len=None):
    """(out, lse, p, spread, size): p[r][h] the probabilities of the row's slots (attended() order);
    spread[r, h] the largest scale * sum |q_i k_i| over them and size[r, h] the vector sum p |v|,
    which error bounds are made of."""
    pages, heads, ps, D = k_cache.shape
    R, Q, _ = q.shape
    out, size = np.zeros((R, Q, D)), np.zeros((R, Q, D))
    lse, spread = np.full((R, Q), -np.inf), np.zeros((R, Q))
    probs = []
    for r, (s, slots) in enumerate(attended(table, length, ps, pages, seq, max_len)):
        probs.append([np.zeros(0)] * Q)
        if not slots:
            continue
        t = np.array(slots)
        pg, pl = table[s][t // ps], t % ps
        for h in range(Q):
            kv = h // (Q // heads)
            K, V = k_cache[pg, kv, pl], v_cache[pg, kv, pl]
            x = scale * (K @ q[r, h])
            m = x.max()
            e = np.exp(x - m)
            lse[r, h] = m + math.log(e.sum())
            p = e / e.sum()
            probs[r][h] = p
            out[r, h] = p @ V
            size[r, h] = p @ np.abs(V)
            spread[r, h] = abs(scale) * (np.abs(K) @ np.abs(q[r, h])).max()
    return out, lse, probs, spread, size


def kept_slots(weight, position, keep, first, recent, newest):
    """Source slot of each kept place of one sequence and head: weight and position of its length."""
    L = len(weight)
    n = min(L, keep)

    def rank(t):
        held = position is not None and (position[t] < first or (recent > 0 and position[t] > newest - recent))
        w = weight[t]
        return (0, 0, 0.0, t) if held else (1, 1 if w != w else 0, 0.0 if w != w else -float(w), t)
    best = set(sorted(range(L), key=rank)[:n])
    tail = iter(t for t in range(n, L) if t in best)
    return [t if t in best else next(tail) for t in range(n)]


def evict(k_cache, v_cache, table, length, keep, *, weight, position=None, newest=None, first=0, recent=0,
          out_table=None, out_weight=None, out_position=None, n=None):
    """(k_cache, v_cache, length, weight, position, source) after the eviction, of the types given."""
    pages, heads, ps, _ = k_cache.shape
    R = len(length)
    k_new, v_new = k_cache.copy(), v_cache.copy()
    to = table if out_table is None else out_table
    out_weight, out_position = out_weight.copy(), None if position is None else out_position.copy()
    out_length, source = np.array(length), np.full((R, heads, keep), -1, np.int32)
    for r in range(R if n is None else min(n, R)):
        L = min(max(int(length[r]), 0), table.shape[1] * ps)
        out_length[r] = min(L, keep)
        for h in range(heads):
            src = kept_slots(weight[r, h, :L], None if position is None else position[r, h, :L], keep, first, recent,
                             0 if newest is None else int(newest[r]))
            for i, t in enumerate(src):
                a, b = slot_place(table[r], t, ps, pages), slot_place(to[r], i, ps, pages)
                if a is not None and b is not None:
                    k_new[b[0], h, b[1]] = k_cache[a[0], h, a[1]]
                    v_new[b[0], h, b[1]] = v_cache[a[0], h, a[1]]
                out_weight[r, h, i] = weight[r, h, t]
                if position is not None:
                    out_position[r, h, i] = position[r, h, t]
            source[r, h, :len(src)] = src
    return k_new, v_new, out_length, out_weight, out_position, source
