"""What the decode loops hand to a decoder, with the library's calls replaced by host ones: tokens are always rows of its
embedding, also where a step has no word to give (-1 of the k-best, 2^31 - 1 of the argmax); a budget that the search
never comes to takes no memory; weights are float32 whatever torch's default type."""
import pytest
import torch

pytest.importorskip("paper_1805_09863_amd")
from paper_1805_09863_amd import decode  # noqa: E402

V, H = 11, 8


class Decoder:
    def __init__(self):
        self.embed, self.H, self.kv_heads, self.seen = torch.zeros(V, H), H, 1, []

    def cache(self, pages, page_size):
        return tuple(torch.zeros(pages, 1, page_size, 8) for _ in range(2))

    def step(self, token, pos, length, k_cache, v_cache, table, *, out=None, weight=None, **kw):
        self.seen.append(token.clone())
        self.weight = weight
        return self.embed[token.long()] if out is None else out


def test_beam_search_feeds_words_where_there_is_none(monkeypatch):
    def gather_rows(src, idx, *, n_dev, n_max, out, stream):
        n = min(n_max, int(n_dev[0]))
        out[:n] = src[idx[:n].long()]
    monkeypatch.setattr(decode.kbb, "gather_rows", gather_rows)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    dec = Decoder()
    states = decode._CachedStates(dec, i32(3, 4), 4, 5, None)
    out = torch.zeros(8, H)
    states.first(out)
    # sentence 0 has two continuations, sentence 1 one; all entries stay alive
    tok, par = i32(7, 2, -1, -1, 9, -1, -1, -1), i32(0, 0, 0, 0, 1, 1, 1, 1)
    states.next(1, 8, i32(8), tok, par, torch.arange(8, dtype=torch.int32), None, out)
    assert dec.seen[1].tolist() == [7, 2, 0, 0, 9, 0, 0, 0]


def test_greedy_search_feeds_words_where_there_is_none(monkeypatch):
    def argmax_step(h, W, b, *, out, ws, stream):
        out[0].copy_(torch.tensor([2 ** 31 - 1, 4], dtype=torch.int32))
    monkeypatch.setattr(decode.kbb, "argmax_step", argmax_step)
    monkeypatch.setattr(decode, "_check_decoder", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: None)
    dec = Decoder()
    res = decode.greedy_search(dec, torch.zeros(H, V), torch.zeros(V), torch.tensor([1, 2], dtype=torch.int32), 4, 3)
    assert res.steps == 4 and len(dec.seen) == 4
    for token in dec.seen:
        assert int(token.min()) >= 0 and int(token.max()) < V
    assert int(res.tokens.max()) < V


def test_greedy_search_with_a_budget_past_all_memory(monkeypatch):
    def argmax_step(h, W, b, *, out, ws, stream):
        out[0].fill_(5)
    monkeypatch.setattr(decode.kbb, "argmax_step", argmax_step)
    monkeypatch.setattr(decode, "_check_decoder", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: None)
    start = torch.tensor([1, 2], dtype=torch.int32)
    res = decode.greedy_search(Decoder(), torch.zeros(H, V), torch.zeros(V), start, 4, 3, keep=10 ** 13)
    assert res.tokens.tolist() == [[5] * 4] * 2 and res.evictions == 0


def test_greedy_search_under_another_default_type(monkeypatch):
    def argmax_step(h, W, b, *, out, ws, stream):
        out[0].fill_(5)
    monkeypatch.setattr(decode.kbb, "argmax_step", argmax_step)
    monkeypatch.setattr(decode, "_check_decoder", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: None)
    dec, W, b = Decoder(), torch.zeros(H, V), torch.zeros(V)
    torch.set_default_dtype(torch.float64)
    try:
        decode.greedy_search(dec, W, b, torch.tensor([1, 2], dtype=torch.int32), 4, 3, keep=3, every=9)
    finally:
        torch.set_default_dtype(torch.float32)
    assert dec.weight.dtype == torch.float32
