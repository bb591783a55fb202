"""The decode loops over a decoder where words are masked until a sentence has fewer continuations than its beam, and
where its states are no numbers: the searches end, and what can be said of their results holds."""
import numpy as np
import pytest
import torch

from tests.gpu_util import TOL
from tests.test_gpu_cached_decode import EOS, V, f64, log_probs, make, states

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


@pytest.mark.parametrize("words,k,T", [([17], 3, 6), ([17, 401], 4, 6), ([2, 3, 499], 7, 8)])
def test_few_words_left(kb, words, k, T):
    """Each translation is of the words that are left, and its score is the sum of its tokens' log-probabilities among
    them, to the output layer's tolerance a token; greedy search takes the best of them at every step."""
    from paper_1805_09863_amd.decode import beam_search, greedy_search
    dec, W, b = make(seed=k, eos_bias=0.0)
    mask = torch.full((V,), -float("inf"))
    mask[words] = 0
    b = b + mask.cuda()
    start = torch.tensor([5, 9, 0], dtype=torch.int32, device="cuda")
    res = beam_search(None, W, b, k, T, EOS, decoder=dec, start=start)
    one = greedy_search(dec, W, b, start, T, EOS)
    torch.cuda.synchronize()
    Wx, bx = W[:, words].contiguous(), b[words]
    for tokens, length, score in ((res.tokens, res.length, res.score), (one.tokens, one.length, None)):
        for s in range(len(start)):
            n = int(length[s])
            tok = tokens[s, :n].tolist()
            assert set(tok) <= set(words) and (n == T or tok[-1] == EOS)
            lp = log_probs(states(dec, [int(start[s])] + tok[:-1]), Wx, bx)
            at = [words.index(w) for w in tok]
            if score is None:
                assert all(lp[i, a] >= lp[i].max() - 2 * TOL["f32"] for i, a in enumerate(at))
            else:
                assert abs(sum(lp[i, a] for i, a in enumerate(at)) - float(score[s])) <= TOL["f32"] * n


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 40])
def test_states_that_are_no_numbers(kb, dtype, rows):
    """A sentence that starts from a token whose embedding is NaN ends after T tokens at most, all of them words or
    none (-1); the others are what they are without it."""
    from paper_1805_09863_amd.decode import beam_search, greedy_search
    dec, W, b = make(dtype, seed=4)
    g = torch.Generator().manual_seed(rows)
    start = torch.randint(10, V, (rows,), generator=g).to(torch.int32).cuda()
    b[7] = -float("inf")                                     # (no other sentence comes to it)
    T = 9
    runs = []
    for bad in (False, True):
        if bad:
            dec.embed[7] = float("nan")
            start[1] = 7
        runs.append((beam_search(None, W, b, 4, T, EOS, decoder=dec, start=start), greedy_search(dec, W, b, start, T, EOS)))
    torch.cuda.synchronize()
    for c in runs[1]:
        assert int(c.tokens.min()) >= -1 and int(c.tokens.max()) < V
        assert int(c.length.max()) <= T
    # a best score may be off by a step's tolerance at each of its steps, in either run (the number of rows picks the
    # projection's kernel, and other kernels sum in another order)
    others = [s for s in range(rows) if s != 1]
    a, c = (f64(r[0].score)[others] for r in runs)
    assert np.abs(a - c).max() <= 2 * T * TOL["f32" if dtype == torch.float32 else "bf16"]


def test_searches_over_a_modules_parameters(kb):
    """The decoder's weights and W as a trained module holds them: the same searches."""
    from paper_1805_09863_amd.decode import beam_search, greedy_search
    from paper_1805_09863_amd.decoder import CachedDecoder
    dec, W, b = make(seed=6)
    module = CachedDecoder(*(torch.nn.Parameter(x.clone()) for x in (dec.embed, dec.Wqkv, dec.Wo)), dec.q_heads,
                           dec.kv_heads)
    start = torch.tensor([5, 9, 11], dtype=torch.int32, device="cuda")
    runs = []
    for d, w, c in ((dec, W, b), (module, torch.nn.Parameter(W.clone()), torch.nn.Parameter(b.clone()))):
        r, o = beam_search(None, w, c, 3, 12, EOS, decoder=d, start=start), greedy_search(d, w, c, start, 12, EOS, keep=6)
        runs.append((r.tokens, r.score, o.tokens))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and not y.requires_grad for x, y in zip(*runs))
