"""CachedDecoder's own products on the host, the cache's operators replaced by host ones."""
import pytest
import torch

pytest.importorskip("paper_1805_09863_amd")
from paper_1805_09863_amd import decoder  # noqa: E402

V, H, Q, KV, D = 11, 24, 4, 2, 8


@pytest.mark.parametrize("with_out", [False, True])
@pytest.mark.parametrize("trained", [False, True])
def test_a_step_with_a_trained_models_weights(monkeypatch, with_out, trained):
    """Weights may be a module's parameters: a step records nothing for a backward pass, and its states may be written
    to memory of the caller's."""
    monkeypatch.setattr(decoder.kbb, "cache_append", lambda k_cache, v_cache, table, length, k, v, *, q, **kw: q.contiguous())
    monkeypatch.setattr(decoder.kbb, "cache_attend", lambda q, *a, **kw: q * 2)
    g = torch.Generator().manual_seed(1)
    w = [torch.randn(s, generator=g) for s in ((V, H), (H, (Q + 2 * KV) * D), (Q * D, H))]
    if trained:
        w = [torch.nn.Parameter(x) for x in w]
    dec = decoder.CachedDecoder(*w, Q, KV, freq=torch.ones(D // 2, dtype=torch.float64))
    token = torch.tensor([3, 10, 3], dtype=torch.int32)
    out = torch.zeros(3, H) if with_out else None
    h = dec.step(token, None, None, None, None, None, out=out)
    assert not h.requires_grad and (out is None or h is out)
    embed, Wqkv, Wo = (x.detach() for x in w)
    x = embed[token.long()]
    want = x + 2 * (x @ Wqkv)[:, :Q * D] @ Wo
    assert torch.allclose(h, want, rtol=1e-5, atol=1e-5)
