"""A decoder that attends to its own past, for the decode loops of decode.py.

One layer, x = embed[token], h = x + attention(x) Wo, with rotary positions and the
keys and values of every hypothesis in the attention cache (include/kbest_cache.h).
It stands where the table of states stands in the synthetic loops: what it computes
is a decoder's step, its weights are the caller's.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as kbb


class CachedDecoder:
    """``embed``: V x H, ``Wqkv``: H x (q_heads + 2 kv_heads) * dim (queries, keys, values),
    ``Wo``: q_heads * dim x H, all float32 or all bfloat16 on the GPU.  ``freq`` and
    ``interleaved`` as cache_append takes them (by default the whole head is turned)."""

    def __init__(self, embed: torch.Tensor, Wqkv: torch.Tensor, Wo: torch.Tensor, q_heads: int, kv_heads: int, *,
                 freq: Optional[torch.Tensor] = None, interleaved: bool = False):
        H = embed.shape[1]
        if q_heads < 1 or kv_heads < 1 or q_heads % kv_heads or Wo.dim() != 2 or Wo.shape[0] % q_heads:
            raise ValueError(f"{q_heads} query and {kv_heads} key-value heads, Wo {tuple(Wo.shape)}")
        self.dim = Wo.shape[0] // q_heads
        if Wqkv.shape != (H, (q_heads + 2 * kv_heads) * self.dim) or Wo.shape[1] != H:
            raise ValueError("shape mismatch among embed, Wqkv, Wo")
        if not embed.dtype == Wqkv.dtype == Wo.dtype or not embed.device == Wqkv.device == Wo.device:
            raise ValueError("embed, Wqkv and Wo must have one type and device")
        self.embed, self.Wqkv, self.Wo = embed, Wqkv, Wo
        self.q_heads, self.kv_heads = q_heads, kv_heads
        self.freq = kbb.rotary_frequencies(self.dim, device=embed.device) if freq is None else freq
        self.interleaved = interleaved

    @property
    def H(self) -> int:
        return self.embed.shape[1]

    def cache(self, pages: int, page_size: int):
        """Keys and values of an empty cache: (k, v), each pages x kv_heads x page_size x dim."""
        shape = (pages, self.kv_heads, page_size, self.dim)
        return tuple(torch.empty(shape, dtype=self.embed.dtype, device=self.embed.device) for _ in range(2))

    @torch.no_grad()
    def step(self, token: torch.Tensor, pos: torch.Tensor, length: torch.Tensor, k_cache, v_cache, table, *,
             max_len: Optional[int] = None, n_dev: Optional[torch.Tensor] = None,
             position: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """States (rows x H) of one new token a row, its keys and values appended to the cache at
        slot ``length[r] - 1``.  Runs on the current stream.  ``weight`` is added to in place
        (what eviction goes by); rows from ``n_dev[0]`` on append nothing and their states
        mean nothing.  ``token`` holds row numbers of ``embed`` in all rows.  Nothing is recorded
        for a backward pass."""
        x = self.embed.index_select(0, token)
        qkv = (x @ self.Wqkv).view(x.shape[0], -1, self.dim)
        q, k, v = qkv.split([self.q_heads, self.kv_heads, self.kv_heads], 1)
        q = kbb.cache_append(k_cache, v_cache, table, length, k, v, q=q, pos=pos, freq=self.freq,
                             interleaved=self.interleaved, n_dev=n_dev, position=position, weight=weight)
        o = kbb.cache_attend(q, k_cache, v_cache, table, length, max_len=max_len, n_dev=n_dev, weight_in=weight,
                             weight_out=weight)
        return torch.addmm(x, o.view(x.shape[0], -1), self.Wo, out=out)
