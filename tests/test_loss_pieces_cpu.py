"""That the bounds of loss_pieces.py hold for operands in all their pieces, and tell when one is lost: a model of the
products on the CPU."""
import numpy as np
import pytest
import torch

import loss_pieces as lp

SIX = [(0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0)]


def pieces(x, n):
    out, r = [], torch.as_tensor(x, dtype=torch.float32)
    for _ in range(n):
        out.append(r.to(torch.bfloat16).float())
        r = r - out[-1]
    return out


def products(a, b, pairs):
    """Sums of the pieces' products, rounded to float32 at each step."""
    s = torch.zeros(())
    for i, j in pairs:
        if i < len(a) and j < len(b):
            s = s + a[i] * b[j]
    return s


def dlogits(N, V):
    g = torch.Generator().manual_seed(3)
    return torch.randn(N, generator=g)[:, None] * torch.softmax(2 * torch.randn((N, V), generator=g), 1)


@pytest.mark.parametrize("N,H,V", [(20, 96, 700), (100, 160, 777)])
def test_float32_in_three_pieces(N, H, V):
    h, W, b, row, word = lp.problem(1, torch.float32, N, H, V)
    G = dlogits(N, V)
    k = np.arange(H)
    assert torch.equal(sum(pieces(G, 3)), G)   # exact
    for want, x, y in zip(lp.exact(h.double().numpy(), W.double().numpy(), G.double().numpy(), row, word),
                          (G[:, word], h[row, k][:, None].expand(H, V)), (W[k, word][None].expand(N, H), G[row])):
        lim = lp.bound(want, False)
        whole = products(pieces(x, 3), pieces(y, 3), SIX).double().numpy()
        assert (np.abs(whole - want) <= lim).all()
        for lost in (dict(a=2), dict(b=2), dict(a=1), dict(b=1)):
            got = products(pieces(x, lost.get("a", 3)), pieces(y, lost.get("b", 3)), SIX).double().numpy()
            assert (np.abs(got - want) > lim).mean() > 0.3, lost
        for lost in SIX:
            got = products(pieces(x, 3), pieces(y, 3), [p for p in SIX if p != lost]).double().numpy()
            assert (np.abs(got - want) > lim).mean() > 0.3, f"without the product {lost}"


@pytest.mark.parametrize("N,H,V", [(20, 96, 700), (100, 160, 777)])
def test_bf16_with_dlogits_in_two_pieces(N, H, V):
    h, W, b, row, word = lp.problem(1, torch.bfloat16, N, H, V)
    G = dlogits(N, V)
    k = np.arange(H)
    for want, x, y in zip(lp.exact(h.double().numpy(), W.double().numpy(), G.double().numpy(), row, word),
                          (G[:, word], G[row]), (W[k, word][None].expand(N, H), h[row, k][:, None].expand(H, V))):
        lim = lp.bound(want, True)
        for n, right in ((2, True), (1, False)):
            got = products(pieces(x, n), [y.float()], [(i, 0) for i in range(n)]).to(torch.bfloat16).double().numpy()
            off = np.abs(got - want) > lim
            assert not off.any() if right else off.mean() > 0.1
