"""Problems whose gradients are single products, so that a lost piece of an operand shows: every state is held by one row
and leads to one word.

With h[n, k] = 0 but for n = row(k) and W[k, v] = 0 but for v = word(k), and dlogits G,

    dW[k, v] = h[row(k), k] G[row(k), v]        dh[n, k] = G[n, word(k)] W[k, word(k)],

whatever is summed besides is zero.  An operand in float32 is x = x0 + x1 + x2 in bf16 (8 + 8 + 8 significand bits, exact);
|x1| <= 2^-8 |x|, |x2| <= 2^-17 |x|.

float32 results: the six products (0,0) (0,1) (1,0) (1,1) (0,2) (2,0), each exact in float32; left out are (1,2) (2,1) (2,2),
2^-25 + 2^-25 + 2^-34 of the whole.  They are added in six steps, the parts of a split sum (zeros) do not round: six
roundings of at most a unit, 2^-23 each, of what is never above 1 + 2^-6 of the whole.  Together below 14 x 2^-24, and so below
2^-20; a third piece is up to 2^-17.

bf16 results with G in two pieces: G is off by 2^-17, the sums by two units, 2^-22; 2^-16 covers it and the binade's edge.
Rounding the result takes half a unit of its binade, 2^(e - 8).  Of G in one piece, 2^-8, there would be two such halves.
"""
import numpy as np
import torch


def problem(seed, dtype, N, H, V):
    """(h, W, b, row, word) on the CPU."""
    g = torch.Generator().manual_seed(seed)
    k = torch.arange(H)
    row, word = k % N, torch.randint(0, V, (H,), generator=g)
    h, W = torch.zeros(N, H), torch.zeros(H, V)
    h[row, k] = torch.randn(H, generator=g)
    W[k, word] = torch.randn(H, generator=g)
    return h.to(dtype), W.to(dtype), 0.5 * torch.randn(V, generator=g), row.numpy(), word.numpy()


def exact(h, W, G, row, word):
    """(dh, dW) of dlogits G (N x V), in 64 bits."""
    k = np.arange(h.shape[1])
    return G[:, word] * W[k, word][None], h[row, k][:, None] * G[row]


def bound(want, bf16):
    size = np.abs(want)
    if not bf16:
        return 2.0 ** -20 * size + 2.0 ** -126
    return 2.0 ** (np.floor(np.log2(np.maximum(size, 2.0 ** -126))) - 8) + 2.0 ** -16 * size
