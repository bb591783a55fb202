"""Values at which the output layer's losses can go wrong, against the fp64 oracle with its bounds (the bounds of the
gradients are those of test_gpu_loss.py)."""
import math

import numpy as np
import pytest
import torch

import loss_pieces as lp
import test_gpu_loss as base
from oracle import loss_oracle as lo
from test_gpu_loss import kb  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
f64 = base.f64


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", base.PATHS)
@pytest.mark.parametrize("smoothing", [2.0 ** -149, 1e-41, 1e-30])
def test_smoothing_of_next_to_nothing(kb, dtype, N, H, V, smoothing):  # noqa: F811
    """smoothing / V is 0 in float32, or the least values there are.  Without words that are left out it makes no
    difference; where the smoothed labels name one, the loss is +inf and the gradient p - q as ever."""
    _, h, W, b, target, grad = base.make(25, dtype, N, H, V)
    target[0], target[1] = 1, -1
    for masked in (False, True):
        if masked:
            b[2] = b[V - 1] = -math.inf
            target[(target == 2) | (target == V - 1)] = 1
        hd, Wd, bd, td, gd = base.dev(h, W, b, target, grad)
        loss, lse = kb.cross_entropy(hd, Wd, bd, td, smoothing=smoothing)
        outs = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, smoothing=smoothing)
        o = lo.cross_entropy(f64(h), f64(W), f64(b), target.numpy(), float(np.float32(smoothing)))
        what = f"smoothing {smoothing}, {'with' if masked else 'no'} words left out"
        if masked:
            assert np.isposinf(o.loss[o.used]).all()
            assert np.isposinf(f64(loss)[o.used]).all() and (f64(loss)[~o.used] == 0).all(), what
            o.loss[:] = 0.0  # compared above
            loss = torch.zeros(N)
        bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad))
        base.check_rows(o, bnd, loss, lse, what)
        base.check_grads(o, bnd, h, W, grad, outs, dtype, what)


def rows_alone(kb, h, W, b, target, lse, grad):  # noqa: F811
    """The dlogits in float32, as the kernels have them before they are cut into pieces: db of every row by itself."""
    out = []
    for n in range(h.shape[0]):
        alone = torch.full_like(target, -1)
        alone[n] = target[n]
        out.append(kb.cross_entropy_grad(h, W, b, alone, lse, grad, out=(None, None, torch.empty_like(b)))[2])
    return f64(torch.stack(out))


# every row tile; bf16 above 128 rows rounds its dlogits once
PIECES = [(F32, N, H, V) for N, H, V in ((20, 96, 700), (60, 100, 60001), (100, 160, 777), (300, 320, 1536), (700, 300, 6000))]
PIECES += [(BF16, N, H, V) for N, H, V in ((6, 1200, 48000), (20, 96, 700), (60, 100, 6001), (64, 512, 60000), (100, 160, 777),
                                          (128, 512, 1536))]


@pytest.mark.parametrize("dtype,N,H,V", PIECES)
def test_all_pieces_of_the_operands(kb, dtype, N, H, V):  # noqa: F811
    """Gradients that are single products: to 2^-20 in float32, rounded once in bf16 (loss_pieces.py)."""
    h, W, b, row, word = lp.problem(7, dtype, N, H, V)
    g = torch.Generator().manual_seed(8)
    target, grad = torch.randint(0, V, (N,), generator=g, dtype=torch.int32), torch.randn(N, generator=g)
    hd, Wd, bd, td, gd = base.dev(h, W, b, target, grad)
    _, lse = kb.cross_entropy(hd, Wd, bd, td)
    dh, dW, _ = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd)
    G = rows_alone(kb, hd, Wd, bd, td, lse, gd)
    o = lo.cross_entropy(f64(h), f64(W), f64(b), target.numpy())
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad))
    assert (np.abs(G - o.dlogits(f64(grad))) <= bnd.dx + 2.0 ** -24 * np.abs(G)).all()
    for name, got, want in zip(("dh", "dW"), (dh, dW), lp.exact(f64(h), f64(W), G, row, word)):
        bad = ~(np.abs(f64(got) - want) <= lp.bound(want, dtype == BF16))
        assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.size} are off, the first at {tuple(np.argwhere(bad)[0])}"


@pytest.mark.parametrize("N", [20, 60, 100, 300, 700])
def test_all_pieces_of_a_logit(kb, N):  # noqa: F811
    """A vocabulary of one word and one state a row: lse is the logit x, a single product, to 2^-20, and the logarithm of
    one exponential: x log2(e) is rounded before x log2(e) less that is taken, so its exponent is not 0 but up to 2^-24
    |x| log2(e); it is off by 2^-22 itself; and the sum of both rounds, 2^-24 |x|."""
    H = 64
    g = torch.Generator().manual_seed(9)
    h, W = torch.zeros(N, H), torch.randn((H, 1), generator=g)
    k = torch.randint(0, H, (N,), generator=g)
    h[torch.arange(N), k] = torch.randn(N, generator=g)
    hd, Wd, bd, td = base.dev(h, W, torch.zeros(1), torch.zeros(N, dtype=torch.int32))
    loss, lse = kb.cross_entropy(hd, Wd, bd, td)
    want = (f64(h) @ f64(W))[:, 0]
    one = 2.0 ** -23 * np.abs(want) + 2.0 ** -22
    assert (np.abs(f64(lse) - want) <= 2.0 ** -20 * np.abs(want) + one).all()
    assert (np.abs(f64(loss)) <= one + 2.0 ** -23 * np.abs(want)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", base.PATHS)
@pytest.mark.parametrize("T", [1e-6, 1e-2, 1e2, 1e6])
@pytest.mark.parametrize("scaled", [False, True])
def test_temperatures(kb, dtype, N, H, V, T, scaled):  # noqa: F811
    """From the least to the greatest, with logits of the usual size and of the temperature's.  Usual logits over 1e-6 are
    millions: their exponents are off by whole numbers in float32, so that a probability has no bound; it is finite.

    The oracle's bounds take the teacher's exponents y = logit / T as small.  Here they are not: 1 / T and the product are
    a rounding each, 2 u |y|, of the entry's and the greatest one's, and their difference one more, u (|y| + |top|): an
    exponential is off by 3 u (|y| + |top|) <= 6 u max |y| of itself, and so is their sum, a probability by both."""
    T = float(np.float32(T))
    g, h, W, b, _, grad = base.make(27, dtype, N, H, V)
    token, logit = base.teacher(g, N, V, 9)
    if scaled:
        s = 2.0 ** round(math.log2(T))
        W, b, logit = W * s, b * s, logit * s
    hd, Wd, bd, td, ld, gd = base.dev(h, W, b, token, logit, grad)
    loss, lse = kb.distill(hd, Wd, bd, td, ld, temperature=T)
    outs = kb.distill_grad(hd, Wd, bd, td, ld, lse, gd, temperature=T)
    o = lo.distill(f64(h), f64(W), f64(b), token.numpy(), f64(logit), T)
    with np.errstate(over="ignore", invalid="ignore"):
        bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad), 9)
        off = o.q * np.expm1(12 * base.U * np.abs(f64(logit)).max(1) / T)[:, None]
        x = np.where(np.isneginf(o.x), 0.0, np.abs(o.x))
        bnd.dx += np.abs(f64(grad))[:, None] * T * np.where(o.used[:, None], off, 0.0)
        bnd.loss += np.where(o.used, T * T * (off * (np.abs(np.log(np.where(o.q > 0, o.q, 1.0))) + 2 + x
                                                     + np.abs(o.lse)[:, None])).sum(1), 0.0)
    what = f"temperature {T}, scaled: {scaled}"
    base.check_rows(o, bnd, loss, lse, what)
    if scaled or T > 1e-3:
        base.check_grads(o, bnd, h, W, grad, outs, dtype, what)
    else:
        assert all(torch.isfinite(t).all() for t in outs) and (f64(outs[0])[~o.used] == 0).all(), what


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [3, 20, 140])
def test_most_states(kb, dtype, N):  # noqa: F811
    """65,536 states: a piece of W is 256 words, and there are 256 tiles of them."""
    base.check_ce(kb, dtype, N, 65536, 300, smoothing=0.1)
    base.check_kd(kb, dtype, N, 65536, 264, 5, 2.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", base.PATHS)
@pytest.mark.parametrize("mask", [-math.inf, torch.finfo(F32).min])
def test_most_words_left_out_in_one_run(kb, dtype, N, H, V, mask):  # noqa: F811
    """Whole tiles and whole shares of the vocabulary without a word, by -inf or by the lowest value there is: the same."""
    _, h, W, b, target, grad = base.make(29, dtype, N, H, V)
    lo_, hi = V // 10, V - V // 20
    target[(target >= lo_) & (target < hi)] = hi
    out = torch.arange(V)
    out = (out >= lo_) & (out < hi)
    hd, Wd, td, gd = base.dev(h, W, target, grad)
    bd = b.masked_fill(out, mask).cuda()
    loss, lse = kb.cross_entropy(hd, Wd, bd, td)
    outs = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd)
    b = f64(b.masked_fill(out, -math.inf))
    o = lo.cross_entropy(f64(h), f64(W), b, target.numpy())
    bnd = lo.bounds(o, f64(h), f64(W), b, dtype == F32, f64(grad))
    base.check_rows(o, bnd, loss, lse, f"left out by {mask}")
    base.check_grads(o, bnd, h, W, grad, outs, dtype, f"left out by {mask}")
    assert (f64(outs[1])[:, out.numpy()] == 0).all() and (f64(outs[2])[out.numpy()] == 0).all()
