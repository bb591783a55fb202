"""The output layer's losses on the GPU against the fp64 oracle (oracle/loss_oracle.py, which derives the bounds of
loss, lse and dlogits).

The gradients, elementwise, from bounds e of the dlogits G and one rounding of them to the operands' type (r = 2^-8 for
bf16, 2^-24 for float32 in three pieces, and as much for the pieces' products that are left out, of either operand):

* dh: sum_v (e + r |G|) |W|, V + 80 additions of sum |G W| (float32: six times as many products), and the rounding of
  the result;
* dW: the same over the rows;
* db: sum_n e, N + 80 additions of sum |G|.
"""
import math

import numpy as np
import pytest
import torch

from oracle import loss_oracle as lo

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


def f64(t):
    return t.detach().cpu().double().numpy()


def make(seed, dtype, N, H, V, pad=0.2, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn((N, H), generator=g).to(dtype)
    W = (scale * torch.randn((H, V), generator=g) / math.sqrt(H)).to(dtype)
    b = 0.5 * torch.randn(V, generator=g)
    target = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    target[torch.rand(N, generator=g) < pad] = -1
    grad = torch.randn(N, generator=g)
    return g, h, W, b, target, grad


def teacher(g, N, V, K, pad=0.2):
    token = torch.randint(0, V, (N, K), generator=g, dtype=torch.int32)
    logit = 3 * torch.randn((N, K), generator=g)
    token[torch.rand((N, K), generator=g) < 0.1] = -1
    token[torch.rand(N, generator=g) < pad] = -1
    return token, logit


def check_rows(o, bd, loss, lse, what):
    for name, got, want, tol in (("lse", lse, o.lse, bd.lse), ("loss", loss, o.loss, bd.loss)):
        err = np.abs(f64(got) - want)
        bad = ~(err <= tol)
        assert not bad.any(), f"{what}: {name} of row {int(np.argmax(bad))} off by {err[bad][0]:.3g} > {tol[bad][0]:.3g}"


def check_grads(o, bd, h, W, grad, outs, dtype, what):
    dh, dW, db = outs
    G = o.dlogits(f64(grad))
    hd = np.where(o.used[:, None], f64(h), 0.0)
    Wd = f64(W)
    r = ROUND[dtype]
    six = 6 if dtype == F32 else 1
    left_out = 2.0 ** -23 if dtype == F32 else 0.0
    e = bd.dx + (r + left_out) * np.abs(G) + 2.0 ** -126
    N, V = G.shape
    for name, got, want, tol, out in (
            ("dh", dh, G @ Wd.T, e @ np.abs(Wd).T + six * (V + 80) * U * (np.abs(G) @ np.abs(Wd).T), r),
            ("dW", dW, hd.T @ G, np.abs(hd).T @ e + six * (N + 80) * U * (np.abs(hd).T @ np.abs(G)), r),
            ("db", db, G.sum(0), bd.dx.sum(0) + (N + 80) * U * np.abs(G).sum(0), U)):
        if got is None:
            continue
        assert got.dtype == (F32 if name == "db" else dtype)
        err = np.abs(f64(got) - want)
        lim = tol + out * (np.abs(want) + tol) + 2.0 ** -126
        bad = ~(err <= lim)
        assert not bad.any(), (f"{what}: {name}{tuple(np.argwhere(bad)[0])} off by {err[bad][0]:.3g} > "
                               f"{lim[bad][0]:.3g}, {int(bad.sum())} of {bad.size}")
    if dh is not None and (~o.used).any():
        assert (f64(dh)[~o.used] == 0).all(), f"{what}: rows left out have a gradient"


def dev(*ts):
    return tuple(t.cuda() for t in ts)


def check_ce(kb, dtype, N, H, V, seed=1, smoothing=0.0, pad=0.2, out=None, b=None, target=None, edit=None, grads=True):
    _, h, W, bias, tg, grad = make(seed, dtype, N, H, V, pad)
    b = bias if b is None else b
    tg = tg if target is None else target
    if edit:
        edit(h, W, b, tg, grad)
    what = f"cross entropy {dtype} {N} x {H} x {V} smoothing {smoothing}"
    hd, Wd, bd, td, gd = dev(h, W, b, tg, grad)
    loss, lse = kb.cross_entropy(hd, Wd, bd, td, smoothing=smoothing)
    o = lo.cross_entropy(f64(h), f64(W), f64(b), tg.numpy(), float(np.float32(smoothing)))
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad))
    check_rows(o, bnd, loss, lse, what)
    if grads:
        outs = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, smoothing=smoothing, out=out)
        check_grads(o, bnd, h, W, grad, outs, dtype, what)


def check_kd(kb, dtype, N, H, V, K, T=1.0, seed=1, pad=0.2, edit=None):
    g, h, W, b, _, grad = make(seed, dtype, N, H, V)
    token, logit = teacher(g, N, V, K, pad)
    if edit:
        edit(token, logit)
    what = f"distillation {dtype} {N} x {H} x {V} of {K} at {T}"
    hd, Wd, bd, td, ld, gd = dev(h, W, b, token, logit, grad)
    loss, lse = kb.distill(hd, Wd, bd, td, ld, temperature=T)
    o = lo.distill(f64(h), f64(W), f64(b), token.numpy(), f64(logit), T)
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad), K)
    check_rows(o, bnd, loss, lse, what)
    outs = kb.distill_grad(hd, Wd, bd, td, ld, lse, gd, temperature=T)
    check_grads(o, bnd, h, W, grad, outs, dtype, what)


# one tile and less, every row tile, several row and word tiles, ragged in every direction
SHAPES = [(2, 300, 515), (8, 1024, 640), (4, 17, 130), (3, 2500, 300), (9, 64, 384), (1, 32, 256), (1, 64, 1000), (5, 256, 2000), (33, 96, 1024), (64, 128, 512), (100, 160, 777), (128, 512, 1536),
          (200, 64, 300), (257, 320, 2304), (600, 128, 4000)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", SHAPES)
def test_cross_entropy(kb, dtype, N, H, V):
    check_ce(kb, dtype, N, H, V)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(2900, 32, 14000), (1300, 64, 20001), (100, 32, 70000), (20, 64, 140001), (60, 32, 140000)])
def test_tiles_in_turn(kb, dtype, N, H, V):
    # a workgroup takes several word tiles, the next one's stages under way while a tile's logits are worked on
    check_ce(kb, dtype, N, H, V, pad=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(7, 1, 1), (3, 5, 2), (9, 31, 255), (40, 33, 257), (70, 200, 1001), (300, 130, 8), (1, 7, 3000)])
def test_odd_sizes(kb, dtype, N, H, V):
    check_ce(kb, dtype, N, H, V)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(5, 64, 1000), (100, 128, 700), (300, 64, 1536)])
def test_smoothing(kb, dtype, N, H, V):
    check_ce(kb, dtype, N, H, V, smoothing=0.1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V,K,T", [(1, 64, 300, 1, 1.0), (5, 256, 2000, 5, 1.0), (40, 128, 512, 12, 2.0), (100, 100, 999, 33, 0.5),
                                       (300, 64, 1536, 64, 4.0), (60, 96, 400, 128, 1.0)])
def test_distill(kb, dtype, N, H, V, K, T):
    check_kd(kb, dtype, N, H, V, K, T)
