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


# chunks of 8 and of 16 threads, several of a workgroup; bf16 of a large W in tiles of 32 rows
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(1, 70, 16384), (2, 33, 16385), (4, 100, 8193), (3, 260, 9001), (8, 96, 40001), (7, 40, 70000), (1, 24, 140003), (8, 712, 32001), (3, 1200, 33000)])
def test_few_rows(kb, dtype, N, H, V):
    check_ce(kb, dtype, N, H, V, smoothing=0.1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(8, 48, 30000), (2, 65, 6001), (5, 800, 40000)])
def test_few_rows_of_a_teacher(kb, dtype, N, H, V):
    check_kd(kb, dtype, N, H, V, 128, 2.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(2900, 32, 14000), (1300, 64, 20001), (100, 32, 70000), (20, 64, 140001), (60, 32, 140000)])
def test_tiles_in_turn(kb, dtype, N, H, V):
    # a workgroup takes several word tiles, the next one's stages under way while a tile's logits are worked on
    check_ce(kb, dtype, N, H, V, pad=0.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(9, 100, 3001), (13, 64, 1000), (16, 256, 30000), (17, 64, 1000)])
def test_a_few_rows_more(kb, dtype, N, H, V):
    check_ce(kb, dtype, N, H, V, smoothing=0.1)
    check_kd(kb, dtype, N, H, V, 70, 2.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(180, 40, 60001), (192, 32, 60000), (570, 64, 30000), (570, 300, 30001)])
def test_tiles_of_192_rows(kb, dtype, N, H, V):
    """Row tiles that are no power of two: one, and several; states of one tile, and of more (dh and dW in one launch)."""
    check_ce(kb, dtype, N, H, V, smoothing=0.1)
    check_kd(kb, dtype, N, H, V, 20, 2.0)


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


def bits(t):
    return t.detach().cpu().view(torch.int16 if t.dtype == BF16 else torch.int32).numpy()


# few rows, small tiles, tiles of 64, 128 and 256 rows
PATHS = [(6, 96, 700), (40, 96, 2000), (60, 64, 60000), (120, 32, 52000), (700, 64, 26000)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_rows_left_out(kb, dtype, N, H, V):
    def edit(h, W, b, target, grad):
        target[0] = V                  # one past the vocabulary
        target[1] = -2 ** 31
        target[2] = 2 ** 31 - 1
        target[N - 1] = -100
        out = (target < 0) | (target >= V)
        h[out] = math.nan              # whatever they hold
        h[1] = math.inf
        grad[out] = math.nan
    check_ce(kb, dtype, N, H, V, edit=edit)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_no_row_counts(kb, dtype, N, H, V):
    _, h, W, b, _, grad = make(3, dtype, N, H, V)
    target = torch.full((N,), -1, dtype=torch.int32)
    hd, Wd, bd, td, gd = dev(h, W, b, target, grad)
    loss, lse = kb.cross_entropy(hd, Wd, bd, td, smoothing=0.2)
    for t in (loss, lse, *kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, smoothing=0.2)):
        assert (f64(t) == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_masked_words(kb, dtype, N, H, V):
    def edit(h, W, b, target, grad):
        b[::3] = -math.inf             # a shortlist: two words of three
        b[V - 1] = -math.inf
        ok = (target >= 0) & torch.isinf(b[target.clamp_min(0).long()])
        target[ok] = 1
    check_ce(kb, dtype, N, H, V, edit=edit)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_masked_words_of_a_teacher(kb, dtype, N, H, V):
    """Teacher and student leave the same words out, the teacher by the lowest finite logit: probabilities of 0 for a
    word whose logit is -inf.  And a target that is left out: a loss of +inf, with a gradient all the same."""
    g, h, W, b, target, grad = make(23, dtype, N, H, V)
    K = 6
    token = torch.arange(K, dtype=torch.int32).expand(N, K).contiguous()
    logit = torch.randn((N, K), generator=g)
    logit[:, 4:] = torch.finfo(F32).min
    b[4:6] = -math.inf
    hd, Wd, bd, td, ld, gd = dev(h, W, b, token, logit, grad)
    loss, lse = kb.distill(hd, Wd, bd, td, ld)
    o = lo.distill(f64(h), f64(W), f64(b), token.numpy(), f64(logit))
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad), K)
    check_rows(o, bnd, loss, lse, "masked by teacher and student")
    check_grads(o, bnd, h, W, grad, kb.distill_grad(hd, Wd, bd, td, ld, lse, gd), dtype, "masked by teacher and student")
    target[0] = 5
    loss, lse = kb.cross_entropy(hd, Wd, bd, target.cuda())
    o = lo.cross_entropy(f64(h), f64(W), f64(b), target.numpy())
    assert loss[0].item() == math.inf and np.isposinf(o.loss[0])
    outs = kb.cross_entropy_grad(hd, Wd, bd, target.cuda(), lse, gd)
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad))
    bnd.loss[0] = 1.0  # compared above
    o.loss[0] = 0.0
    loss[0] = 0.0
    check_rows(o, bnd, loss, lse, "a target that is left out")
    check_grads(o, bnd, h, W, grad, outs, dtype, "a target that is left out")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_large_logits(kb, dtype, N, H, V):
    # a word far above all others, and states of very different sizes
    def edit(h, W, b, target, grad):
        h *= torch.logspace(-3, 1.5, N)[:, None].to(dtype)
        b[V // 2] = 60.0
        b[V // 3] = -3e4
    check_ce(kb, dtype, N, H, V, edit=edit)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_teachers_entries(kb, dtype, N, H, V, T):
    def edit(token, logit):
        token[0] = 5                              # one word again and again
        token[1, ::2] = token[1, 0]
        logit[2] = -math.inf                      # a row without an entry
        logit[3, 1:] = -math.inf                  # one entry
        token[4] = torch.arange(40)               # neighbours
        token[5] = torch.tensor([-1, V, 2 ** 31 - 1, -2 ** 31] * 10)
        logit[:, 7] = -80.0                       # nearly nothing
    check_kd(kb, dtype, N, H, V, 40, T, edit=edit)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(8, 64, 2000), (30, 64, 2000), (64, 64, 60000), (128, 32, 52000), (600, 32, 30000)])
def test_all_entries_in_one_place(kb, dtype, N, H, V):
    # every row's 128 words in the same 128: thousands of entries in one wave's part of a tile, 1,024 in a block
    def edit(token, logit):
        token[:] = torch.stack([torch.randperm(128) for _ in range(N)]).to(torch.int32) + 256
    check_kd(kb, dtype, N, H, V, 128, 2.0, pad=0.0, edit=edit)


@pytest.mark.parametrize("N", [8193, 9000])
def test_many_rows(kb, N):
    check_ce(kb, BF16, N, 32, 300, pad=0.5)
    check_kd(kb, BF16, N, 32, 300, 3)


def test_most_rows(kb):
    """KB_LOSS_MAX_N rows, against float64 on the GPU: offsets of states, dlogits and parts past 2^31 bytes."""
    N, H, V = 4194304, 8, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn((N, H), generator=g, device="cuda").to(BF16)
    W = (torch.randn((H, V), generator=g, device="cuda") / 3).to(BF16)
    b = torch.randn(V, generator=g, device="cuda")
    target = torch.randint(-1, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.randn(N, generator=g, device="cuda")
    loss, lse = kb.cross_entropy(h, W, b, target)
    dh, dW, db = kb.cross_entropy_grad(h, W, b, target, lse, grad)
    used = target >= 0
    t = target.long().clamp_min(0)[:, None]
    x = h.double() @ W.double() + b.double()
    norm = torch.logsumexp(x, 1)
    size = h.double().abs() @ W.double().abs() + b.double().abs()
    # a logit: H + 3 roundings of what it sums; exponentials 2^-22, exponents 4 u of |x| twice, the sum V, the logarithm
    off = (H + 3) * U * size.amax(1) + 8 * U * x.abs().amax(1) + 2.0 ** -22 + (V + 4) * U * (1 + norm.abs())
    assert ((lse - norm).abs() <= off)[used].all() and (lse[~used] == 0).all()
    want = norm - x.gather(1, t).squeeze(1)
    assert ((loss - want).abs() <= 2 * off + 2 * U * want.abs())[used].all() and (loss[~used] == 0).all()
    p = torch.exp(x - norm[:, None])
    G = (p - torch.zeros_like(p).scatter_(1, t, 1.0)) * (grad.double() * used)[:, None]
    e = (grad.double().abs() * used)[:, None] * p * torch.expm1(3 * off + 2.0 ** -21)[:, None] + 4 * U * G.abs() + 2.0 ** -126
    r = 2.0 ** -8
    Wd = W.double()
    for name, got, want, tol, out in (
            ("dh", dh, G @ Wd.t(), (e + (r + (V + 80) * U) * G.abs()) @ Wd.t().abs(), r),
            # sums in 256 parts and 16 of them at a time: chains of N / 256 and 16 + 16 (db: 32 of a tile, then N / 2048 + 16)
            ("dW", dW, h.double().t() @ G, h.double().abs().t() @ (e + (r + (N / 256 + 80) * U) * G.abs()), r),
            ("db", db, G.sum(0), (e + (N / 2048 + 80) * U * G.abs()).sum(0), U)):
        lim = tol + out * (want.abs() + tol) + 2.0 ** -126
        err = (got.double() - want).abs()
        assert (err <= lim).all(), f"{name}: off by {err.max().item()}"
    assert (dh[~used] == 0).all()


@pytest.mark.parametrize("N,H,V", [(5, 32, 262144), (40, 32, 262144), (2000, 32, 262144)])
def test_largest_vocabulary(kb, N, H, V):
    _, h, W, b, target, grad = make(5, BF16, N, H, V, pad=0.0)
    target[:3] = torch.tensor([0, V - 1, V - 2])
    hd, Wd, bd, td, gd = dev(h, W, b, target, grad)
    loss, lse = kb.cross_entropy(hd, Wd, bd, td)
    dh, dW, db = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd)
    # the first rows and the last against the oracle; of the sums over rows, the columns of some words
    rows = np.r_[0:4, N - 1]
    o = lo.cross_entropy(f64(h)[rows], f64(W), f64(b), target.numpy()[rows])
    bnd = lo.bounds(o, f64(h)[rows], f64(W), f64(b), False, f64(grad)[rows])
    check_rows(o, bnd, loss[rows], lse[rows], f"{N} x {H} x {V}")
    check_grads(o, bnd, h[rows], W, grad[rows], (dh[rows], None, None), BF16, f"{N} x {H} x {V}")
    words = np.r_[0:8, 100000:100008, V - 8:V]
    x = f64(h) @ f64(W)[:, words] + f64(b)[words]
    p = np.exp(x - f64(lse)[:, None])
    G = f64(grad)[:, None] * (p - (target.numpy()[:, None] == words[None]))
    # a probability is off by what its exponent is: lse's float32 (3 u of it), the logit's (H + 3) u of sum |h W| + |b| and
    # their difference's rounding
    size = np.abs(f64(h)) @ np.abs(f64(W)[:, words]) + np.abs(f64(b)[words])
    off = 3 * U * np.abs(f64(lse))[:, None] + (H + 5) * U * size + 4 * U * (np.abs(x) + np.abs(f64(lse))[:, None]) + 2.0 ** -22
    dp = np.abs(f64(grad))[:, None] * p * (np.exp(off) - 1) + 4 * U * np.abs(f64(grad))[:, None] * (p + 1)
    e = dp + 2.0 ** -8 * np.abs(G) + 2.0 ** -126
    ah, aG = np.abs(f64(h)), np.abs(G)
    want, lim = f64(h).T @ G, ah.T @ e + (N + 80) * U * (ah.T @ aG)
    assert (np.abs(f64(dW)[:, words] - want) <= lim + 2.0 ** -8 * (np.abs(want) + lim)).all()
    want, lim = G.sum(0), dp.sum(0) + (N + 80) * U * aG.sum(0)
    assert (np.abs(f64(db)[words] - want) <= lim + U * np.abs(want)).all()


def test_logits_beyond_32_bits(kb):
    # 20,000 x 131,072: 2.6e9 logits; some rows against 64 bits
    N, H, V = 20000, 32, 131072
    g = torch.Generator(device="cuda").manual_seed(11)
    h = torch.randn((N, H), generator=g, device="cuda").to(BF16)
    W = (torch.randn((H, V), generator=g, device="cuda") / 6).to(BF16)
    b = torch.randn(V, generator=g, device="cuda")
    target = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.randn(N, generator=g, device="cuda")
    loss, lse = kb.cross_entropy(h, W, b, target)
    dh, dW, db = kb.cross_entropy_grad(h, W, b, target, lse, grad)
    rows = torch.tensor([0, 255, 256, 16383, 16384, 19998, 19999], device="cuda")
    hr, tr = h[rows].cpu(), target[rows].cpu().numpy()
    o = lo.cross_entropy(f64(hr), f64(W), f64(b), tr)
    bnd = lo.bounds(o, f64(hr), f64(W), f64(b), False, f64(grad[rows]))
    check_rows(o, bnd, loss[rows], lse[rows], "2.6e9 logits")
    check_grads(o, bnd, hr, W.cpu(), grad[rows].cpu(), (dh[rows], None, None), BF16, "2.6e9 logits")
    # every row's dlogits add up to zero, and so does db: to the rounding of N x V float32 terms
    assert abs(f64(db).sum()) <= 1e-3 * f64(grad.abs()).sum() / math.sqrt(N)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_wanted_gradients_only(kb, dtype, N, H, V):
    _, h, W, b, target, grad = make(7, dtype, N, H, V)
    hd, Wd, bd, td, gd = dev(h, W, b, target, grad)
    _, lse = kb.cross_entropy(hd, Wd, bd, td)
    whole = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd)
    for want in range(1, 7):
        out = tuple(torch.full_like(t, math.nan) if want >> i & 1 else None for i, t in enumerate((hd, Wd, bd)))
        got = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, out=out)
        for x, y, z in zip(got, out, whole):
            assert x is y
            if x is not None:
                err = (x.double() - z.double()).abs().max()  # dh and dW apart may be split otherwise than together
                assert err <= 2 * ROUND[x.dtype if x.dim() == 2 else F32] * z.double().abs().max()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", PATHS)
def test_same_bits_whatever_the_workspace_held(kb, dtype, N, H, V):
    g, h, W, b, _, grad = make(9, dtype, N, H, V)
    token, logit = teacher(g, N, V, 9)
    hd, Wd, bd, td, yd, gd = dev(h, W, b, token, logit, grad)
    code = kb.KB_BF16 if dtype == BF16 else kb.KB_F32
    seen = []
    for fill in (0, 0xFF, 0x7F):
        ws = torch.full((kb.loss_workspace_bytes(code, N, H, V, 9),), fill, dtype=torch.uint8, device="cuda")
        wg = torch.full((kb.loss_grad_workspace_bytes(code, N, H, V, 9),), fill, dtype=torch.uint8, device="cuda")
        out = tuple(torch.full((N,), math.nan, device="cuda") for _ in range(2))
        loss, lse = kb.distill(hd, Wd, bd, td, yd, temperature=1.5, ws=ws, out=out)
        assert loss is out[0] and lse is out[1]
        seen.append([bits(t) for t in (loss, lse, *kb.distill_grad(hd, Wd, bd, td, yd, lse, gd, temperature=1.5, ws=wg))])
    for other in seen[1:]:
        assert all((x == y).all() for x, y in zip(seen[0], other))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(6, 96, 704), (40, 96, 2000), (300, 64, 1536)])
def test_any_address(kb, dtype, N, H, V):
    # operands one value past an allocation's start, results as well
    _, h, W, b, target, grad = make(13, dtype, N, H, V)

    def shifted(t, by=1):
        buf = torch.zeros(t.numel() + by, dtype=t.dtype, device="cuda")
        buf[by:] = t.flatten().cuda()
        return buf[by:].view(t.shape)

    hd, Wd, bd, td, gd = (shifted(t) for t in (h, W, b, target, grad))
    loss, lse = kb.cross_entropy(hd, Wd, bd, td, out=tuple(shifted(torch.zeros(N)) for _ in range(2)))
    out = tuple(shifted(torch.zeros_like(t)) for t in (h, W, b))
    outs = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, out=out)
    o = lo.cross_entropy(f64(h), f64(W), f64(b), target.numpy())
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad))
    check_rows(o, bnd, loss, lse, "shifted")
    check_grads(o, bnd, h, W, grad, outs, dtype, "shifted")


def test_no_rows(kb):
    h, W, b = (torch.zeros(s, device="cuda") for s in ((0, 16), (16, 300), (300,)))
    target = torch.zeros(0, dtype=torch.int32, device="cuda")
    loss, lse = kb.cross_entropy(h, W, b, target)
    assert loss.shape == (0,) and lse.shape == (0,)
    out = (torch.empty_like(h), torch.full_like(W, math.nan), torch.full_like(b, math.nan))
    kb.cross_entropy_grad(h, W, b, target, lse, loss, out=out)
    assert (f64(out[1]) == 0).all() and (f64(out[2]) == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", [(6, 96, 700), (70, 64, 3000), (300, 64, 3000)])
def test_captured_and_replayed(kb, dtype, N, H, V):
    """A training step in a graph, replayed on new inputs between eager calls of the same size."""
    g, h, W, b, target, grad = make(17, dtype, N, H, V)
    token, logit = teacher(g, N, V, 6)
    hd, Wd, bd, td, kd, yd, gd = dev(h, W, b, target, token, logit, grad)

    def step(ws=None):
        loss, lse = kb.cross_entropy(hd, Wd, bd, td, smoothing=0.1)
        l2, s2 = kb.distill(hd, Wd, bd, kd, yd, temperature=2.0)
        return (loss, lse, l2, s2, *kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, smoothing=0.1),
                *kb.distill_grad(hd, Wd, bd, kd, yd, s2, gd, temperature=2.0))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for turn in range(4):
        for t, like in ((hd, h), (bd, b), (gd, grad), (yd, logit)):
            t.copy_(torch.randn(like.shape, generator=g).to(like.dtype))
        td.copy_(torch.randint(-1, V, (N,), generator=g, dtype=torch.int32))  # other rows left out
        kd.copy_(torch.randint(-1, V, kd.shape, generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(captured, eager)):
            assert (bits(x) == bits(y)).all(), f"turn {turn}: result {i}"


def test_two_streams_at_once(kb):
    jobs = []
    for seed, (dtype, N, H, V) in enumerate([(BF16, 300, 128, 9000), (F32, 200, 64, 5000), (BF16, 7, 64, 3000)]):
        _, h, W, b, target, grad = make(seed, dtype, N, H, V)
        jobs.append(dev(h, W, b, target, grad))

    def step(j, stream):
        h, W, b, target, grad = j
        loss, lse = kb.cross_entropy(h, W, b, target, stream=stream)
        return (loss, lse, *kb.cross_entropy_grad(h, W, b, target, lse, grad, stream=stream))

    alone = [[bits(t) for t in step(j, None)] for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[] for _ in jobs]
    for _ in range(5):
        for i, (j, s) in enumerate(zip(jobs, streams)):
            got[i].append(step(j, s))
    torch.cuda.synchronize()
    for want, runs in zip(alone, got):
        for run in runs:
            assert all((x == bits(t)).all() for x, t in zip(want, run))


@pytest.mark.parametrize("N,H,V", [(4, 24, 90), (20, 24, 400), (140, 32, 600)])
def test_gradient_is_that_of_the_loss(kb, N, H, V):
    """Against central differences of the float32 loss along random directions.  A step of e leaves e^2 / 6 of the third
    derivative, a third central moment of the logits' change over a row: at most its spread cubed; and the rounding of
    the two losses, 2^-20 of their size and of the log-sum-exp's, at most 8 here, over 2 e."""
    g, h, W, b, target, grad = make(21, F32, N, H, V)
    token, logit = teacher(g, N, V, 5)
    eps = 2.0 ** -6
    hd, Wd, bd, td, kd, yd, gd = dev(h, W, b, target, token, logit, grad)
    losses = {
        "cross entropy": (lambda h_, W_, b_: kb.cross_entropy(h_, W_, b_, td, smoothing=0.1)[0],
                          lambda: kb.cross_entropy_grad(hd, Wd, bd, td, kb.cross_entropy(hd, Wd, bd, td, smoothing=0.1)[1],
                                                        gd, smoothing=0.1)),
        "distillation": (lambda h_, W_, b_: kb.distill(h_, W_, b_, kd, yd, temperature=2.0)[0],
                         lambda: kb.distill_grad(hd, Wd, bd, kd, yd, kb.distill(hd, Wd, bd, kd, yd, temperature=2.0)[1], gd,
                                                 temperature=2.0))}
    for name, (loss, gradient) in losses.items():
        grads = gradient()
        for i, t in enumerate((hd, Wd, bd)):
            v = torch.randn(t.shape, generator=g).cuda()
            v /= v.norm() / math.sqrt(t.shape[0])
            args = [hd, Wd, bd]
            args[i] = t + eps * v
            up = loss(*args)
            args[i] = t - eps * v
            down = loss(*args)
            size = ((up.abs() + down.abs() + 16) * gd.abs()).double().sum().item()
            diff = ((up.double() - down.double()) * gd.double()).sum().item() / (2 * eps)
            want = (grads[i].double() * v.double()).sum().item()
            dx = {0: lambda: v @ Wd, 1: lambda: hd @ v, 2: lambda: v[None].expand(N, V)}[i]().double()
            spread = (dx.max(1).values - dx.min(1).values) ** 3
            lim = eps ** 2 / 6 * (gd.abs().double() * spread).sum().item() + 2.0 ** -20 * size / (2 * eps)
            assert abs(diff - want) <= lim, f"{name}, argument {i}: {diff} and {want}, {lim}"


def test_student_learns_from_a_teacher_through_the_step(kb):
    """As they are used together: a teacher's step gives every row's best words, the student is distilled from them, and
    the update goes down the gradient."""
    N, H, V, k = 96, 64, 3000, 8
    g = torch.Generator().manual_seed(31)
    ht, Wt = torch.randn((N, 128), generator=g).to(BF16).cuda(), (torch.randn((128, V), generator=g) / 11).to(BF16).cuda()
    bt = torch.zeros(V, device="cuda")
    _, h, W, b, _, _ = make(32, BF16, N, H, V)
    hd, Wd, bd = dev(h, W, b)
    off = torch.arange(N + 1, dtype=torch.int32, device="cuda")
    token, parent, score = kb.kbest_step(ht, Wt, bt, torch.zeros(N, device="cuda"), off, k)
    assert (parent == off[:N, None]).all()
    loss, lse = kb.distill(hd, Wd, bd, token, score, temperature=2.0)
    grad = torch.full((N,), 1.0 / N, device="cuda")
    dh, dW, db = kb.distill_grad(hd, Wd, bd, token, score, lse, grad, temperature=2.0)
    o = lo.distill(f64(h), f64(W), f64(b), token.cpu().numpy(), f64(score), 2.0)
    bnd = lo.bounds(o, f64(h), f64(W), f64(b), False, f64(grad), k)
    check_rows(o, bnd, loss, lse, "student")
    check_grads(o, bnd, h, W, grad.cpu(), (dh, dW, db), BF16, "student")
    # the greedy step's logit less the cross entropy's lse is the best word's log-probability
    best, x = kb.argmax_step(hd, Wd, bd)
    ce, lse1 = kb.cross_entropy(hd, Wd, bd, best)
    assert (ce - (lse1 - x)).abs().max() <= 1e-4
