"""The output layer's losses at the sizes that their header still allows, against float64 on the GPU, a stretch of rows at
a time."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


def test_most_rows_of_many_states(kb):
    """4,194,304 rows of 1,024 states: dh's parts are joined by 2^22 workgroups of 1,024 threads, 2^32 threads in all.

    Bounds as for the smaller sizes: a logit is off by (H + 3) u of what it sums, a probability by what its exponent is
    (lse's and the logit's error, 2^-21 for the exponential), a dlogit by one rounding to bf16, and sums by their
    additions: dh's V + 80; db's and dW's N at most, in any order."""
    N, H, V, step = 4194304, 1024, 8, 1 << 17
    g = torch.Generator(device="cuda").manual_seed(41)
    h = torch.empty((N, H), dtype=BF16, device="cuda")
    for r0 in range(0, N, step):
        h[r0:r0 + step] = torch.randn((step, H), generator=g, device="cuda").to(BF16)
    W = (torch.randn((H, V), generator=g, device="cuda") / 32).to(BF16)
    b = torch.randn(V, generator=g, device="cuda")
    target = torch.randint(-1, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.randn(N, generator=g, device="cuda")
    loss, lse = kb.cross_entropy(h, W, b, target)
    out = (torch.full_like(h, float("nan")), torch.full_like(W, float("nan")), torch.full_like(b, float("nan")))
    dh, dW, db = kb.cross_entropy_grad(h, W, b, target, lse, grad, out=out)
    r = 2.0 ** -8
    Wd, bd = W.double(), b.double()
    sums = {name: [torch.zeros(shape, dtype=torch.float64, device="cuda") for _ in range(2)]
            for name, shape in (("dW", (H, V)), ("db", (V,)))}
    for r0 in range(0, N, step):
        rows = slice(r0, r0 + step)
        hd, used = h[rows].double(), target[rows] >= 0
        t = target[rows].long().clamp_min(0)[:, None]
        x = hd @ Wd + bd
        norm = torch.logsumexp(x, 1)
        size = (hd.abs() @ Wd.abs() + bd.abs()).amax(1)
        off = (H + 3) * U * size + 8 * U * x.abs().amax(1) + 2.0 ** -22 + (V + 4) * U * (1 + norm.abs())
        assert ((lse[rows] - norm).abs() <= off)[used].all() and (lse[rows][~used] == 0).all(), f"lse from row {r0} on"
        want = norm - x.gather(1, t).squeeze(1)
        assert ((loss[rows] - want).abs() <= 2 * off + 2 * U * want.abs())[used].all(), f"loss from row {r0} on"
        p = torch.exp(x - norm[:, None])
        ga = (grad[rows].double() * used)[:, None]
        G = (p - torch.zeros_like(p).scatter_(1, t, 1.0)) * ga
        e = ga.abs() * p * torch.expm1(3 * off + 2.0 ** -21)[:, None] + 4 * U * G.abs() + 2.0 ** -126
        want, tol = G @ Wd.t(), (e + (r + (V + 80) * U) * G.abs()) @ Wd.t().abs()
        lim = tol + r * (want.abs() + tol) + 2.0 ** -126
        assert ((dh[rows].double() - want).abs() <= lim).all(), f"dh from row {r0} on"
        assert (dh[rows][~used] == 0).all(), f"rows left out from row {r0} on"
        for name, value, size in (("dW", hd.t() @ G, hd.abs().t() @ (e + (r + N * U) * G.abs())),
                                  ("db", G.sum(0), (e + N * U * G.abs()).sum(0))):
            sums[name][0] += value
            sums[name][1] += size
    for name, got, out in (("dW", dW, r), ("db", db, U)):
        want, tol = sums[name]
        assert ((got.double() - want).abs() <= tol + out * (want.abs() + tol)).all(), name
