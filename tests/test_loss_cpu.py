"""The output layer's losses without a GPU: the oracle against autograd in 64 bits and closed forms, and what the C entry
points and the binding refuse (nothing is launched on a refusal)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import loss_oracle as lo
from paper_1805_09863_amd import binding

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BASE = 1 << 20     # an address that nothing reads: every call here is refused before


@pytest.fixture(scope="module")
def L():
    if not binding.os.path.exists(binding.LIB_PATH):
        pytest.skip("libkbest.so is not built")
    return binding.lib()


# ---------------------------------------------------------------- the oracle

def layer(seed, N, H, V):
    g = torch.Generator().manual_seed(seed)
    h, W, b = (torch.randn(s, generator=g, dtype=torch.float64, requires_grad=True) for s in ((N, H), (H, V), (V,)))
    return g, h, W, b, torch.randn(N, generator=g, dtype=torch.float64)


def numpy(*ts):
    return tuple(t.detach().numpy() for t in ts)


def same_gradients(o, loss, h, W, b, grad):
    (loss * grad).sum().backward()
    G = o.dlogits(grad.numpy())
    hd, Wd = numpy(h, W)
    assert np.allclose(o.loss, loss.detach().numpy(), atol=1e-12)
    assert np.allclose(G @ Wd.T, h.grad.numpy(), atol=1e-12)
    assert np.allclose(hd.T @ G, W.grad.numpy(), atol=1e-12)
    assert np.allclose(G.sum(0), b.grad.numpy(), atol=1e-12)


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 0.7])
def test_cross_entropy_oracle(smoothing):
    g, h, W, b, grad = layer(1, 9, 5, 13)
    target = torch.tensor([0, 12, -1, 5, 5, 13, 3, -100, 1])
    used = (target >= 0) & (target < 13)
    logp = torch.log_softmax(h @ W + b, dim=1)
    picked = logp.gather(1, torch.where(used, target, 0)[:, None])[:, 0]
    loss = torch.where(used, -(1 - smoothing) * picked - smoothing * logp.mean(1), 0.0)
    same_gradients(lo.cross_entropy(*numpy(h, W, b), target.numpy(), smoothing), loss, h, W, b, grad)


@pytest.mark.parametrize("T", [1.0, 0.5, 3.0])
def test_distill_oracle(T):
    g, h, W, b, grad = layer(2, 6, 4, 11)
    token = torch.tensor([[1, 2, 3], [4, 4, 0], [-1, -1, -1], [10, -1, 7], [11, 5, 6], [8, 9, 8]])
    logit = torch.randn(6, 3, generator=g, dtype=torch.float64)
    logit[3, 0] = -math.inf
    q = torch.zeros(6, 11, dtype=torch.float64)
    for n in range(6):
        kept = [(int(t), float(y)) for t, y in zip(token[n], logit[n]) if 0 <= t < 11 and y > -math.inf]
        for t, y in kept:
            q[n, t] += math.exp(y / T) / sum(math.exp(z / T) for _, z in kept)
    used = q.sum(1) > 0
    logp = torch.log_softmax((h @ W + b) / T, dim=1)
    loss = torch.where(used, T * T * (torch.xlogy(q, q) - q * logp).sum(1), 0.0)
    o = lo.distill(*numpy(h, W, b), token.numpy(), logit.numpy(), T)
    assert o.used.tolist() == [True, True, False, True, True, True]
    same_gradients(o, loss, h, W, b, grad)


def test_closed_forms():
    # equal logits: ln V whatever the target; ln 1 .. ln 4: probabilities 1/10 .. 4/10
    o = lo.cross_entropy(np.zeros((1, 2)), np.zeros((2, 8)), np.zeros(8), np.array([3]))
    assert np.isclose(o.loss[0], math.log(8))
    b = np.log(np.arange(1.0, 5.0))
    o = lo.cross_entropy(np.zeros((1, 2)), np.zeros((2, 4)), b, np.array([2]))
    assert np.allclose([o.loss[0], o.lse[0]], [-math.log(0.3), math.log(10)])
    assert np.allclose(o.dlogits(np.ones(1)), [[0.1, 0.2, -0.7, 0.4]])
    # a teacher that agrees costs nothing
    o = lo.distill(np.zeros((1, 2)), np.zeros((2, 4)), b, np.array([[3, 1, 0, 2]]), b[[3, 1, 0, 2]][None] + 5.0)
    assert np.isclose(o.loss[0], 0.0) and np.allclose(o.dlogits(np.ones(1)), 0.0)


# ---------------------------------------------------------------- what is refused

CE = dict(dtype=1, N=10, H=64, V=512, h=BASE, W=BASE, b=BASE, target=BASE, smoothing=0.1, loss=BASE, lse=BASE, ws=BASE,
          ws_bytes=1 << 40, stream=None)
CG = dict(dtype=1, N=10, H=64, V=512, h=BASE, W=BASE, b=BASE, target=BASE, smoothing=0.1, lse=BASE, grad=BASE, dh=BASE,
          dW=BASE, db=BASE, ws=BASE, ws_bytes=1 << 40, stream=None)
KD = dict(dtype=1, N=10, H=64, V=512, K=8, h=BASE, W=BASE, b=BASE, token=BASE, logit=BASE, temperature=2.0, loss=BASE,
          lse=BASE, ws=BASE, ws_bytes=1 << 40, stream=None)
KG = dict(dtype=1, N=10, H=64, V=512, K=8, h=BASE, W=BASE, b=BASE, token=BASE, logit=BASE, temperature=2.0, lse=BASE,
          grad=BASE, dh=BASE, dW=BASE, db=BASE, ws=BASE, ws_bytes=1 << 40, stream=None)
CALLS = {"kb_cross_entropy": CE, "kb_cross_entropy_grad": CG, "kb_distill": KD, "kb_distill_grad": KG}

SIZES = [(dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(N=-1), INVALID), (dict(H=0), INVALID), (dict(V=0), INVALID),
         (dict(V=262145), UNSUPPORTED), (dict(H=65537), UNSUPPORTED), (dict(N=4194305), UNSUPPORTED)]
POINTERS = [(dict(h=None), INVALID), (dict(W=None), INVALID), (dict(b=None), INVALID), (dict(h=BASE + 1), INVALID),
            (dict(W=BASE + 1), INVALID), (dict(b=BASE + 2), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=BASE + 128), WORKSPACE),
            (dict(ws_bytes=0), WORKSPACE), (dict(dtype=0, h=BASE + 2), INVALID)]
SMOOTH = [(dict(smoothing=x), INVALID) for x in (-0.1, 1.0, math.nan, math.inf)]
HEAT = [(dict(temperature=x), INVALID) for x in (0.0, -1.0, math.nan, math.inf, 1e-7, 1e7)]
TEACH = [(dict(K=0), INVALID), (dict(K=129), INVALID), (dict(token=None), INVALID), (dict(logit=None), INVALID),
         (dict(token=BASE + 2), INVALID), (dict(logit=BASE + 2), INVALID), (dict(K=128, N=4194304 * 2 + 1), UNSUPPORTED),
         (dict(K=128, N=4194304, H=1), OK)]
TARGET = [(dict(target=None), INVALID), (dict(target=BASE + 2), INVALID)]
FORWARD = [(dict(loss=None), INVALID), (dict(lse=None), INVALID), (dict(loss=BASE + 2), INVALID), (dict(lse=BASE + 1), INVALID)]
BACKWARD = [(dict(lse=None), INVALID), (dict(grad=None), INVALID), (dict(lse=BASE + 2), INVALID), (dict(grad=BASE + 2), INVALID),
            (dict(dh=None, dW=None, db=None), INVALID), (dict(dh=BASE + 1), INVALID), (dict(dW=BASE + 1), INVALID),
            (dict(db=BASE + 2), INVALID)]
REFUSED = ([(n, c, s) for n in CALLS for c, s in SIZES + POINTERS]
           + [(n, c, s) for n in ("kb_cross_entropy", "kb_cross_entropy_grad") for c, s in SMOOTH + TARGET]
           + [(n, c, s) for n in ("kb_distill", "kb_distill_grad") for c, s in HEAT + TEACH if s != OK]
           + [(n, c, s) for n in ("kb_cross_entropy", "kb_distill") for c, s in FORWARD]
           + [(n, c, s) for n in ("kb_cross_entropy_grad", "kb_distill_grad") for c, s in BACKWARD])


@pytest.mark.parametrize("name,change,status", REFUSED, ids=lambda x: str(x).replace(" ", "") if not isinstance(x, int) else "")
@pytest.mark.parametrize("N", [5, 10, 100, 3000])   # every kind of plan
def test_refusals(L, name, change, status, N):
    args = dict(CALLS[name])
    args["N"] = N
    args.update(change)
    got = getattr(L, name)(*args.values())
    assert got == status, L.kb_last_error().decode()
    assert L.kb_last_error() != b""


def test_no_rows_is_no_work(L):
    assert L.kb_cross_entropy(1, 0, 64, 512, *[None] * 4, 0.1, None, None, None, 0, None) == OK
    assert L.kb_distill(1, 0, 64, 512, 4, *[None] * 5, 1.0, None, None, None, 0, None) == OK
    # also then something has to be asked for
    assert L.kb_cross_entropy_grad(1, 0, 64, 512, *[None] * 4, 0.1, *[None] * 6, 0, None) == INVALID


def test_workspace_sizes(L):
    for f in (L.kb_loss_workspace_bytes, L.kb_loss_grad_workspace_bytes):
        assert f(1, 0, 64, 512, 1) == 0
        for bad in ((3, 1, 1, 1, 1), (1, -1, 64, 512, 1), (1, 1, 0, 512, 1), (1, 1, 64, 262145, 1), (1, 1, 64, 512, 0),
                    (1, 1, 64, 512, 129), (1, 4194304, 64, 512, 128 * 3)):
            assert f(*bad) == 0
    # the logits are never kept, whole or in part: a gradient's workspace stays below a fourth of theirs in float32
    N, V = 8192, 90000
    assert L.kb_loss_grad_workspace_bytes(1, N, 1024, V, 1) < N * V * 4 // 4
    assert L.kb_loss_workspace_bytes(1, N, 1024, V, 1) < N * V * 4 // 16
    rng = np.random.default_rng(0)
    for _ in range(200):
        a = [int(rng.integers(0, 2)), int(10 ** rng.uniform(0, 4)), int(10 ** rng.uniform(0, 3.3)), int(10 ** rng.uniform(0, 5.4)),
             int(rng.integers(1, 129))]
        assert L.kb_loss_workspace_bytes(*a) > 0 and L.kb_loss_grad_workspace_bytes(*a) > 0


def test_binding_refuses_what_is_not_on_the_gpu():
    h, W, b = torch.zeros(4, 8), torch.zeros(8, 20), torch.zeros(20)
    t, y = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    k = torch.zeros((4, 3), dtype=torch.int32)
    for call in (lambda: binding.cross_entropy(h, W, b, t), lambda: binding.cross_entropy_grad(h, W, b, t, y, y),
                 lambda: binding.distill(h, W, b, k, torch.zeros(4, 3)),
                 lambda: binding.distill_grad(h, W, b, k, torch.zeros(4, 3), y, y),
                 lambda: binding.cross_entropy(None, W, b, t), lambda: binding.cross_entropy([1.0], W, b, t)):
        with pytest.raises(TypeError):
            call()


def test_header_limits_match():
    import re
    text = open(binding.os.path.join(binding._HERE, "..", "include", "kbest_loss.h")).read()
    limits = dict(re.findall(r"#define (KB_LOSS_MAX_\w) (\d+)", text))
    assert limits == {"KB_LOSS_MAX_V": "262144", "KB_LOSS_MAX_H": "65536", "KB_LOSS_MAX_N": "4194304", "KB_LOSS_MAX_K": "128"}
    assert ctypes.sizeof(ctypes.c_int) == 4
