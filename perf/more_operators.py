"""The performance cases of the output layer's losses: what training the layer, or asking it what it makes of given
translations, has it do.

Two losses of logits = h W + b, each through the package's public entry points, neither keeping the rows x vocabulary
logits:

  cross_entropy   -log of the probability of each row's target word, with label smoothing where a case says so
  distill         a teacher's best words and their logits for each row against the student's whole softmax, at a temperature

and of each two kinds of call:

  score           the losses and log-sum-exps of all rows (``cross_entropy``, ``distill``): translations rescored, a
                  model's loss on held-out text
  train           those and then the gradients of h, W and b (``cross_entropy_grad``, ``distill_grad``): the output
                  layer's part of a training step

States are N(0, 1), weights N(0, 1 / H), the bias falls with the word's rank as its frequency does, and targets are
drawn by it.  A part of the rows is padding (target -1, or no teacher entry) and has neither loss nor gradient.  All
inputs are drawn on the GPU.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one sentence's beam rescored under another model: latency
        dict(name="ce_score_f32_5x256x8000", loss="cross_entropy", train=False, dtype="f32", N=5, H=256, V=8000, pad=0.0,
             smoothing=0.0),
        # the translations of 128 sentences at beam 5 rescored, a word each
        dict(name="ce_score_bf16_640x1024x60000", loss="cross_entropy", train=False, dtype="bf16", N=640, H=1024, V=60000,
             pad=0.0, smoothing=0.0),
        # held-out text in one call; a vocabulary of an odd size, and padding
        dict(name="ce_score_bf16_5000x512x32001", loss="cross_entropy", train=False, dtype="bf16", N=5000, H=512, V=32001,
             pad=0.1, smoothing=0.0),
        # a few sentences to adapt a model with, between translations
        dict(name="ce_train_bf16_60x1024x50000", loss="cross_entropy", train=True, dtype="bf16", N=60, H=1024, V=50000,
             pad=0.0, smoothing=0.1),
        # a small model in 32 bits
        dict(name="ce_train_f32_640x512x30000", loss="cross_entropy", train=True, dtype="f32", N=640, H=512, V=30000,
             pad=0.15, smoothing=0.1),
        # a training batch of ordinary size, a part of it padding
        dict(name="ce_train_bf16_4096x1024x50000", loss="cross_entropy", train=True, dtype="bf16", N=4096, H=1024, V=50000,
             pad=0.15, smoothing=0.1),
        # the largest: a batch over the largest vocabulary
        dict(name="ce_train_bf16_8192x1024x90000", loss="cross_entropy", train=True, dtype="bf16", N=8192, H=1024, V=90000,
             pad=0.0, smoothing=0.0),
        # one sentence against its teacher: latency
        dict(name="kd_train_f32_5x256x8000", loss="distill", train=True, dtype="f32", N=5, H=256, V=8000, pad=0.0, K=5,
             temperature=1.0),
        # how far a student is from its teacher on held-out text
        dict(name="kd_score_bf16_2000x512x30000", loss="distill", train=False, dtype="bf16", N=2000, H=512, V=30000, pad=0.1,
             K=12, temperature=1.0),
        # a training batch of a student; vocabulary and states of odd sizes, soft targets
        dict(name="kd_train_bf16_1111x500x32001", loss="distill", train=True, dtype="bf16", N=1111, H=500, V=32001, pad=0.2,
             K=8, temperature=2.0),
        # a large one, with many of the teacher's words
        dict(name="kd_train_bf16_4096x1024x60000", loss="distill", train=True, dtype="bf16", N=4096, H=1024, V=60000, pad=0.0,
             K=64, temperature=2.0),
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "bf16"])
    H = rng.choice([64, 128, 256, 256, 500, 512, 512, 640, 1000, 1024, 1024])
    V = _between(rng, 500, 90000)
    if rng.random() < 0.6:
        V = max(8, V // 8 * 8)
    # at most the largest listed one's products; those of 32 bits take the place of several of 16
    most = 8192 * 1024 * 90000 // (8 if dtype == "f32" else 1) // (H * V)
    c = dict(loss=rng.choice(["cross_entropy", "distill"]), train=rng.random() < 0.6, dtype=dtype,
             N=_between(rng, 1, max(1, min(8192, most))), H=H, V=V, pad=rng.choice([0.0, 0.0, 0.1, 0.3]))
    if c["loss"] == "distill":
        c.update(K=rng.choice([1, 4, 5, 8, 12, 16, 33, 64]), temperature=rng.choice([1.0, 1.0, 2.0, 4.0]))
    else:
        c.update(smoothing=rng.choice([0.0, 0.0, 0.1]))
    return c


# ---------------------------------------------------------------- inputs

def _by_frequency(u, V):
    """Words of ranks spread as their frequency falls: u in [0, 1)."""
    return (torch.exp(u.double() * math.log(V)).long() - 1).clamp(0, V - 1)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    N, H, V, dtype = c["N"], c["H"], c["V"], DTYPES[c["dtype"]]
    s = dict(case=c)
    s["h"] = torch.randn((N, H), generator=g, device="cuda").to(dtype)
    s["W"] = (torch.randn((H, V), generator=g, device="cuda") / math.sqrt(H)).to(dtype)
    rank = torch.arange(V, device="cuda", dtype=torch.float32)
    s["b"] = -0.5 * torch.log1p(rank) + 0.1 * torch.randn(V, generator=g, device="cuda")
    # which rows are padding: about the given part, never the first
    padding = torch.rand(N, generator=g, device="cuda") < c["pad"]
    padding[0] = False
    if c["loss"] == "cross_entropy":
        s["target"] = _by_frequency(torch.rand(N, generator=g, device="cuda"), V).masked_fill(padding, -1).to(torch.int32)
    else:
        # the teacher's best words, all different, best first, as its own output layer finds them
        K = c["K"]
        at = torch.arange(K, device="cuda")
        word = _by_frequency((at + torch.rand((N, K), generator=g, device="cuda")) / K, V)
        word = torch.minimum(torch.cummax(word - at, dim=1).values + at, V - K + at)
        word = word.gather(1, torch.argsort(torch.rand((N, K), generator=g, device="cuda"), dim=1))
        logit = 2.0 * torch.randn((N, K), generator=g, device="cuda")
        s["logit"] = torch.sort(logit, dim=1, descending=True).values
        # some rows have fewer words than the rest
        short = torch.rand(N, generator=g, device="cuda") < 0.05
        absent = (short[:, None] & (at >= (K + 1) // 2)) | padding[:, None]
        s["token"] = word.masked_fill(absent, -1).to(torch.int32)
    # the mean over the rows that count, each with a weight of its own
    weight = 0.5 + torch.rand(N, generator=g, device="cuda")
    s["grad"] = weight / (~padding).sum()
    return s


# ---------------------------------------------------------------- the plain forms

def _plain(s):
    c = s["case"]
    V = c["V"]
    h, W = s["h"].float(), s["W"].float()
    x = h @ W + s["b"]
    scale = 1.0
    if c["loss"] == "cross_entropy":
        eps = c["smoothing"]
        counts = s["target"] >= 0
        word = s["target"].long().clamp_min(0)[:, None]
        part = torch.full(word.shape, 1.0 - eps, device=x.device)
        rest, known = eps / V, 0.0
    else:
        t = c["temperature"]
        x = x / t
        scale = t * t
        present = s["token"] >= 0
        counts = present.any(1)
        word = s["token"].long().clamp_min(0)
        y = (s["logit"] / t).masked_fill(~present, -math.inf)
        y = y - torch.where(counts, y.amax(1), 0.0)[:, None]
        e = torch.exp(y)
        total = torch.where(counts, e.sum(1), 1.0)[:, None]
        part = e / total
        known = torch.where(present, part * (y - torch.log(total)), 0.0).sum(1)
        rest = 0.0
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    loss = lse + known - (part * x.gather(1, word)).sum(1)
    if rest:
        loss = loss - rest * x.sum(1)
    loss = torch.where(counts, scale * loss, 0.0)
    lse = torch.where(counts, lse, 0.0)
    if not c["train"]:
        return loss, lse
    d = e / total - rest
    d.scatter_add_(1, word, -part)
    d = d * torch.where(counts, s["grad"] * math.sqrt(scale), 0.0)[:, None]
    return loss, lse, (d @ W.t()).to(s["h"].dtype), (h.t() @ d).to(s["W"].dtype), d.sum(0)


# ---------------------------------------------------------------- the framework's operators

def _own(s):
    import paper_1805_09863_amd as kb
    c, h, W, b = s["case"], s["h"], s["W"], s["b"]
    if c["loss"] == "cross_entropy":
        loss, lse = kb.cross_entropy(h, W, b, s["target"], smoothing=c["smoothing"])
        if not c["train"]:
            return loss, lse
        dh, dW, db = kb.cross_entropy_grad(h, W, b, s["target"], lse, s["grad"], smoothing=c["smoothing"])
        return loss, lse, dh, dW, db
    loss, lse = kb.distill(h, W, b, s["token"], s["logit"], temperature=c["temperature"])
    if not c["train"]:
        return loss, lse
    dh, dW, db = kb.distill_grad(h, W, b, s["token"], s["logit"], lse, s["grad"], temperature=c["temperature"])
    return loss, lse, dh, dW, db


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    """By the definition: a distribution q over the whole vocabulary for each row, and what it and log p give."""
    s = prepare(case, seed)
    N, H, V = case["N"], case["H"], case["V"]
    W, b = s["W"].double(), s["b"].double()
    t = case.get("temperature", 1.0)
    loss, lse = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(2))
    dh = torch.zeros((N, H), dtype=torch.float64, device="cuda")
    dW, db = torch.zeros_like(W), torch.zeros_like(b)
    step = max(1, 2 ** 28 // V)
    for r0 in range(0, N, step):
        rows = slice(r0, min(N, r0 + step))
        h = s["h"][rows].double()
        n = h.shape[0]
        q = torch.zeros((n, V), dtype=torch.float64, device="cuda")
        if case["loss"] == "cross_entropy":
            target = s["target"][rows].long()
            used = (target >= 0).nonzero().squeeze(1)
            q[used] = case["smoothing"] / V
            q[used, target[used]] += 1.0 - case["smoothing"]
        else:
            token = s["token"][rows].long()
            r, k = (token >= 0).nonzero(as_tuple=True)
            teacher = torch.full((n, V), -math.inf, dtype=torch.float64, device="cuda")
            teacher[r, token[r, k]] = s["logit"][rows].double()[r, k] / t
            used = torch.unique(r)
            q[used] = torch.softmax(teacher[used], dim=1)
            del teacher
        x = (h @ W + b) / t
        norm = torch.logsumexp(x, dim=1)
        logp = x - norm[:, None]
        del x
        seen = torch.zeros(n, dtype=torch.bool, device="cuda")
        seen[used] = True
        if case["loss"] == "cross_entropy":
            value = -(q * logp).sum(1)
        else:
            value = t * t * (torch.special.xlogy(q, q) - q * logp).sum(1)
        loss[rows] = torch.where(seen, value, 0.0)
        lse[rows] = torch.where(seen, norm, 0.0)
        if case["train"]:
            d = (logp.exp() - q) * (t * s["grad"][rows].double() * seen)[:, None]
            dh[rows] = d @ W.t()
            dW += h.t() @ d
            db += d.sum(0)
        del q, logp
    return (loss, lse, dh, dW, db) if case["train"] else (loss, lse)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    z = SIZE[c["dtype"]]
    N, H, V = c["N"], c["H"], c["V"]
    rows = max(1.0, N * (1.0 - c["pad"]))
    read = rows * H * z + H * V * z + 4 * V + (N * 4 if c["loss"] == "cross_entropy" else 8 * N * c["K"])
    wrote = 8 * N
    products = 1
    if c["train"]:
        read += 4 * N  # the gradients of the losses
        wrote += N * H * z + H * V * z + 4 * V
        products = 3  # the logits, and the gradients of h and of W
    return {"bytes": read + wrote, "flops": 2.0 * products * rows * H * V}
