"""The performance cases of the attention cache: what a decoder with attention has it do in a decode step.

Three kinds of call, each through the package's public entry points:

  append   the step's new tokens, one row each: rotary positions on queries and keys, keys and values
           into their pages (``cache_append``); prompts go in the same way, a row for each token
  attend   attention of one new token a row over its cached keys and values (``cache_attend``), where
           the cache is to be thinned out later also the sums of its weights
  evict    caches longer than their budget keep the slots of greatest accumulated weight
           (``cache_evict``), in place or into pages of their own

Queries, keys and values are N(0, 1) before the scale 1 / sqrt(D); lengths are those of a batch in
which sequences have run for different times.  Pages lie scattered, in the order in which a server
hands them out.  All inputs are drawn on the GPU.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one sentence at beam 5, every token of a hypothesis in a page of its own (beams share their past): latency
        dict(name="append_f32_5x16x64", kind="append", dtype="f32", rows=5, q_heads=16, kv_heads=16, dim=64, rot=64,
             style="half", page=1, length=60, prompt=False),
        # 128 sentences at beam 5, half of each head turned
        dict(name="append_bf16_640_part", kind="append", dtype="bf16", rows=640, q_heads=8, kv_heads=8, dim=128, rot=64,
             style="pairs", page=1, length=60, prompt=False),
        # prompts of different lengths at once, positions far beyond the trained length
        dict(name="append_bf16_prompts", kind="append", dtype="bf16", rows=8200, q_heads=32, kv_heads=8, dim=128,
             rot=128, style="half", page=16, length=2500, prompt=True, far=True),
        # one sentence at beam 5: latency
        dict(name="attend_f32_5x60", kind="attend", dtype="f32", rows=5, q_heads=16, kv_heads=16, dim=64, page=1,
             length=60, ragged=True),
        # 128 sentences at beam 5, each somewhere within its 60 tokens
        dict(name="attend_bf16_640x60", kind="attend", dtype="bf16", rows=640, q_heads=8, kv_heads=8, dim=128, page=1,
             length=60, ragged=True),
        # one reader, one very long text: nothing but the length to share out
        dict(name="attend_bf16_1x131072", kind="attend", dtype="bf16", rows=1, q_heads=32, kv_heads=8, dim=128, page=64,
             length=131072, ragged=False),
        # a served batch of mixed lengths, some places empty, weights wanted for eviction
        dict(name="attend_bf16_64x8192_weights", kind="attend", dtype="bf16", rows=64, q_heads=32, kv_heads=8, dim=128,
             page=16, length=8192, ragged=True, weights=True),
        # single precision, a head size and a number of shared heads that are no power of two
        dict(name="attend_f32_odd17x3001", kind="attend", dtype="f32", rows=17, q_heads=15, kv_heads=5, dim=80, page=32,
             length=3001, ragged=True, weights=True),
        # a full offline batch
        dict(name="attend_bf16_128x4096", kind="attend", dtype="bf16", rows=128, q_heads=64, kv_heads=8, dim=128,
             page=64, length=4096, ragged=False),
        # every step of a small batch drops the token that its cache is over budget by
        dict(name="evict_f32_16x257", kind="evict", dtype="f32", rows=16, kv_heads=8, dim=64, page=16, length=257,
             keep=256, place=True, ragged=False),
        # every so often a larger batch goes back to its budget
        dict(name="evict_bf16_64x1100", kind="evict", dtype="bf16", rows=64, kv_heads=8, dim=128, page=16, length=1100,
             keep=512, place=True, ragged=True),
        # after long prompts: their best tokens move to pages of their own, the prompts' pages are given back
        dict(name="evict_bf16_4x32768", kind="evict", dtype="bf16", rows=4, kv_heads=8, dim=128, page=64, length=32768,
             keep=2048, place=False, ragged=False),
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "evict"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    dim = rng.choice([32, 64, 72, 80, 96, 128, 128, 192, 256])
    kv = rng.choice([1, 2, 3, 4, 5, 8, 16])
    group = rng.choice([1, 1, 2, 3, 4, 7, 8])
    page = rng.choice([1, 8, 16, 32, 64, 128])
    if kind == "append":
        rot = rng.choice([dim, dim // 2, dim // 4])
        per_row = (kv * group + 2 * kv) * dim
        rows = _between(rng, 1, max(2, min(8200, 8200 * 48 * 128 // per_row)))
        return dict(kind=kind, dtype=dtype, rows=rows, q_heads=kv * group, kv_heads=kv, dim=dim, rot=rot,
                    style=rng.choice(["half", "pairs"]), page=page, length=_between(rng, 60, 4000),
                    prompt=rng.random() < 0.4, far=rng.random() < 0.3)
    if kind == "attend":
        length = _between(rng, 1, 40000)
        # at most a quarter of the largest listed one's cache, as the plain form lays it out
        most = 128 * 4096 * 8 * 128 // 4 // (length * kv * dim)
        rows = _between(rng, 1, max(1, min(1000, most)))
        return dict(kind=kind, dtype=dtype, rows=rows, q_heads=kv * group, kv_heads=kv, dim=dim, page=page,
                    length=length, ragged=rng.random() < 0.7, weights=rng.random() < 0.4)
    length = _between(rng, 20, 30000)
    rows = _between(rng, 1, max(1, min(100, 4 * 30000 * 8 * 128 // (length * kv * dim))))
    keep = max(8, int(length * rng.uniform(0.05, 0.999)))
    return dict(kind=kind, dtype=dtype, rows=rows, kv_heads=kv, dim=dim, page=page, length=length, keep=keep,
                place=rng.random() < 0.6, ragged=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=DTYPES[dtype])


def _lengths(g, rows, most, ragged, empty=False):
    """Lengths up to ``most`` (the first row's), spread over their logarithm; ``empty``: one row in 16 has none."""
    if not ragged:
        return torch.full((rows,), most, dtype=torch.int32, device="cuda")
    u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
    n = torch.exp(u * math.log(most + 0.999)).floor().to(torch.int32).clamp(1, most)
    if empty:
        n[15::16] = 0
    n[0] = most
    return n


def _table(g, rows, page, cap):
    """(table, pages): ``rows`` sequences of ``cap`` slots, in pages of their own that lie scattered."""
    cols = -(-cap // page)
    pages = rows * cols
    return torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(rows, cols), pages


def _frequencies(rot, far):
    """Radians a position of each pair: base 10,000; far beyond the trained length, pairs that have not
    turned once by its end are slowed down eight times, those that turned 32 times are left, and the ones
    between are blended."""
    half = torch.arange(rot // 2, dtype=torch.float64)
    w = 10000.0 ** (-2.0 * half / rot)
    if far:
        turns = 8192.0 * w / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        w = w * keep + w / 8.0 * (1.0 - keep)
    return w.cuda()


def prepare(case, seed):
    c, g = case, _gen(seed)
    kind, dtype, R, KV, D, ps = c["kind"], c["dtype"], c["rows"], c["kv_heads"], c["dim"], c["page"]
    s = dict(case=c)
    if kind == "append":
        Q = c["q_heads"]
        if c["prompt"]:
            # rows are the tokens of ragged prompts: sequence r's first, second, ... one after the other
            lens, left = [], R
            k = 0
            while left > 0:
                n = min(left, max(1, c["length"] * (1 + k % 4) // 4))
                lens.append(n)
                left -= n
                k += 1
            lt = torch.tensor(lens, device="cuda")
            seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lt)
            first = torch.cumsum(lt, 0) - lt
            s["length"] = (torch.arange(R, device="cuda") - first[seq] + 1).to(torch.int32)
            s["seq"] = seq.to(torch.int32)
            seqs, cap = len(lens), max(lens)
        else:
            s["length"] = _lengths(g, R, c["length"], True)
            s["seq"] = None
            seqs, cap = R, c["length"]
        s["table"], pages = _table(g, seqs, ps, cap)
        s["pos"] = s["length"] - 1 + (1000000 if c.get("far") else 0)
        s["freq"] = _frequencies(c["rot"], c.get("far"))
        s["amplitude"] = 1.2079 if c.get("far") else 1.0  # 0.1 ln 8 + 1
        # as one fused projection leaves them
        s["qkv"] = _randn(g, (R, (Q + 2 * KV) * D), dtype)
        s["k_cache"] = _randn(g, (pages, KV, ps, D), dtype)
        s["v_cache"] = _randn(g, (pages, KV, ps, D), dtype)
        s["position"] = torch.full((seqs, KV, s["table"].shape[1] * ps), -1, dtype=torch.int32, device="cuda")
        return s
    if kind == "attend":
        L = c["length"]
        s["length"] = _lengths(g, R, L, c["ragged"], empty=c.get("weights", False))
        if ps == 1 and L <= 60 and R % 5 == 0:
            # a beam's hypotheses: each slot's page is one of the five that the sentence wrote at that step
            s["table"] = (torch.arange(L, device="cuda")[None, :] * R + torch.arange(R, device="cuda")[:, None] // 5 * 5
                          + torch.randint(0, 5, (R, L), generator=g, device="cuda")).to(torch.int32)
            pages = R * L
        else:
            s["table"], pages = _table(g, R, ps, L)
        s["q"] = _randn(g, (R, c["q_heads"], D), dtype)
        s["k_cache"] = _randn(g, (pages, KV, ps, D), dtype)
        s["v_cache"] = _randn(g, (pages, KV, ps, D), dtype)
        if c.get("weights"):
            cap = s["table"].shape[1] * ps
            s["weight_in"] = torch.rand((R, KV, cap), generator=g, device="cuda") * 3
            s["weight_out"] = torch.zeros((R, KV, cap), device="cuda")
        return s
    L, keep = c["length"], c["keep"]
    s["length"] = _lengths(g, R, L, c["ragged"])
    s["table"], pages = _table(g, R, ps, L)
    cap = s["table"].shape[1] * ps
    if c["place"]:
        s["out_table"] = s["table"]
    else:
        t, more = _table(g, R, ps, keep)
        s["out_table"] = t + pages
        pages += more
    out_cap = s["out_table"].shape[1] * ps
    s["k_cache"] = _randn(g, (pages, KV, ps, D), dtype)
    s["v_cache"] = _randn(g, (pages, KV, ps, D), dtype)
    # few tokens hold most of the weight
    s["weight"] = torch.rand((R, KV, cap), generator=g, device="cuda").clamp_min(1e-6).pow(-0.7)
    # earlier evictions have left the slots out of their order in time
    s["position"] = torch.argsort(torch.rand((R, KV, cap), generator=g, device="cuda"), dim=-1).to(torch.int32)
    s["newest"] = torch.full((R,), cap - 1, dtype=torch.int32, device="cuda")
    s["first"], s["recent"] = min(4, keep // 4), keep // 4
    s["out"] = (torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros((R, KV, out_cap), device="cuda"),
                torch.full((R, KV, out_cap), -1, dtype=torch.int32, device="cuda"),
                torch.full((R, KV, keep), -1, dtype=torch.int32, device="cuda"))
    return s


# ---------------------------------------------------------------- the plain forms

def _split(s):
    c = s["case"]
    return s["qkv"].view(c["rows"], -1, c["dim"]).split([c["q_heads"], c["kv_heads"], c["kv_heads"]], dim=1)


def _turn(x, cos, sin, rot, style):
    """x: rows x heads x dim in 32 bits; cos, sin: rows x rot / 2."""
    cos, sin = cos[:, None], sin[:, None]
    head, rest = x[..., :rot], x[..., rot:]
    if style == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], dim=-1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), rest], dim=-1)


def _plain_append(s):
    c = s["case"]
    q, k, v = _split(s)
    angle = s["pos"].double()[:, None] * s["freq"]
    cos = (angle.cos() * s["amplitude"]).float()
    sin = (angle.sin() * s["amplitude"]).float()
    seq = torch.arange(c["rows"], device="cuda") if s["seq"] is None else s["seq"].long()
    slot = s["length"].long() - 1
    page, place = s["table"][seq, slot // c["page"]].long(), slot % c["page"]
    s["k_cache"][page, :, place] = _turn(k.float(), cos, sin, c["rot"], c["style"]).to(k.dtype)
    s["v_cache"][page, :, place] = v
    s["position"][seq, :, slot] = s["pos"][:, None].expand(-1, c["kv_heads"])
    q_out = _turn(q.float(), cos, sin, c["rot"], c["style"]).to(q.dtype)
    return q_out, s["k_cache"], s["v_cache"], s["position"]


def _pages_of(cache, table, most):
    """rows x heads x most x dim in 32 bits."""
    ps = cache.shape[2]
    x = cache[table[:, :-(-most // ps)].long()]
    R, n, H, _, D = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(R, H, n * ps, D)[:, :, :most].float()


def _plain_attend(s):
    c = s["case"]
    R, KV, D, L = c["rows"], c["kv_heads"], c["dim"], c["length"]
    k = _pages_of(s["k_cache"], s["table"], L)
    score = s["q"].float().view(R, KV, -1, D) @ k.transpose(-1, -2) / math.sqrt(D)
    seen = torch.arange(L, device="cuda") < s["length"][:, None]
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).view(R, -1)
    p = p / torch.where(total == 0, 1.0, total)
    out = (p @ _pages_of(s["v_cache"], s["table"], L)).view(R, -1, D).to(s["q"].dtype)
    if not c.get("weights"):
        return out, lse
    new = s["weight_in"][..., :L] + p.sum(2)
    s["weight_out"][..., :L] = torch.where(seen[:, None], new, s["weight_out"][..., :L])
    return out, lse, s["weight_out"]


def _plain_evict(s):
    c = s["case"]
    R, KV, ps, keep, L = c["rows"], c["kv_heads"], c["page"], c["keep"], c["length"]
    slot = torch.arange(L, device="cuda")
    seen = (slot < s["length"][:, None])[:, None]
    pos = s["position"][..., :L]
    held = (pos < s["first"]) | (pos > (s["newest"] - s["recent"])[:, None, None])
    key = s["weight"][..., :L].masked_fill(held, math.inf).masked_fill(~seen, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order))
    n = s["length"].clamp(max=keep)[:, None, None]
    kept = rank < n
    # kept slots from n on, in order, before all others
    tail = torch.sort((~(kept & (slot >= n))).to(torch.int8), dim=-1, stable=True).indices
    width = min(keep, L)
    hole = ~kept[..., :width] & (slot[:width] < n)
    nth = (hole.long().cumsum(-1) - 1).clamp_min(0)
    source = torch.where(hole, tail.gather(-1, nth), slot[:width])
    used = (slot[:width] < n).expand_as(source)
    length, weight, position, out_source = s["out"]
    r, h, i = used.nonzero(as_tuple=True)
    j = source[r, h, i]
    frm, to = s["table"][r, j // ps].long(), s["out_table"][r, i // ps].long()
    for cache in (s["k_cache"], s["v_cache"]):
        cache[to, h, i % ps] = cache[frm, h, j % ps]
    weight[r, h, i] = s["weight"][r, h, j]
    position[r, h, i] = s["position"][r, h, j]
    out_source.fill_(-1)[..., :width] = torch.where(used, source, -1).to(torch.int32)
    length.copy_(n.view(-1))
    return s["k_cache"], s["v_cache"], length, weight, position, out_source


# ---------------------------------------------------------------- the framework's operators

def _own_append(s):
    import paper_1805_09863_amd as kb
    q, k, v = _split(s)
    q_out = kb.cache_append(s["k_cache"], s["v_cache"], s["table"], s["length"], k, v, q=q, pos=s["pos"],
                            freq=s["freq"], interleaved=s["case"]["style"] == "pairs", amplitude=s["amplitude"],
                            seq=s["seq"], position=s["position"])
    return q_out, s["k_cache"], s["v_cache"], s["position"]


def _own_attend(s):
    import paper_1805_09863_amd as kb
    lse = torch.empty((s["case"]["rows"], s["case"]["q_heads"]), device="cuda")
    if not s["case"].get("weights"):
        return kb.cache_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["length"], lse=lse), lse
    out = kb.cache_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["length"], lse=lse,
                          weight_in=s["weight_in"], weight_out=s["weight_out"])
    return out, lse, s["weight_out"]


def _own_evict(s):
    import paper_1805_09863_amd as kb
    kb.cache_evict(s["k_cache"], s["v_cache"], s["table"], s["length"], s["case"]["keep"], weight=s["weight"],
                   position=s["position"], newest=s["newest"], first=s["first"], recent=s["recent"],
                   out_table=s["out_table"], out=s["out"])
    return (s["k_cache"], s["v_cache"]) + s["out"]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "evict": _own_evict}[kind](state)
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[kind](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c, e = case, SIZE[case["dtype"]]
    R, KV, D = c["rows"], c["kv_heads"], c["dim"]
    if c["kind"] == "append":
        heads = c["q_heads"] + 2 * KV
        # position and length of each row in, the slots' positions out, three operations a turned value
        return {"bytes": 2 * R * heads * D * e + R * (8 + 4 * KV),
                "flops": 3 * R * (c["q_heads"] + KV) * c["rot"]}
    s = prepare(dict(c, rows=R, kv_heads=1, dim=8, **({"q_heads": 1} if "q_heads" in c else {})), 0)
    n = s["length"].double()
    if c["kind"] == "attend":
        total = float(n.sum())
        if c["page"] == 1 and c["length"] <= 60 and R % 5 == 0:
            # the pages that the rows of a beam share are read once
            seen = torch.arange(c["length"], device="cuda") < s["length"][:, None]
            pages = int(torch.unique(s["table"][seen]).numel())
        else:
            pages = total
        b = pages * KV * 2 * D * e + 2 * R * c["q_heads"] * D * e + R * c["q_heads"] * 4
        b += total * KV * 8 if c.get("weights") else 0
        return {"bytes": b, "flops": 4.0 * total * c["q_heads"] * D}
    over = n - n.clamp(max=c["keep"])
    # in place, a kept slot past the budget fills a hole: as the weights do not depend on the slot,
    # keep / length of the slots past it are kept; elsewhere every kept slot moves
    moved = float((n.clamp(max=c["keep"]) * over / n).sum()) if c["place"] else float(n.clamp(max=c["keep"]).sum())
    b = float(n.sum()) * KV * 8 + moved * KV * 4 * D * e + float(n.clamp(max=c["keep"]).sum()) * KV * 12
    return {"bytes": b, "flops": 2.0 * float(n.sum()) * KV}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _slot_rows(s, r, n):
    """Page and place of the first n slots of table row r."""
    ps = s["case"]["page"]
    t = torch.arange(n, device="cuda")
    return s["table"][r][torch.div(t, ps, rounding_mode="floor")].long(), t % ps


def _exact_append(s):
    c = s["case"]
    R, Q, KV, D, rot = c["rows"], c["q_heads"], c["kv_heads"], c["dim"], c["rot"]
    x = s["qkv"].double().view(R, Q + 2 * KV, D)
    i = torch.arange(rot // 2, device="cuda")
    lo, hi = (i, i + rot // 2) if c["style"] == "half" else (2 * i, 2 * i + 1)
    # a turn in the plane of each pair, as a product of complex numbers
    z = torch.complex(x[..., lo], x[..., hi])
    a = s["pos"].double()[:, None, None] * s["freq"]
    z = z * torch.polar(torch.full_like(a, s["amplitude"]), a)
    y = x.clone()
    y[..., lo], y[..., hi] = z.real, z.imag
    k_cache, v_cache, position = s["k_cache"].double(), s["v_cache"].double(), s["position"].clone()
    slots = s["length"].tolist()
    seqs = list(range(R)) if s["seq"] is None else s["seq"].tolist()
    table = s["table"].tolist()
    page = torch.tensor([table[q][(n - 1) // c["page"]] for q, n in zip(seqs, slots)], device="cuda")
    place = torch.tensor([(n - 1) % c["page"] for n in slots], device="cuda")
    for h in range(KV):
        k_cache[page, h, place] = y[:, Q + h]
        v_cache[page, h, place] = x[:, Q + KV + h]
        position[torch.tensor(seqs, device="cuda"), h, s["length"].long() - 1] = s["pos"]
    return y[:, :Q].contiguous(), k_cache, v_cache, position


def _exact_attend(s):
    c = s["case"]
    R, Q, KV, D = c["rows"], c["q_heads"], c["kv_heads"], c["dim"]
    out = torch.zeros((R, Q, D), dtype=torch.float64, device="cuda")
    lse = torch.full((R, Q), -math.inf, dtype=torch.float64, device="cuda")
    weight = s["weight_out"].double() if c.get("weights") else None
    for r, n in enumerate(s["length"].tolist()):
        if n == 0:
            continue
        page, place = _slot_rows(s, r, n)
        k, v = s["k_cache"][page, :, place].double(), s["v_cache"][page, :, place].double()  # n x KV x D
        for h in range(KV):
            mine = slice(h * Q // KV, (h + 1) * Q // KV)
            score = (s["q"][r, mine].double() @ k[:, h].T.contiguous()) * D ** -0.5
            lse[r, mine] = torch.logsumexp(score, dim=-1)
            p = torch.softmax(score, dim=-1)
            out[r, mine] = p @ v[:, h]
            if weight is not None:
                weight[r, h, :n] = s["weight_in"][r, h, :n].double() + p.sum(0)
    return (out, lse) if weight is None else (out, lse, weight)


def _exact_evict(s):
    c = s["case"]
    keep = c["keep"]
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    k_from, v_from = s["k_cache"], s["v_cache"]
    length, weight, position, source = (x.clone() for x in s["out"])
    weight = weight.double()
    k_to, v_to = k_cache, v_cache
    w_host, p_host = s["weight"].cpu(), s["position"].cpu()
    ps = c["page"]
    for r, L in enumerate(s["length"].tolist()):
        n = min(L, keep)
        length[r] = n
        newest = int(s["newest"][r])
        for h in range(c["kv_heads"]):
            w, p = w_host[r, h, :L].double(), p_host[r, h, :L]
            w = torch.where((p < s["first"]) | (p > newest - s["recent"]), torch.full_like(w, math.inf), w)
            order = torch.argsort(-w, stable=True)[:n]
            stay = torch.zeros(L, dtype=torch.bool)
            stay[order] = True
            src = torch.arange(n)
            src[~stay[:n]] = torch.nonzero(stay[n:]).view(-1) + n
            src = src.cuda()
            to = torch.arange(n, device="cuda")
            fp, tp = s["table"][r][src // ps].long(), s["out_table"][r][to // ps].long()
            k_to[tp, h, to % ps] = k_from[fp, h, src % ps].double()
            v_to[tp, h, to % ps] = v_from[fp, h, src % ps].double()
            weight[r, h, :n] = s["weight"][r, h][src].double()
            position[r, h, :n] = s["position"][r, h][src]
            source[r, h, :n] = src.to(torch.int32)
    return k_cache, v_cache, length, weight, position, source


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["kind"]](s)
