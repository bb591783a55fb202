"""Calls of the output layer on a side stream that allocate for themselves: their results are those of the current
stream, and they take no memory that the current stream has freed but still reads."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


def _calls(kb):
    g = torch.Generator().manual_seed(3)
    S, beam, H, V, k = 40, 4, 128, 3000, 4          # (a shape that the unfused baseline takes too)
    N = S * beam
    h, W = torch.randn(N, H, generator=g).bfloat16().cuda(), (torch.randn(H, V, generator=g) / 8).bfloat16().cuda()
    b, prev = torch.randn(V, generator=g).cuda() * 0.1, -torch.rand(N, generator=g).cuda()
    off = torch.arange(0, N + 1, beam, dtype=torch.int32, device="cuda")
    alive = (torch.rand(S * k, generator=g) < 0.6).to(torch.uint8).cuda()
    sent = (torch.arange(S * k) // k).to(torch.int32).cuda()
    idx = torch.randint(0, N, (N,), generator=g).to(torch.int32).cuda()
    P = kb.shard_splits(h, W, b, k)
    stats, lists = torch.zeros(P, N, 2, device="cuda"), torch.zeros((P, N, k, 2), dtype=torch.int32, device="cuda")
    T = 3
    fin = (torch.ones(S, dtype=torch.int32, device="cuda"), -torch.rand(S * k, generator=g).cuda(),
           torch.full((S * k,), 2, dtype=torch.int32, device="cuda"),
           torch.arange(S * k, dtype=torch.int32, device="cuda") + S * k)
    hist = (torch.randint(0, V, (T * S * k,), generator=g).to(torch.int32).cuda(),
            torch.cat([torch.full((S * k,), -1), torch.arange(2 * S * k)]).to(torch.int32).cuda())

    def shards(stream=None):
        kb.shard_partials(h, W, b, k, 0, stats, lists, stream=stream)
        return kb.merge_partials(stats, lists, P, V, k, prev, off, stream=stream)

    return [lambda stream=None: kb.kbest_step(h, W, b, prev, off, k, stream=stream),
            lambda stream=None: kb.argmax_step(h, W, b, stream=stream),
            lambda stream=None: kb.kbest_step_unfused(h, W, b, prev, off, k, stream=stream),
            lambda stream=None: kb.compact_batch(alive, sent, stream=stream),
            lambda stream=None: kb.compact_beams(alive, S, k, stream=stream),
            lambda stream=None: (kb.gather_rows(h, idx, stream=stream),), shards,
            lambda stream=None: kb.binding.beam_backtrace(S, k, T, 0.5, fin, *hist, stream=stream)], S, k


def test_calls_beside_a_busy_stream(kb):
    calls, S, k = _calls(kb)
    want = [c() for c in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    read = [torch.ones(1 << n, device="cuda") for n in range(7, 22) for _ in range(6)]
    copies = [torch.empty_like(x) for x in read]
    torch.cuda.synchronize()
    torch.cuda._sleep(60_000_000)          # about 30 ms of the current stream
    for x, y in zip(read, copies):
        y.copy_(x)
    del read, x
    got = [c(side) for c in calls]
    side.synchronize()
    host = [[t.to("cpu") for t in r] for r in got]
    torch.cuda.synchronize()
    assert all(bool((y == 1).all()) for y in copies)
    for i, (a, c) in enumerate(zip(want, host)):
        a = [t.cpu() for t in a]
        if i in (3, 4):                    # only the first kept entries and kept sentences mean anything
            kept, sents = int(a[1]), int(a[-1])
            cut = [kept, 1, sents + 1] + ([1] if i == 3 else [sents, 1])
            a, c = [t[:n] for t, n in zip(a, cut)], [t[:n] for t, n in zip(c, cut)]
        assert len(a) == len(c) and all(torch.equal(x, y) for x, y in zip(a, c)), i
