"""The decode loops on a stream of the caller's while the current stream is busy: nothing of theirs waits for it, lies
in its memory or is filled by it."""
import pytest
import torch

from synth import workloads as wl

pytestmark = pytest.mark.gpu
H, V, Q, KV, D = 64, 500, 4, 2, 16
EOS = 3


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


def _decoder():
    from paper_1805_09863_amd.decoder import CachedDecoder
    g = torch.Generator().manual_seed(21)
    r = lambda *s: torch.randn(s, generator=g).cuda()  # noqa: E731
    dec = CachedDecoder(r(V, H), r(H, (Q + 2 * KV) * D) / H ** 0.5, r(Q * D, H) / (Q * D) ** 0.5, Q, KV)
    return dec, r(H, V) / H ** 0.5, r(V) * 0.1, torch.tensor([5, 9, 5, 77, 0, 31], dtype=torch.int32, device="cuda")


def _loops():
    """name -> a call that takes a stream and on_step and returns tensors."""
    from paper_1805_09863_amd.decode import beam_search, decode_loop, greedy_search
    dec, W, b, start = _decoder()
    k, T = 4, 12
    table = torch.randn(len(start) * T * k, H, device="cuda")
    work = wl.make_loop_workload(S=20, V=1001, H=64, T=8, Lmin=1, Lmax=8, seed=5)
    bf16 = lambda a: torch.from_numpy(a.view("int16")).view(torch.bfloat16).cuda()  # noqa: E731
    loop = (bf16(work.h_table().reshape(-1, work.H)), bf16(work.W), torch.from_numpy(work.b).cuda(),
            torch.from_numpy(work.lengths).cuda(), torch.from_numpy(work.prev0).cuda(), work.k, work.T)

    def beams(h_table, decoder, **kw):
        res = beam_search(h_table, W, b, k, T, EOS, decoder=decoder, start=start if decoder else None, alpha=0.6, **kw)
        return res.tokens, res.length, res.score, res.norm

    def greedy(**kw):
        res = greedy_search(dec, W, b, start, 30, EOS, keep=10, every=3, **kw)
        return res.tokens, res.length

    def batch(compact, stream=None, on_step=None):
        got = []

        def each(t, st):
            got.extend((st["token"].clone(), st["score"].clone()))
            if on_step is not None:
                on_step(t, st)
        decode_loop(*loop, compact=compact, stream=stream, on_step=each)
        return got

    return {"beams_of_a_decoder": lambda **kw: beams(None, dec, **kw), "beams_of_a_table": lambda **kw: beams(table, None, **kw),
            "greedy": greedy, "compacted": lambda **kw: batch(True, **kw), "constant": lambda **kw: batch(False, **kw)}


@pytest.mark.parametrize("name", ["beams_of_a_decoder", "beams_of_a_table", "greedy", "compacted", "constant"])
def test_a_loop_beside_a_busy_stream(kb, name):
    call = _loops()[name]
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    # memory of the current stream in every size that the loops ask for, freed while copies of it are still to run
    read = [torch.ones(1 << n, device="cuda") for n in range(7, 21) for _ in range(4)]
    copies = [torch.empty_like(x) for x in read]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)         # about 50 ms of the current stream
    for x, y in zip(read, copies):
        y.copy_(x)
    del read, x
    seen = []
    got = call(stream=side, on_step=lambda t, st: seen.append(torch.cuda.current_stream() == side))
    side.synchronize()
    assert seen and all(seen)
    assert len(got) == len(want) and all(torch.equal(a.to("cpu"), b.to("cpu")) for a, b in zip(got, want))
    torch.cuda.synchronize()
    assert all(bool((y == 1).all()) for y in copies)


def test_a_compacted_loop_writes_nothing_once_it_has_returned(kb):
    """Its last step, launched for a batch that turns out to be empty, is held up on the device: the pinned memory of
    its counts, given back when the loop returns, keeps what the next owner writes."""
    from paper_1805_09863_amd.decode import decode_loop
    work = wl.make_loop_workload(S=6, V=1001, H=64, T=8, Lmin=3, Lmax=3, seed=6)
    bf16 = lambda a: torch.from_numpy(a.view("int16")).view(torch.bfloat16).cuda()  # noqa: E731
    args = (bf16(work.h_table().reshape(-1, work.H)), bf16(work.W), torch.from_numpy(work.b).cuda(),
            torch.from_numpy(work.lengths).cuda(), torch.from_numpy(work.prev0).cuda(), work.k, work.T)
    decode_loop(*args)
    torch.cuda.synchronize()
    steps = []

    def on_step(t, st):
        steps.append(t)
        if t == 2:
            torch.cuda._sleep(40_000_000)      # about 20 ms before the step after the last
    decode_loop(*args, on_step=on_step)
    assert steps == [0, 1, 2]
    owned = [torch.full((3,), -5, dtype=torch.int32, pin_memory=True) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(x.tolist() == [-5] * 3 for x in owned)
