"""Sizes that take the attention cache's kernels through turns and variants of theirs that ordinary ones do not: splits
at every built head size and with weights, one workgroup a (row, head) in their join, a second turn of the weights' slots
and of the append's pieces, longer caches of few heads in a captured eviction."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from tests.test_gpu_cache import ROUND, bits, check_attend, f64, host, make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


def batch(g, dtype, R, heads, dim, page, most, long):
    """Short rows, empty ones among them, and some of 900 to 2,500 slots; pages of one sequence shared by none."""
    n = torch.randint(0, most + 1, (R,), generator=g).to(torch.int32)
    at = torch.randperm(R, generator=g)[:long]
    n[at] = torch.randint(900, 2500, (long,), generator=g).to(torch.int32)
    n[at[0]] = 2500
    # short rows share the few pages that they use: the pool stays small
    k, v, table = make_cache(g, dtype, long, heads, dim, page, 2500, spare=40, dirty=False)
    wide = torch.randint(0, k.shape[0], (R, table.shape[1]), generator=g).to(torch.int32)
    wide[at] = table
    return k, v, wide, n


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("q_heads,heads,dim,page", [
    (1, 1, 24, 16), (1, 1, 128, 8), (1, 1, 256, 32),      # up to 2,048 (row, head)s: a workgroup each in the join
    (4, 2, 72, 1), (3, 1, 192, 64), (34, 2, 64, 16),      # more: several in one
])
def test_splits(kb, dtype, q_heads, heads, dim, page):
    g = torch.Generator().manual_seed(dim + q_heads)
    R = 1030
    k, v, table, n = batch(g, dtype, R, heads, dim, page, 12, 3)
    q = torch.randn((R, q_heads, dim), generator=g).to(dtype)
    w = torch.rand((R, heads, table.shape[1] * page), generator=g)
    check_attend(kb, q, k, v, table, n, weights=True, weight_in=w)
    check_attend(kb, q, k, v, table, n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("R,q_heads,heads", [(600, 4, 4), (300, 20, 10), (1025, 6, 6)])
def test_weights_of_many_heads(kb, dtype, R, q_heads, heads):
    """A block of the second launch takes its row's slots in several turns."""
    g = torch.Generator().manual_seed(R)
    k, v, table, n = batch(g, dtype, R, heads, 16, 8, 10, 4)
    q = torch.randn((R, q_heads, 16), generator=g).to(dtype)
    check_attend(kb, q, k, v, table, n, weights=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("q_heads,heads,dim,rot", [(64, 8, 256, 256), (120, 16, 128, 128), (96, 96, 192, 96)])
def test_append_of_many_heads(kb, dtype, pairs, q_heads, heads, dim, rot):
    """More than 1,024 pieces a row."""
    g = torch.Generator().manual_seed(q_heads)
    R, page, cap = 3, 4, 12
    k_cache, v_cache, table = make_cache(g, dtype, R, heads, dim, page, cap, dirty=False)
    x = torch.randn((R, q_heads + 2 * heads, dim), generator=g).to(dtype)
    length = torch.tensor([1, 12, 7], dtype=torch.int32)
    pos = torch.tensor([0, 5000, 6], dtype=torch.int32)
    freq = kb.rotary_frequencies(rot, device="cpu")
    q, k, v = x.split([q_heads, heads, heads], 1)
    dk, dv, dx = k_cache.cuda(), v_cache.cuda(), x.cuda()
    dq, dkn, dvn = dx.split([q_heads, heads, heads], 1)
    out = kb.cache_append(dk, dv, table.cuda(), length.cuda(), dkn, dvn, q=dq, pos=pos.cuda(), freq=freq.cuda(),
                          interleaved=pairs)
    torch.cuda.synchronize()
    ref = co.append(f64(k_cache), f64(v_cache), table.numpy(), length.numpy(), f64(k), f64(v), q=f64(q),
                    pos=pos.numpy(), freq=freq.numpy(), interleaved=pairs)
    # a turned pair is within 2^-21 + 3 * 2^-53 |pos| of |x| + |y|, and rounded once
    big = (2.0 ** -21 + 3 * 2.0 ** -53 * 5000) * 2 * float(x.abs().max())
    for got, want in ((out, ref[0]), (dk, ref[1])):
        assert np.all(np.abs(f64(got) - want) <= ROUND[dtype] * np.abs(want) + big)
    assert np.array_equal(f64(dv), ref[2])
    assert np.array_equal(f64(out)[..., rot:], f64(q)[..., rot:])


@pytest.mark.parametrize("cap,keep", [(2500, 2100), (40000, 3000)])
def test_long_evictions_in_a_graph(kb, cap, keep):
    """Caches whose keys take more than 64 KB of LDS, or none of it: captured once, replayed over other weights."""
    g = torch.Generator().manual_seed(cap)
    R, heads, page = 3, 2, 64
    k, v, table = (x.cuda() for x in make_cache(g, torch.bfloat16, R, heads, 64, page, cap, dirty=False))
    slots = table.shape[1] * page
    n = torch.tensor([cap, keep + 1, keep - 1], dtype=torch.int32, device="cuda")
    w = torch.rand((R, heads, slots), generator=g).cuda()

    def results():
        return (torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros((R, heads, slots), device="cuda"), None,
                torch.zeros((R, heads, keep), dtype=torch.int32, device="cuda"))
    kk, vv, out = k.clone(), v.clone(), results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kb.cache_evict(kk, vv, table, n, keep, weight=w, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kb.cache_evict(kk, vv, table, n, keep, weight=w, out=out)
    for i in range(5):
        w.copy_(torch.rand((R, heads, slots), generator=g))
        kk.copy_(k), vv.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        k2, v2, want = k.clone(), v.clone(), results()
        want[1].copy_(out[1])                      # places from n on are left as they were
        kb.cache_evict(k2, v2, table, n, keep, weight=w, out=want)
        torch.cuda.synchronize()
        assert np.array_equal(bits(kk), bits(k2)) and np.array_equal(bits(vv), bits(v2)), f"replay {i}"
        for a, b in ((out[0], want[0]), (out[1], want[1]), (out[3], want[3])):
            assert np.array_equal(host(a), host(b)), f"replay {i}"
