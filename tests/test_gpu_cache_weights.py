"""Weights of attention whose slots all have one score, large against 1: each is one part of its row's slots, to the
rounding of that, by every path of the pass (a wave or a workgroup a row, equal shares, splits) and both of the join."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1805_09863_amd as kb
    kb.lib()
    return kb


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("value", [2.71, -3.3])
@pytest.mark.parametrize("R,q_heads,heads,dim,page,most", [
    (3, 4, 2, 64, 16, 1), (3, 6, 2, 80, 4, 300), (600, 4, 2, 64, 1, 40), (5, 40, 2, 64, 16, 3000), (1, 8, 1, 128, 64, 9000),
    (1030, 2, 1, 16, 8, 1500), (1100, 1, 1, 8, 16, 2100),
])
def test_equal_scores(kb, dtype, value, R, q_heads, heads, dim, page, most):
    g = torch.Generator().manual_seed(R + most)
    cols = -(-most // page)
    n = torch.randint(1, most + 1, (R,), generator=g).to(torch.int32)
    n[0] = most
    q = torch.full((R, q_heads, dim), value).to(dtype).cuda()
    k = torch.full((R * cols, heads, page, dim), 9.1).to(dtype).cuda()   # scores of about 200 to 290 and below 0
    v = torch.randn(k.shape, generator=g).to(dtype).cuda()
    table = torch.randperm(R * cols, generator=g).to(torch.int32).view(R, cols).cuda()
    w = torch.full((R, heads, cols * page), -1.0, device="cuda")
    kb.cache_attend(q, k, v, table, n.cuda(), weight_out=w)
    torch.cuda.synchronize()
    group = q_heads // heads
    slot = torch.arange(cols * page)
    seen = (slot < n[:, None])[:, None].expand(-1, heads, -1)
    want = (group / n.double())[:, None, None].expand(seen.shape)
    # exponentials of 0 are 1 and sums of ones exact: a reciprocal's rounding, and one a head that is added
    err = (w.cpu().double() - want).abs()[seen] / want[seen]
    assert float(err.max()) <= (group + 1) * U, float(err.max()) / U
    assert bool((w.cpu()[~seen] == -1).all())
