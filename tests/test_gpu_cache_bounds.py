"""The attention cache on the GPU at the ends of its arguments' ranges, and with memory laid out otherwise than it
asks for."""
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


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("page", [1, 16])
@pytest.mark.parametrize("turned", [True, False])
def test_append_stores_no_token_without_a_slot(kb, dtype, page, turned):
    """Lengths of none, below none and past the table, to the ends of int32: queries are turned, nothing is stored."""
    lengths = [0, -1, -3, -2 ** 31, -2 ** 31 + 1, 33, 2 ** 31 - 1, 5]
    R, heads, dim, cap = len(lengths), 2, 64, 32
    g = torch.Generator().manual_seed(page)
    x = torch.randn((R, 4 + 2 * heads, dim), generator=g).to(dtype).cuda()
    q, k, v = x.split([4, heads, heads], 1)
    table = torch.arange(R * cap // page, dtype=torch.int32, device="cuda").view(R, -1)
    kc, vc = (torch.full((R * cap // page, heads, page, dim), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    position = torch.full((R, heads, cap), -9, dtype=torch.int32, device="cuda")
    weight = torch.full((R, heads, cap), 5.0, device="cuda")
    more = dict(pos=i32(*range(R)), freq=torch.zeros(dim // 2, dtype=torch.float64, device="cuda")) if turned else {}
    out = kb.cache_append(kc, vc, table, i32(*lengths), k, v, q=q, position=position, weight=weight, **more)
    torch.cuda.synchronize()
    assert torch.equal(out, q)                       # angles of 0
    at = table[R - 1].long()[4 // page]
    assert torch.equal(kc[at, :, 4 % page], k[R - 1]) and torch.equal(vc[at, :, 4 % page], v[R - 1])
    kc[at, :, 4 % page] = vc[at, :, 4 % page] = 3
    assert bool((kc == 3).all()) and bool((vc == 3).all())
    assert bool((position[R - 1, :, 4] == (R - 1 if turned else 4)).all()) and bool((weight[R - 1, :, 4] == 0).all())
    position[R - 1, :, 4], weight[R - 1, :, 4] = -9, 5
    assert bool((position == -9).all()) and bool((weight == 5).all())


def test_weights_of_another_row_length_are_refused(kb):
    """A table of 50 slots and weights of 64 a row: refused, not addressed at 50; flat memory is taken as it lies."""
    R, heads, dim, page, cols = 3, 2, 32, 2, 25
    k, v = (torch.randn(R * cols, heads, page, dim, device="cuda") for _ in range(2))
    table = torch.arange(R * cols, dtype=torch.int32, device="cuda").view(R, cols)
    n = i32(50, 7, 33)
    q = torch.randn(R, 4, dim, device="cuda")
    want = torch.zeros(R, heads, 50, device="cuda")
    kb.cache_attend(q, k, v, table, n, weight_out=want)
    with pytest.raises(ValueError, match="rows of 2 x 50"):
        kb.cache_attend(q, k, v, table, n, weight_out=torch.zeros(R, heads, 64, device="cuda"))
    with pytest.raises(ValueError, match="rows of 2 x 50"):
        kb.cache_evict(k, v, table, n, 10, weight=torch.zeros(R, heads, 64, device="cuda"))
    for shape in ((R * heads * 50 + 3,), (R, heads, cols, page), (R * heads, 50)):
        got = torch.zeros(shape, device="cuda")
        kb.cache_attend(q, k, v, table, n, weight_out=got)
        assert torch.equal(got.flatten()[:R * heads * 50], want.flatten())


def test_an_evictions_own_results_under_another_default_type(kb):
    k, v = (torch.randn(6, 1, 4, 16, device="cuda") for _ in range(2))
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    w = torch.rand(2, 1, 12, device="cuda")
    want = w.topk(5).values.sort().values
    torch.set_default_dtype(torch.float64)
    try:
        n, weight, position, source = kb.cache_evict(k, v, table, i32(12, 12), 5, weight=w)
    finally:
        torch.set_default_dtype(torch.float32)
    assert n.tolist() == [5, 5] and position is None and weight.dtype == torch.float32
    assert torch.equal(weight[:, :, :5].sort().values, want)
