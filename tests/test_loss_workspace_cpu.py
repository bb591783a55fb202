"""What the workspaces of the output layer's losses promise, without a GPU: one for the most rows serves all smaller
batches, and it grows no faster than the header says.  Nothing is launched: the calls lack a result or an input, which they
find after they have looked at the workspace."""
import random

import pytest

from paper_1805_09863_amd import binding

INVALID, WORKSPACE = 1, 3
BASE = 1 << 20
MiB = 1 << 20


@pytest.fixture(scope="module")
def L():
    if not binding.os.path.exists(binding.LIB_PATH):
        pytest.skip("libkbest.so is not built")
    return binding.lib()


def rows(rng, most):
    """Every batch up to 600, then some of each size."""
    n = 0
    while n < most:
        n = n + 1 if n < 600 else n + rng.randint(1, n // 40)
        yield min(n, most)


# layers of the sizes that users have, odd ones, and the largest
LAYERS = [(0, 512, 30000, 1), (1, 1024, 90000, 1), (1, 512, 32001, 8), (0, 297, 106808, 1), (1, 942, 43623, 2), (0, 64, 8, 12),
          (1, 256, 500, 128), (0, 1024, 60000, 1), (1, 3000, 262144, 1), (0, 65536, 1000, 4)]


@pytest.mark.parametrize("dtype,H,V,K", LAYERS)
def test_more_rows_never_take_less(L, dtype, H, V, K):
    rng = random.Random(H + V)
    for f in (L.kb_loss_workspace_bytes, L.kb_loss_grad_workspace_bytes):
        last = 0
        for N in rows(rng, 20000):
            size = f(dtype, N, H, V, K)
            assert size >= last, f"{f.__name__}: {N} rows take {size}, {last} with fewer"
            last = size
        # whatever was asked for before: the same
        some = [(N, f(dtype, N, H, V, K)) for N in (17, 20000, 5, 640, 4097)]
        f(1 - dtype, 100, H, V, K)
        assert some == [(N, f(dtype, N, H, V, K)) for N, _ in some]


@pytest.mark.parametrize("dtype,H,V,K", LAYERS)
def test_the_largest_batchs_workspace_serves_all(L, dtype, H, V, K):
    rng = random.Random(H + V + 1)
    most = 9000
    score, grad = L.kb_loss_workspace_bytes(dtype, most, H, V, K), L.kb_loss_grad_workspace_bytes(dtype, most, H, V, K)
    for N in rows(rng, most):
        for W in (BASE, BASE + 4):   # aligned to 16 bytes and not
            head = (dtype, N, H, V)
            got = [L.kb_distill(*head, K, BASE, W, BASE, BASE, BASE, 1.0, None, None, BASE, score, None),
                   L.kb_distill_grad(*head, K, BASE, W, BASE, BASE, BASE, 1.0, None, None, BASE, BASE, BASE, BASE, grad, None)]
            if K == 1:
                got += [L.kb_cross_entropy(*head, BASE, W, BASE, BASE, 0.1, None, None, BASE, score, None),
                        L.kb_cross_entropy_grad(*head, BASE, W, BASE, BASE, 0.1, None, None, BASE, BASE, BASE, BASE, grad, None)]
            assert got == [INVALID] * len(got), f"{N} rows: {got}, {L.kb_last_error().decode()}"
            # and the batch's own is looked at
            assert L.kb_distill(*head, K, BASE, W, BASE, BASE, BASE, 1.0, BASE, BASE, BASE, 0, None) == WORKSPACE


def test_growth(L):
    """The header's terms, for rows rounded up to the next step (a 32nd or 32 of them more) and a tile (255 more); the
    states' and words' numbers to 256.  Beside them: lists and maps of the rows, at most 768 + 341 parts of a gradient's
    tiles of 256 KiB, the scores' statistics (12 bytes for every row of a round's tiles, 65,536 at least, and piece)."""
    rng = random.Random(5)
    for _ in range(3000):
        dtype, K = rng.randint(0, 1), rng.choice([1, 1, 5, 128])
        H, V = int(10 ** rng.uniform(0, 4.8)), int(10 ** rng.uniform(0, 5.41))
        N = int(10 ** rng.uniform(0, 6.6))
        n, Hp, Vp = N * 33 // 32 + 32 + 255, (H + 255) // 256 * 256, (V + 255) // 256 * 256
        planes = 3 if dtype == 0 else 1
        both = n * Hp * 2 * planes + n * (24 * K + 64) + n * Vp // 512 + 4 * Vp + 8192
        piece_w, piece_g = (max(256 * MiB, 512 * planes * (rows_ + 31)) for rows_ in (H, n))
        pieces = 1 + Vp // 256 // max(1, (4 if dtype else 64) * MiB // (512 * planes * (H + 31)))
        few = 512 * 8 * 4 * (H + 4 + K)  # at most eight rows: 512 workgroups' parts
        score, grad = L.kb_loss_workspace_bytes(dtype, N, H, V, K), L.kb_loss_grad_workspace_bytes(dtype, N, H, V, K)
        assert score <= both + piece_w + pieces * 12 * max(65536, n) + few, (dtype, N, H, V, K)
        assert grad <= both + 4 * n * Hp + n * Vp // 8 + piece_w + piece_g + (768 + 341) * 256 * 1024 + few, (dtype, N, H, V, K)
