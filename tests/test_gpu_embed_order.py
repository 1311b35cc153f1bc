"""The order in which the rows of a token are added, by the bits of the sums."""
import numpy as np
import pytest
import torch

from rows_util import matrix, rounded, values
from test_gpu_embed_sorted import gradient, ids_of

pytestmark = pytest.mark.gpu


def in_order(ids, a, v, scale):
    """fp32 sums of a token's rows one after the other, then the scale."""
    g = np.zeros((v, a.shape[1]), np.float32)
    for i, row in zip(ids, a.astype(np.float32)):
        if 0 <= i < v:
            g[i] += row
    return g * np.float32(scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["words", "all equal", "outside", "even"])
@pytest.mark.parametrize("n,d,v", [(2, 1, 3), (65, 3, 5), (129, 33, 9), (200, 650, 30), (256, 70, 40), (256, 8, 3)])
def test_few_ids(n, d, v, kind, dtype):
    rng = np.random.default_rng(n)
    ids, a = ids_of(kind, n, v, rng), rounded(rng.standard_normal((n, d)) * 10.0 ** rng.integers(-3, 4, (n, 1)), dtype)
    assert np.array_equal(values(gradient(ids, matrix(a, dtype), v, 0.7)), in_order(ids, a, v, 0.7))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,v,more", [(256, 70, 40, 1), (100, 33, 9, 157), (256, 650, 40, 8000), (256, 66, 40, 9000)])
def test_ids_of_padding_change_nothing(n, d, v, more, dtype):
    """Tokens with up to 64 rows each: alike without a sort, sorted by one block and sorted by several."""
    rng = np.random.default_rng(n + more)
    ids, a = np.concatenate([rng.integers(0, v, n), np.full(more, -1)]), rounded(rng.standard_normal((n + more, d)) * 10.0 ** rng.integers(-3, 4, (n + more, 1)), dtype)
    assert np.bincount(ids[:n]).max() <= 64
    got = gradient(ids, matrix(a, dtype), v, 0.7)
    assert torch.equal(gradient(ids[:n], matrix(a[:n], dtype), v, 0.7), got)
    assert np.array_equal(values(got), in_order(ids, a, v, 0.7))
