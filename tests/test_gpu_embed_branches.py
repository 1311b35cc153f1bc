"""Further branches of the embeddings' gradient: added to another one on every path, and few ids into tables of which a wave has several rows."""
import numpy as np
import pytest
import torch

from oracle import recurrent as R
from rows_util import U, close, matrix, rounded, values
from test_gpu_embed_sorted import gradient, ids_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["words", "all equal", "outside", "none"])
@pytest.mark.parametrize("n", [1, 65, 256, 257, 9001, 20000])
@pytest.mark.parametrize("large", [False, True])             # a table of fewer and of more than twice as many rows as there are ids
def test_added_to_another(n, large, kind, dtype):
    d, v, scale = 21, 2 * n + 37 if large else max(1, n // 3), 0.7
    rng = np.random.default_rng(n + large)
    ids, a, before = ids_of(kind, n, v, rng), rounded(rng.standard_normal((n, d)), dtype), rng.standard_normal((v, d)).astype(np.float32)
    want, bound = R.embed_scaled_bwd(ids, a, v, np.float32(scale))
    got = gradient(ids, matrix(a, dtype), v, scale, accumulate=True, before=before)
    # (one rounding for the product and the sum)
    close(values(got), want + before, bound + U * (np.abs(want + before) + bound))
    none = np.bincount(ids[(ids >= 0) & (ids < v)], minlength=v) == 0
    assert np.array_equal(values(got)[none], before[none])
    again = gradient(ids, matrix(a, dtype, 3, 1), v, scale, accumulate=True, before=before, pad=5, shift=3, stride=2, dtype=torch.int32)
    assert torch.equal(again, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["words", "all equal", "outside", "even"])
@pytest.mark.parametrize("n,d,v", [(1, 650, 10000), (256, 5, 40001), (200, 3, 300007), (130, 700, 16389), (0, 9, 70001)])
def test_few_ids_into_large_tables(n, d, v, kind, dtype):
    E = 4 if dtype == "f32" else 8
    chunks = -(-d // (64 * E))
    rows = min(16, max(1, v * chunks // 8192))
    assert rows > 1 and (v % rows or v == 10000)             # several rows to a wave, the last wave with fewer
    rng = np.random.default_rng(n)
    ids, a = ids_of(kind, n, v, rng), rounded(rng.standard_normal((n, d)), dtype)
    if n:
        ids[-1] = v - 1
    want, bound = R.embed_scaled_bwd(ids, a, v, np.float32(2.5))
    got = gradient(ids, matrix(a, dtype), v, 2.5)
    close(values(got), want, bound)
    before = rng.standard_normal((v, d)).astype(np.float32)
    more = gradient(ids, matrix(a, dtype), v, 2.5, accumulate=True, before=before)
    close(values(more), want + before, bound + U * (np.abs(want + before) + bound))
