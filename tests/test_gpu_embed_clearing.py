"""The embeddings' gradient on both sides of the limits from which a table is cleared beside the sort: every row is written, whoever does it."""
import numpy as np
import pytest

from oracle import recurrent as R
from rows_util import close, matrix, rounded, values
from test_gpu_embed_sorted import gradient, ids_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["words", "even", "outside"])
@pytest.mark.parametrize("n,d,v", [(9000, 5, 17999), (9000, 5, 18000), (9000, 5, 71999), (9000, 5, 72000), (2 ** 15, 3, 2 ** 18), (2 ** 15 + 1, 3, 2 ** 18 + 8), (8200, 2048, 2 ** 16 - 1), (8200, 2048, 2 ** 16)])
def test_both_sides(n, d, v, kind, dtype):
    rng = np.random.default_rng(n)
    ids = ids_of(kind, n, v, rng)
    if d < 100:
        a = rounded(rng.standard_normal((n, d)), dtype)
        want, bound = R.embed_scaled_bwd(ids, a, v, np.float32(0.7))
        close(values(gradient(ids, matrix(a, dtype), v, 0.7)), want, bound)
    else:                                                # (the same four columns many times over)
        a = rounded(rng.standard_normal((n, 4)), dtype)
        want, bound = R.embed_scaled_bwd(ids, a, v, np.float32(0.7))
        got = gradient(ids, matrix(np.tile(a, d // 4), dtype), v, 0.7)
        assert bool((got.view(v, d // 4, 4) == got[:, None, :4]).all())
        close(values(got[:, :4]), want, bound)
