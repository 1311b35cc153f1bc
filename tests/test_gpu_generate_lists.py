"""Lists of biases and masks that `generate` takes as arrays on the device, of both ranks and types."""
import numpy as np
import pytest
import torch

from paper_1908_00213_amd import tape as T
from recurrent_backend import gated_params

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("penalty", [{}, {"repetition": 1.3, "presence": 0.25}])
@pytest.mark.parametrize("ids_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("rank", [1, 2])
def test_arrays_on_the_device(rank, ids_type, penalty):
    F = T.backend()
    rng = np.random.default_rng(4)
    n, Bn, V, more = 4, 5, 300, 6
    P = {k: F.from_numpy(np.float32(v)) for k, v in gated_params(rng, V, 24).items()}
    ids, u = F.from_numpy(rng.integers(0, V, n * Bn)), F.from_numpy(rng.random((more, Bn), dtype=np.float32))
    lists = {"bias_ids": np.arange(40) * 7, "bias": np.float32(3 * rng.standard_normal(40)), "allowed": rng.integers(-2 ** 31, 2 ** 31, (V + 31) // 32).astype(np.int32)}
    model = T.GatedLanguageModel(P)
    want, _ = model.generate(ids, n, u, **lists, **penalty)
    device = {k: F.from_numpy(v if rank == 1 else np.tile(v, (Bn, 1))) for k, v in lists.items()}
    device["bias_ids"] = device["bias_ids"].to(ids_type)
    got, _ = model.generate(ids, n, u, **device, **penalty)
    assert torch.equal(got, want)
    got, _ = model.generate(ids, n, u, **dict(lists, bias_ids=device["bias_ids"]), **penalty)
    assert torch.equal(got, want)
