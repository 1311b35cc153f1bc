"""LSTMLanguageModel.generate on the GPU: the same tokens by numbers and vectors of every kind."""
import numpy as np
import pytest
import torch

from paper_1908_00213_amd import tape as T
from paper_1908_00213_amd import workloads as W

pytestmark = pytest.mark.gpu


def test_numbers_and_vectors_of_every_kind():
    F = T.backend()
    w = W.config4(vocab=500, embed=64, hidden=64, batch=12, bptt=5)
    model = T.LSTMLanguageModel({k: F.from_numpy(v) for k, v in w.params.items()}, n_step=True)
    ids, u = F.from_numpy(w.ids.reshape(-1)), F.from_numpy(np.random.default_rng(9).random((5, 12), dtype=np.float32))
    want, _ = model.generate(ids, w.bptt, u, temperature=0.8, top_k=20, top_p=0.9, min_p=0.01)
    for f, i in ((np.float32, np.int32), (np.float64, np.int64), (np.array, np.array), (lambda v: np.full(12, v), lambda v: np.full(12, v, np.int32)), (lambda v: [v] * 12, lambda v: [v] * 12),
                 (lambda v: torch.full((12,), v, device="cuda"), lambda v: torch.full((12,), v, device="cuda", dtype=torch.int32))):
        got, _ = model.generate(ids, w.bptt, u, temperature=f(0.8), top_k=i(20), top_p=f(0.9), min_p=f(0.01))
        assert torch.equal(got, want)
    with pytest.raises(ValueError):
        model.generate(ids, w.bptt, u, temperature=[0.5] * 11)
