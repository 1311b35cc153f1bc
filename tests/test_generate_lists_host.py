"""Lists of biases and masks that `generate` takes as arrays of the backend's, which are no NumPy arrays, without a GPU."""
import numpy as np
import pytest
import torch

from paper_1908_00213_amd import tape as T
from recurrent_backend import RecurrentBackend, gated_params


class ListsBackend(RecurrentBackend):
    """Looks at what reaches the entry point: lists of a row for each sequence, tokens and biases' ids of one type."""

    def logits_adjust(self, logits, out, **k):
        for name in ("bias_ids", "bias", "allowed"):
            if k.get(name) is not None:
                assert len(k[name].shape) == 2 and k[name].shape[0] == logits.shape[0], name
                k[name] = np.asarray(k[name])
        if k.get("tokens") is not None and k.get("bias_ids") is not None:
            assert k["tokens"].dtype == k["bias_ids"].dtype
        super().logits_adjust(logits, out, **k)


@pytest.mark.parametrize("penalty", [{}, {"repetition": 1.3}])
@pytest.mark.parametrize("ids_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("ranks", [(1, 1, 1), (2, 2, 2), (1, 2, 1), (2, 1, 2)])
def test_arrays_of_the_backend(ranks, ids_type, penalty):
    rng = np.random.default_rng(4)
    n, Bn, V, more = 4, 3, 11, 6
    ids, u = rng.integers(0, V, n * Bn), rng.random((more, Bn))
    lists = {"bias_ids": np.array([2, 7, 2]), "bias": np.array([0.5, -2.0, 0.25]), "allowed": np.array([0b11111011111], np.int32)}
    types = {"bias_ids": ids_type, "bias": torch.float64, "allowed": torch.int32}
    with T.using_backend(ListsBackend()):
        model = T.GatedLanguageModel(gated_params(rng))
        want, _ = model.generate(ids, n, u, **lists, **penalty)
        device = {k: torch.from_numpy(v if r == 1 else np.tile(v, (Bn, 1))).to(types[k]) for (k, v), r in zip(lists.items(), ranks)}
        got, _ = model.generate(ids, n, u, **device, **penalty)
        assert np.array_equal(got, want) and (got != 5).all()


@pytest.mark.parametrize("penalty", [{}, {"repetition": 1.3}])
def test_lists_of_other_shapes_reach_the_entry_point_as_they_are(penalty):
    """Which refuses them: ids of (2 B, M) are not those of (B, 2 M)."""
    rng = np.random.default_rng(4)
    n, Bn, V = 4, 2, 11
    seen = []

    class Backend(RecurrentBackend):
        def logits_adjust(self, logits, out, **k):
            seen.append(tuple(k["bias_ids"].shape))
            raise ValueError("refused")
    for shape in ((4, 3), (1, 4), (2, 3, 1)):
        with T.using_backend(Backend()):
            model = T.GatedLanguageModel(gated_params(rng))
            with pytest.raises(ValueError, match="refused"):
                model.generate(rng.integers(0, V, n * Bn), n, rng.random((1, Bn)), bias_ids=torch.zeros(shape, dtype=torch.int64), bias=torch.zeros(2, 6), **penalty)
        assert seen.pop() == shape
