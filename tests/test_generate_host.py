"""What LSTMLanguageModel.generate takes for its parameters, without a GPU."""
import numpy as np
import pytest

from paper_1908_00213_amd import tape as T
from rows_backend import RowsBackend
from test_tape_rows_host import lm_params


class Own(np.ndarray):
    """An array of the backend's own: what its kernels take, as the GPU's take no NumPy."""


class Strict(RowsBackend):
    def from_numpy(self, a, dtype=None):
        return super().from_numpy(a, dtype).view(Own)

    def sample(self, logits, u, out, temperature=None, top_k=None, top_p=None, min_p=None):
        for p in (temperature, top_k, top_p, min_p):
            assert p is None or isinstance(p, Own) and p.shape == u.shape
        super().sample(logits, u, out, temperature, top_k, top_p, min_p)


def model_of():
    return T.LSTMLanguageModel(lm_params(np.random.default_rng(6)), n_step=True)


FORMS = [np.float32, np.float64, float, lambda v: np.array(v), lambda v: np.full(3, v), lambda v: [v] * 3, lambda v: (v,) * 3, lambda v: np.array([v])]


@pytest.mark.parametrize("form", FORMS)
def test_numbers_and_vectors_of_every_kind(form):
    rng = np.random.default_rng(1)
    prompt, u = rng.integers(0, 11, 12), rng.random((4, 3))
    with T.using_backend(Strict()) as F:
        model = model_of()
        want, _ = model.generate(prompt, 4, u, temperature=0.8, top_k=5, top_p=0.9, min_p=0.05)
        got, _ = model.generate(prompt, 4, u, temperature=form(0.8), top_k=5, top_p=form(0.9), min_p=form(0.05))
        assert np.array_equal(got, want)
        for k in (np.int32(5), np.array(5), np.full(3, 5, np.int32), [5, 5, 5]):
            assert np.array_equal(model.generate(prompt, 4, u, temperature=0.8, top_k=k, top_p=0.9, min_p=0.05)[0], want)
        own = F.from_numpy(np.array([0.8, 0.8, 0.8], np.float32))
        assert np.array_equal(model.generate(prompt, 4, u, temperature=own, top_k=5, top_p=0.9, min_p=0.05)[0], want)


def test_vectors_that_do_not_fit_are_refused():
    with T.using_backend(Strict()):
        model = model_of()
        for bad in (np.full(2, 0.5), [0.5] * 4, np.full((3, 1), 0.5)):
            with pytest.raises(ValueError):
                model.generate(np.zeros(12, np.int64), 4, np.zeros((2, 3)), temperature=bad)
