"""What LSTMLanguageModel.generate leaves of its model, without a GPU."""
import numpy as np

from paper_1908_00213_amd import tape as T
from rows_backend import RowsBackend
from test_tape_rows_host import lm_params


class Watch(RowsBackend):
    def sample(self, *args):
        self.seen = self.model.train
        super().sample(*args)


def test_a_model_that_trains_meanwhile_sees_no_change():
    rng = np.random.default_rng(2)
    with T.using_backend(Watch()) as F:
        F.model = model = T.LSTMLanguageModel(lm_params(np.random.default_rng(6)), n_step=True, ratio=0.5, masks=T.Masks(3))
        sites = model.masks.sites
        a, _ = model.generate(rng.integers(0, 11, 12), 4, rng.random((3, 3)), top_k=4)
        assert F.seen is True and model.train is True                # never switched, not even inside
        assert model.masks.sites == sites and "dropout" not in [c[0] for c in F.calls]
