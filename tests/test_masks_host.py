"""Seeds of every kind that name 64 bits, without a GPU."""
import numpy as np
import pytest

from paper_1908_00213_amd import tape as T
from rows_backend import RowsBackend


@pytest.mark.parametrize("seed,bits", [(5, 5), (-1, 2 ** 64 - 1), (2 ** 64 - 1, 2 ** 64 - 1), (2 ** 63, 2 ** 63), (np.int64(5), 5), (np.int64(-7), 2 ** 64 - 7), (np.int32(-7), 2 ** 64 - 7),
                                       (np.uint64(2 ** 64 - 1), 2 ** 64 - 1), (np.uint32(9), 9), (np.random.default_rng(1).integers(2 ** 62), int(np.random.default_rng(1).integers(2 ** 62)))])
def test_seeds(seed, bits):
    with T.using_backend(RowsBackend()):
        rng = T.Masks(seed, np.int64(3)).rng
        assert int(rng[0]) % 2 ** 64 == bits and int(rng[1]) == 3
