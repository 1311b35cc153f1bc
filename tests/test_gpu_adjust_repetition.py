"""Repetitions at the ends of fp32's range."""
import numpy as np
import pytest

from test_gpu_logits_adjust import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("v", [9, 300, 40000])
def test_tiny_and_huge_repetitions(v):
    """Quotients of a logit and a repetition whose reciprocal, or whose product with the logit, is out of range where the quotient is not."""
    r = np.array([1e-45, 1e-39, 2.9e-39, 3e-39, 1e-38, 1e-30, 1.0, 1e30, 8e37, 3.4e38], np.float32)
    z = np.tile(np.array([1e-3, -1e-3, 0.0, 2.0 ** -20, 1.0, -5.0, 1e-12, 3.0, 100.0]), (len(r), -(-v // 9)))[:, :v].astype(np.float32)
    wide = z.astype(np.float64)
    result = np.abs(np.where(z > 0, wide / r[:, None], wide * r[:, None]))
    z[(result < 2.0 ** -126) | (result > 3e38)] = 0.0        # (results in the normal range, of which the bound is a part)
    assert (z[1] != 0).any() and (z[-1] != 0).any()
    tokens = np.tile(np.arange(v), (len(r), 1))
    check(z, tokens=tokens, repetition=r)
