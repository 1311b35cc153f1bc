"""Residual blocks on the tape that are handed gradients of another type than their arrays', on the GPU against the oracle's kernels in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1908_00213_amd import tape as T
from test_gpu_tape_norm_views import C, N, arrays, both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["y", "s", "both"])
def test_residual_norm_takes_gradients_of_another_type(which):
    """A function that hands fp32 gradients to its bfloat16 input, behind either output of a block in bfloat16."""
    def run(F):
        x, res, w, ws, gamma, beta = arrays(6, (N, C), (N, C), (N, C), (N, C), (C,), (C,))
        rnd = lambda a: torch.from_numpy(a).bfloat16().float().numpy()
        low = lambda a: T.Variable(F.from_numpy(rnd(a), "bf16"))
        xv, rv = low(x), low(res)
        gv, bv = T.Variable(F.from_numpy(gamma)), T.Variable(F.from_numpy(beta))
        y, s = T.residual_norm(xv, rv, gv, bv)
        parts = []
        for v, f, name in ((y, w, "y"), (s, ws, "s")):
            if which in (name, "both"):
                wide = T.dropout(v, 0.0, out_dtype="f32", gx_dtype="f32")
                parts.append(T.sum_all(T.mul(wide, T.Variable(F.from_numpy(rnd(f)), False))))
        (parts[0] if len(parts) == 1 else T.add(*parts)).backward()
        return [xv.grad, rv.grad] + ([gv.grad, bv.grad] if which != "s" else [])
    # stored in bfloat16: the sum, which is normalised, and each gradient
    both(run, 4 * 2.0 ** -8)
