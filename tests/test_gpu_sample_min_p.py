"""Sampled tokens whose weight is next to min_p: the same ones are kept, whichever way a row goes."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_1908_00213_amd import binding as B

pytestmark = pytest.mark.gpu

# (logit below a largest one of 0, temperature, min_p, whether the weight exp(logit / temperature) is at least min_p).  The weights are
# 2e-14 to 1.1e-13 of themselves away from min_p: far more than the 1e-15 that an exponential in 64 bits is off by, and
# less than the 2e-13 by which the exponential that sums are made of may be.
NEAR = [(*map(float.fromhex, c[:3]), c[3]) for c in [
        ("-0x1.17262ap-3", "0x1.6bdbdap+0", "0x1.d12e3ep-1", True), ("-0x1.9f2becp-5", "0x1.12486ap-2", "0x1.a7bd18p-1", False),
        ("-0x1.9f69b4p-4", "0x1.56f3cep+0", "0x1.daab76p-1", False), ("-0x1.75d634p-5", "0x1.dcea1ep-1", "0x1.e78556p-1", True),
        ("-0x1.a34bep-1", "0x1.c5a00ep+0", "0x1.4284fp-1", True), ("-0x1.cc5666p-4", "0x1.e197b6p-1", "0x1.c6568ap-1", True),
        ("-0x1.9fc502p-5", "0x1.d0b13p-1", "0x1.e4279ep-1", False), ("-0x1.ea8ba8p-3", "0x1.31e536p+0", "0x1.a2ffe2p-1", True),
        ("-0x1.d01edp-1", "0x1.37732ep+0", "0x1.e614c4p-2", True), ("-0x1.5eb6dcp-4", "0x1.74826p+0", "0x1.e2bdd6p-1", False),
        ("-0x1.c8a18ep-2", "0x1.cade14p+0", "0x1.8f3b6ep-1", False), ("-0x1.4abf3ep-2", "0x1.f29ea4p+0", "0x1.b1c2c6p-1", False),
        ("-0x1.58be02p+0", "0x1.809de4p+0", "0x1.a1dc08p-2", True), ("-0x1.384af2p+1", "0x1.94b616p+0", "0x1.b59ca2p-3", True)]]


def vec(a, dtype=np.float32):
    return torch.from_numpy(np.asarray(a, dtype)).cuda()


def draw(z, u, ws=True, **params):
    out = torch.full((z.shape[0],), -7, device="cuda", dtype=torch.int64)
    w = torch.empty(max(256, B.sample_workspace_bytes(z)), dtype=torch.uint8, device="cuda").fill_(0xA5) if ws else None
    B.sample(z, u, out, ws=w, **params)
    return out.cpu().numpy()


@pytest.mark.parametrize("v", [9, 256, 300, 5000, 40000])
@pytest.mark.parametrize("more", [{}, {"top_k": 5}, {"top_p": 0.9999}, {"top_k": 5, "top_p": 0.9999}])
def test_min_p_is_decided_in_64_bits_on_every_path(v, more):
    n = len(NEAR)
    z = np.full((n, v), -60.0, np.float32)
    z[:, 2] = 0.0
    z[:, v - 2] = [c[0] for c in NEAR]
    params = dict(temperature=vec([c[1] for c in NEAR]), min_p=vec([c[2] for c in NEAR]))
    params.update({k: vec([q] * n, np.int32 if k == "top_k" else np.float32) for k, q in more.items()})
    want = np.where([c[3] for c in NEAR], v - 2, 2)      # the last token that is kept, as u is next to 1
    for u in (1.0 - 2.0 ** -24, 1.0):                    # (a sum, and the end of the range)
        u = np.full(n, u, np.float32)
        assert np.array_equal(R.sample(z, u, *(None if params.get(k) is None else params[k].cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p"))), want)
        for ws in (True, False):
            assert np.array_equal(draw(vec(z), vec(u), ws, **params), want), (ws, u[0])
