"""Sampling from rows in chunks: top-k of any size, and vocabularies of more parts than are looked at together."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_1908_00213_amd import binding as B

pytestmark = pytest.mark.gpu


def vec(a, dtype=np.float32):
    return torch.from_numpy(np.asarray(a, dtype)).cuda()


def draw(z, u, ws=True, **params):
    out = torch.full((z.shape[0],), -7, device="cuda", dtype=torch.int64)
    w = torch.empty(max(256, B.sample_workspace_bytes(z)), dtype=torch.uint8, device="cuda").fill_(0xA5) if ws else None
    B.sample(z, u, out, ws=w, **params)
    return out.cpu().numpy()


@pytest.mark.parametrize("v", [32776, 32783, 50257, 70001, 131072, 262144])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_in_chunks_have_as_many_bounds_as_a_block_has_threads(v, dtype):
    """The k-th largest of the extremes that the first launch leaves of a row's parts is what spares a top-k the passes over its row: there are 1024 of
    each kind at the least, and so they serve any k that a block which has the whole row narrows."""
    g = torch.Generator().manual_seed(v)
    z = torch.randn(2, v, generator=g).to(dtype)
    z[z == 0] = 1.0                                      # (a zero that is found is no extreme)
    dev, u = z.cuda(), torch.rand(2, generator=g).cuda()
    ws = torch.empty(B.sample_workspace_bytes(dev), dtype=torch.uint8, device="cuda").fill_(0xA5)
    assert ws.numel() > 0                                # in chunks
    out, k = torch.empty(2, dtype=torch.int64, device="cuda"), torch.tensor([100, 1000], device="cuda", dtype=torch.int32)
    B.sample(dev, u, out, top_k=k, ws=ws)
    assert np.array_equal(out.cpu().numpy(), R.sample(z.float().numpy(), u.cpu().numpy(), None, k.cpu().numpy()))
    for row, part in zip(z.float().numpy(), np.split(ws.cpu().numpy().view(np.float32), 2)):
        assert np.isin(part, row).sum() >= 2 * 1024


@pytest.mark.parametrize("v", [32768, 32771, 32776, 50257, 65541])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_top_k_of_rows_in_chunks(v, dtype):
    """Any k, also where most of a row's parts hold nothing and where the best tokens are neighbours."""
    g = torch.Generator().manual_seed(v)
    n = 12
    z = torch.randn(n, v, generator=g) * 2
    z[1, : v - 100] = -torch.inf                         # what is left lies in a few parts
    z[2, 7:] = float("nan")
    z[3, -5:] += 50.0                                    # the last tokens, behind the last whole unit among them
    z[4, 1000:1300] += 30.0
    z[5, ::2] = -torch.inf
    z = z.to(dtype)
    z[6] = (z[6].float() * 2).round().to(dtype) / 2      # ties
    u = torch.rand(n, generator=g)
    for k in ([64, 80, 65, 129, 100, 1000] * 2, [1, 90, 5, 4, 300, 1024, 513, 1023, 1024, 1025, 2000, v - 1], [128, 128, 7, 6, 301, 257, 255, 256, 511, 512, 33, 2]):
        for p in (None, [0.9] * n):
            params = dict(top_k=vec(k, np.int64), **({} if p is None else {"top_p": vec(p)}))
            want = R.sample(z.float().numpy(), u.numpy(), None, np.array(k), None if p is None else np.asarray(p, np.float32))
            for ws in (True, False):
                assert np.array_equal(draw(z.cuda(), u.cuda(), ws, **params), want), (k, p, ws)


@pytest.mark.parametrize("v", [600001, 1048576])
def test_rows_of_more_parts_than_are_looked_at_together(v):
    """Rows in chunks of more than 2048 parts: greedy, with top-k, with top-p, mixed, the best tokens in the last parts and in the first."""
    g = torch.Generator().manual_seed(v)
    n = 8
    z = torch.randn(n, v, generator=g) * 2
    z[0, v - 1] = z[1, v - 70] = 25.0
    z[1, 3] = 25.0                                       # the first of two equals
    z[2, v - 3000:] += 4.0
    z[3, :10] += 9.0
    z[3, -10:] += 9.0
    z[4, : v // 2] = -torch.inf
    u = torch.rand(n, generator=g)
    dev = z.cuda()
    assert B.sample_workspace_bytes(dev) > 0
    t = np.array([0, 0, 0.8, 1, 0, 1, 1.3, 0.7], np.float32)
    k = np.array([0, 5, 50, 20, 3, 0, 1000, 0], np.int64)
    p = np.array([1, 1, 0.9, 1, 1, 0.8, 0.95, 0.999], np.float32)
    m = np.array([0, 0, 0, 0, 0, 0, 0.01, 0.001], np.float32)
    host = z.numpy()
    for params in (dict(temperature=t), dict(top_k=k), dict(top_p=p), dict(temperature=t, top_k=k, top_p=p, min_p=m)):
        want = R.sample(host, u.numpy(), **params)
        for ws in (True, False):
            assert np.array_equal(draw(dev, u.cuda(), ws, **{q: torch.from_numpy(a).cuda() for q, a in params.items()}), want), (sorted(params), ws)


def test_a_row_that_a_block_holds_in_its_registers_is_not_cut():
    """bfloat16 rows of 32768 tokens are four pieces of 16 bytes a thread, with up to seven tokens behind them; fp32 rows of as many are eight."""
    for v, cut in ((32768, False), (32775, False), (32776, True)):
        assert (B.sample_workspace_bytes(torch.empty(1, v, dtype=torch.bfloat16)) > 0) == cut
        assert B.sample_workspace_bytes(torch.empty(1, v)) > 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_longest_row(dtype):
    """2^30 equal logits: the token is u times their number, and one that stands out."""
    v = 2 ** 30
    z = torch.zeros(1, v, device="cuda", dtype=dtype)
    for u in (0.3, 1.0 - 2.0 ** -24):
        assert draw(z, vec([u]))[0] == int(float(np.float32(u)) * v), u
    z[0, v - 3] = z[0, v - 1] = 40.0                     # two that outweigh all others together
    assert draw(z, vec([0.5]), temperature=vec([0.0]))[0] == v - 3
    assert draw(z, vec([0.6]))[0] == v - 1 and draw(z, vec([0.9]), top_k=vec([1], np.int32))[0] == v - 3
