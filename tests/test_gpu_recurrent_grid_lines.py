"""More blocks than a line of the grid has (2^20): the recurrence, the embeddings' gradient and adjusted logits."""
import numpy as np
import pytest
import torch

from paper_1908_00213_amd import binding as B
from rows_util import U

pytestmark = pytest.mark.gpu


def test_recurrence_of_many_columns():
    D = 70_000_001                                       # 64 to a block
    g = torch.Generator(device="cuda").manual_seed(1)
    gate, x = (torch.randn(2, 1, D, device="cuda", generator=g) for _ in range(2))
    y, h0, last = torch.empty_like(x), torch.randn(1, D, device="cuda", generator=g), torch.empty(1, D, device="cuda")
    B.gated_scan_fwd(gate, x, y, h0=h0, h_last=last)
    h = h0.double()
    for t in range(2):
        a = torch.sigmoid(gate[t].double())
        m = a * h.abs() + (1 - a) * x[t].abs().double()
        h = a * h + (1 - a) * x[t].double()
        # 12 roundings of the magnitudes of each step, as in oracle/recurrent.py, and those of the step before
        assert ((y[t].double() - h).abs() <= 26 * U * (m + 6)).all()     # (|h0| and |x| stay below 6)
    assert torch.equal(last, y[1])


def test_gradient_of_many_rows():
    V, n = 80_000_000, 5000                              # 16 rows to a wave, 4 waves to a block
    g = torch.Generator(device="cuda").manual_seed(2)
    ids, dout = torch.randint(0, V, (n,), device="cuda", generator=g), torch.randn(n, 1, device="cuda", generator=g)
    ids[:300] = ids[300:600]
    ids[600:900] = V - 1
    ids[900] = 0
    table = torch.full((V, 1), float("nan"), device="cuda")
    ws = torch.empty(B.embed_sorted_workspace_bytes(ids, table), dtype=torch.uint8, device="cuda").fill_(0x55)
    B.embed_sorted_bwd(ids, dout, table, 2.0, ws=ws)
    want = torch.zeros(V, 1, device="cuda", dtype=torch.float64).index_add_(0, ids, dout.double() * 2)
    size = torch.zeros(V, 1, device="cuda").index_add_(0, ids, dout.abs() * 2)
    assert ((table.double() - want).abs() <= 90 * U * size).all()        # 64 places, then 5 pieces, 20 further


def test_logits_of_many_rows():
    n, v = 1_100_000, 3
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn(n, v, device="cuda", generator=g)
    tokens = torch.randint(-1, v + 1, (n, 4), device="cuda", generator=g)
    f = torch.rand(n, device="cuda", generator=g)
    allowed = torch.randint(0, 8, (n, 1), device="cuda", generator=g, dtype=torch.int32)
    o = B.logits_adjust(z, torch.empty_like(z), tokens=tokens, frequency=f, allowed=allowed)
    count = torch.stack([(tokens == k).sum(1) for k in range(v)], 1)
    want = z.double() - f.double()[:, None] * count
    on = (allowed >> torch.arange(v, device="cuda", dtype=torch.int32)) & 1 > 0
    assert torch.equal(torch.isneginf(o), ~on)
    assert ((o.double() - want).abs()[on] <= (4 * U * (z.abs().double() + 4))[on]).all()
