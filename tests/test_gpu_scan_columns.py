"""Columns whose products leave fp32's range, or hold a NaN or an infinity, change no bit of the columns beside them."""
import pytest
import torch

from paper_1908_00213_amd import binding as B
from rows_util import DT
from test_gpu_gated_scan import workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [700, 2048, 5000])
def test_neighbours_keep_their_bits(T, dtype):
    Bn, D = 2, 77
    gen = torch.Generator(device="cuda").manual_seed(T)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    gate, x, dy = (1.0 + 0.01 * normal(T, Bn, D)).to(DT[dtype]), normal(T, Bn, D).to(DT[dtype]), normal(T, Bn, D).to(DT[dtype])
    h0, dlast = normal(Bn, D), normal(Bn, D)
    ws = workspace(gate)

    def both(g, xx, d):
        y, dg, dx = (torch.empty_like(g) for _ in range(3))
        hl, d0, st = torch.empty_like(h0), torch.empty_like(h0), torch.empty(B.gated_scan_states_shape(T, Bn, D), device="cuda")
        B.gated_scan_fwd(g, xx, y, h0=h0, h_last=hl, states=st, kind="decay", ws=ws)
        B.gated_scan_bwd(g, xx, st, d, dg, dx, dh_last=dlast, dh0=d0, kind="decay", ws=ws)
        return y, hl, st, dg, dx, d0
    want = both(gate, x, dy)
    odd = torch.zeros(Bn, D, dtype=torch.bool, device="cuda")
    g, xx, d = gate.clone(), x.clone(), dy.clone()
    for b, c, what in ((0, 0, "grow"), (0, 40, "nan"), (1, 5, "inf"), (1, 75, "grow"), (1, 76, "nan")):
        odd[b, c] = True
        if what == "grow":
            g[:, b, c], xx[:, b, c], d[:, b, c] = 2.5, 0.0, 0.0
        else:
            xx[T // 3, b, c] = d[T // 2, b, c] = float(what)
    got = both(g, xx, d)
    for a, w in zip(got, want):
        assert torch.equal(a[..., ~odd], w[..., ~odd])
    assert torch.isnan(got[0][T // 3:, 0, 40]).all() and torch.isnan(got[4][:T // 2 + 1, 0, 40]).all()
