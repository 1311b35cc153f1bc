"""Recurrences of more tiles than a line of the grid has blocks (2^20) and more than one piece of 128 steps: the line's further blocks have no work."""
import pytest
import torch

from paper_1908_00213_amd import binding as B

pytestmark = pytest.mark.gpu


def test_more_tiles_than_a_line_and_two_pieces():
    """Gates of 1 and -1 and small whole numbers: every sum is exact in fp32 in whatever order, every state and gradient of a state below 256, so exact in
    bfloat16 too.  One row of gates, inputs and gradients for all steps."""
    T, D = 129, 2 ** 27 + 131                                # two columns to a lane, 64 lanes to a tile
    assert (D + 127) // 128 > 2 ** 20
    g = torch.Generator(device="cuda").manual_seed(4)
    whole = lambda m, *s: torch.randint(-m, m + 1, s, device="cuda", generator=g, dtype=torch.int8)
    gate = (whole(0, 1, 1, D) + 1).bfloat16()
    gate[:, :, 1::3] = -1.0
    x, dy, h0, dlast = whole(1, 1, 1, D).bfloat16(), whole(1, 1, 1, D).bfloat16(), whole(3, 1, D).float(), whole(3, 1, D).float()
    every = lambda a: a.expand(T, 1, D)
    y = torch.empty(T, 1, D, device="cuda", dtype=torch.bfloat16)
    last, states = torch.empty(1, D, device="cuda"), torch.empty(B.gated_scan_states_shape(T, 1, D), device="cuda")
    assert B.gated_scan_workspace_bytes(y) == 0              # (a block walks through its tile's pieces)
    B.gated_scan_fwd(every(gate), every(x), y, h0=h0, h_last=last, states=states, kind="decay")
    parts = [slice(a, min(a + 2 ** 24, D)) for a in range(0, D, 2 ** 24)]
    for p in parts:
        h, a, u = h0[0, p], gate[0, 0, p].float(), x[0, 0, p].float()
        for t in range(T):
            if t % 16 == 0:
                assert torch.equal(states[t // 16, 0, p], h), (p.start, t)
            h = a * h + u
            assert torch.equal(y[t, 0, p].float(), h), (p.start, t)
        assert torch.equal(last[0, p], h), p.start
    del y
    dgate, dx = (torch.empty(T, 1, D, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    d0 = torch.empty(1, D, device="cuda")
    B.gated_scan_bwd(every(gate), every(x), states, every(dy), dgate, dx, dh_last=dlast, dh0=d0, kind="decay")
    for p in parts:
        h, a, u, v = h0[0, p], gate[0, 0, p].float(), x[0, 0, p].float(), dy[0, 0, p].float()
        before = []
        for t in range(T):
            before.append(h.to(torch.int16))
            h = a * h + u
        G = dlast[0, p]
        for t in range(T - 1, -1, -1):
            G = G + v
            assert torch.equal(dx[t, 0, p].float(), G), (p.start, t)
            assert torch.equal(dgate[t, 0, p], (before[t].float() * G).bfloat16()), (p.start, t)
            G = a * G
        assert torch.equal(d0[0, p], G), p.start
    del dgate, dx, states
    torch.cuda.empty_cache()
