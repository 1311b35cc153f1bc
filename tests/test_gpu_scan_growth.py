"""Decays above 1, whose products over a few hundred steps leave fp32's range where the states do not: the same results whichever way pieces are joined."""
import numpy as np
import pytest
import torch

from oracle import recurrent as R
from paper_1908_00213_amd import binding as B
from rows_util import HALF, close, rounded, values
from test_gpu_gated_scan import dev, steps, workspace

pytestmark = pytest.mark.gpu
KINDS = 7


def columns(T, dtype, back):
    """gate and x (or, for the way back, what comes to each step's gradient) of seven kinds of columns, (T, 1, KINDS)."""
    gate, u = np.full((T, KINDS), 0.9), np.zeros((T, KINDS))
    t = np.arange(T)
    gate[:, 0] = 2.0                                         # nothing, all the way
    gate[:, 1] = 2.0                                         # nothing but at the end
    u[0 if back else T - 1, 1] = 1.0
    gate[:, 2] = np.where(t // 150 % 2 == 0, 2.5, 0.4)       # up by 10^59 and down again; a piece of 128 steps leaves the range
    u[149 if back else 0::300, 2] = 1e-30
    gate[:, 3] = np.where(t // 200 % 2 == 0, 1.9, 1 / 1.9)   # up by 10^55 and down again; two pieces leave the range, one does not
    u[199 if back else 0::400, 3] = 1e-25
    gate[:, 4] = 1.7                                         # up by 10^34 before a decay of zero
    gate[::500, 4] = 0.0
    u[:, 4] = np.where(t % 500 < 150 if back else t % 500 > 350, 1e-20, 0.0)
    u[:, 5] = np.sin(t)                                      # an ordinary one
    gate[:, 6] = -2.0
    return rounded(gate[:, None], dtype), rounded(u[:, None], dtype)


def below(a, u, first):
    """What the states h <- a h + u are off by beside the roundings of numbers in the normal range, before each step and behind the last one.

    Joined steps multiply decays first.  Wherever such a product of decays, or a state, is rounded below the normal range it is off by 2^-150 and not by a part of itself; of a state
    that is multiplied with it by 2^-150 of that state, which is at most M, the largest magnitude so far.  From there on it goes through the decays that follow.  A product
    and a sum to a step: 2^-149 (M + 1), and nothing while all is zero.  A product with a decay of zero is exact: M begins again there."""
    z, m, M = np.zeros_like(first), np.abs(first), np.abs(first)
    out = [z]
    with np.errstate(over="ignore"):
        for at, ut in zip(np.abs(a), np.abs(u)):
            m = at * m + ut
            M = np.where(at == 0, m, np.maximum(M, m))
            z = at * z + 2.0 ** -149 * (M + (M > 0))
            out.append(z)
    return np.stack(out)


def one(T, dtype, copies):
    gate, x = columns(T, dtype, False)
    dy = columns(T, dtype, True)[1]
    h0, dlast = np.zeros((1, KINDS), np.float32), np.zeros((1, KINDS), np.float32)
    h0[0, 2], h0[0, 5], dlast[0, 3], dlast[0, 5] = 1e-30, 1.0, 1e-25, 1.0
    want, states, bound = R.gated_scan(gate, x, h0, "decay")
    (wg, wx, w0), (bg, bx, b0) = R.gated_scan_bwd(gate, x, h0, dy, dlast, "decay")
    assert all(np.abs(v).max() < 1e37 for v in (want, wg, wx, w0))
    d = lambda v: np.asarray(v, np.float64)
    zh = below(d(gate), d(x), d(h0))
    # G_t = dy_t + a_{t+1} G_{t+1}: what flows into a step is a (dy + what flows into the next one)
    zc = below(d(gate)[::-1], np.abs(d(gate)[::-1] * d(dy)[::-1]), d(dlast))[::-1]
    with np.errstate(over="ignore"):
        zg = zc[1:] + 2.0 ** -149
        zd = zg * (np.abs(states[:T]) + zh[:T]) + zh[:T] * np.abs(wx)
    bound, bx, bg, b0 = bound + zh, bx + zg, bg + zd, b0 + zc[0]
    wide = lambda a: np.tile(a, copies)
    g, xx, dyd = (steps(wide(a), dtype) for a in (gate, x, dy))
    D = KINDS * copies
    y, dgate, dx = (steps(np.zeros((T, 1, D)), dtype) for _ in range(3))
    st, d0, ws = torch.full(B.gated_scan_states_shape(T, 1, D), 7.0, device="cuda"), torch.full((1, D), 7.0, device="cuda"), workspace(g)
    assert (ws.numel() > 256) == (copies == 1)               # pieces that wait for each other, or blocks that walk
    h = dev(wide(h0))
    B.gated_scan_fwd(g, xx, y, h0=h, h_last=h, states=st, kind="decay", ws=ws)
    half = lambda v, b: HALF[dtype] * (np.abs(v) + b)
    tiny = 2.0 ** -126                                       # (a stored number, below the normal range)
    close(values(y), wide(want), wide(bound[1:] + half(want, bound[1:]) + tiny), "y")
    close(values(h), wide(states[T]), wide(bound[T] + tiny), "h_last")
    close(values(st), wide(states[:T:16]), wide(bound[:T:16] + tiny), "states")
    B.gated_scan_bwd(g, xx, st, dyd, dgate, dx, dh_last=dev(wide(dlast)), dh0=d0, kind="decay", ws=ws.fill_(0x5A))
    close(values(dx), wide(wx), wide(bx + half(wx, bx) + tiny), "dx")
    close(values(dgate), wide(wg), wide(bg + half(wg, bg) + tiny), "dgate")
    close(values(d0), wide(w0), wide(b0 + tiny), "d0")
    again, h = torch.empty_like(y), dev(wide(h0))
    B.gated_scan_fwd(g, xx, again, h0=h, h_last=torch.empty_like(h), kind="decay", ws=ws)
    assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [150, 300, 2048, 2049, 2500, 6000])
def test_pieces_that_wait_for_each_other(T, dtype):
    one(T, dtype, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [300, 1100])
def test_blocks_that_walk(T, dtype):
    one(T, dtype, 10000)


def test_an_infinity_stays_one():
    """A state that leaves the range by itself, alike in both ways."""
    T, got = 3000, []
    for copies in (1, 40000):
        D = copies
        gate, x = torch.full((T, 1, D), 1.25, device="cuda"), torch.zeros(T, 1, D, device="cuda")
        x[7] = 1.0
        y, last = torch.empty_like(x), torch.empty(1, D, device="cuda")
        B.gated_scan_fwd(gate, x, y, h_last=last, kind="decay", ws=workspace(gate))
        assert (y == y[:, :, :1]).all() and (last == last[:, :1]).all()
        got.append(values(y[:, :, :1]))
    want, _, bound = R.gated_scan(np.full((T, 1, 1), 1.25), values(x[:, :, :1]), None, "decay")
    ok = np.abs(want) + bound[1:] < 3.4e38
    for y in got:
        close(y[ok], want[ok], bound[1:][ok] + R.U * np.abs(want[ok]))
        assert np.isposinf(y[want > 3.5e38]).all()
