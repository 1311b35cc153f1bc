"""The gated recurrence, scaled embeddings and adjusted logits without a GPU: what the entry points refuse before anything is launched, and the
oracle's gradients against differences."""
import ctypes as C

import numpy as np

from oracle import recurrent as R
from paper_1908_00213_amd import binding as B
from test_rows_host import d, r

NULL = None


def scan(fwd=True, kind=0, gate=None, x=None, h0=None, lengths=None, y=None, h_last=None, states=None, dy=None, dgate=None, dx=None, ws=None, nbytes=0, T=40, Bn=3, D=8):
    f = lambda a, shape, t=B.F32: d(shape, t) if a is None else None if a is False else a
    gate, x, y = f(gate, (T, Bn, D)), f(x, (T, Bn, D)), f(y, (T, Bn, D))
    h0, h_last = f(h0, (Bn, D)), f(h_last, (Bn, D))
    states = f(states, (-(-T // 16), Bn, D))
    if fwd:
        return B.lib().chn_gated_scan_fwd(kind, r(gate), r(x), r(h0), r(lengths), r(y), r(h_last), r(states), ws, nbytes, None)
    dy, dgate, dx = f(dy, (T, Bn, D)), f(dgate, (T, Bn, D)), f(dx, (T, Bn, D))
    return B.lib().chn_gated_scan_bwd(kind, r(gate), r(x), r(states), r(lengths), r(dy), r(h_last), r(dgate), r(dx), r(h0), ws, nbytes, None)


def test_scan_refuses():
    T, Bn, D = 40, 3, 8
    for fwd in (True, False):
        assert scan(fwd, kind=2) == -6 and scan(fwd, kind=-1) == -6
        assert scan(fwd, gate=False) == -1 and scan(fwd, x=False) == -1
        assert scan(fwd, gate=d((T, Bn * D))) == -2
        assert scan(fwd, x=d((T, Bn, D + 1))) == -4 and scan(fwd, x=d((T, Bn, D), B.BF16)) == -3
        assert scan(fwd, gate=d((T, Bn, D), B.I32), x=d((T, Bn, D), B.I32)) == -3
        assert scan(fwd, gate=d((T, Bn, D), strides=[Bn * D * 8, D * 8, 8])) == -5        # inner stride 2
        assert scan(fwd, gate=d((T, Bn, D), strides=[-96, 32, 4])) == -5
        assert scan(fwd, h0=d((Bn, D), B.BF16)) == -3 and scan(fwd, h0=d((Bn, D + 1))) == -4
        assert scan(fwd, h_last=d((Bn + 1, D))) == -4 and scan(fwd, h_last=d((D,))) == -2
        assert scan(fwd, lengths=d((Bn,))) == -3 and scan(fwd, lengths=d((Bn + 1,), B.I64)) == -4
        assert scan(fwd, states=d((2, Bn, D))) == -4 and scan(fwd, states=d((3, Bn, D), B.BF16)) == -3
        assert scan(fwd, states=d((3, Bn, D), strides=[Bn * D * 8, D * 4, 4])) == -4       # not contiguous
    assert scan(y=False) == -1 and scan(y=d((T, Bn, D), B.I64)) == -3 and scan(y=d((T, Bn, D), strides=[0, 32, 4])) == -5
    assert scan(y=d((T, Bn, D), strides=[64, 32, 4])) == -5                                # rows over each other
    assert scan(False, states=False) == -1 and scan(False, dy=False) == -1
    assert scan(False, dgate=d((T, Bn, D), B.BF16)) == -3 and scan(False, dx=d((T, Bn, D), B.BF16)) == -3
    assert scan(False, dx=d((T, Bn, D), strides=[96, 16, 4])) == -5
    big = d((1, 1, 2 ** 30))
    assert B.lib().chn_gated_scan_fwd(0, r(big), r(big), None, None, r(big), None, None, None, 0, None) == -4
    big = d((2 ** 31, 1, 1))
    assert B.lib().chn_gated_scan_fwd(0, r(big), r(big), None, None, r(big), None, None, None, 0, None) == -4
    assert B.gated_scan_states_shape(0, 2, 3) == (0, 2, 3) and B.gated_scan_states_shape(16, 2, 3)[0] == 1 and B.gated_scan_states_shape(17, 2, 3)[0] == 2


def test_scan_of_nothing():
    assert scan(Bn=0) == 0 and scan(D=0) == 0 and scan(False, Bn=0) == 0


def test_scan_asks_for_its_workspace():
    T, Bn, D = 70000, 1, 1024
    gate = d((T, Bn, D))
    need = B.gated_scan_workspace_bytes(gate)
    assert need > 0
    for fwd in (True, False):
        assert scan(fwd, T=T, Bn=Bn, D=D) == -8
        assert scan(fwd, T=T, Bn=Bn, D=D, ws=4096, nbytes=need - 1) == -8
        assert scan(fwd, T=T, Bn=Bn, D=D, ws=4096 + 64, nbytes=need) == -8
    assert B.gated_scan_workspace_bytes(d((1, 128, 650))) == 0


def embed(bwd=True, ids=None, rows=None, table=None, ws=None, nbytes=0, accumulate=0, N=10, V=6, D=4):
    ids = d((N,), B.I64) if ids is None else ids
    rows, table = d((N, D)) if rows is None else rows, d((V, D)) if table is None else table
    if bwd:
        return B.lib().chn_embed_sorted_bwd(r(ids), r(rows), 1.0, r(table), accumulate, ws, nbytes, None)
    return B.lib().chn_embed_scaled_fwd(r(table), r(ids), 1.0, r(rows), None)


def test_embed_refuses():
    for bwd in (True, False):
        assert embed(bwd, ids=d((10,))) == -3 and embed(bwd, ids=d((10, 1), B.I64)) == -2
        assert embed(bwd, rows=d((9, 4))) == -4 and embed(bwd, rows=d((10, 5))) == -4 and embed(bwd, rows=d((10, 4), B.I32)) == -3
        assert embed(bwd, table=d((6, 4), B.I64)) == -3
        assert embed(bwd, table=d((6, 4), strides=[32, 8])) == -5 and embed(bwd, rows=d((10, 4), strides=[8, 4])) == -5
        assert embed(bwd, ids=d((2 ** 31,), B.I32), rows=d((2 ** 31, 4))) == -4
        assert embed(bwd, table=d((2 ** 31, 4))) == -4
    assert embed(table=d((6, 4), B.BF16)) == -3
    assert embed(table=d((6, 4), strides=[0, 4])) == -5 and embed(False, rows=d((10, 4), strides=[0, 4])) == -5
    assert B.embed_sorted_workspace_bytes(d((10,), B.I64), d((6, 4))) == 0           # (few ids are not sorted)
    many = dict(ids=d((5000,), B.I64), rows=d((5000, 4)))
    need = B.embed_sorted_workspace_bytes(many["ids"], d((6, 4)))
    assert need > 0 and embed(**many) == -8 and embed(ws=4096, nbytes=need - 1, **many) == -8 and embed(ws=4100, nbytes=need, **many) == -8
    assert embed(V=0) == 0 and embed(D=0) == 0 and embed(False, N=0) == 0


def adjust(N=3, V=50, L=9, M=4, logits=None, out=None, **k):
    names = ["tokens", "lengths", "prompt", "repetition", "frequency", "presence", "bias_ids", "bias", "allowed"]
    assert set(k) <= set(names)
    return B.lib().chn_logits_adjust(r(d((N, V)) if logits is None else logits), *[r(k.get(n)) for n in names], r(d((N, V)) if out is None else out), None)


def test_adjust_refuses():
    t = d((3, 9), B.I64)
    p, i = d((3,)), d((3,), B.I64)
    assert adjust(logits=d((3, 50), B.I32)) == -3 and adjust(out=d((3, 50), B.I64)) == -3 and adjust(out=d((3, 49))) == -4 and adjust(out=d((2, 50))) == -4
    assert adjust(logits=d((150,))) == -2 and adjust(logits=d((3, 50), strides=[400, 8])) == -5
    assert adjust(out=d((3, 50), strides=[0, 4])) == -5
    for name in ("repetition", "frequency", "presence"):
        assert adjust(tokens=t, **{name: i}) == -3 and adjust(tokens=t, **{name: d((4,))}) == -4 and adjust(tokens=t, **{name: d((3, 1))}) == -4
    for name in ("lengths", "prompt"):
        assert adjust(tokens=t, **{name: p}) == -3 and adjust(tokens=t, **{name: d((2,), B.I64)}) == -4
    assert adjust(tokens=d((3, 9))) == -3 and adjust(tokens=d((2, 9), B.I64)) == -4 and adjust(tokens=d((27,), B.I64)) == -2
    assert adjust(tokens=d((3, 9), B.I64, strides=[144, -16])) == -5 and adjust(tokens=d((3, 2 ** 30), B.I32)) == -4
    b, bi = d((3, 4)), d((3, 4), B.I64)
    assert adjust(bias=b) == -1 and adjust(bias_ids=bi) == -1
    assert adjust(bias=bi, bias_ids=bi) == -3 and adjust(bias=b, bias_ids=b) == -3 and adjust(bias=d((3, 5)), bias_ids=bi) == -4
    assert adjust(tokens=t, bias=b, bias_ids=d((3, 4), B.I32)) == -3
    assert adjust(allowed=d((3, 2), B.I64)) == -3 and adjust(allowed=d((3, 3), B.I32)) == -4 and adjust(allowed=d((2, 2), B.I32)) == -4
    assert adjust(logits=d((1, 2 ** 31)), out=d((1, 2 ** 31))) == -4
    assert adjust(N=0) == 0 and adjust(V=0) == 0


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(3)
    T, Bn, D = 9, 3, 2
    gate, x, h0, w, wl = (rng.standard_normal(s) for s in ((T, Bn, D), (T, Bn, D), (Bn, D), (T, Bn, D), (Bn, D)))
    lengths = [0, 5, 9]
    for kind in ("sigmoid", "decay"):
        def f(g, xx, h):
            y, states, _ = R.gated_scan(g, xx, h, kind, lengths)
            return (y * w).sum() + (states[T] * wl).sum()
        grads, _ = R.gated_scan_bwd(gate, x, h0, w, wl, kind, lengths)
        h = 1e-5                                         # error of the differences about h^2 and 1e-15 / h
        for k, a in enumerate((gate, x, h0)):
            for i in np.ndindex(a.shape):
                d_ = []
                for s in (h, -h):
                    args = [gate.copy(), x.copy(), h0.copy()]
                    args[k][i] += s
                    d_.append(f(*args))
                assert abs((d_[0] - d_[1]) / (2 * h) - grads[k][i]) < 1e-8, (kind, k, i)


def test_the_recurrence_of_ones_is_a_running_sum():
    x = np.random.default_rng(0).standard_normal((20, 2, 3))
    y, _, _ = R.gated_scan(np.ones_like(x), x, None, "decay")
    assert np.allclose(y, np.cumsum(x, 0), rtol=0, atol=1e-13)
