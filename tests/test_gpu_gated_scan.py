"""The gated linear recurrence and its gradients against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import recurrent as R
from paper_1908_00213_amd import binding as B
from rows_util import DT, HALF, close, rounded, values

pytestmark = pytest.mark.gpu


def steps(a, dtype, pad=0, batch_first=False, fill=7.0):
    """(T,B,D) on the device inside rows `pad` elements longer, time or batch outermost; the rest holds `fill`."""
    T, Bn, D = a.shape
    buf = torch.full((Bn, T, D + pad) if batch_first else (T, Bn, D + pad), fill, device="cuda", dtype=DT[dtype])
    v = (buf.transpose(0, 1) if batch_first else buf)[:, :, :D]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda())
    v.whole = buf
    return v


def around(v):
    """Whether what lies behind the rows still holds 7."""
    return bool((v.whole[..., v.shape[2]:] == 7.0).all())


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def workspace(gate):
    n = B.gated_scan_workspace_bytes(gate)
    return torch.empty(max(256, n), dtype=torch.uint8, device="cuda").fill_(0xA5)


def inputs(T, Bn, D, kind, dtype, seed):
    rng = np.random.default_rng(seed)
    gate = rng.standard_normal((T, Bn, D)) * 2 + 1
    if kind == "decay":
        gate = np.where(rng.random((T, Bn, 1)) < 0.02, 0.0, 1 / (1 + np.exp(-gate - 1))) * np.where(rng.random((T, Bn, D)) < 0.1, -1, 1)
    r = lambda a, t: rounded(a, t)
    return (r(gate, dtype), r(rng.standard_normal((T, Bn, D)), dtype), rng.standard_normal((Bn, D)).astype(np.float32),
            rng.standard_normal((T, Bn, D)) * 0.1, (rng.standard_normal((Bn, D)) * 0.1).astype(np.float32))


def check(T, Bn, D, kind, dtype, out, lengths=None, pad=0, batch_first=False, h0=True, last=True, seed=0, same=False):
    gate, x, first, dy, dlast = inputs(T, Bn, D, kind, dtype, seed + T * 131 + D)
    dy = rounded(dy, out)
    first, dlast = first if h0 else None, dlast if last else None
    want, states, bound = R.gated_scan(gate, x, first, kind, lengths)
    (wg, wx, w0), (bg, bx, b0) = R.gated_scan_bwd(gate, x, first, dy, dlast, kind, lengths)
    if lengths is not None:                              # what lies behind a sequence's end is not looked at
        gate, x, dy = (np.where(np.arange(T)[:, None, None] < np.asarray(lengths)[None, :, None], v, np.nan) for v in (gate, x, dy))
    g, xx = steps(gate, dtype, pad, batch_first), steps(x, dtype, pad, batch_first)
    y = steps(np.zeros_like(want), out, pad, batch_first)
    ln = None if lengths is None else torch.tensor(lengths, device="cuda", dtype=torch.int64 if T % 2 else torch.int32)
    hl, st = torch.full((Bn, D), 7.0, device="cuda"), torch.full(B.gated_scan_states_shape(T, Bn, D), 7.0, device="cuda")
    ws = workspace(g)
    B.gated_scan_fwd(g, xx, y, h0=dev(first), h_last=hl, states=st, lengths=ln, kind=kind, ws=ws)
    half = lambda t, v, b: HALF[t] * (np.abs(v) + b)
    tiny = 1e-36
    close(values(y), want, bound[1:] + half(out, want, bound[1:]) + tiny, "y")
    close(values(hl), states[T], bound[T] + tiny, "h_last")
    close(values(st), states[:T:16], bound[:T:16] + tiny, "states")
    dgate, dx = steps(np.zeros_like(want), dtype, pad, batch_first), steps(np.zeros_like(want), dtype, pad, batch_first)
    d0 = torch.full((Bn, D), 7.0, device="cuda")
    dyd = steps(dy, out, pad, batch_first)
    args = dict(dh_last=dev(dlast), lengths=ln, kind=kind)
    B.gated_scan_bwd(g, xx, st, dyd, dgate, dx, dh0=d0, ws=ws.fill_(0x5A), **args)
    close(values(dx), wx, bx + half(dtype, wx, bx) + tiny, "dx")
    close(values(dgate), wg, bg + half(dtype, wg, bg) + tiny, "dgate")
    close(values(d0), w0, b0 + tiny, "dh0")
    for v in (y, dgate, dx):
        assert around(v)
    if same:                                             # the same bits again, and in place
        y2, hl2, st2 = torch.empty_like(y), torch.empty_like(hl), torch.empty_like(st)
        B.gated_scan_fwd(g, xx, y2, h0=dev(first), h_last=hl2, states=st2, lengths=ln, kind=kind, ws=ws)
        assert torch.equal(y2, y) and torch.equal(hl2, hl) and torch.equal(st2, st)
        h = torch.zeros(Bn, D, device="cuda") if first is None else dev(first)
        xc = steps(x, dtype, pad, batch_first)
        yc = xc if out == dtype else y2
        B.gated_scan_fwd(g, xc, yc, h0=h, h_last=h, lengths=ln, kind=kind, ws=ws)
        assert torch.equal(h, hl) and torch.equal(yc, y)
        gc, xc = steps(gate, dtype, pad, batch_first), steps(x, dtype, pad, batch_first)
        B.gated_scan_bwd(gc, xc, st, dyd, gc, xc, ws=ws, **args)
        assert torch.equal(gc, dgate) and torch.equal(xc, dx)
    return g, xx, y


KINDS = ["sigmoid", "decay"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("T,Bn,D", [(1, 1, 1), (1, 3, 65), (2, 2, 2), (3, 5, 7), (15, 2, 64), (16, 1, 130), (17, 3, 33), (33, 2, 129), (64, 1, 512), (127, 2, 31), (128, 1, 66),
                                    (129, 2, 100), (257, 1, 257), (500, 3, 9)])
def test_scan(T, Bn, D, dtype, out, kind):
    check(T, Bn, D, kind, dtype, out, same=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("batch_first", [False, True])
def test_scan_of_ragged_batches(dtype, kind, pad, batch_first):
    T = 150
    check(T, 6, 45, kind, dtype, dtype, lengths=[0, 1, 149, 150, 16, 129], pad=pad, batch_first=batch_first, same=True)
    check(T + 1, 6, 45, kind, dtype, "f32", lengths=[-5, 151, 1000, 32, 33, 128], pad=pad, batch_first=batch_first, h0=False, last=False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,Bn,D", [(5000, 1, 70), (2100, 2, 130), (4097, 3, 64), (20000, 1, 3)])
def test_scan_of_long_sequences(T, Bn, D, kind):
    check(T, Bn, D, kind, "f32", "f32", same=True)
    check(T, Bn, D, kind, "bf16", "bf16", lengths=[T - 700] * Bn, batch_first=True, seed=1)


@pytest.mark.parametrize("Bn,D", [(300, 650), (1, 70000), (2000, 3)])
def test_scan_of_wide_batches(Bn, D):
    check(3, Bn, D, "sigmoid", "f32", "f32", same=True)
    check(20, Bn, D, "decay", "bf16", "bf16", lengths=list(np.arange(Bn) % 22), batch_first=True)


def test_scan_of_many_tiles_and_pieces():
    """More than 512 tiles: a block walks through the pieces of its tile."""
    Bn, D = 1000, 66
    check(261, Bn, D, "sigmoid", "f32", "f32", lengths=list(np.arange(Bn) % 270), same=True)
    check(261, Bn, D, "decay", "bf16", "bf16", batch_first=True, pad=1)
    check(130, 1100, 65, "sigmoid", "bf16", "f32", same=True)


def test_halves_of_one_product_and_repeated_gates():
    T, Bn, D = 200, 3, 50
    gate, x, first, _, _ = inputs(T, Bn, D, "sigmoid", "f32", 5)
    want, states, bound = R.gated_scan(gate, x, first, "sigmoid")
    z = torch.empty(T, Bn, 2 * D + 1, device="cuda")
    z[:, :, :D], z[:, :, D:2 * D] = torch.from_numpy(gate).cuda(), torch.from_numpy(x).cuda()
    y = torch.empty(T, Bn, D, device="cuda")
    B.gated_scan_fwd(z[:, :, :D], z[:, :, D:2 * D], y, h0=dev(first), ws=workspace(y))
    close(values(y), want, bound[1:] + R.U * np.abs(want))
    # one gate for all sequences, one for all steps
    for g in (gate[:, :1], gate[:1], gate[:1, :1]):
        whole = np.broadcast_to(g, gate.shape)
        want, _, bound = R.gated_scan(whole, x, first, "sigmoid")
        gd = torch.from_numpy(np.ascontiguousarray(g)).cuda().expand(T, Bn, D)
        B.gated_scan_fwd(gd, z[:, :, D:2 * D], y, h0=dev(first), ws=workspace(gd))
        close(values(y), want, bound[1:] + R.U * np.abs(want))


@pytest.mark.parametrize("T", [1, 40, 700])
def test_states_inside_wider_rows(T):
    """First and last states as columns of a wider array, the last one in the first one's place; the columns beside them stay."""
    Bn, D = 3, 37
    gate, x, first, dy, dlast = inputs(T, Bn, D, "sigmoid", "f32", 11)
    dy = np.float32(dy)
    want, states, bound = R.gated_scan(gate, x, first, "sigmoid")
    (_, _, w0), (_, _, b0) = R.gated_scan_bwd(gate, x, first, dy, dlast, "sigmoid")
    wide = torch.full((Bn, D + 6), 7.0, device="cuda")
    h = wide[:, 2:D + 2]
    h.copy_(dev(first))
    g, xx = dev(gate), dev(x)
    y, st = torch.empty_like(g), torch.empty(B.gated_scan_states_shape(T, Bn, D), device="cuda")
    ws = workspace(g)
    B.gated_scan_fwd(g, xx, y, h0=h, h_last=h, states=st, ws=ws)
    close(values(y), want, bound[1:] + R.U * np.abs(want))
    close(values(h), states[T], bound[T] + 1e-36)
    h.copy_(dev(dlast))
    B.gated_scan_bwd(g, xx, st, dev(dy), torch.empty_like(g), torch.empty_like(g), dh_last=h, dh0=h, ws=ws)
    close(values(h), w0, b0 + 1e-36)
    assert (wide[:, :2] == 7).all() and (wide[:, D + 2:] == 7).all()


def test_gates_at_the_ends_of_the_range():
    big = np.float32(3e38)
    g = np.array([0, 1e-30, 20, -20, 88, -88, 104, -104, 1000, -1000, big, -big, np.inf, -np.inf], np.float32)
    T, D = len(g), len(g)
    gate = np.stack([np.roll(g, i) for i in range(T)])[:, None, :]
    x = np.random.default_rng(0).standard_normal((T, 1, D)).astype(np.float32)
    want, states, bound = R.gated_scan(gate, x, None, "sigmoid")
    y = torch.empty(T, 1, D, device="cuda")
    st = torch.empty(B.gated_scan_states_shape(T, 1, D), device="cuda")
    gd, xd = torch.from_numpy(gate).cuda(), torch.from_numpy(x).cuda()
    B.gated_scan_fwd(gd, xd, y, states=st, ws=workspace(y))
    close(values(y), want, bound[1:] + R.U * np.abs(want) + 1e-36)
    dy = np.random.default_rng(1).standard_normal((T, 1, D)).astype(np.float32)
    (wg, wx, w0), (bg, bx, b0) = R.gated_scan_bwd(gate, x, None, dy, None, "sigmoid")
    dg, dx = torch.empty_like(y), torch.empty_like(y)
    B.gated_scan_bwd(gd, xd, st, torch.from_numpy(dy).cuda(), dg, dx, ws=workspace(y))
    close(values(dg), wg, bg + R.U * np.abs(wg) + 1e-36)
    close(values(dx), wx, bx + R.U * np.abs(wx) + 1e-36)


def test_a_decay_of_zero_ends_what_was_before():
    T, D = 300, 5
    gate = np.full((T, 1, D), 0.5, np.float32)
    gate[200] = 0.0
    x = np.zeros((T, 1, D), np.float32)
    x[10], x[250] = 3e38, 1.0
    y = torch.empty(T, 1, D, device="cuda")
    B.gated_scan_fwd(torch.from_numpy(gate).cuda(), torch.from_numpy(x).cuda(), y, kind="decay", ws=workspace(y))
    want, _, bound = R.gated_scan(gate, x, None, "decay")
    close(values(y), want, bound[1:] + 1e-36)
    assert (values(y)[200:250] == 0).all()


def test_nan_and_infinity_stay_in_their_column_and_sequence():
    T, Bn, D = 400, 2, 6
    gate, x, first, _, _ = inputs(T, Bn, D, "sigmoid", "f32", 9)
    x[150, 0, 2], x[150, 1, 3] = np.nan, np.inf
    y = torch.empty(T, Bn, D, device="cuda")
    B.gated_scan_fwd(torch.from_numpy(gate).cuda(), torch.from_numpy(x).cuda(), y, h0=dev(first), ws=workspace(y))
    got = values(y)
    assert np.isnan(got[150:, 0, 2]).all() and not np.isfinite(got[150:, 1, 3]).any()
    got[150:, 0, 2] = got[150:, 1, 3] = 0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("D", [2, 3])
def test_sequences_further_apart_than_32_bits(D):
    """66 sequences, 2^25 elements and more from one to the next, everything interleaved in one block of memory."""
    T, Bn, apart = 150, 66, (1 << 25) + 24
    buf = torch.empty(Bn * apart, device="cuda", dtype=torch.bfloat16)
    view = lambda k: buf.as_strided((T, Bn, D), (20, apart, 1), k * D)
    gate, x, first, dy, dlast = inputs(T, Bn, D, "sigmoid", "bf16", 4)
    dy = rounded(dy, "bf16")
    g, xx, dyd, y, dg, dx = (view(k) for k in range(6))
    for v, a in ((g, gate), (xx, x), (dyd, dy)):
        v.copy_(torch.from_numpy(a).cuda())
    ws = workspace(g)
    st, hl, d0 = torch.empty(B.gated_scan_states_shape(T, Bn, D), device="cuda"), torch.empty(Bn, D, device="cuda"), torch.empty(Bn, D, device="cuda")
    B.gated_scan_fwd(g, xx, y, h0=dev(first), h_last=hl, states=st, ws=ws)
    B.gated_scan_bwd(g, xx, st, dyd, dg, dx, dh_last=dev(dlast), dh0=d0, ws=ws)
    got = [values(v) for v in (y, hl, dg, dx, d0)]
    near = lambda a: torch.from_numpy(a).cuda().bfloat16()
    g, xx, dyd = near(gate), near(x), near(dy)
    y, dg, dx, hl, d0 = (torch.empty_like(v) for v in (g, g, g, hl, d0))
    B.gated_scan_fwd(g, xx, y, h0=dev(first), h_last=hl, states=st, ws=ws)
    B.gated_scan_bwd(g, xx, st, dyd, dg, dx, dh_last=dev(dlast), dh0=d0, ws=ws)
    for a, b in zip(got, (y, hl, dg, dx, d0)):
        assert np.array_equal(a, values(b))
    want, _, bound = R.gated_scan(gate, x, first, "sigmoid")
    close(got[0], want, bound[1:] + HALF["bf16"] * (np.abs(want) + bound[1:]))


def test_no_steps_no_columns():
    h0 = torch.randn(3, 5, device="cuda")
    e = torch.empty(0, 3, 5, device="cuda")
    last = torch.full((3, 5), 7.0, device="cuda")
    B.gated_scan_fwd(e, e, torch.empty_like(e), h0=h0, h_last=last, states=torch.empty(0, 3, 5, device="cuda"))
    assert torch.equal(last, h0)
    B.gated_scan_fwd(e, e, torch.empty_like(e), h_last=last)
    assert (last == 0).all()
    B.gated_scan_bwd(e, e, e, e, torch.empty_like(e), torch.empty_like(e), dh_last=h0, dh0=last)
    assert torch.equal(last, h0)
    z = torch.empty(4, 3, 0, device="cuda")
    B.gated_scan_fwd(z, z, torch.empty_like(z), h_last=torch.empty(3, 0, device="cuda"))


def test_another_stream_and_a_captured_graph():
    T, Bn, D = 1500, 2, 300
    gate, x, first, dy, dlast = inputs(T, Bn, D, "sigmoid", "bf16", 3)
    g, xx, dyd, f, dl = steps(gate, "bf16"), steps(x, "bf16"), steps(rounded(dy, "bf16"), "bf16"), dev(first), dev(dlast)

    def call(y, hl, st, dg, dx, d0, ws):
        B.gated_scan_fwd(g, xx, y, h0=f, h_last=hl, states=st, ws=ws)
        B.gated_scan_bwd(g, xx, st, dyd, dg, dx, dh_last=dl, dh0=d0, ws=ws)

    def outputs():
        e = lambda *s, dt="f32": torch.full(s, 7.0, device="cuda", dtype=DT[dt])
        return e(T, Bn, D, dt="bf16"), e(Bn, D), e(*B.gated_scan_states_shape(T, Bn, D)), e(T, Bn, D, dt="bf16"), e(T, Bn, D, dt="bf16"), e(Bn, D)
    want, ws = outputs(), workspace(g)
    call(*want, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, ws2 = outputs(), workspace(g)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(*got, ws2)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*got, ws2)
    for k in range(4):
        for o in got:
            o.fill_(float(k))
        ws2.fill_(17 * k)
        graph.replay()
        call(*want, ws)                                  # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_two_streams_at_once():
    """Two recurrences whose pieces wait for each other, and products beside them: more blocks than run at once."""
    T, Bn, D = 6000, 4, 1024
    gate, x, first, _, _ = inputs(T, Bn, D, "sigmoid", "bf16", 7)
    g, xx, f = steps(gate, "bf16"), steps(x, "bf16"), dev(first)
    want, ws = torch.empty_like(g), workspace(g)
    B.gated_scan_fwd(g, xx, want, h0=f, ws=ws)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs, spaces = [torch.empty_like(g) for _ in range(2)], [workspace(g) for _ in range(2)]
    m = torch.randn(2048, 2048, device="cuda")
    for k in range(5):
        torch.cuda.synchronize()
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for s, o, w in zip(streams, outs, spaces):
                with torch.cuda.stream(s):
                    B.gated_scan_fwd(g, xx, o, h0=f, ws=w)
            with torch.cuda.stream(streams[2]):
                torch.mm(m, m)
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs), k


def test_gradients_against_differences():
    """Differences of the fp32 results: a step of 2^-6 is off by its square times third derivatives below 1, and by 2 roundings of the sum over its size."""
    T, Bn, D = 40, 2, 3
    gate, x, first, w, wl = inputs(T, Bn, D, "sigmoid", "f32", 12)
    w, wl = w.astype(np.float32), wl.astype(np.float32)

    def f(g, xx, h):
        y, hl = torch.empty(T, Bn, D, device="cuda"), torch.empty(Bn, D, device="cuda")
        B.gated_scan_fwd(dev(g), dev(xx), y, h0=dev(h), h_last=hl, ws=workspace(y))
        return float((values(y) * w).sum() + (values(hl) * wl).sum())
    st = torch.empty(B.gated_scan_states_shape(T, Bn, D), device="cuda")
    y, dg, dx, d0 = (torch.empty(T, Bn, D, device="cuda") for _ in range(4))
    d0 = torch.empty(Bn, D, device="cuda")
    B.gated_scan_fwd(dev(gate), dev(x), y, h0=dev(first), states=st, ws=workspace(y))
    B.gated_scan_bwd(dev(gate), dev(x), st, dev(w), dg, dx, dh_last=dev(wl), dh0=d0, ws=workspace(y))
    h = 2.0 ** -6
    scale = (np.abs(w).sum() + np.abs(wl).sum()) * 4
    for k, (a, da) in enumerate(((gate, values(dg)), (x, values(dx)), (first, values(d0)))):
        for at in [(0, 0, 0), (7, 1, 2), (16, 0, 1), (39, 1, 0)] if k < 2 else [(0, 0), (1, 2)]:
            args = [gate, x, first]
            up, down = a.copy(), a.copy()
            up[at] += h
            down[at] -= h
            d = []
            for v in (up, down):
                args[k] = v
                d.append(f(*args))
            assert abs((d[0] - d[1]) / (float(up[at]) - float(down[at])) - da[at]) < h ** 2 * 4 + 16 * R.U * scale / h, (k, at)
