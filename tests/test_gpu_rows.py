"""Layer normalisation, dropout and their fusion in a residual block, against the definitions in 64 bits (bounds: rows_util.py)."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_1908_00213_amd import binding as B
from rows_util import DT, HALF, U, bwd_bounds, close, matrix, norm_bounds, rounded, untouched, values

pytestmark = pytest.mark.gpu
SEED, OFFSET, SITE = 0x1234567890ABCDEF, 41, 3
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 100), (130, 64), (33, 100), (7, 129), (2, 650), (70, 1000), (9, 2049), (5, 4096), (3, 5003), (2, 8200), (3, 16400),
          (2, 40007), (300, 19), (530, 33), (77, 300), (40, 1030), (33, 1100), (40, 2300), (9, 6000), (5, 8191)]


def rng_state(seed=SEED, offset=OFFSET):
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def vec(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def workspace(x):
    return torch.empty(max(256, B.layer_norm_bwd_workspace_bytes(x)), dtype=torch.uint8, device="cuda")


def data(shape, dtype, seed, scale=1.0, shift=0.0):
    return rounded(np.random.default_rng(seed).standard_normal(shape) * scale + shift, dtype)


# ---- dropout: every result has its definition's bits --------------------------------------------------------------
@pytest.mark.parametrize("tx,ty", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("ratio", [0.0, 0.3, 0.9])
def test_dropout(shape, tx, ty, ratio):
    x, res = data(shape, tx, 1), data(shape, ty, 2)
    for pad, shift in ((0, 0), (3, 1)):
        xd, rd, y, z = matrix(x, tx, pad, shift), matrix(res, ty, pad, shift), matrix(x * 0, ty, pad, shift), matrix(x * 0, ty, pad, shift)
        B.dropout(xd, y, ratio, rng_state() if ratio else None, SITE)
        B.dropout(xd, z, ratio, rng_state() if ratio else None, SITE, residual=rd)
        assert np.array_equal(values(y), rounded(R.dropout(x, ratio, SEED, OFFSET, SITE), ty))
        assert np.array_equal(values(z), rounded(R.dropout(x, ratio, SEED, OFFSET, SITE, res), ty))
        assert untouched(y, pad, shift) and untouched(z, pad, shift) and np.array_equal(values(xd), x)


def test_dropout_of_views():
    g = np.random.default_rng(5)
    ratio, want = 0.5, lambda a, r=None: R.dropout(a, ratio, SEED, OFFSET, SITE, r)
    cube = g.standard_normal((6, 5, 22)).astype(np.float32)
    c = torch.from_numpy(cube).cuda()
    cases = {"3-d": c, "3-d, middle axis sliced": c[:, 1:4], "permuted": c.permute(2, 0, 1), "transposed": c[0].t(), "every second column": c[:, :, ::2],
             "a row repeated": c[0, 0].expand(9, 22), "a column repeated": c[0, :, :1].expand(5, 8), "one number": c[0, 0, 0], "one axis": c[1, 2],
             "no columns": c[:, :, :0], "a single column": c[:, 0, :1], "five axes": c.reshape(3, 2, 5, 11, 2).permute(3, 0, 4, 1, 2)}
    for name, v in cases.items():
        a = v.cpu().numpy()
        for out in (torch.zeros(v.shape, device="cuda"), torch.zeros(tuple(v.shape)[::-1], device="cuda").permute(tuple(range(v.dim() - 1, -1, -1)))):
            B.dropout(v, out, ratio, rng_state(), SITE)
            assert np.array_equal(out.cpu().numpy(), want(a)), name
            if v.dim() == 3:
                B.dropout(v, out, ratio, rng_state(), SITE, residual=v)
                assert np.array_equal(out.cpu().numpy(), want(a, a)), name
    flat = c.reshape(-1).clone()                        # in place
    B.dropout(flat, flat, ratio, rng_state(), SITE)
    assert np.array_equal(flat.cpu().numpy(), want(cube.reshape(-1)))


def test_dropped_elements_are_zero_whatever_they_were():
    x = np.full((4, 64), np.nan, np.float32)
    x[1], x[2] = np.inf, -np.inf
    y = torch.empty(4, 64, device="cuda")
    B.dropout(vec(x), y, 0.5, rng_state(), SITE)
    keep = R.mask(4, 64, 0.5, SEED, OFFSET, SITE)
    got = y.cpu().numpy()
    assert np.all(got[~keep] == 0) and np.array_equal(np.isnan(got), keep & np.isnan(x)) and np.array_equal(np.isinf(got), keep & np.isinf(x))


def test_sites_offsets_and_seeds_draw_other_masks_and_advance_counts():
    x, state = torch.ones(64, 256, device="cuda"), rng_state()
    draw = lambda site=SITE, state=state: B.dropout(x, torch.empty_like(x), 0.5, state, site).cpu().numpy() != 0
    first = draw()
    assert np.array_equal(first, R.mask(64, 256, 0.5, SEED, OFFSET, SITE)) and np.array_equal(draw(), first)
    assert np.array_equal(draw(2 ** 32 - 1), R.mask(64, 256, 0.5, SEED, OFFSET, 2 ** 32 - 1))
    B.rng_advance(state, 9)
    assert state.tolist() == [SEED, OFFSET + 9] and np.array_equal(draw(), R.mask(64, 256, 0.5, SEED, OFFSET + 9, SITE))
    wide = rng_state(-3, 2 ** 32 + 7)                    # a negative number is the same 64 bits, the offset counts by its low ones
    assert np.array_equal(draw(state=wide), R.mask(64, 256, 0.5, (-3) % 2 ** 64, 7, SITE))


# ---- layer normalisation --------------------------------------------------------------------------------------------
def check_norm(x, tx, ty, gamma, beta, eps=1e-5, pad=0, shift=0, dy=None):
    n, c = x.shape
    opt = lambda a: None if a is None else vec(a)
    xd, y, mean, rstd = matrix(x, tx, pad, shift), matrix(x * 0, ty, pad, shift), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    B.layer_norm_fwd(xd, y, opt(gamma), opt(beta), eps, mean, rstd)
    wy, wm, wr = R.layer_norm(x, gamma, beta, eps)
    by, bm, br = norm_bounds(x.astype(np.float64), wm, wr, wy, gamma, beta, ty)
    close(values(mean), wm, bm, "mean")
    close(values(rstd), wr, br, "rstd")
    close(values(y), wy, by, "y")
    assert untouched(y, pad, shift)
    if dy is None:
        return
    sm, sr = values(mean), values(rstd)                  # the backward pass is judged by the statistics that it is given
    dyd, dx = matrix(dy, ty, pad, shift), matrix(x * 0, tx, pad, shift)
    dg, db = torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
    B.layer_norm_bwd(dyd, xd, mean, rstd, dx, opt(gamma), dg, db, ws=workspace(xd))
    wdx, wdg, wdb = R.layer_norm_bwd(dy, x, sm, sr, gamma)
    bdx, bdg, bdb = bwd_bounds(dy.astype(np.float64), x.astype(np.float64), sm, sr, gamma, tx)
    close(values(dx), wdx, bdx + HALF[tx] * (1 + 2 ** -6) * (np.abs(wdx) + bdx), "dx")
    close(values(dg), wdg, bdg + U * np.abs(wdg), "dgamma")
    close(values(db), wdb, bdb + U * np.abs(wdb), "dbeta")
    assert untouched(dx, pad, shift)
    # without the weights' gradients: the same dx, and a workspace for long rows only
    dx2 = matrix(x * 0, tx, pad, shift)
    B.layer_norm_bwd(dyd, xd, mean, rstd, dx2, opt(gamma), ws=workspace(xd) if c > 8192 else None)
    assert torch.equal(dx2, dx)


@pytest.mark.parametrize("tx,ty", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_layer_norm(shape, tx, ty):
    n, c = shape
    gamma, beta = 1 + 0.3 * data((c,), "f32", 11), data((c,), "f32", 12)
    check_norm(data(shape, tx, 13, 1.5, 0.5), tx, ty, gamma, beta, dy=data(shape, ty, 14))
    check_norm(data(shape, tx, 15, 1.5, 0.5), tx, ty, gamma, None, pad=5, shift=1, dy=data(shape, ty, 16))


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 255, 257, 1023, 2049, 5000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_by_rows(rows, dtype):
    shape = (rows, 72)
    check_norm(data(shape, dtype, 21), dtype, dtype, None, data((72,), "f32", 22), pad=3, dy=data(shape, dtype, 23))


def test_layer_norm_keeps_the_digits_of_a_small_spread():
    x = data((40, 777), "f32", 31, 1.0, 1e4)
    check_norm(x, "f32", "f32", None, None, dy=data(x.shape, "f32", 32))
    check_norm(data((3, 30011), "f32", 33, 0.1, -1e3), "f32", "f32", None, None)


def test_layer_norm_of_constant_rows_and_large_values():
    x = np.full((5, 130), 3.0, np.float32)
    y, rstd = torch.empty(5, 130, device="cuda"), torch.empty(5, device="cuda")
    B.layer_norm_fwd(vec(x), y, None, vec(np.arange(130)), 1e-5, None, rstd)
    assert np.array_equal(y.cpu().numpy(), np.broadcast_to(np.arange(130, dtype=np.float32), (5, 130)))      # h = 0 exactly: 3 is the mean of threes
    check_norm(data((4, 130), "f32", 41, 1e15), "f32", "f32", None, None)
    bad = data((3, 130), "f32", 42)
    bad[1, 7] = np.nan
    B.layer_norm_fwd(vec(bad), (out := torch.empty(3, 130, device="cuda")))
    got = out.cpu().numpy()
    assert np.isnan(got[1]).all() and not np.isnan(got[[0, 2]]).any()


def test_layer_norm_without_rows():
    dg, db = torch.full((9,), 5.0, device="cuda"), torch.full((9,), 5.0, device="cuda")
    x, n = torch.empty(0, 9, device="cuda"), torch.empty(0, device="cuda")
    B.layer_norm_fwd(x, x)
    B.layer_norm_bwd(x, x, n, n, x, None, dg, db, ws=workspace(x))
    assert not dg.any() and not db.any()


def test_layer_norm_in_place():
    x, dy = data((50, 300), "f32", 51), data((50, 300), "f32", 52)
    mean, rstd, y = torch.empty(50, device="cuda"), torch.empty(50, device="cuda"), torch.empty(50, 300, device="cuda")
    xd, dyd = vec(x), vec(dy)
    B.layer_norm_fwd(xd, y, None, None, 1e-5, mean, rstd)
    dx, grads = torch.empty_like(y), [torch.empty(300, device="cuda") for _ in range(4)]
    B.layer_norm_bwd(dyd, xd, mean, rstd, dx, None, *grads[:2], ws=workspace(xd))
    for over in (0, 1):                                  # dx over dy, dx over x
        a, b = dyd.clone(), xd.clone()
        B.layer_norm_bwd(a, b, mean, rstd, (a, b)[over], None, *grads[2:], ws=workspace(xd))
        assert torch.equal((a, b)[over], dx) and torch.equal(grads[0], grads[2]) and torch.equal(grads[1], grads[3])
    again = xd.clone()
    B.layer_norm_fwd(again, again)
    assert torch.equal(again, y)


# ---- residual + dropout + normalisation -------------------------------------------------------------------------------
def check_residual(shape, tl, ts, ratio, pad=0, shift=0, with_ds=True):
    n, c = shape
    x, res, dy, ds = data(shape, tl, 61), data(shape, ts, 62, 1.0, 0.5), data(shape, tl, 63), data(shape, ts, 64)
    gamma, beta = 1 + 0.3 * data((c,), "f32", 65), data((c,), "f32", 66)
    new = lambda t: matrix(np.zeros(shape), t, pad, shift)
    xd, rd, s, y = matrix(x, tl, pad, shift), matrix(res, ts, pad, shift), new(ts), new(tl)
    mean, rstd, g, b = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), vec(gamma), vec(beta)
    drop = dict(ratio=ratio, rng=rng_state() if ratio else None, site=SITE)
    B.residual_norm_fwd(xd, rd, s, y, g, b, 1e-5, mean, rstd, **drop)
    ws_ = rounded(R.dropout(x, ratio, SEED, OFFSET, SITE, res), ts)
    assert np.array_equal(values(s), ws_)                # the sum has chn_dropout's bits
    wy, wm, wr = R.layer_norm(ws_, gamma, beta)
    by, bm, br = norm_bounds(ws_.astype(np.float64), wm, wr, wy, gamma, beta, tl)
    close(values(mean), wm, bm, "mean")
    close(values(rstd), wr, br, "rstd")
    close(values(y), wy, by, "y")
    sm, sr = values(mean), values(rstd)
    dyd, dsd, dres, dx = matrix(dy, tl, pad, shift), matrix(ds, ts, pad, shift) if with_ds else None, new(ts), new(tl)
    dg, db = torch.zeros(c, device="cuda"), torch.zeros(c, device="cuda")
    B.residual_norm_bwd(dyd, dsd, s, mean, rstd, dres, dx, g, dg, db, ws=workspace(s), **drop)
    wt, wdg, wdb = R.layer_norm_bwd(dy, ws_, sm, sr, gamma)
    bt, bdg, bdb = bwd_bounds(dy.astype(np.float64), ws_.astype(np.float64), sm, sr, gamma, ts)
    if with_ds:
        wt = wt + ds
    bt = bt + U * (np.abs(wt) + bt)
    close(values(dres), wt, bt + HALF[ts] * (1 + 2 ** -6) * (np.abs(wt) + bt), "dresidual")
    factor = R.mask(n, c, ratio, SEED, OFFSET, SITE) / (1 - ratio) if ratio else np.ones(shape)
    close(values(dx), wt * factor, factor * (bt + (3 * U + HALF[tl] * (1 + 2 ** -6)) * (np.abs(wt) + bt)), "dx")
    close(values(dg), wdg, bdg + U * np.abs(wdg), "dgamma")
    close(values(db), wdb, bdb + U * np.abs(wdb), "dbeta")
    assert all(untouched(m, pad, shift) for m in (s, y, dres, dx))
    # either gradient by itself
    only, other = new(ts), new(tl)
    long = workspace(s) if c > 8192 else None
    B.residual_norm_bwd(dyd, dsd, s, mean, rstd, only, None, g, ws=long, **drop)
    B.residual_norm_bwd(dyd, dsd, s, mean, rstd, None, other, g, ws=long, **drop)
    assert torch.equal(only, dres) and torch.equal(other, dx)
    # over their inputs
    B.residual_norm_fwd(xd, rd, rd, xd, g, b, 1e-5, None, None, **drop)
    assert torch.equal(rd, s) and torch.equal(xd, y)
    if with_ds:
        B.residual_norm_bwd(dyd, dsd, s, mean, rstd, dsd, dyd, g, dg, db, ws=workspace(s), **drop)
        assert torch.equal(dsd, dres) and torch.equal(dyd, dx)


@pytest.mark.parametrize("tl,ts", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_residual_norm(shape, tl, ts):
    check_residual(shape, tl, ts, 0.3)
    check_residual(shape, tl, ts, 0.0, pad=7, shift=1, with_ds=False)


def test_residual_norm_without_rows():
    x, n, v = torch.empty(0, 8, device="cuda"), torch.empty(0, device="cuda"), torch.ones(8, device="cuda")
    B.residual_norm_fwd(x, x, x, x, v, v, ratio=0.5, rng=rng_state())
    B.residual_norm_bwd(x, None, x, n, n, x, x, v, v, v.clone(), ratio=0.5, rng=rng_state(), ws=workspace(x))
    assert not v.any()


# ---- how the calls meet a program -------------------------------------------------------------------------------------
def test_calls_follow_the_stream_and_replay_in_a_graph():
    n, c = 300, 520
    x, res, dy = vec(data((n, c), "f32", 71)), vec(data((n, c), "f32", 72)), vec(data((n, c), "f32", 73))
    gamma, beta, state = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda"), rng_state()

    class Buffers:
        def __init__(self):
            self.s, self.y, self.dr, self.dx, self.z = (torch.zeros(n, c, device="cuda") for _ in range(5))
            self.mean, self.rstd, self.dg, self.db = (torch.zeros(k, device="cuda") for k in (n, n, c, c))
            self.ws = workspace(x)

        def step(self, state):
            B.rng_advance(state)
            B.residual_norm_fwd(x, res, self.s, self.y, gamma, beta, 1e-5, self.mean, self.rstd, ratio=0.4, rng=state, site=1)
            B.residual_norm_bwd(dy, None, self.s, self.mean, self.rstd, self.dr, self.dx, gamma, self.dg, self.db, ratio=0.4, rng=state, site=1, ws=self.ws)
            B.dropout(self.y, self.z, 0.4, state, 2)
            return [t.clone() for t in (self.s, self.y, self.dr, self.dx, self.z, self.dg, self.db)]

    eager, a = Buffers(), rng_state()
    want = [eager.step(a) for _ in range(4)]
    assert not torch.equal(want[0][0], want[1][0])       # other masks in every step
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                        # on another stream than the tensors' own
        other, b = Buffers(), rng_state()
        got = [other.step(b) for _ in range(2)]
    side.synchronize()
    assert all(torch.equal(p, q) for w, g in zip(want, got) for p, q in zip(w, g))
    graphed, graph = Buffers(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = graphed.step(state)
    state.copy_(rng_state())
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want[k], out)), k
        eager.step(rng_state())                          # eager work between the replays
    assert state.tolist() == [SEED, OFFSET + 4]


def test_arrays_of_the_host_are_refused():
    x = torch.ones(4, 8)
    with pytest.raises(ValueError):
        B.dropout(x, torch.empty(4, 8, device="cuda"), 0.0)
    with pytest.raises(ValueError):
        B.layer_norm_fwd(torch.ones(4, 8, device="cuda"), torch.empty(4, 8, device="cuda"), torch.ones(8))
    with pytest.raises(ValueError):
        B.sample(x.cuda(), torch.ones(4), torch.empty(4, dtype=torch.int64, device="cuda"))


def test_more_rows_than_a_line_of_the_grid_has_blocks():
    n, c = 2 ** 24 + 37, 3                               # sixteen rows to a block
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(n, c, device="cuda", generator=g)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    B.layer_norm_fwd(x, y, None, None, 1e-2, mean, rstd)
    d = x.double()
    m = d.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(((d - m) ** 2).mean(1, keepdim=True) + 1e-2)
    # three terms: a handful of roundings of values of at most 1 / sqrt(eps) times the spread
    assert float((y - (d - m) * r).abs().max()) < 16 * U * 10 * float(x.abs().max())
    z = torch.empty_like(x)
    B.dropout(x, z, 0.5, rng_state(), SITE)
    tail = torch.arange(n - 5, n)
    for row in tail.tolist() + [0, 2 ** 20, 2 ** 24]:
        words = R.philox4x32([0, row, OFFSET, SITE], [SEED & R.LOW, SEED >> 32], 7)[:3]
        want = [float(v) * 2 if w >= 2 ** 31 else 0.0 for v, w in zip(x[row].tolist(), words)]
        assert z[row].tolist() == want, row


def test_a_workspace_of_the_host_is_refused():
    x, v = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda")
    m = torch.ones(4, device="cuda")
    with pytest.raises(ValueError):
        B.layer_norm_bwd(x, x, m, m, torch.empty_like(x), v, v.clone(), v.clone(), ws=torch.empty(1 << 16, dtype=torch.uint8))


def test_more_columns_than_a_line_of_the_grid_has_blocks():
    n, c = 2, 2 ** 27 + 41                               # 64 column sums to a block, 2 c of them
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn(n, c, device="cuda", generator=g) for _ in range(2))
    mean, rstd = torch.tensor([0.25, -0.5], device="cuda"), torch.tensor([0.5, 2.0], device="cuda")
    dgamma, dbeta = (torch.full((c,), 7.0, device="cuda") for _ in range(2))
    ws = torch.empty(B.layer_norm_bwd_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    B.layer_norm_bwd(dy, x, mean, rstd, torch.empty_like(x), None, dgamma, dbeta, ws)
    assert torch.equal(dbeta, dy[0] + dy[1])             # (one rounding either way)
    for a in range(0, c, 2 ** 25):
        p, q = (t[:, a:a + 2 ** 25].double() for t in (x, dy))
        t = (p - mean.double()[:, None]) * rstd.double()[:, None] * q
        # a difference (the scales are powers of two), a product and a sum
        assert bool(((dgamma[a:a + 2 ** 25] - t.sum(0)).abs() <= 4 * U * (t.abs().sum(0) + 1e-30)).all()), a


@pytest.mark.parametrize("shape", [(0, 40), (1, 7), (3, 100), (8, 1000), (9, 1000), (5, 1500), (1, 5000), (2, 5000), (4, 8200), (5, 8200), (300, 30)])
def test_each_weight_gradient_by_itself(shape):
    n, c = shape
    x, dy, gamma = data(shape, "f32", 51), data(shape, "f32", 52), vec(1 + 0.3 * data((c,), "f32", 53))
    xd, dyd = matrix(x, "f32", 1, 0), matrix(dy, "f32")
    mean, rstd = vec(data((n,), "f32", 54)), vec(1 + 0.1 * np.abs(data((n,), "f32", 55)))
    both = [torch.full((c,), 9.0, device="cuda") for _ in range(2)]
    dx = matrix(x * 0, "f32")
    B.layer_norm_bwd(dyd, xd, mean, rstd, dx, gamma, *both, ws=workspace(xd))
    wdx, wdg, wdb = R.layer_norm_bwd(dy, x, values(mean), values(rstd), values(gamma))
    bdx, bdg, bdb = bwd_bounds(dy.astype(np.float64), x.astype(np.float64), values(mean), values(rstd), values(gamma), "f32")
    close(values(both[0]), wdg, bdg + U * np.abs(wdg), "dgamma")
    close(values(both[1]), wdb, bdb + U * np.abs(wdb), "dbeta")
    for k in range(2):
        one, around, dx1 = [None, None], torch.full((c + 8,), 9.0, device="cuda"), matrix(x * 0, "f32")
        one[k] = around[4:4 + c]
        B.layer_norm_bwd(dyd, xd, mean, rstd, dx1, gamma, *one, ws=workspace(xd))
        assert torch.equal(one[k], both[k]) and torch.equal(dx1, dx) and bool((around[:4] == 9.0).all()) and bool((around[4 + c:] == 9.0).all())
