"""Scaled embeddings and their gradient by sorted tokens against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import recurrent as R
from paper_1908_00213_amd import binding as B
from rows_util import HALF, U, close, matrix, rounded, untouched, values

pytestmark = pytest.mark.gpu


def ids_of(kind, n, v, rng):
    if kind == "words":
        return np.minimum(np.exp(rng.random(n) * np.log(v + 1)).astype(np.int64) - 1, v - 1)
    if kind == "all equal":
        return np.full(n, v - 1)
    if kind == "outside":
        return np.where(rng.random(n) < 0.5, rng.integers(0, v, n), rng.choice([-1, v, v + 1, -2 ** 31, 2 ** 31 - 1], n))
    if kind == "none":
        return np.full(n, -1)
    return rng.integers(0, v, n)


def gradient(ids, dout, v, scale, accumulate=False, pad=0, shift=0, stride=1, dtype=torch.int64, before=None):
    """The device's gradient inside rows `pad` elements longer; what lies around it stays."""
    d = dout.shape[1]
    table = matrix(np.zeros((v, d)) if before is None else before, "f32", pad, shift)
    if before is None:
        table.fill_(np.nan)
    buf = torch.full((len(ids) * stride,), -3, device="cuda", dtype=dtype)
    idd = buf[::stride]
    idd.copy_(torch.from_numpy(np.asarray(ids)).to(dtype).cuda())
    n = B.embed_sorted_workspace_bytes(idd, table)
    B.embed_sorted_bwd(idd, dout, table, scale, accumulate=accumulate, ws=torch.empty(max(256, n), dtype=torch.uint8, device="cuda").fill_(0xA5))
    assert untouched(table, pad, shift)
    return table


SIZES = [(1, 1, 1), (1, 5, 3), (3, 4, 1), (63, 8, 7), (64, 1, 64), (65, 2, 65), (100, 33, 257), (257, 16, 255), (1000, 650, 100), (4096, 12, 513), (5000, 9, 3), (9001, 66, 1000),
         (70000, 5, 70000), (33000, 130, 300), (20000, 3, 200000), (9001, 2, 300000), (5000, 2, 300000)]


@pytest.mark.parametrize("kind", ["words", "all equal", "outside", "none", "even"])
@pytest.mark.parametrize("n,d,v", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient(n, d, v, dtype, kind):
    rng = np.random.default_rng(n + d)
    ids, scale = ids_of(kind, n, v, rng), 3.7
    a = rounded(rng.standard_normal((n, d)), dtype)
    want, bound = R.embed_scaled_bwd(ids, a, v, np.float32(scale))
    got = gradient(ids, matrix(a, dtype, 0), v, scale)
    close(values(got), want, bound)
    again = gradient(ids, matrix(a, dtype, 3, 1), v, scale, pad=5, shift=3, stride=2, dtype=torch.int32)
    assert torch.equal(again, got)                       # the same bits whatever the strides


@pytest.mark.parametrize("n,d,v", [(700, 20, 90), (5000, 66, 40)])
def test_gradient_added_to_another(n, d, v):
    rng = np.random.default_rng(n)
    ids, a, before = ids_of("words", n, v, rng), rng.standard_normal((n, d)).astype(np.float32), rng.standard_normal((v, d)).astype(np.float32)
    want, bound = R.embed_scaled_bwd(ids, a, v, 0.5)
    got = values(gradient(ids, matrix(a, "f32"), v, 0.5, accumulate=True, before=before))
    close(got, want + before, bound + U * np.abs(want + before))
    assert np.array_equal(got[np.bincount(ids, minlength=v) == 0], before[np.bincount(ids, minlength=v) == 0])


def test_small_tables_and_nothing_at_all():
    a = matrix(np.ones((5, 4)), "f32")
    assert values(gradient(np.array([0, 0, 0, -1, 1]), a, 1, 2.0)).tolist() == [[6.0] * 4]
    e = torch.empty(0, 4, device="cuda")
    assert (values(gradient(np.zeros(0, np.int64), e, 3, 1.0)) == 0).all()
    t = torch.empty(0, 4, device="cuda")
    B.embed_sorted_bwd(torch.zeros(5, dtype=torch.int64, device="cuda"), a, t, ws=torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))


def test_rows_of_others_stay_out_of_a_rows_sum():
    """A row of NaN and infinities shows in its own token's row alone; a row without a token shows nowhere."""
    n, d, v = 300, 10, 20
    rng = np.random.default_rng(0)
    ids, a = rng.integers(0, v, n), rng.standard_normal((n, d)).astype(np.float32)
    ids[17], ids[40], ids[41] = 5, -1, v
    a[17], a[40], a[41] = np.nan, np.inf, np.nan
    got = values(gradient(ids, matrix(a, "f32"), v, 1.0))
    assert np.isnan(got[5]).all() and np.isfinite(np.delete(got, 5, 0)).all()


@pytest.mark.parametrize("table", ["f32", "bf16"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,v,pad", [(1, 1, 1, 0), (5, 3, 2, 1), (100, 8, 7, 0), (33, 650, 100, 3), (257, 1001, 50, 5), (9, 4099, 3, 0)])
def test_lookup(n, d, v, pad, table, out):
    rng = np.random.default_rng(n)
    w = rounded(rng.standard_normal((v, d)), table)
    ids = ids_of("outside", n, v, rng)
    scale = float(np.sqrt(d))
    want = R.embed_scaled(w, ids, np.float32(scale))
    for dt in (torch.int32, torch.int64):
        o = matrix(np.zeros((n, d)), out, pad, pad)
        o.fill_(np.nan)
        B.embed_scaled_fwd(matrix(w, table, pad, 1), torch.from_numpy(ids).to(dt).cuda(), o, scale)
        close(values(o), want, (U + HALF[out] * (1 + U)) * np.abs(want))
        assert untouched(o, pad, pad)


def test_lookup_of_scale_one_copies_bits():
    t, ids = torch.randn(50, 33, device="cuda"), torch.randint(0, 50, (70,), device="cuda")
    o, p = torch.empty(70, 33, device="cuda"), torch.empty(70, 33, device="cuda")
    assert torch.equal(B.embed_scaled_fwd(t, ids, o), B.embed_fwd(t, ids, p))


def test_gradient_against_differences():
    """The lookup is linear: a difference is the gradient's product with a direction, up to the roundings of both."""
    n, d, v = 200, 12, 30
    rng = np.random.default_rng(2)
    ids, w, dout, delta = rng.integers(0, v, n), rng.standard_normal((v, d)), rng.standard_normal((n, d)).astype(np.float32), rng.standard_normal((v, d))
    w, delta = rounded(w, "bf16"), rounded(delta, "bf16")          # w + delta is exact in fp32 to 2^-23 of their sizes
    out = lambda t: values(B.embed_scaled_fwd(matrix(t, "f32"), torch.from_numpy(ids).cuda(), torch.empty(n, d, device="cuda"), 2.5))
    up = np.float32(w + delta)
    change = ((out(up) - out(w)) * dout).sum()
    g = values(gradient(ids, matrix(dout, "f32"), v, 2.5))
    size = (np.abs(dout) * 2.5 * (np.abs(w[ids]) + np.abs(delta[ids]))).sum()
    assert abs(change - (g * (up.astype(np.float64) - w)).sum()) < 100 * U * size


def test_another_stream_and_a_captured_graph():
    n, d, v = 20000, 70, 3000
    rng = np.random.default_rng(4)
    ids = torch.from_numpy(ids_of("words", n, v, rng)).cuda()
    dout = matrix(rng.standard_normal((n, d)), "bf16")
    new = lambda: (torch.empty(v, d, device="cuda"), torch.empty(B.embed_sorted_workspace_bytes(ids, torch.empty(v, d, device="cuda")) + 256, dtype=torch.uint8, device="cuda"))
    want, ws = new()
    B.embed_sorted_bwd(ids, dout, want, 2.0, ws=ws)
    got, ws2 = new()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.embed_sorted_bwd(ids, dout, got, 2.0, ws=ws2)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.embed_sorted_bwd(ids, dout, got, 2.0, ws=ws2)
    for k in range(4):                                   # other ids and other gradients from replay to replay
        ids.copy_(torch.from_numpy(ids_of("words" if k % 2 else "outside", n, v, rng)).cuda())
        dout.copy_(torch.from_numpy(rng.standard_normal((n, d))).cuda())
        got.fill_(5.0)
        graph.replay()
        B.embed_sorted_bwd(ids, dout, want, 2.0, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(got, want), k
