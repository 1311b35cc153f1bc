"""Sampled tokens against the definition in 64 bits: equal, token by token."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_1908_00213_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(z, u, out_dtype=torch.int64, ws=True, **params):
    out = torch.full((z.shape[0],), -7, device="cuda", dtype=out_dtype)
    w = torch.empty(max(256, B.sample_workspace_bytes(z)), dtype=torch.uint8, device="cuda").fill_(0xA5) if ws else None
    B.sample(z, u, out, ws=w, **params)
    return out.cpu().numpy()


def check(z, u, **params):
    """z: device logits; parameters: NumPy vectors."""
    n = z.shape[0]
    dev = {k: torch.from_numpy(np.asarray(v, np.int32 if k == "top_k" else np.float32)).cuda() for k, v in params.items()}
    u = np.asarray(u, np.float32)
    want = R.sample(z.float().cpu().numpy(), u, **{k: v.cpu().numpy() for k, v in dev.items()})
    ud = torch.from_numpy(u).cuda()
    got = draw(z, ud, **dev)
    assert np.array_equal(got, want), (got, want)
    assert np.array_equal(draw(z, ud, torch.int32, ws=False, **dev), want)
    return want


def logits(n, v, dtype, seed, spread=2.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, v + pad, generator=g) * spread).to(DT[dtype]).cuda()[:, :v]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v,pad", [(1, 0), (2, 1), (7, 0), (64, 3), (100, 0), (255, 1), (256, 0), (257, 0), (500, 3), (513, 0), (1000, 8), (1025, 0), (4099, 5), (10000, 0)])
@pytest.mark.parametrize("which", ["", "t", "k", "p", "m", "tkpm"])
def test_sample(v, pad, dtype, which):
    n = 13
    rng = np.random.default_rng(v + pad)
    z, u = logits(n, v, dtype, v, 2.0, pad), rng.random(n, dtype=np.float32)
    u[0], u[1] = 0.0, np.float32(1) - np.float32(2.0 ** -24)
    params = {}
    if "t" in which:
        params["temperature"] = rng.choice([0.0, 0.1, 0.7, 1.0, 1.9], n)
    if "k" in which:
        params["top_k"] = rng.choice([0, 1, 2, 5, 50, v - 1, v, v + 1], n)
    if "p" in which:
        params["top_p"] = rng.choice([0.0, 0.05, 0.5, 0.9, 0.99, 1.0, 2.0], n)
    if "m" in which:
        params["min_p"] = rng.choice([0.0, 0.01, 0.1, 0.6, 1.0, 3.0], n)
    check(z, u, **params)


@pytest.mark.parametrize("v", [32768, 50001, 65536, 131072, 262145])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_of_large_vocabularies(v, dtype):
    n = 6
    rng = np.random.default_rng(v)
    z = logits(n, v, dtype, v, 1.5, 3)
    u = rng.random(n, dtype=np.float32)
    check(z, u)
    check(z, u, temperature=[0.8] * n, top_k=[0, 1, 40, 1000, v // 2, v - 1], top_p=[1, 0.9, 0.999, 0.5, 0.9, 0.3], min_p=[0, 0, 0.001, 0, 0.01, 0])


def test_equal_logits_go_by_index():
    n, v = 9, 1000
    for value in (0.0, -3.5, 100.0):
        z = torch.full((n, v), value, device="cuda")
        u = np.linspace(0, 0.999, n).astype(np.float32)
        assert np.array_equal(check(z, u), (u.astype(np.float64) * v).astype(int))
        assert check(z, u, top_k=[10] * n).max() < 10
        assert check(z, u, top_p=[0.25] * n).max() < 250
        check(z, u, top_k=[500] * n, top_p=[0.1] * n, min_p=[1.0] * n)
    z = torch.zeros(2, v, device="cuda")
    z[:, ::2] = -0.0                                     # equal to zero
    check(z, [0.1, 0.9], top_k=[3, 4])
    z = torch.randint(-2, 3, (40, 3000), device="cuda").float()      # many ties at every border
    rng = np.random.default_rng(1)
    check(z, rng.random(40), top_k=rng.integers(1, 3000, 40), top_p=rng.random(40))
    check(z, rng.random(40), temperature=[0.0] * 40)


def test_masked_rows_and_values():
    n, v = 8, 500
    z = logits(n, v, "f32", 3).contiguous()
    z[0] = -np.inf                                       # nothing is left
    z[1] = np.nan
    z[2, 5:] = -np.inf
    z[3] = -np.inf
    z[3, 499] = -2.0                                     # one token
    z[4, 7] = np.inf
    z[4, 9] = np.inf
    z[5, 100] = np.nan
    z[6] = torch.finfo(torch.float32).min                # a mask of the type's lowest value, everywhere
    z[7] = torch.finfo(torch.float32).min
    z[7, 33] = 1.0
    rng = np.random.default_rng(4)
    for _ in range(4):
        u = rng.random(n).astype(np.float32)
        got = check(z, u)
        assert got[0] == got[1] == -1 and got[2] < 5 and got[3] == 499 and got[4] in (7, 9) and got[7] == 33
        check(z, u, temperature=[0.9] * n, top_k=[3] * n, top_p=[0.8] * n, min_p=[0.05] * n)
        check(z, u, temperature=[0.0] * n)
    check(logits(3, 2000, "bf16", 9), [0.2, 0.5, 0.9], temperature=[1e-30, 1e30, np.inf])


def test_numbers_outside_their_range():
    z = logits(6, 300, "f32", 5)
    u = np.array([-1.0, np.nan, 1.0, 2.0, np.inf, 0.0], np.float32)
    got = draw(z, torch.from_numpy(u).cuda(), top_k=torch.full((6,), 4, device="cuda", dtype=torch.int64))
    host = z.cpu().numpy()
    for n, t in enumerate(got):
        best = sorted(sorted(range(300), key=lambda i: (-host[n, i], i))[:4])
        assert t == (best[-1] if u[n] >= 1 else best[0])
    nan = torch.full((6,), float("nan"), device="cuda")
    ok = torch.full((6,), 0.5, device="cuda")
    first = host.argmax(1)
    assert np.array_equal(draw(z, ok, temperature=nan), first)                       # not above 0: the best token
    assert np.array_equal(draw(z, ok, top_p=nan, min_p=nan), draw(z, ok))
    assert np.array_equal(draw(z, ok, top_k=torch.full((6,), -2 ** 40, device="cuda", dtype=torch.int64)), draw(z, ok))
    assert np.array_equal(draw(z, ok, top_k=torch.full((6,), 2 ** 40, device="cuda", dtype=torch.int64)), draw(z, ok))


def test_one_parameter_for_all_rows():
    z, u = logits(20, 700, "f32", 6), torch.rand(20, device="cuda")
    one = lambda x, dt=torch.float32: torch.tensor([x], device="cuda", dtype=dt).expand(20)
    full = lambda x, dt=torch.float32: torch.full((20,), x, device="cuda", dtype=dt)
    a = draw(z, u, temperature=one(0.7), top_k=one(9, torch.int64), top_p=one(0.8), min_p=one(0.02))
    assert np.array_equal(a, draw(z, u, temperature=full(0.7), top_k=full(9, torch.int32), top_p=full(0.8), min_p=full(0.02)))
    every = torch.rand(40, device="cuda")[::2]           # a view of every second number
    assert np.array_equal(draw(z, every), draw(z, every.contiguous()))


def test_tokens_come_as_often_as_their_weights_say():
    # 20000 draws from five tokens: each count within five standard deviations
    p = np.array([0.4, 0.3, 0.15, 0.1, 0.05])
    n = 20000
    z = torch.log(torch.from_numpy(p)).float().cuda().expand(n, 5)
    z = z.contiguous()
    g = torch.Generator(device="cuda").manual_seed(8)
    counts = np.bincount(draw(z, torch.rand(n, generator=g, device="cuda")), minlength=5)
    assert np.all(np.abs(counts - n * p) < 5 * np.sqrt(n * p * (1 - p)))


@pytest.mark.parametrize("v", [30000, 100000])           # a block for a row, and rows in chunks
def test_sample_on_a_stream_and_in_a_graph(v):
    z, u = logits(5, v, "f32", 10).contiguous(), torch.rand(5, device="cuda")
    k = torch.tensor([20, 0, 20, 0, 1], device="cuda", dtype=torch.int32)
    want = []
    inputs = [(logits(5, v, "f32", 20 + i).contiguous(), torch.rand(5, device="cuda")) for i in range(3)]
    for zi, ui in inputs:
        want.append(draw(zi, ui, top_k=k))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = draw(*inputs[0], top_k=k)
    assert np.array_equal(got, want[0])
    out, ws = torch.empty(5, dtype=torch.int64, device="cuda"), torch.empty(max(256, B.sample_workspace_bytes(z)), dtype=torch.uint8, device="cuda")
    B.sample(z, u, out, top_k=k, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sample(z, u, out, top_k=k, ws=ws)
    for (zi, ui), w in zip(inputs, want):
        z.copy_(zi)
        u.copy_(ui)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), w)
        B.sample(torch.zeros(2, 9, device="cuda"), torch.rand(2, device="cuda"), torch.empty(2, dtype=torch.int64, device="cuda"))


@pytest.mark.parametrize("v", [32769, 65536, 70003, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_every_kind_in_one_batch(v, dtype):
    """Long rows are cut in chunks where the call brings a workspace: every way a row can go, beside all the others, and the same tokens without."""
    n = 24
    rng = np.random.default_rng(v)
    z = logits(n, v, dtype, v + 1, 2.0, 1)
    z[0] = -np.inf                                       # nothing to choose from
    z[1] = 0.25                                          # all equal
    z[2, 10:] = float("nan")
    z[3, ::3] = np.inf                                   # equal infinities
    z[4] = torch.finfo(z.dtype).min
    z[5, :-1] = -np.inf                                  # one token, the last
    z[6] = torch.round(z[6] * 2) / 2                     # few values, many ties at every border
    z[7] = torch.round(z[7] * 2) / 2
    z[8] = z[8] * 1e-3                                   # nearly flat
    z[9] = z[9] * 1e4
    z[10, 100] = np.inf                                  # one infinity
    params = dict(temperature=rng.choice([0.0, 0.5, 1.0, 1.7], n), top_k=rng.choice([0, 0, 1, 50, 600, 5000, v], n),
                  top_p=rng.choice([1.0, 0.0, 0.3, 0.9, 0.999], n), min_p=rng.choice([0.0, 0.0, 0.01, 0.3, 1.0], n))
    params["temperature"][:12] = 0.9
    u = rng.random(n, dtype=np.float32)
    u[12], u[13] = 0.0, np.nextafter(np.float32(1), np.float32(0))
    for names in ((), ("top_k",), ("top_p",), ("min_p",), ("temperature", "top_p", "min_p"), ("temperature", "top_k", "top_p", "min_p")):
        check(z, u, **{k: params[k] for k in names})


def test_two_calls_at_once_have_their_own_workspaces():
    v = 131072
    a, b = logits(3, v, "f32", 31).contiguous(), logits(5, v, "f32", 32).contiguous()
    ua, ub = torch.rand(3, device="cuda"), torch.rand(5, device="cuda")
    p = torch.full((5,), 0.9, device="cuda")
    alone = draw(a, ua, top_p=p[:3]), draw(b, ub, top_p=p)
    torch.cuda.synchronize()
    streams, outs, spaces = [torch.cuda.Stream() for _ in range(2)], [], []
    for s, z, u in zip(streams, (a, b), (ua, ub)):
        spaces.append(torch.empty(B.sample_workspace_bytes(z), dtype=torch.uint8, device="cuda"))
        outs.append(torch.empty(z.shape[0], dtype=torch.int64, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(4):
        for s, z, u, o, w in zip(streams, (a, b), (ua, ub), outs, spaces):
            with torch.cuda.stream(s):
                B.sample(z, u, o, top_p=p[:z.shape[0]], ws=w)
    torch.cuda.synchronize()
    assert np.array_equal(outs[0].cpu().numpy(), alone[0]) and np.array_equal(outs[1].cpu().numpy(), alone[1])


def test_a_row_for_every_block_beyond_a_line_of_the_grid():
    n = 2 ** 20 + 3
    z = torch.randn(n, 3, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    u = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    out = torch.empty(n, dtype=torch.int32, device="cuda")
    B.sample(z, u, out)
    w = torch.exp(z.double() - z.double().max(1, keepdim=True).values)
    cum = torch.cumsum(w, 1)
    want = (cum > u.double()[:, None] * cum[:, -1:]).to(torch.uint8).argmax(1).int()
    assert torch.equal(out, want)


@pytest.mark.parametrize("v", [5000, 70001])
def test_more_tokens_in_the_bin_of_a_border_than_are_ordered_by_comparing(v):
    """Bins have equal width between the largest and the smallest logit: one that lies far off leaves all others in one bin."""
    n = 10
    rng = np.random.default_rng(v)
    z = logits(n, v, "f32", v + 2, 1e-3).contiguous()
    z[:5, v // 2] = -500.0
    z[5:, v // 3] = 12.0
    z[1] = z[1].bfloat16().float()                       # ties
    z[2, : v // 2] = 0.0                                 # equals only, up to the one far off
    z[2, v // 2 + 1:] = 0.0
    z[6] = torch.where(z[6] == 12.0, 12.0, -0.5)
    z[7] = z[7].bfloat16().float()
    z[3, ::7] = -np.inf
    z[8, ::7] = float("nan")
    u, k = rng.random(n, dtype=np.float32), rng.integers(1500, v - v // 6, n)
    p, t = rng.uniform(0.2, 0.95, n), rng.choice([0.7, 1.0, 1.6], n)
    for _ in range(3):
        check(z, u, top_k=k)
        check(z, u, top_p=p)
        check(z, u, temperature=t, top_k=k, top_p=p)
        check(z, u, temperature=t, top_k=k, top_p=p, min_p=[0.999] * 5 + [1e-5] * 5)
        u, k, p = np.roll(u, 1), np.roll(k, 1), np.roll(p, 1)


@pytest.mark.parametrize("v", [5, 61, 255, 256, 257, 300, 512])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_short_rows_of_every_kind_in_one_batch(v, dtype):
    n = 31
    rng = np.random.default_rng(v)
    z = logits(n, v, dtype, v + 5, 2.0, 1)
    z[0] = -np.inf                                       # nothing to choose from
    z[1] = 0.25                                          # all equal
    z[2, 2:] = float("nan")
    z[3, ::3] = np.inf                                   # equal infinities
    z[4] = torch.finfo(z.dtype).min
    z[5, :-1] = -np.inf                                  # one token, the last
    z[6] = torch.round(z[6])                             # ties at every border
    z[7] = torch.round(z[7])
    z[8] = z[8] * 1e-3                                   # nearly flat
    z[9] = z[9] * 1e4
    z[10, v // 2] = np.inf                               # one infinity
    z[11, ::2] = -0.0                                    # equal to zero
    z[11, 1::2] = 0.0
    u = rng.random(n, dtype=np.float32)
    u[12], u[13] = 0.0, np.nextafter(np.float32(1), np.float32(0))
    for _ in range(4):
        params = dict(temperature=rng.choice([0.0, 0.5, 1.0, 1.7], n), top_k=rng.choice([0, 0, 1, 2, 5, v // 2, v - 1, v, v + 7], n),
                      top_p=rng.choice([1.0, 0.0, 0.3, 0.9, 0.999], n), min_p=rng.choice([0.0, 0.0, 0.01, 0.3, 1.0], n))
        params["temperature"][:12] = 0.9
        for names in ((), ("top_k",), ("top_p",), ("min_p",), ("top_k", "top_p"), ("temperature", "top_p", "min_p"), ("temperature", "top_k", "top_p", "min_p")):
            check(z, u, **{k: params[k] for k in names})
        u = rng.random(n, dtype=np.float32)


@pytest.mark.parametrize("v", [9, 200, 400])
def test_the_ends_of_the_range_in_short_rows(v):
    z = logits(12, v, "f32", v + 6)
    z[0, 0] = z[1, v - 1] = -150.0                       # weights that are zero in sums, and the lightest token all the same
    z[2] = -np.inf
    z[3, 1] = np.inf
    u = np.array([-1.0, 2.0, 1.0, 1.0, 1.0, np.nan, 0.0, np.inf, -np.inf, 1.5, 1.0, -3.0], np.float32)
    got = draw(z, torch.from_numpy(u).cuda())
    host = z.double().cpu().numpy()
    for n, t in enumerate(got):
        some = np.flatnonzero(host[n] == np.inf) if n == 3 else np.flatnonzero(host[n] > -np.inf)
        assert t == (-1 if n == 2 else some[-1] if u[n] >= 1 else some[0]), n
    k = torch.full((12,), 3, device="cuda", dtype=torch.int32)
    got = draw(z, torch.from_numpy(u).cuda(), top_k=k)
    for n, t in enumerate(got):
        if n in (2, 3):
            assert t == (-1 if n == 2 else 1), n
        else:
            best = sorted(sorted(range(v), key=lambda i: (-host[n, i], i))[:3])
            assert t == (best[-1] if u[n] >= 1 else best[0]), n


@pytest.mark.parametrize("n,v", [(2 ** 22 + 5, 3), (2 ** 20 + 3, 260)])      # four rows to a block, and a block for each
def test_more_rows_than_a_line_of_the_grid_has_blocks(n, v):
    z = torch.randint(-3, 4, (n, v), device="cuda", dtype=torch.int8, generator=torch.Generator(device="cuda").manual_seed(4)).to(torch.bfloat16)
    out = torch.empty(n, dtype=torch.int32, device="cuda")
    B.sample(z, torch.full((n,), 0.5, device="cuda"), out, temperature=torch.zeros(n, device="cuda"))
    for a in range(0, n, 2 ** 18):                       # the first of the largest
        part = z[a:a + 2 ** 18].float()
        assert torch.equal(out[a:a + 2 ** 18], (part == part.max(1, keepdim=True).values).to(torch.uint8).argmax(1).int()), a
