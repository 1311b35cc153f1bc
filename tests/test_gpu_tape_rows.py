"""Residual blocks, dropout, layer normalisation and generation as the tape's models use them, on the GPU: against the same models on the oracle's
kernels in 64 bits (the masks are the same, bit for bit), and captured in a graph."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_1908_00213_amd import tape as T
from paper_1908_00213_amd import workloads as W
from rows_backend import RowsBackend
from util import bf16r, check, host

pytestmark = pytest.mark.gpu


def cmp(got, ref, tol, what):
    ref = np.asarray(ref, dtype=np.float64)
    check(host(got), ref, tol, float(np.max(np.abs(ref))) if ref.size else 0.0, what)


def mlp_data(sizes, batch, seed, exact=False):
    rng = np.random.default_rng(seed)
    f32 = lambda a: bf16r(a) if exact else np.asarray(a, np.float32)
    params = [(f32(rng.standard_normal((o, i)) / np.sqrt(i)), np.asarray(0.1 * rng.standard_normal(o), np.float32)) for i, o in zip(sizes[:-1], sizes[1:])]
    norms = [(np.asarray(1 + 0.2 * rng.standard_normal(o), np.float32), np.asarray(0.2 * rng.standard_normal(o), np.float32)) for o in sizes[1:-1]]
    return params, norms, f32(rng.standard_normal((batch, sizes[0]))), rng.integers(0, sizes[-1], batch)


def mlp(F, data, lowp, norms=True):
    params, ns, _, _ = data
    put = lambda pairs: [(F.from_numpy(a), F.from_numpy(b)) for a, b in pairs]
    return T.MLP(put(params), "gelu", lowp, norms=put(ns) if norms else None, ratio=0.2, masks=T.Masks(77, 5))


# fp32: the bar of the other tape tests.  bf16: every layer stores five values of the longest path (its output, its normalisation, and three
# gradients), each off by half a step, 2^-8, and operands are rounded once more on either side of three layers.
@pytest.mark.parametrize("lowp,tol", [(False, 1e-4), (True, 21 * 2.0 ** -8)])
@pytest.mark.parametrize("sizes,batch", [((40, 96, 96, 96, 10), 64), ((33, 65, 65, 130, 7), 50)])
@pytest.mark.parametrize("norms", [True, False])
def test_residual_mlp(sizes, batch, lowp, tol, norms):
    if lowp:
        sizes = tuple((s + 7) // 8 * 8 for s in sizes)
    data = mlp_data(sizes, batch, 1, lowp)

    def step(F):
        model = mlp(F, data, lowp and not isinstance(F, RowsBackend), norms)
        x = F.from_numpy(data[2], "bf16" if lowp else None)
        loss = model.loss(T.Variable(x, False), F.from_numpy(data[3]))
        loss.backward()
        return loss, model
    loss, model = step(T.backend())
    assert T.live_function_nodes() == 0
    with T.using_backend(RowsBackend()) as O:
        want, ref = step(O)
    assert abs(float(loss.array.cpu()) - float(want.array)) <= tol * max(1.0, abs(float(want.array)))
    assert len(model.params()) == len(ref.params()) == (14 if norms else 8)
    for k, (p, q) in enumerate(zip(model.params(), ref.params())):
        assert p.grad.dtype == torch.float32
        cmp(p.grad, q.grad, tol, "parameter %d" % k)


@pytest.mark.parametrize("n_step,lowp,tol", [(False, False, 1e-4), (True, False, 1e-4), (True, True, 21 * 2.0 ** -8)])
def test_regularised_language_model(n_step, lowp, tol):
    w = W.config4(vocab=300, embed=72, hidden=96, batch=16, bptt=6)
    P = {k: (bf16r(v) if lowp else v) for k, v in w.params.items()}
    rng = np.random.default_rng(8)
    P["gamma"], P["beta"] = np.asarray(1 + 0.1 * rng.standard_normal(96), np.float32), np.asarray(0.1 * rng.standard_normal(96), np.float32)

    def step(F):
        low = lowp and not isinstance(F, RowsBackend)
        model = T.LSTMLanguageModel({k: F.from_numpy(v) for k, v in P.items()}, n_step, low, ratio=0.3, masks=T.Masks(4))
        model.masks.advance()
        loss, _ = model.loss(F.from_numpy(w.ids.reshape(-1)), F.from_numpy(w.targets.reshape(-1)), w.bptt)
        loss.backward()
        return loss, model
    loss, model = step(T.backend())
    assert T.live_function_nodes() == 0
    with T.using_backend(RowsBackend()) as O:
        want, ref = step(O)
    assert abs(float(loss.array.cpu()) - float(want.array)) <= tol * abs(float(want.array))
    for k in P:
        cmp(model.P[k].grad, ref.P[k].grad, tol, "d" + k)


@pytest.mark.parametrize("n_step,lowp", [(False, False), (True, False), (True, True)])
def test_generation(n_step, lowp):
    """Every token is the oracle's choice from the model's own logits."""
    F = T.backend()
    w = W.config4(vocab=500, embed=64, hidden=64, batch=12, bptt=5)
    model = T.LSTMLanguageModel({k: F.from_numpy(v) for k, v in w.params.items()}, n_step, lowp, ratio=0.5, masks=T.Masks(1))
    rng = np.random.default_rng(9)
    n, ids = 7, F.from_numpy(w.ids.reshape(-1))
    u = rng.random((n, 12), dtype=np.float32)
    filters = dict(temperature=np.asarray(rng.choice([0.0, 0.7, 1.2], 12), np.float32), top_k=rng.integers(0, 60, 12), top_p=np.full(12, 0.95, np.float32), min_p=None)
    dev = {k: None if v is None else F.from_numpy(v) for k, v in filters.items()}
    tokens, (c, h) = model.generate(ids, w.bptt, F.from_numpy(u), **dev)
    assert tokens.shape == (n, 12) and tokens.dtype == torch.int64 and model.train
    got = F.to_numpy(tokens)
    model.train = False
    text, steps, state = ids, w.bptt, None
    for t in range(n):
        with T.no_backprop_mode():
            hs, state = model._hidden(text, steps, state)
            last = model._logits(T.Variable(hs.array[-12:], False)).array
        assert np.array_equal(got[t], R.sample(last.float().cpu().numpy(), u[t], **filters)), t
        text, steps = tokens[t], 1
    one, _ = model.generate(ids, w.bptt, F.from_numpy(u), temperature=0.0, top_k=3)
    assert np.array_equal(F.to_numpy(one)[0], F.to_numpy(model._logits(model._hidden(ids, w.bptt, None)[0]).array)[-12:].argmax(1))


@pytest.mark.parametrize("lowp", [False, True])
def test_a_captured_step_draws_new_masks_at_every_replay(lowp):
    F = T.backend()
    data = mlp_data((64, 128, 128, 128, 16), 96, 3, True)
    x, t = F.from_numpy(data[2], "bf16" if lowp else None), F.from_numpy(data[3])

    def run(model):
        model.masks.advance()
        loss = model.loss(T.Variable(x, False), t)
        loss.backward()
        opt = T.SGD(model.params(), 0.05)
        opt.update()
        opt.cleargrads()
        return loss.array
    eager = mlp(F, data, lowp)
    losses = [float(run(eager)) for _ in range(4)]
    assert len(set(losses)) == 4
    graphed, graph = mlp(F, data, lowp), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = run(graphed)
    other = mlp(F, data, lowp)
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert float(out) == losses[k], k
        run(other)                                       # eager work between the replays
    for p, q in zip(eager.params(), graphed.params()):
        assert torch.equal(p.array, q.array)
