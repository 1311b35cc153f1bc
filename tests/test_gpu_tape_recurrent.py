"""The gated language model on the GPU: against the same model on the oracle's kernels in 64 bits, trained in a captured graph, answering token by token."""
import numpy as np
import pytest
import torch

from oracle import recurrent as R
from oracle import rows
from paper_1908_00213_amd import tape as T
from recurrent_backend import RecurrentBackend, gated_params
from util import bf16r, check, host

pytestmark = pytest.mark.gpu


def cmp(got, ref, tol, what):
    ref = np.asarray(ref, dtype=np.float64)
    check(host(got), ref, tol, float(np.max(np.abs(ref))) if ref.size else 0.0, what)


def data(V, H, n, Bn, exact, seed=1):
    rng = np.random.default_rng(seed)
    f32 = lambda k, a: bf16r(a) if exact and (k == "E" or k[0] == "W") else np.asarray(a, np.float32)
    P = {k: f32(k, v) for k, v in gated_params(rng, V, H).items()}
    ids, targets = rng.integers(0, V, n * Bn), rng.integers(0, V, n * Bn)
    return P, ids, targets


# fp32: the bar of the other tape tests.  bf16: the longest path stores a normalised value, gates and inputs, and states in each of two layers, and the gradient of each of
# them (12), the first normalisation and its gradient, and the logits' gradient (3), each off by half a step, 2^-8; operands are rounded once more on either side of three products (6).
@pytest.mark.parametrize("lowp,tol", [(False, 1e-4), (True, 21 * 2.0 ** -8)])
@pytest.mark.parametrize("V,H,n,Bn,ragged", [(300, 64, 9, 16, False), (77, 40, 150, 3, True), (50, 24, 300, 2, False)])
def test_model(V, H, n, Bn, ragged, lowp, tol):
    P, ids, targets = data(V, H, n, Bn, lowp)
    lengths = np.array([n, n // 2, 17][:Bn]) if ragged else None
    if ragged:
        targets[(np.arange(n)[:, None] >= lengths[None]).reshape(-1)] = -1

    def step(F):
        low = lowp and not isinstance(F, RecurrentBackend)
        model = T.GatedLanguageModel({k: F.from_numpy(v) for k, v in P.items()}, low, ratio=0.2, masks=T.Masks(3))
        model.masks.advance()
        loss, state = model.loss(F.from_numpy(ids), F.from_numpy(targets), n, lengths=None if lengths is None else F.from_numpy(lengths))
        loss.backward()
        return loss, model, state
    loss, model, state = step(T.backend())
    assert T.live_function_nodes() == 0
    with T.using_backend(RecurrentBackend()) as O:
        want, ref, end = step(O)
    assert abs(float(loss.array.cpu()) - float(want.array)) <= tol * abs(float(want.array))
    for a, b in zip(state, end):
        assert a.array.dtype == torch.float32
        cmp(a.array, b.array, tol, "state")
    for k in P:
        assert model.P[k].grad.dtype == torch.float32
        cmp(model.P[k].grad, ref.P[k].grad, tol, "d" + k)


@pytest.mark.parametrize("lowp", [False, True])
def test_a_captured_training_step(lowp):
    F = T.backend()
    P, ids, targets = data(500, 64, 140, 4, lowp)
    ids, targets = F.from_numpy(ids), F.from_numpy(targets)

    def make():
        return T.GatedLanguageModel({k: F.from_numpy(v) for k, v in P.items()}, lowp, ratio=0.1, masks=T.Masks(9))

    def run(model):
        model.masks.advance()
        loss, _ = model.loss(ids, targets, 140)
        loss.backward()
        opt = T.SGD(model.params(), 0.1)
        opt.update()
        opt.cleargrads()
        return loss.array
    eager = make()
    losses = [float(run(eager)) for _ in range(4)]
    assert len(set(losses)) == 4
    graphed, graph = make(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = run(graphed)
    other = make()
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert float(out) == losses[k], k
        run(other)                                       # eager work between the replays
    for p, q in zip(eager.params(), graphed.params()):
        assert torch.equal(p.array, q.array)


@pytest.mark.parametrize("lowp", [False, True])
def test_generation(lowp):
    """Every token is the oracle's choice from the model's own logits, as the definition adjusts them."""
    F = T.backend()
    n, Bn, V, more = 5, 12, 700, 8
    P, ids, _ = data(V, 64, n, Bn, lowp)
    model = T.GatedLanguageModel({k: F.from_numpy(v) for k, v in P.items()}, lowp, ratio=0.3, masks=T.Masks(1))
    rng = np.random.default_rng(2)
    u = rng.random((more, Bn), dtype=np.float32)
    words = rng.integers(-2 ** 31, 2 ** 31, (V + 31) // 32).astype(np.int32)
    k = dict(repetition=np.float32(1.25), frequency=np.asarray(rng.random(Bn), np.float32), presence=0.5, bias_ids=np.arange(20) * 7, bias=np.float32(rng.standard_normal(20)),
             allowed=words)
    tokens, state = model.generate(F.from_numpy(ids), n, F.from_numpy(u), temperature=0.8, top_k=40, **k)
    got = F.to_numpy(tokens)
    assert got.shape == (more, Bn) and model.train and len(state) == 2
    # (generate's own logits: the same calls, prompt at once and then step by step)
    text, steps, st = F.from_numpy(ids), n, None
    for t in range(more):
        with T.no_backprop_mode():
            y, st = model._hidden(text, steps, st, 0.0)
            z = model._logits(T.Variable(y.array[-Bn:], False), 0.0).array
        history = np.concatenate([ids.reshape(n, Bn), got[:t]]).T
        want, bound = R.adjust(host(z), history, None, np.full(Bn, n), np.full(Bn, np.float32(1.25)), k["frequency"], np.full(Bn, 0.5), np.tile(k["bias_ids"], (Bn, 1)),
                               np.tile(k["bias"], (Bn, 1)), np.tile(words, (Bn, 1)))
        adjusted = torch.empty_like(z)
        rep = lambda a: F.from_numpy(np.tile(a, (Bn, 1)))
        F.logits_adjust(z, adjusted, tokens=F.from_numpy(np.ascontiguousarray(history)), prompt=F.from_numpy(np.full(Bn, n)), repetition=F.from_numpy(np.full(Bn, np.float32(1.25))),
                        frequency=F.from_numpy(k["frequency"]), presence=F.from_numpy(np.full(Bn, np.float32(0.5))), bias_ids=rep(k["bias_ids"]), bias=rep(k["bias"]), allowed=rep(words))
        ok = ~np.isneginf(want)
        a = host(adjusted)
        assert np.array_equal(np.isneginf(a), ~ok) and (np.abs(a[ok] - want[ok]) <= bound[ok] + R.U * np.abs(want[ok])).all()
        assert np.array_equal(rows.sample(a, u[t], np.full(Bn, np.float32(0.8)), np.full(Bn, 40)), got[t]), t
        text, steps = tokens[t], 1


def test_a_sequence_at_once_and_step_by_step():
    """The recurrence's states over 300 steps are those of 300 calls of one step each, up to the roundings of both ways of grouping them."""
    F = T.backend()
    P, ids, _ = data(60, 48, 300, 2, False)
    model = T.GatedLanguageModel({k: F.from_numpy(v) for k, v in P.items()})
    d = F.from_numpy(ids)
    with T.no_backprop_mode():
        whole, after = model._hidden(d, 300, None)
        state, ys = None, []
        for t in range(300):
            y, state = model._hidden(d[t * 2:(t + 1) * 2], 1, state)
            ys.append(y.array)
    cmp(torch.cat(ys), host(whole.array), 1e-4, "hidden")
    for a, b in zip(state, after):
        cmp(a.array, host(b.array), 1e-4, "state")


def test_gradients_of_the_gpus_own_types():
    """Gradients that come in fp32 for bfloat16 states, and arrays that are views of others."""
    F = T.backend()
    rng = np.random.default_rng(6)
    n, Bn, H = 40, 3, 10
    wide = F.from_numpy(rng.standard_normal((n * Bn, 2 * H + 3)).astype(np.float32), "bf16")
    z, h0 = T.Variable(wide[:, 1:2 * H + 1]), T.Variable(F.from_numpy(rng.standard_normal((H, Bn)).astype(np.float32)).T)
    w = F.from_numpy(rng.standard_normal((n * Bn, H)).astype(np.float32))
    h, hs = T.gated_scan(h0, z, n, out_dtype="f32")
    T.add(T.sum_all(T.mul(hs, T.Variable(w, False))), T.sum_all(h)).backward()
    zz = host(z.array).reshape(n, Bn, 2 * H)
    (dg, dx, d0), _ = R.gated_scan_bwd(zz[:, :, :H], zz[:, :, H:], host(h0.array), host(w).reshape(n, Bn, H), np.ones((Bn, H)), "sigmoid")
    assert z.grad.dtype == torch.bfloat16
    cmp(z.grad, np.concatenate([dg, dx], 2).reshape(n * Bn, 2 * H), 2.0 ** -8, "dz")
    cmp(h0.grad, d0, 1e-4, "dh0")
