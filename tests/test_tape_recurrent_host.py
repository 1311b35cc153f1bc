"""The gated language model and its functions on the tape, without a GPU: gradients against differences, gradients of gradients, what is kept and released,
what generation hands to its kernels, what is refused."""
import numpy as np
import pytest

from oracle import recurrent as R
from oracle import rows
from paper_1908_00213_amd import tape as T
from recurrent_backend import RecurrentBackend, gated_params
from test_tape_rows_host import check_against_differences, lm_params


@pytest.mark.parametrize("lengths", [None, [4, 0, 6]])
@pytest.mark.parametrize("ratio", [0.0, 0.3])
def test_model_gradients(ratio, lengths):
    rng = np.random.default_rng(1)
    P = gated_params(rng)
    n, Bn = 6, 3
    ids, targets = rng.integers(-1, 11, n * Bn), rng.integers(0, 11, n * Bn)
    if lengths is not None:
        targets[(np.arange(n)[:, None] >= np.array(lengths)[None]).reshape(-1)] = -1
    h = [rng.standard_normal((Bn, 6)) for _ in range(2)]
    with T.using_backend(RecurrentBackend()) as F:
        model = T.GatedLanguageModel(P, ratio=ratio, masks=T.Masks(5) if ratio else None)
        start = [T.Variable(a) for a in h]
        ln = None if lengths is None else np.array(lengths)

        def run():
            if ratio:
                model.masks.sites = 0
            loss, after = model.loss(ids, targets, n, start, ln)
            return T.add(loss, T.add(T.sum_all(after[0]), T.sum_all(after[1])))
        l = run()
        l.backward()
        assert T.live_function_nodes() == 0
        ps = model.params() + start
        assert all(p.grad is not None for p in ps)
        check_against_differences(lambda: float(run().array), [p.array for p in ps], [p.grad.copy() for p in ps], rng)
        assert ("embed_sorted_bwd", False) in F.calls


@pytest.mark.parametrize("kind", ["sigmoid", "decay"])
def test_scan_node(kind):
    rng = np.random.default_rng(2)
    n, Bn, H = 5, 2, 3
    z, h0 = T.Variable(rng.standard_normal((n * Bn, 2 * H))), T.Variable(rng.standard_normal((Bn, H)))
    with T.using_backend(RecurrentBackend()) as F:
        h, hs = T.gated_scan(h0, z, n, kind)
        assert np.array_equal(h.array, hs.array[-Bn:])
        # only the last state, only the others, and both
        for pick in (lambda h, hs: T.sum_all(T.mul(h, h)), lambda h, hs: T.sum_all(T.mul(hs, hs)), lambda h, hs: T.add(T.sum_all(T.mul(h, h)), T.sum_all(hs))):
            z.cleargrad(), h0.cleargrad()
            loss = lambda: pick(*T.gated_scan(h0, z, n, kind))
            loss().backward()
            check_against_differences(lambda: float(loss().array), [z.array, h0.array], [z.grad.copy(), h0.grad.copy()], rng)
        # nothing is kept for a backward pass that will not come
        F.calls.clear()
        with T.no_backprop_mode():
            T.gated_scan(h0, z, n, kind)
        T.gated_scan(T.Variable(h0.array, False), T.Variable(z.array, False), n, kind)
        assert [c[1] for c in F.calls] == [False, False]
        for bad in (lambda: T.gated_scan(h0, z, 4, kind), lambda: T.gated_scan(h0, z, 0, kind), lambda: T.gated_scan(h0, z, n, kind, np.zeros(3, np.int64))):
            with pytest.raises(ValueError):
                bad()


def test_lookup_used_twice_and_its_gradients_gradient():
    rng = np.random.default_rng(3)
    table, a, b = T.Parameter(rng.standard_normal((5, 4))), rng.integers(-1, 6, 7), rng.integers(0, 5, 3)
    with T.using_backend(RecurrentBackend()) as F:
        y = T.add(T.sum_all(T.mul(T.embed_scaled(a, table, 3.0), T.embed_scaled(a, table, 3.0))), T.sum_all(T.embed_scaled(b, table, 0.5)))
        y.backward()
        want = R.embed_scaled_bwd(a, 2 * R.embed_scaled(table.array, a, 3.0), 5, 3.0)[0] + R.embed_scaled_bwd(b, np.ones((3, 4)), 5, 0.5)[0]
        assert np.allclose(table.grad, want, rtol=0, atol=1e-12)
        assert ("embed_sorted_bwd", True) in F.calls                 # the second one adds to the first
        y = T.embed_scaled(a, table, 2.0)
        g, = T.grad([T.sum_all(T.mul(y, T.mul(y, y)))], [table], enable_double_backprop=True)
        table.cleargrad()
        T.sum_all(T.mul(g, g)).backward()
        # d/dt of the sum of (2 * 3 y^2 summed by rows)^2
        e = R.embed_scaled(table.array, a, 2.0)
        first = R.embed_scaled_bwd(a, 3 * e * e, 5, 2.0)[0]
        want = R.embed_scaled_bwd(a, R.embed_scaled(2 * first, a, 2.0) * 6 * e, 5, 2.0)[0]
        assert np.allclose(table.grad, want, rtol=1e-10, atol=1e-10)


def sequence(model, F, ids, n, lengths=None):
    with T.no_backprop_mode():
        y, _ = model._hidden(ids, n, None, 0.0, lengths) if lengths is not None else model._hidden(ids, n, None, 0.0)
        return model._logits(y, 0.0).array


@pytest.mark.parametrize("which", ["gated", "lstm"])
def test_generation_with_penalties(which):
    """Every token is the oracle's choice from the logits that the definition makes of the text so far."""
    rng = np.random.default_rng(4)
    n, Bn, V, more = 4, 3, 11, 6
    ids, u = rng.integers(0, V, n * Bn), rng.random((more, Bn))
    allowed = np.array([0b11111011111], np.int32)
    with T.using_backend(RecurrentBackend()) as F:
        model = T.GatedLanguageModel(gated_params(rng)) if which == "gated" else T.LSTMLanguageModel(lm_params(rng), n_step=True)
        k = dict(repetition=1.4, frequency=np.array([0.3, 0.0, 1.0]), presence=[0.5] * Bn, bias_ids=[2, 7, 2], bias=[0.5, -2.0, 0.25], allowed=allowed)
        tokens, _ = model.generate(ids, n, u, temperature=0.9, top_k=5, **k)
        text = np.concatenate([ids.reshape(n, Bn), tokens])
        assert (tokens != 5).all()
        for t in range(more):
            z = sequence(model, F, text[:n + t].reshape(-1), n + t)[-Bn:]
            z, _ = R.adjust(z, text[:n + t].T, None, np.full(Bn, n), np.full(Bn, 1.4), k["frequency"], np.full(Bn, 0.5), np.tile([2, 7, 2], (Bn, 1)),
                            np.tile([0.5, -2.0, 0.25], (Bn, 1)), np.tile(allowed, (Bn, 1)))
            assert np.array_equal(rows.sample(z, u[t], np.full(Bn, 0.9), np.full(Bn, 5)), tokens[t])
        # a mask alone asks for no text
        F.calls.clear()
        got, _ = model.generate(ids, n, u, allowed=np.array([1 << 3], np.int32))
        assert (got == 3).all() and F.calls.count(("logits_adjust", None)) == more
        F.calls.clear()
        plain, _ = model.generate(ids, n, u)
        assert ("logits_adjust", None) not in F.calls
        again, _ = model.generate(ids, n, u, repetition=1.0)
        assert np.array_equal(plain, again)


def test_a_sequence_at_once_and_step_by_step():
    rng = np.random.default_rng(5)
    n, Bn, V = 7, 2, 11
    ids = rng.integers(0, V, n * Bn)
    with T.using_backend(RecurrentBackend()) as F:
        model = T.GatedLanguageModel(gated_params(rng))
        whole = sequence(model, F, ids, n)
        state = None
        for t in range(n):
            with T.no_backprop_mode():
                y, state = model._hidden(ids[t * Bn:(t + 1) * Bn], 1, state)
                assert np.allclose(model._logits(y).array, whole[t * Bn:(t + 1) * Bn], rtol=0, atol=1e-12)


def test_model_refuses():
    with T.using_backend(RecurrentBackend()):
        P = gated_params(np.random.default_rng(0))
        for bad in ({k: v for k, v in P.items() if k != "b1"}, {k: v for k, v in P.items() if k != "gamma"}, dict(P, U=P["E"]),
                    {k: v for k, v in P.items() if not k[-1].isdigit()}):
            with pytest.raises(ValueError):
                T.GatedLanguageModel(bad)
        with pytest.raises(ValueError):
            T.GatedLanguageModel(P, ratio=0.1)
        model = T.GatedLanguageModel(P)
        with pytest.raises(ValueError, match="GatedLanguageModel"):
            model.generate(np.zeros(5, np.int64), 2, np.zeros((1, 2)))
