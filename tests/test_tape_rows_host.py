"""Layer normalisation, dropout, residual blocks and generation on the tape, without a GPU: gradients against differences, the masks' places,
what is released, what is refused."""
import numpy as np
import pytest

from paper_1908_00213_amd import tape as T
from rows_backend import RowsBackend

H = 1e-6                     # of the differences: their error is about H^2 times a third derivative and 1e-16 / H


def mlp_params(rng, sizes=(6, 8, 8, 5, 4)):
    return [(rng.standard_normal((o, i)) / np.sqrt(i), 0.1 * rng.standard_normal(o)) for i, o in zip(sizes[:-1], sizes[1:])]


def lm_params(rng, V=11, E=5, Hn=6, norm=True):
    P = {"E": rng.standard_normal((V, E)), "W": rng.standard_normal((E, 4 * Hn)) / 2, "U": rng.standard_normal((Hn, 4 * Hn)) / 2,
         "b": 0.1 * rng.standard_normal(4 * Hn), "W_out": rng.standard_normal((V, Hn)), "b_out": 0.1 * rng.standard_normal(V)}
    if norm:
        P.update(gamma=1 + 0.1 * rng.standard_normal(Hn), beta=0.1 * rng.standard_normal(Hn))
    return P


def check_against_differences(loss, arrays, grads, rng, tol=2e-6):
    """d loss / d array at a few places of every array."""
    for a, g in zip(arrays, grads):
        for _ in range(4):
            i = tuple(rng.integers(0, n) for n in a.shape)
            keep = a[i]
            a[i] = keep + H
            up = loss()
            a[i] = keep - H
            down = loss()
            a[i] = keep
            assert abs((up - down) / (2 * H) - g[i]) < tol * (1 + abs(g[i])), (a.shape, i)


@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("ratio", [0.0, 0.3])
def test_mlp_gradients(norms, ratio):
    rng = np.random.default_rng(1)
    params = mlp_params(rng)
    ng = [(1 + 0.2 * rng.standard_normal(W.shape[0]), 0.2 * rng.standard_normal(W.shape[0])) for W, _ in params[:-1]] if norms else None
    x, t = rng.standard_normal((7, 6)), rng.integers(0, 4, 7)
    with T.using_backend(RowsBackend()) as F:
        model = T.MLP(params, act="gelu", norms=ng, ratio=ratio, masks=T.Masks(5) if ratio else None)

        def loss():
            if ratio:
                model.masks.sites = 0                    # the same step again
            return model.loss(T.Variable(x, False), t)
        l = loss()
        l.backward()
        assert T.live_function_nodes() == 0
        ps = model.params()
        assert len(ps) == 8 + (6 if norms else 0) and all(p.grad is not None for p in ps)
        grads = [p.grad.copy() for p in ps]
        check_against_differences(lambda: float(loss().array), [p.array for p in ps], grads, rng)
        names = [c[0] for c in F.calls]
        if norms:                                        # widths 8, 8, 5: one block continues the stream
            assert names.count("residual_norm_bwd") == 1 and names.count("layer_norm_bwd") == 2


@pytest.mark.parametrize("n_step", [False, True])
def test_language_model_gradients(n_step):
    rng = np.random.default_rng(2)
    ids, targets = rng.integers(0, 11, 12), rng.integers(0, 11, 12)
    with T.using_backend(RowsBackend()):
        model = T.LSTMLanguageModel(lm_params(rng), n_step=n_step, ratio=0.25, masks=T.Masks(9))

        def loss():
            model.masks.sites = 0
            return model.loss(ids, targets, 4)[0]
        l = loss()
        l.backward()
        grads = [p.grad.copy() for p in model.params()]
        check_against_differences(lambda: float(loss().array), [p.array for p in model.params()], grads, rng)
        model.train = False
        assert abs(float(loss().array) - float(loss().array)) == 0 and model.masks.sites == 0


def test_functions_by_themselves():
    rng = np.random.default_rng(3)
    with T.using_backend(RowsBackend()):
        masks = T.Masks(-7)
        x, r, w = (T.Variable(rng.standard_normal((5, 9))) for _ in range(3))
        gamma, beta = T.Variable(rng.standard_normal(9)), T.Variable(rng.standard_normal(9))
        for use in ((True, True), (True, False), (False, True)):       # either output, and both
            def loss():
                masks.sites = 3
                y, s = T.residual_norm(x, r, gamma, beta, 0.4, masks)
                parts = [T.sum_all(T.mul(v, w)) for v, on in zip((y, s), use) if on]
                return parts[0] if len(parts) == 1 else T.add(*parts)
            l = loss()
            l.backward()
            vs = [x, r] + ([gamma, beta] if use[0] else [])
            check_against_differences(lambda: float(loss().array), [v.array for v in vs], [v.grad.copy() for v in vs], rng)
            for v in (x, r, gamma, beta, w):
                v.cleargrad()
        # dropout keeps, scales and drops the same places in both directions, and is differentiable any number of times
        y = T.dropout(x, 0.5, masks)
        g, = T.grad([T.sum_all(T.mul(y, T.mul(y, y)))], [x], enable_double_backprop=True)
        gg, = T.grad([T.sum_all(g)], [x])
        kept = y.array != 0
        assert np.allclose(g.array, np.where(kept, 24 * x.array ** 2, 0)) and np.allclose(gg.array, np.where(kept, 48 * x.array, 0))
        with pytest.raises(NotImplementedError):
            z = T.layer_norm(x, gamma, beta)
            T.grad([T.sum_all(T.mul(z, z))], [x], enable_double_backprop=True)


def test_places_steps_and_refusals():
    rng = np.random.default_rng(4)
    with T.using_backend(RowsBackend()):
        masks = T.Masks(1)
        x = T.Variable(np.ones((40, 50)))
        a, b = T.dropout(x, 0.5, masks), T.dropout(x, 0.5, masks)
        assert not np.array_equal(a.array, b.array)      # two places
        masks.advance()
        c = T.dropout(x, 0.5, masks)
        assert not np.array_equal(a.array, c.array) and masks.steps == 1 and masks.sites == 1
        c.grad = np.ones((40, 50))
        c.backward()
        assert np.array_equal(x.grad, c.array)
        a.grad = np.ones((40, 50))
        with pytest.raises(RuntimeError, match="advance"):
            a.backward()                                 # its masks are gone
        assert T.dropout(x, 0.0).array is not None       # nothing to draw
        with pytest.raises(ValueError, match="Masks"):
            T.dropout(x, 0.5)
        with pytest.raises(ValueError):
            T.MLP(mlp_params(rng), ratio=0.5)
        with pytest.raises(ValueError):
            T.MLP(mlp_params(rng), norms=[])
        with pytest.raises(ValueError):
            T.LSTMLanguageModel(lm_params(rng), ratio=0.5)
        P = lm_params(rng)
        del P["beta"]
        with pytest.raises(ValueError):
            T.LSTMLanguageModel(P)


def test_generate_follows_the_model():
    rng = np.random.default_rng(6)
    Bn, n = 3, 5
    prompt, u = rng.integers(0, 11, 4 * Bn), rng.random((n, Bn))
    with T.using_backend(RowsBackend()) as F:
        model = T.LSTMLanguageModel(lm_params(rng), n_step=True, ratio=0.5, masks=T.Masks(3))
        tokens, state = model.generate(prompt, 4, u, temperature=0.8, top_k=5, top_p=0.9, min_p=np.array([0.0, 0.1, 0.3]))
        assert tokens.shape == (n, Bn) and model.train and T.live_function_nodes() == 0
        assert ("dropout", 0) not in F.calls
        # the same from the whole text every time
        text = prompt
        model.train = False
        for t in range(n):
            with T.no_backprop_mode():
                hs, _ = model._hidden(text, len(text) // Bn, None)
                logits = model._logits(hs).array[-Bn:]
            want = np.zeros(Bn, np.int64)
            F.sample(logits, u[t], want, np.full(Bn, 0.8), np.full(Bn, 5), np.full(Bn, 0.9), np.array([0.0, 0.1, 0.3]))
            assert np.array_equal(tokens[t], want)
            text = np.concatenate([text, want])
        greedy, _ = model.generate(prompt, 4, u, temperature=0.0)
        assert np.array_equal(greedy[0], model._logits(model._hidden(prompt, 4, None)[0]).array[-Bn:].argmax(1))


def test_generate_refuses_a_prompt_that_does_not_fit():
    with T.using_backend(RowsBackend()):
        model = T.LSTMLanguageModel(lm_params(np.random.default_rng(6)), n_step=True)
        for ids, steps, u in ((12, 4, (2, 4)), (12, 4, (0, 3)), (0, 0, (2, 3)), (13, 4, (2, 3)), (12, 4, (3,))):
            with pytest.raises(ValueError):
                model.generate(np.zeros(ids, np.int64), steps, np.zeros(u, np.float32))
