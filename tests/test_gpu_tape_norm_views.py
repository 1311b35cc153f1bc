"""Normalisations on the tape of what other functions hand on: views, repeated rows, on the GPU against the same on the oracle's
kernels in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1908_00213_amd import tape as T
from rows_backend import RowsBackend
from util import check, host

pytestmark = pytest.mark.gpu
N, C = 24, 40


def cmp(got, ref, tol, what):
    ref = np.asarray(ref, np.float64)
    check(host(got), ref, tol, float(np.max(np.abs(ref))), what)


def both(run, tol=1e-4):
    """What `run` returns on the GPU against what it returns on the oracle's kernels."""
    got = run(T.backend())
    with T.using_backend(RowsBackend()) as O:
        want = run(O)
    assert T.live_function_nodes() == 0
    for k, (g, w) in enumerate(zip(got, want)):
        cmp(g, w, tol, "result %d" % k)


def arrays(seed, *shapes):
    rng = np.random.default_rng(seed)
    return [np.asarray(rng.standard_normal(s), np.float32) for s in shapes]


def columns(v, lo, hi):
    return T.SliceCols(lo, hi).apply((v,))[0]


@pytest.mark.parametrize("where", ["input", "gradient", "both"])
def test_layer_norm_of_transposed_arrays(where):
    def run(F):
        x, w, gamma, beta = arrays(1, (N, C) if where == "gradient" else (C, N), (N, C) if where == "input" else (C, N), (C,), (C,))
        xv, gv, bv, wv = (T.Variable(F.from_numpy(a)) for a in (x, gamma, beta, w))
        y = T.layer_norm(xv if where == "gradient" else T.transpose(xv), gv, bv)
        T.sum_all(T.mul(y if where == "input" else T.transpose(y), wv)).backward()
        return y.array, xv.grad, gv.grad, bv.grad
    both(run)


@pytest.mark.parametrize("which", ["x", "residual", "y", "s", "all"])
def test_residual_norm_of_transposed_arrays(which):
    def run(F):
        t = lambda name, v: T.transpose(v) if which in (name, "all") else v
        shape = lambda name: (C, N) if which in (name, "all") else (N, C)
        x, res, w, ws, gamma, beta = arrays(2, shape("x"), shape("residual"), shape("y"), shape("s"), (C,), (C,))
        xv, rv, gv, bv, wv, sv = (T.Variable(F.from_numpy(a)) for a in (x, res, gamma, beta, w, ws))
        y, s = T.residual_norm(t("x", xv), t("residual", rv), gv, bv)
        T.add(T.sum_all(T.mul(t("y", y), wv)), T.sum_all(T.mul(t("s", s), sv))).backward()
        return y.array, s.array, xv.grad, rv.grad, gv.grad, bv.grad
    both(run)


def test_columns_of_a_wider_array_are_taken_as_they_lie():
    def run(F):
        x, w, gamma, beta = arrays(3, (N, C + 9), (N, C), (C,), (C,))
        xv, gv, bv = (T.Variable(F.from_numpy(a)) for a in (x, gamma, beta))
        y = T.layer_norm(columns(xv, 5, 5 + C), gv, bv)
        T.sum_all(T.mul(y, T.Variable(F.from_numpy(w), False))).backward()
        return y.array, xv.grad, gv.grad, bv.grad
    both(run)


def test_a_row_that_is_repeated_without_a_copy():
    F = T.backend()
    row, gamma, beta = (F.from_numpy(a) for a in arrays(4, (C,), (C,), (C,)))
    params = T.Variable(gamma, False), T.Variable(beta, False)
    y = T.layer_norm(T.Variable(row[None].expand(N, C), False), *params)
    want = T.layer_norm(T.Variable(row[None].repeat(N, 1), False), *params)
    assert torch.equal(y.array, want.array)
    a, b = T.residual_norm(T.Variable(row[None].expand(N, C), False), T.Variable(row[None].expand(N, C), False), *params)
    p, q = T.residual_norm(T.Variable(row[None].repeat(N, 1), False), T.Variable(row[None].repeat(N, 1), False), *params)
    assert torch.equal(a.array, p.array) and torch.equal(b.array, q.array)


def test_sampling_from_a_transposed_view():
    F = T.backend()
    z, u = F.from_numpy(arrays(5, (50, 7))[0]), F.from_numpy(np.linspace(0.05, 0.95, 7).astype(np.float32))
    a, b = F.empty((7,), "i64"), F.empty((7,), "i64")
    F.sample(z.t(), u, a)
    F.sample(z.t().contiguous(), u, b)
    assert torch.equal(a, b)
