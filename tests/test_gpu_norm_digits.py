"""Gradients of rows whose mean is far above their spread, against the definition with the statistics in 64 bits (not those that a forward
pass left): the backward pass is given the mean with what its rounding left of it, or takes the mean as it is rounded."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from paper_1908_00213_amd import binding as B
from paper_1908_00213_amd import tape as T
from rows_util import DEPTH, HALF, U, bwd_bounds, close, matrix, rounded, untouched, values

pytestmark = pytest.mark.gpu
# every geometry of the backward pass: 4, 8 and 16 lanes, a wave, three to sixteen waves, two launches
SHAPES = [(300, 19), (70, 100), (40, 250), (40, 777), (33, 1100), (9, 2049), (5, 4096), (3, 8000), (6, 8200), (3, 16400)]


def exact_bounds(dy, x, mean, rstd, gamma):
    """Bounds for dx, dgamma and dbeta where the kernels computed the statistics too.  What is left of an element after the subtractions of the mean's
    two parts is off as in the forward pass (rows_util.norm_bounds), `dh`, and rstd by `rel`; both reach dx and dgamma besides the roundings that
    bwd_bounds counts."""
    bdx, bdg, bdb = bwd_bounds(dy, x, mean, rstd, gamma, "f32")
    h = np.abs((x - mean[:, None]) * rstd[:, None])
    delta = DEPTH * U * np.abs(x).mean(1, keepdims=True) * rstd[:, None]
    dev, rel = h + delta, (DEPTH + 8) * U * (1 + delta ** 2) / 2 + 4 * U
    dh = 3 * U * dev + DEPTH * U * dev.mean(1, keepdims=True) + rel * h
    g = np.abs(dy if gamma is None else dy * gamma)
    mg, mgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    bdx = bdx + rstd[:, None] * (rel * (g + mg + h * mgh) + dh * mgh + h * (g * dh).mean(1, keepdims=True))
    return bdx, bdg + (np.abs(dy) * dh).sum(0), bdb


def data(shape, seed, scale=1.0, shift=0.0, dtype="f32"):
    return rounded(np.random.default_rng(seed).standard_normal(shape) * scale + shift, dtype)


def vec(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def check(dx, dg, db, dy, x, gamma, extra=None, tx="f32"):
    x64, dy64, g64 = x.astype(np.float64), dy.astype(np.float64), gamma.astype(np.float64)
    _, mean, rstd = R.layer_norm(x64)
    wdx, wdg, wdb = R.layer_norm_bwd(dy64, x64, mean, rstd, g64)
    bdx, bdg, bdb = exact_bounds(dy64, x64, mean, rstd, g64)
    if extra is not None:
        wdx, bdx = wdx + extra, bdx + U * np.abs(wdx + extra)
    if dx is not None:
        close(values(dx), wdx, bdx + HALF[tx] * (1 + 2 ** -6) * (np.abs(wdx) + bdx), "dx")
    close(values(dg), wdg, bdg + U * np.abs(wdg), "dgamma")
    close(values(db), wdb, bdb + U * np.abs(wdb), "dbeta")


@pytest.mark.parametrize("shift", [0.75, 1e4, -1e5])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients_on_the_tape_keep_their_digits(shape, shift):
    n, c = shape
    x, res, w, ws = data(shape, 1, 1.0, shift), data(shape, 2), data(shape, 3), data(shape, 4)
    gamma, beta = 1 + 0.3 * data((c,), 5), data((c,), 6)
    F = T.backend()
    new = lambda a: T.Variable(F.from_numpy(np.asarray(a, np.float32)))
    xv, gv, bv = new(x), new(gamma), new(beta)
    T.sum_all(T.mul(T.layer_norm(xv, gv, bv), T.Variable(F.from_numpy(w), False))).backward()
    check(xv.grad, gv.grad, bv.grad, w, x, gamma)
    # a residual block: the stream carries the mean
    xv, rv, gv, bv = new(res), new(x), new(gamma), new(beta)
    y, s = T.residual_norm(xv, rv, gv, bv)
    T.add(T.sum_all(T.mul(y, T.Variable(F.from_numpy(w), False))), T.sum_all(T.mul(s, T.Variable(F.from_numpy(ws), False)))).backward()
    stored = res + x                                     # one rounding to fp32, as the sum is stored
    check(rv.grad, gv.grad, bv.grad, w, stored, gamma, ws.astype(np.float64))
    assert torch.equal(xv.grad, rv.grad)


@pytest.mark.parametrize("ty", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_mean_in_two_parts(shape, ty):
    """What the second part changes, and that it changes nothing else."""
    n, c = shape
    x, dy = data(shape, 7, 1.0, 1e4), data(shape, 8, dtype=ty)
    gamma = 1 + 0.3 * data((c,), 9)
    xd, dyd, g = matrix(x, "f32", 5, 1), matrix(dy, ty, 3, 1), vec(gamma)
    one, two, rstd, rstd2 = (torch.full(s, 7.0, device="cuda") for s in ((n,), (n, 2), (n,), (n,)))
    y, y2 = matrix(x * 0, ty, 2), matrix(x * 0, ty, 2)
    B.layer_norm_fwd(xd, y, g, None, 1e-5, one, rstd)
    B.layer_norm_fwd(xd, y2, g, None, 1e-5, two, rstd2)
    assert torch.equal(y, y2) and torch.equal(rstd, rstd2) and torch.equal(two[:, 0], one)
    # the two parts are the mean to DEPTH + 8 roundings of the spread, the second is at most half a step of the first
    m = x.astype(np.float64).mean(1)
    both = values(two).sum(1)
    spread = np.abs(x - m[:, None]).mean(1)
    # (the first mean is off by DEPTH U mean |x|, and the second sum is over elements that much larger)
    assert np.all(np.abs(both - m) <= (DEPTH + 8) * U * (spread + DEPTH * U * 1e4 * 1.01))
    assert np.all(np.abs(values(two)[:, 1]) <= np.spacing(np.abs(values(one).astype(np.float32))) / 2)
    dx, dg, db = matrix(x * 0, "f32", 2), torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
    ws = torch.empty(max(256, B.layer_norm_bwd_workspace_bytes(xd)), dtype=torch.uint8, device="cuda")
    B.layer_norm_bwd(dyd, xd, two, rstd, dx, g, dg, db, ws=ws)
    check(dx, dg, db, dy, x, gamma)
    assert untouched(dx, 2, 0) and untouched(y2, 2, 0)
    # a second part of zeros is the mean as it is rounded
    dx1, dx2, grads = matrix(x * 0, "f32", 2), matrix(x * 0, "f32", 2), [torch.empty(c, device="cuda") for _ in range(4)]
    zero = torch.stack([one, torch.zeros_like(one)], 1)
    B.layer_norm_bwd(dyd, xd, one, rstd, dx1, g, *grads[:2], ws=ws)
    B.layer_norm_bwd(dyd, xd, zero, rstd, dx2, g, *grads[2:], ws=ws)
    assert torch.equal(dx1, dx2) and torch.equal(grads[0], grads[2]) and torch.equal(grads[1], grads[3])


@pytest.mark.parametrize("shape", SHAPES)
def test_a_residual_block_with_a_mean_in_two_parts(shape):
    n, c = shape
    x, res, dy = data(shape, 11, dtype="bf16"), data(shape, 12, 1.0, 1e4), data(shape, 13, dtype="bf16")
    gamma = 1 + 0.3 * data((c,), 14)
    xd, rd, dyd, g = matrix(x, "bf16"), matrix(res, "f32"), matrix(dy, "bf16"), vec(gamma)
    s, y, dres, dx = matrix(res * 0, "f32", 4), matrix(x * 0, "bf16", 4), matrix(res * 0, "f32", 4), matrix(x * 0, "bf16", 4)
    mean, rstd, dg, db = (torch.full(k, 7.0, device="cuda") for k in ((n, 2), (n,), (c,), (c,)))
    B.residual_norm_fwd(xd, rd, s, y, g, None, 1e-5, mean, rstd)
    B.residual_norm_bwd(dyd, None, s, mean, rstd, dres, dx, g, dg, db, ws=torch.empty(max(256, B.layer_norm_bwd_workspace_bytes(s)), dtype=torch.uint8, device="cuda"))
    check(dres, dg, db, dy, x + res, gamma)
    assert np.array_equal(values(s), (x + res).astype(np.float64)) and all(untouched(m, 4, 0) for m in (s, y, dres, dx))
