"""Shared by the tests of the row operators: matrices inside wider buffers, and error bounds.

U is half a step of fp32, half a step of a stored type t is finfo(t).eps / 2.  A sum of n terms, added by lanes and then in a tree, is off by at
most DEPTH roundings times the sum of magnitudes: no lane adds more than 64 terms one after the other at the sizes tested, and
the tree over at most 1024 lanes and the further additions are less than 16 deep."""
import numpy as np
import torch

U = 2.0 ** -24
DEPTH = 80
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": U, "bf16": 2.0 ** -8}


def matrix(a, dtype, pad=0, shift=0):
    """A device matrix with a's values, rows `pad` elements longer, starting `shift` elements into its memory; the rest holds 7."""
    n, c = a.shape
    buf = torch.full((n * (c + pad) + shift,), 7.0, device="cuda", dtype=DT[dtype])
    m = buf[shift:].view(n, c + pad)[:, :c] if c + pad > 0 else buf[shift:].view(n, c + pad)
    m.copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda())
    m.whole = buf
    return m


def untouched(m, pad, shift):
    """Whether what lies around a matrix made by `matrix` still holds 7."""
    n, c = m.shape
    rest = m.whole[shift:].view(n, c + pad)[:, c:]
    return bool((rest == 7.0).all()) and bool((m.whole[:shift] == 7.0).all())


def values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rounded(a, dtype):
    """The values a becomes when it is stored, as float32."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DT[dtype]).float().numpy()


def close(got, want, bound, what=""):
    got, want, bound = np.asarray(got, np.float64), np.asarray(want, np.float64), np.broadcast_to(np.asarray(bound, np.float64), np.shape(want))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / np.maximum(bound, 1e-300), 0)), want.shape)
        raise AssertionError("%s: %d of %d beyond their bound; at %s: %r for %r, bound %r" % (what, bad.sum(), want.size, i, got[i], want[i], bound[i]))


def norm_bounds(x, mean, rstd, y, gamma, beta, dtype):
    """Bounds for y, mean and rstd.  With m0 the first mean, off by delta <= DEPTH U mean|x|, the second one corrects it; what is left of an element
    after both subtractions is off by 2 U |d| + DEPTH U mean|d| (d taken about m0, so at most delta larger), the variance by
    DEPTH + 4 roundings of mean d^2 <= var + delta^2, rstd by half of that and 2 roundings; two products and a sum follow, then the store."""
    ax = np.abs(x).mean(1, keepdims=True)
    h = (x - mean[:, None]) * rstd[:, None]
    delta = DEPTH * U * ax * rstd[:, None]                               # in units of the spread
    dev = np.abs(h) + delta
    rel = (DEPTH + 8) * U * (1 + delta ** 2) / 2 + 4 * U                 # of rstd
    dh = 3 * U * dev + DEPTH * U * dev.mean(1, keepdims=True) + rel * np.abs(h)
    g = np.ones(x.shape[1]) if gamma is None else np.abs(gamma)
    b = np.zeros(x.shape[1]) if beta is None else np.abs(beta)
    by = dh * g + 3 * U * (np.abs(h) * g + b) + (HALF[dtype] * (1 + 2 ** -6) if dtype != "f32" else U) * np.abs(y)
    bm = (U * np.abs(mean) + (2 * U * dev + DEPTH * U * dev).mean(1) / rstd + U * np.abs(mean))
    return by, bm, rel[:, 0] * rstd


def bwd_bounds(dy, x, mean, rstd, gamma, dtype):
    """Bounds for dx (before a further addition and the store), dgamma and dbeta: h is off by 3 roundings, the two row sums by DEPTH of the sums of
    magnitudes, five operations follow; a column sum is added by rows in strips of at most 200 and then strip by strip (at most 520)."""
    h = np.abs((x - mean[:, None]) * rstd[:, None])
    g = np.abs(dy if gamma is None else dy * gamma)
    mg, mgh = g.mean(1, keepdims=True), (g * h).mean(1, keepdims=True)
    bdx = rstd[:, None] * U * (6 * (g + mg + h * mgh) + DEPTH * mg + (DEPTH + 8) * h * mgh)
    depth = min(len(dy), 720) + 8
    return bdx, depth * U * (np.abs(dy) * h).sum(0), depth * U * np.abs(dy).sum(0)
