"""Layer normalisation, dropout and sampling without a GPU: the generator against the paper's published words, what the entry points
refuse before anything is launched, and the oracle's gradients against differences."""
import ctypes as C

import numpy as np

from oracle import rows as R
from paper_1908_00213_amd import binding as B

P = 4096          # an aligned address that is never looked at


def d(shape, dtype=B.F32, p=P, strides=None):
    isz = {B.F32: 4, B.BF16: 2, B.I32: 4, B.I64: 8}[dtype]
    if strides is None:
        strides, acc = [], isz
        for n in reversed(shape):
            strides.insert(0, acc)
            acc *= max(n, 1)
    return B.raw_desc(p, shape, strides, dtype)


def r(a):
    return None if a is None else C.byref(a)


def test_generator_gives_the_published_words():
    # known answers of Philox-4x32 with seven and with ten rounds for counter and key of zeros
    assert R.philox4x32([0] * 4, [0] * 2, 7) == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert R.philox4x32([0] * 4, [0] * 2, 10) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    # the mask is built of those words: column block, row, offset, site
    seed, offset, site = 0x0123456789ABCDEF, 77, 5
    keep = R.mask(3, 10, 0.25, seed, offset, site)
    for row in range(3):
        for col in range(10):
            word = R.philox4x32([col // 4, row, offset, site], [seed & R.LOW, seed >> 32], 7)[col % 4]
            assert keep[row, col] == (word >= 2 ** 30)


def test_mask_keeps_its_share_and_repeats_nowhere():
    n, c, ratio = 400, 500, 0.3
    m = R.mask(n, c, ratio, 11, 0, 0)
    # the share of a fair draw: five standard deviations
    assert abs(m.mean() - 0.7) < 5 * (0.21 / (n * c)) ** 0.5
    others = [R.mask(n, c, ratio, 12, 0, 0), R.mask(n, c, ratio, 11, 1, 0), R.mask(n, c, ratio, 11, 0, 1)]
    for o in others:                                     # independent masks agree in 0.7^2 + 0.3^2 = 0.58 of the places
        assert abs((m == o).mean() - 0.58) < 5 * (0.58 * 0.42 / (n * c)) ** 0.5
    assert len({row.tobytes() for row in m}) == n


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, gamma, beta, w = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    f = lambda x, g, b: float((R.layer_norm(x, g, b)[0] * w).sum())
    _, mean, rstd = R.layer_norm(x, gamma, beta)
    dx, dg, db = R.layer_norm_bwd(w, x, mean, rstd, gamma)
    h = 1e-5                                             # error of the differences about h^2 and 1e-16 / h
    for a, da, call in ((x, dx, lambda v: f(v, gamma, beta)), (gamma, dg, lambda v: f(x, v, beta)), (beta, db, lambda v: f(x, gamma, v))):
        for i in np.ndindex(a.shape):
            up, down = a.copy(), a.copy()
            up[i] += h
            down[i] -= h
            assert abs((call(up) - call(down)) / (2 * h) - da[i]) < 1e-7 * (1 + abs(da[i]))


def test_dropout_refusals():
    L = B.lib()
    rng = d((2,), B.I64)
    x = d((4, 6))
    call = lambda x, y, ratio=0.5, rng=rng, site=0, res=None: L.chn_dropout(r(x), r(res), ratio, r(rng), site, r(y), None)
    assert call(None, x) == -1 and call(x, None) == -1
    assert call(x, x, rng=None) == -1                                  # masks need a generator
    for ratio in (-0.1, 1.0, 1.5, float("nan")):
        assert call(x, x, ratio) == -6
    assert call(x, x, site=-1) == -6 and call(x, x, site=2 ** 32) == -6
    assert call(x, d((4, 7))) == -4 and call(x, d((24,))) == -4
    assert call(x, x, res=d((4, 5))) == -4
    assert call(x, x, res=d((4, 6), B.BF16)) == -3                     # the residual has y's type
    assert call(d((4, 6), B.I32), x) == -3 and call(x, d((4, 6), B.I64)) == -3
    assert call(x, d((4, 6), strides=(0, 4))) == -5                    # an output of stride 0
    assert call(x, x, rng=d((3,), B.I64)) == -4 and call(x, x, rng=d((2,), B.I32)) == -3
    assert call(x, x, rng=d((2,), B.I64, strides=(16,))) == -5
    many = d((2 ** 32 + 1, 1), strides=(4, 4))
    assert call(many, many) == -4                                      # more rows than the generator numbers
    assert call(d((0, 6)), d((0, 6))) == 0 and call(d((4, 0)), d((4, 0))) == 0
    assert L.chn_rng_advance(r(d((2,), B.I32)), 1, None) == -3 and L.chn_rng_advance(r(d((3,), B.I64)), 1, None) == -4
    assert L.chn_rng_advance(None, 1, None) == -1


def test_layer_norm_refusals():
    L = B.lib()
    x, v, n = d((4, 6)), d((6,)), d((4,))
    fwd = lambda x=x, g=v, b=v, eps=1e-5, y=x, m=n, s=n: L.chn_layer_norm_fwd(r(x), r(g), r(b), eps, r(y), r(m), r(s), None)
    assert fwd(x=None) == -1 and fwd(y=None) == -1
    assert fwd(g=d((5,))) == -4 and fwd(b=d((4,))) == -4 and fwd(m=d((6,))) == -4 and fwd(s=d((1, 4))) == -4
    assert fwd(g=d((6,), B.BF16)) == -3 and fwd(y=d((4, 6), B.I32)) == -3
    assert fwd(g=d((6,), strides=(8,))) == -5
    assert fwd(y=d((4, 5))) == -4 and fwd(x=d((24,))) == -2
    assert fwd(x=d((4, 6), strides=(4, 16))) == -5                     # a transposed view
    assert fwd(eps=-1e-5) == -6 and fwd(eps=float("nan")) == -6 and fwd(eps=float("inf")) == -6
    assert fwd(x=d((4, 0)), y=d((4, 0)), g=None, b=None) == -4         # rows without elements
    assert fwd(x=d((0, 6)), y=d((0, 6)), m=d((0,)), s=d((0,))) == 0
    need = L.chn_layer_norm_bwd_workspace_bytes(r(x))
    assert need > 0
    bwd = lambda dy=x, x=x, m=n, s=n, g=v, dx=x, dg=v, db=v, ws=P, nb=1 << 30: L.chn_layer_norm_bwd(
        r(dy), r(x), r(m), r(s), r(g), r(dx), r(dg), r(db), C.c_void_p(ws), nb, None)
    assert bwd(m=None) == -1 and bwd(dx=None) == -1 and bwd(dy=None) == -1
    assert bwd(ws=0) == -8 and bwd(nb=need - 1) == -8 and bwd(ws=P + 16) == -8
    assert bwd(dx=d((4, 6), B.BF16)) == -3                             # dx has x's type
    assert bwd(dy=d((4, 5))) == -4 and bwd(dg=d((5,))) == -4
    rng = d((2,), B.I64)
    res = lambda x=x, re=x, ratio=0.5, rng=rng, site=0, s=x, y=x: L.chn_residual_norm_fwd(
        r(x), r(re), ratio, r(rng), site, None, None, 1e-5, r(s), r(y), None, None, None)
    assert res(re=None) == -1 and res(s=None) == -1 and res(rng=None) == -1
    assert res(re=d((4, 6), B.BF16)) == -3 and res(y=d((4, 6), B.BF16)) == -3
    assert res(ratio=1.0) == -6 and res(site=-1) == -6 and res(re=d((4, 5))) == -4
    rb = lambda dy=x, ds=x, s=x, dr=x, dx=x, ratio=0.5, rng=rng, ws=P: L.chn_residual_norm_bwd(
        r(dy), r(ds), r(s), r(n), r(n), r(v), ratio, r(rng), 0, r(dr), r(dx), r(v), r(v), C.c_void_p(ws), 1 << 30, None)
    assert rb(ds=d((4, 6), B.BF16)) == -3 and rb(dr=d((4, 6), B.BF16)) == -3 and rb(dx=d((4, 6), B.BF16)) == -3
    assert rb(rng=None) == -1 and rb(ws=0) == -8 and rb(dx=d((3, 6))) == -4


def test_sample_refusals():
    L = B.lib()
    z, f, i = d((4, 9)), d((4,)), d((4,), B.I32)
    call = lambda z=z, u=f, t=None, k=None, p=None, m=None, out=i: L.chn_sample(r(z), r(u), r(t), r(k), r(p), r(m), r(out), None, 0, None)
    assert call(z=None) == -1 and call(u=None) == -1 and call(out=None) == -1
    assert call(z=d((4, 9), B.I32)) == -3 and call(u=i) == -3 and call(out=f) == -3 and call(k=f) == -3 and call(t=i) == -3
    assert call(u=d((5,))) == -4 and call(p=d((1,))) == -4 and call(out=d((4, 1), B.I32)) == -4 and call(k=d((3,), B.I64)) == -4
    assert call(z=d((4, 9), strides=(4, 16))) == -5 and call(out=d((4,), B.I32, strides=(0,))) == -5 and call(out=d((4,), B.I64, strides=(16,))) == -5
    assert call(z=d((4, 0))) == -4                                     # nothing to choose from
    assert call(z=d((4, 2 ** 30 + 1))) == -4
    assert call(z=d((0, 9)), u=d((0,)), out=d((0,), B.I64)) == 0


def test_a_workspace_that_grew_in_place_is_described_anew():
    import torch
    ws = torch.empty(64, dtype=torch.uint8)
    assert B._ws(ws)[1] == 64
    ws.resize_(1 << 20)
    p, n = B._ws(ws)
    assert p.value == ws.data_ptr() and n == 1 << 20
