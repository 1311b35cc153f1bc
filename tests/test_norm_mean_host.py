"""The mean of layer normalisation in one part or two, without a GPU: which arrays the entry points take."""
import ctypes as C

from paper_1908_00213_amd import binding as B

P = 4096          # an aligned address that is never looked at


def d(shape, strides=None, dtype=B.F32):
    if strides is None:
        strides, acc = [], 4
        for n in reversed(shape):
            strides.insert(0, acc)
            acc *= max(n, 1)
    return B.raw_desc(P, shape, strides, dtype)


def r(a):
    return None if a is None else C.byref(a)


def test_shapes_of_the_mean():
    L = B.lib()
    x, v, none = d((4, 6)), d((6,)), d((0, 6))
    fwd = lambda m, x=x: L.chn_layer_norm_fwd(r(x), r(v), r(v), 1e-5, r(x), r(m), None, None)
    bwd = lambda m, x=x, n=4: L.chn_layer_norm_bwd(r(x), r(x), r(m), r(d((n,))), r(v), r(x), None, None, C.c_void_p(P), 1 << 30, None)
    res = lambda m: L.chn_residual_norm_fwd(r(x), r(x), 0.0, None, 0, None, None, 1e-5, r(x), r(x), r(m), None, None)
    rbw = lambda m: L.chn_residual_norm_bwd(r(x), None, r(x), r(m), r(d((4,))), None, 0.0, None, 0, r(x), None, None, None, C.c_void_p(P), 1 << 30, None)
    for call in (fwd, bwd, res, rbw):
        assert call(d((4, 3))) == -4 and call(d((2, 4))) == -4 and call(d((4, 1))) == -4 and call(d((6,))) == -4 and call(d((4, 2, 1))) == -4
        assert call(d((4, 2), (4, 16))) == -5 and call(d((4, 2), (16, 4))) == -5
        assert call(d((4, 2), dtype=B.I32)) == -3
    assert bwd(None) == -1
    # without rows both shapes are taken, and nothing is launched
    assert fwd(d((0,)), none) == 0 and fwd(d((0, 2)), none) == 0 and bwd(d((0, 2)), none, 0) == 0
