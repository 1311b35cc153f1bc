"""Descriptors that are kept on tensors, without a GPU: they follow what is done to the tensor, and copies of a tensor are free of them."""
import copy
import io
import pickle

import pytest
import torch

from paper_1908_00213_amd import binding as B


def described(t):
    """What a call would be told of a tensor: by both ways that a call takes."""
    a = B.desc(t)
    out = (a.data, tuple(a.shape[:a.ndim]), tuple(a.strides[:a.ndim]), a.dtype)
    for ref in (B._arg(t), B._here(0, t)[0]):
        b = ref._obj
        assert out == (b.data, tuple(b.shape[:b.ndim]), tuple(b.strides[:b.ndim]), b.dtype)
    return out


def as_it_is(t):
    return t.data_ptr(), tuple(t.shape), tuple(s * t.element_size() for s in t.stride()), B._DTYPES[t.dtype]


@pytest.fixture(autouse=True)
def host_is_the_device(monkeypatch):
    monkeypatch.setattr(B, "_raw_device", lambda: -1)


def assign(t, to):
    t.data = to


CHANGES = {"grown": lambda t: t.resize_(4096, 8), "shrunk": lambda t: t.resize_(2, 8), "as many elements": lambda t: t.resize_(16, 4), "transposed": lambda t: t.t_(),
           "axes exchanged": lambda t: t.transpose_(0, 1), "an axis more": lambda t: t.unsqueeze_(0), "strides alone": lambda t: t.as_strided_((8, 8), (1, 1)),
           "another storage": lambda t: t.set_(torch.zeros(3, 5)), "the same storage": lambda t: t.set_(t.view(4, 16)), "out= of another size": lambda t: torch.rand(50, 50, out=t),
           "data": lambda t: assign(t, torch.zeros(9, 2)), "data of the same shape": lambda t: assign(t, torch.zeros(8, 8)), "storage moved": lambda t: t.untyped_storage().resize_(1 << 20),
           "moved through a view": lambda t: t[:2].resize_(5000, 8), "written to": lambda t: t.copy_(torch.ones(8, 8))}


@pytest.mark.parametrize("name", sorted(CHANGES))
def test_descriptors_follow_a_tensor(name):
    t = torch.zeros(8, 8)
    assert described(t) == as_it_is(t)
    CHANGES[name](t)
    assert described(t) == as_it_is(t)
    CHANGES[name](t) if name not in ("as many elements", "the same storage", "strides alone", "written to") else t.zero_()
    assert described(t) == as_it_is(t)


def test_tensors_whose_versions_are_not_counted():
    with torch.inference_mode():
        t = torch.zeros(8, 8)
        for change in (lambda: t.add_(1), lambda: t.t_(), lambda: t.resize_(100, 8), lambda: t.resize_(3, 3)):
            assert described(t) == as_it_is(t) and described(t) == as_it_is(t)
            change()
        assert described(t) == as_it_is(t)
    assert described(t) == as_it_is(t)


def test_a_descriptor_is_made_once():
    t = torch.zeros(8, 8)
    a = B.desc(t)
    t.add_(1)                                            # (written to, not changed otherwise)
    assert B.desc(t) is a and B.desc(t) is a
    t.resize_(2, 2)
    assert B.desc(t) is not a


def test_copies_carry_no_descriptor():
    t = torch.arange(12.0).view(3, 4)
    described(t)
    for other in (copy.deepcopy(t), pickle.loads(pickle.dumps(t)), copy.deepcopy([t])[0]):
        assert torch.equal(other, t) and described(other) == as_it_is(other) and other.data_ptr() != t.data_ptr()
    f = io.BytesIO()
    torch.save({"W": t, "again": t}, f)
    for weights_only in (True, False):
        f.seek(0)
        back = torch.load(f, weights_only=weights_only)
        assert torch.equal(back["W"], t) and described(back["W"]) == as_it_is(back["W"])
    shallow = copy.copy(t)
    assert described(shallow) == as_it_is(shallow)
    shallow.add_(1)
    assert described(shallow) == as_it_is(shallow) and described(t) == as_it_is(t)
    t.t_()
    assert described(t) == as_it_is(t) and described(shallow) == as_it_is(shallow)


def test_arrays_of_pointers_follow_too():
    ts = [torch.zeros(4, 4), None, B.raw_desc(4096, (2,), (4,), B.F32), torch.zeros(3)]
    for _ in range(2):
        p = B._ptrs(ts)
        assert not p[1] and p[2].contents.data == 4096
        for i in (0, 3):
            assert p[i].contents.data == ts[i].data_ptr() and tuple(p[i].contents.shape[:p[i].contents.ndim]) == tuple(ts[i].shape)
        ts[0].resize_(500, 4)
        ts[3].unsqueeze_(0)


def test_arrays_elsewhere_are_refused():
    t = torch.zeros(3, 3)
    described(t)
    B._raw_device = lambda: 0                            # (undone by the fixture)
    for _ in range(2):
        with pytest.raises(ValueError):
            B._here(0, t)
