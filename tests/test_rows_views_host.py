"""Which arrays the GPU backend of the tape copies before a kernel that walks over rows, without a GPU."""
import torch

from paper_1908_00213_amd import tape as T


class Copies:
    """In the binding's place: element-wise copies by torch."""

    def elementwise_broadcast(self, op, inputs, out, scalars=()):
        assert op == "copy"
        return out.copy_(inputs[0])


def test_views_whose_rows_do_not_lie_one_after_the_other_are_copied():
    F = T.GpuBackend.__new__(T.GpuBackend)
    F.torch, F.B = torch, Copies()
    a = torch.arange(60.0).view(6, 10)
    for taken in (a, a[2:5], a[:, 1:7], a[::2], a[:, :1], torch.empty(0, 4), None):
        assert F._rows(taken) is taken
    for view in (a.t(), a[:, ::2], a[0].expand(6, 10), a[:, :1].expand(6, 10), a.bfloat16().t(), a.as_strided((4, 10), (5, 1))):
        copy = F._rows(view)
        assert copy is not view and copy.is_contiguous() and copy.dtype == view.dtype and torch.equal(copy, view)
