"""Normalisations of more rows or columns than a line of the grid has blocks (2^20): every kernel that puts a number together from two of the grid's indexes."""
import pytest
import torch

from paper_1908_00213_amd import binding as B
from rows_util import DEPTH, HALF, U

pytestmark = pytest.mark.gpu


def part(a, n):
    """Rows from a on, and a few thousand at the seam and at the end."""
    return slice(a, min(a + 4096, n))


# fp32 rows of three elements are four lanes' work, 64 to a block of 256; rows of 1030 are a block's
@pytest.mark.parametrize("n,c,dtype,blocks", [(2 ** 26 + 37, 3, torch.float32, (2 ** 26 + 37 + 63) // 64), (2 ** 20 + 3, 1030, torch.bfloat16, 2 ** 20 + 3)])
def test_forward(n, c, dtype, blocks):
    assert blocks > 2 ** 20
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(n, c, device="cuda", generator=g, dtype=dtype)
    y, mean, rstd = torch.full_like(x, 9.0), torch.full((n, 2), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda")
    B.layer_norm_fwd(x, y, None, None, 1e-2, mean, rstd)
    half = HALF["f32" if dtype == torch.float32 else "bf16"]
    for a in (0, 2 ** 19, 2 ** 20 - 2048, 64 * 2 ** 20 - 2048, n - 4096):
        if not 0 <= a < n:
            continue
        rows = part(a, n)
        d = x[rows].double()
        m = d.mean(1)
        r = 1.0 / torch.sqrt(((d - m[:, None]) ** 2).mean(1) + 1e-2)
        h = (d - m[:, None]) * r[:, None]
        # the mean in two parts is off by DEPTH roundings of the spread and of the first mean's error, rstd by half of its variance's and a few, h by both
        size = d.abs().mean(1)
        assert bool(((mean[rows].double().sum(1) - m).abs() <= (DEPTH + 8) * U * size * (1 + DEPTH * U)).all()), a
        rel = ((DEPTH + 8) / 2 + 4) * U
        assert bool(((rstd[rows].double() - r).abs() <= rel * r).all()), a
        bound = rel * h.abs() + 3 * U * h.abs() + (DEPTH + 8) * U * (size * r)[:, None] + half * (1 + 2 ** -6) * (h.abs() + 1e-3)
        assert bool(((y[rows].double() - h).abs() <= bound).all()), a
    for a in range(0, n, 2 ** 22):                       # nothing is left out: the rows' means are found where they are computed in 32 bits too
        k = slice(a, min(a + 2 ** 22, n))
        assert float((mean[k, 0] - x[k].float().mean(1)).abs().max()) < 1e-4, a


def test_backward_of_rows_longer_than_a_block_holds():
    n, c = 2 ** 20 + 3, 8193                             # the first of two launches has a block for each row
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(n, c, device="cuda", generator=g, dtype=torch.bfloat16)
    dy = torch.randn(n, c, device="cuda", generator=g, dtype=torch.bfloat16)
    # statistics that tell the rows apart
    mean = torch.rand(n, device="cuda", generator=g) - 0.5
    rstd = 2.0 ** torch.randint(-2, 3, (n,), device="cuda", generator=g).float()
    dx, dgamma, dbeta = torch.full_like(x, 9.0), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.empty(B.layer_norm_bwd_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    B.layer_norm_bwd(dy, x, mean, rstd, dx, None, dgamma, dbeta, ws=ws)
    for a in (0, 2 ** 19 + 5, 2 ** 20 - 300, n - 256):
        rows = slice(a, min(a + 600, n))
        q, s, m, r = dy[rows].double(), x[rows].double(), mean[rows].double()[:, None], rstd[rows].double()[:, None]
        h = (s - m) * r
        c1, c2 = q.mean(1, keepdim=True), (q * h).mean(1, keepdim=True)
        want = r * (q - c1 - h * c2)
        m1, m2 = q.abs().mean(1, keepdim=True), (q * h).abs().mean(1, keepdim=True)
        bound = r * U * (6 * (q.abs() + m1 + h.abs() * m2) + DEPTH * m1 + (DEPTH + 8) * h.abs() * m2)
        assert bool(((dx[rows].double() - want).abs() <= bound + HALF["bf16"] * (1 + 2 ** -6) * (want.abs() + bound)).all()), a
    sums = [torch.zeros(c, device="cuda", dtype=torch.float64) for _ in range(4)]
    for a in range(0, n, 2 ** 14):
        k = slice(a, min(a + 2 ** 14, n))
        q = dy[k].double()
        t = q * ((x[k].double() - mean[k].double()[:, None]) * rstd[k].double()[:, None])
        for v, w in zip(sums, (t, t.abs(), q, q.abs())):
            v += w.sum(0)
    # a strip has a 64th of the rows, added one after the other, and the strips are added up
    depth = (n + 63) // 64 + 64 + 8
    assert bool(((dgamma.double() - sums[0]).abs() <= depth * U * sums[1]).all()) and bool(((dbeta.double() - sums[2]).abs() <= depth * U * sums[3]).all())


def test_fold_of_more_columns():
    n, c = 5, 2 ** 26 + 41                               # five rows are two strips, whose 2 c sums are folded 64 to a block
    assert (2 * c + 63) // 64 > 2 ** 20
    g = torch.Generator(device="cuda").manual_seed(8)
    x, dy = (torch.randn(n, c, device="cuda", generator=g) for _ in range(2))
    mean, rstd = torch.tensor([0.25, -0.5, 0.0, 1.0, 0.125], device="cuda"), torch.tensor([0.5, 2.0, 1.0, 0.25, 4.0], device="cuda")
    dgamma, dbeta = (torch.full((c,), 7.0, device="cuda") for _ in range(2))
    ws = torch.empty(B.layer_norm_bwd_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    B.layer_norm_bwd(dy, x, mean, rstd, torch.empty_like(x), None, dgamma, dbeta, ws=ws)
    for a in range(0, c, 2 ** 24):
        p, q = (t[:, a:a + 2 ** 24].double() for t in (x, dy))
        t = (p - mean.double()[:, None]) * rstd.double()[:, None] * q
        # a difference (the scales are powers of two), a product and four sums
        assert bool(((dgamma[a:a + 2 ** 24] - t.sum(0)).abs() <= 7 * U * t.abs().sum(0)).all()), a
        assert bool(((dbeta[a:a + 2 ** 24] - q.sum(0)).abs() <= 5 * U * q.abs().sum(0)).all()), a
