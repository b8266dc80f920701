"""Gradients of float16 layers whose dy spans what float16 can hold (GPU).

Sums are held to their own size, not to that of the terms: an output may be as far
from the formula in 64 bits, in the norm, as the formula's value rounded to float16
is, and 2^-14 of the value more.  The slope of SiLU is known to 16 u = 2^-20, a pair
of float16 holds dz to 2^-22, and a sum in float32 whose terms have no common sign
goes wrong by some sqrt(K) u of it, 2^-16 for 65,536 rows; all are below 2^-14.
"""
import pytest
import torch

import paper_2608_19041_amd as dp

pytestmark = pytest.mark.gpu

F64 = torch.float64


def inputs(n, k, m, groups, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1009 + n + 7 * k + 3 * m)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    ids = torch.randint(-1, groups, (n,), generator=g, device="cuda").to(torch.int32)
    return ids, normal(n, k).half(), (normal(groups, k, m) * m ** -0.5).half(), normal(n, m), normal(n, m).half()


def formula(ids, x, w, dy, z):
    x, w, dy, z = (t.to(F64) for t in (x, w, dy, z))
    p = torch.sigmoid(z)
    dz = dy * p * (1 + z * (1 - p))
    dz[ids < 0] = 0
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w[:, 0])
    for t in range(w.shape[0]):
        at = (ids == t).nonzero().flatten()
        dx[at] = dz[at] @ w[t].T
        dw[t] = x[at].T @ dz[at]
        db[t] = dz[at].sum(0)
    return dx, dw, db


def held(got, want, dims, name):
    """Every slice over ``dims`` is as near to ``want`` as rounding leaves it."""
    beyond = want.half().isinf()   # float16 ends at 65,504: the rounded value is an infinity
    assert torch.equal(got[beyond], want.half()[beyond]), name
    got, want = torch.where(beyond, 0, got), torch.where(beyond, 0, want)
    assert torch.isfinite(got).all(), name
    norm = lambda t: t.square().sum(dims).sqrt()
    off, least = norm(got.to(F64) - want), norm(want.half().to(F64) - want)
    bound = 1.01 * least + 2.0 ** -14 * norm(want)
    worst = (off / bound.clamp(min=1e-300)).max().item()
    assert (off <= bound).all(), f"{name}: {worst:.3g} of the bound"


SHAPES = [(4096, 70, 96, 5), (300, 20, 5, 3), (700, 33, 700, 2), (1000, 3, 8, 2), (20000, 130, 260, 3),
          (50000, 64, 40, 1), (1, 40, 40, 1)]


def gradients(ids, x, w, dy, z):
    ptr, order = dp.group_rows(ids, w.shape[0])
    return dp.grouped_linear_backward(dy, x, w, ptr, order, preact=z)


@pytest.mark.parametrize("size", [6e4, 1.0, 1e-3, 1e-4, 1e-5, 1e-6, 2e-7])
@pytest.mark.parametrize("n,k,m,groups", SHAPES)
def test_any_size(n, k, m, groups, size):
    ids, x, w, dy, z = inputs(n, k, m, groups)
    if n == 1:
        ids[:] = 0
    if size > 1e4:   # slopes up to 1.1 carry these beyond float16, and the weights and rows bring them back
        dy, w, x = torch.sign(dy) * size, w * 2.0 ** -6, x * 2.0 ** -11
        z = z + 2.4
    else:
        dy = dy * size
    dy = dy.half()
    want = formula(ids, x, w, dy, z)
    dx, dw, db = gradients(ids, x, w, dy, z)
    held(dx, want[0], (0, 1), "dx")
    held(dw, want[1], (0, 1, 2), "dw")
    if size < 1e4:
        held(db, want[2], (0, 1), "db")
    else:   # sums of such are beyond float16 where they do not cancel
        inside = want[2].abs() < 6e4
        held(torch.where(inside, db, 0), torch.where(inside, want[2], 0), (0, 1), "db")


@pytest.mark.parametrize("n,k,m,groups", [(4096, 70, 96, 12), (700, 33, 700, 9), (20000, 130, 260, 6)])
def test_groups_and_rows_of_different_sizes(n, k, m, groups):
    # groups' dy 2^37 apart: each group's sums keep their own precision
    ids, x, w, dy, z = inputs(n, k, m, groups, seed=1)
    fall = torch.exp2(torch.linspace(12, -22, groups, device="cuda"))
    small = (dy * fall[ids.clamp(min=0).long()][:, None]).half()
    want = formula(ids, x, w, small, z)
    dx, dw, db = gradients(ids, x, w, small, z)
    for t in range(groups):
        held(dx[ids == t], want[0][ids == t], (0, 1), f"dx {t}")
    held(dw, want[1], (1, 2), "dw")
    held(db, want[2], (1,), "db")
    # rows 2^37 apart in one group: dx keeps every row, and the sums are right beside their largest
    fall = torch.exp2(torch.linspace(12, -22, n, device="cuda"))[torch.randperm(n, device="cuda")]
    small = (dy * fall[:, None]).half()
    want = formula(ids, x, w, small, z)
    dx, dw, db = gradients(ids, x, w, small, z)
    # dx of float16 has nothing below 2^-24: of the rows that have bits left
    some = (ids >= 0) & (fall > 2.0 ** -14)
    held(dx[some], want[0][some], (1,), "dx by row")
    held(dw, want[1], (1, 2), "dw")
    held(db, want[2], (1,), "db")


def test_the_smallest_numbers_add_up():
    # 100,000 rows of 2^-24 times a slope near 0.45
    n, k, m = 100000, 8, 16
    x = torch.ones(n, k, device="cuda").half()
    w = torch.ones(1, k, m, device="cuda").half()
    dy = torch.full((n, m), 2.0 ** -24, device="cuda").half()
    z = torch.full((n, m), -0.1, device="cuda").half()
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    want = formula(ids, x, w, dy, z)
    _, dw, db = gradients(ids, x, w, dy, z)
    held(dw, want[1], (0, 1, 2), "dw")
    held(db, want[2], (0, 1), "db")


def test_an_infinity_keeps_to_its_row_and_column():
    n, k, m = 900, 24, 48
    ids, x, w, dy, z = inputs(n, k, m, 2, seed=2)
    dy = (dy * 1e-6).half()
    row = int((ids == 0).nonzero()[5])
    dy[row, 7] = 0
    clean = gradients(ids, x, w, dy, z)
    bad = dy.clone()
    bad[row, 7] = float("inf")
    got = gradients(ids, x, w, bad, z)
    rows = torch.ones(n, dtype=torch.bool, device="cuda")
    rows[row] = False
    cols = torch.ones(2, m, dtype=torch.bool, device="cuda")
    cols[0, 7] = False
    assert torch.equal(got[0][rows], clean[0][rows]) and not torch.isfinite(got[0][row]).any()
    for a, c in ((got[1].transpose(1, 2), clean[1].transpose(1, 2)), (got[2], clean[2])):
        assert torch.equal(a[cols], c[cols])
        assert not torch.isfinite(a[0, 7]).any()
