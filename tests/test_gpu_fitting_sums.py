"""Sums of gradients over very many rows, held to their own size (GPU).

u = 2^-24.  A block's db adds the 32 rows of a step as a tree and the steps in 64 bits, and
blocks are added in 64 bits: 5 roundings of a tree, one of a block's sum and one of the output,
below 8 u of the sum of magnitudes.  A block's dW adds 16 rows at a time in float32, in three
products: 8,192 rows of one sign round 1,536 times at sums that are half of the last on the
average, less than 1,024 u of it; and 2^-22 of each product for its operands' pairs.
"""
import pytest
import torch

import paper_2608_19041_amd as dp

pytestmark = pytest.mark.gpu

F64 = torch.float64
U = 2.0 ** -24


@pytest.mark.parametrize("n", [1000, 20000, 1000000, 70000000])
def test_equal_terms(n):
    # a row for all: roundings that all go one way
    k, m = 8, 16
    x = torch.linspace(0.7, 1.3, k, device="cuda")[None].expand(n, k)
    dy = torch.linspace(0.1, 0.11, m, device="cuda")[None].expand(n, m)
    w = torch.zeros(1, k, m, device="cuda")
    ptr = torch.tensor([0, n], device="cuda")
    _, dw, db = dp.grouped_linear_backward(dy, x, w, ptr, need=(False, True, True))
    one_x, one_dy = x[0].to(F64), dy[0].to(F64)
    want = n * one_dy
    assert ((db[0].to(F64) - want).abs() <= 8 * U * want).all()
    want = n * one_x[:, None] * one_dy[None]
    assert ((dw[0].to(F64) - want).abs() <= (1024 * U + 2.0 ** -22 + 4 * U) * want).all()
