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


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_rows_beyond_32_bits_enter_the_sums(dtype):
    # 2.25e9 entries of x and of dz.  Terms of both signs: the sums are some sqrt(rows) of a term,
    # so a row that is missed or read from elsewhere shows.  Roundings of both signs too: 1,536 of
    # a block's sum come to 2^-18 of it, the slope is off by 2^-20 and the operands by 2^-22 of
    # themselves (pairs of bfloat16 by 2^-16): below 2^-16 of the sum, 2^-15 for bfloat16.
    n, k, m, groups = 5630001, 400, 400, 3
    g = torch.Generator(device="cuda").manual_seed(41)

    def normal(*shape):
        return torch.empty(*shape, dtype=dtype, device="cuda").normal_(generator=g)

    x, dy, z, w = normal(n, k), normal(n, m), normal(n, m), normal(groups, k, m)
    if dtype == torch.float16:
        dy *= 2.0 ** -8
    ids = torch.randint(-1, groups, (n,), generator=g, device="cuda", dtype=torch.int32)
    ptr, order = dp.group_rows(ids, groups)
    _, dw, db = dp.grouped_linear_backward(dy, x, w, ptr, order, preact=z, need=(False, True, True))
    cols = torch.tensor([0, 1, 131, 255, 256, 398, 399], device="cuda")
    want, wb = torch.zeros(groups, k, len(cols), dtype=F64, device="cuda"), torch.zeros(groups, len(cols), dtype=F64,
                                                                                      device="cuda")
    for i in range(0, n, 200000):
        part = slice(i, i + 200000)
        v = z[part][:, cols].to(F64)
        p = torch.sigmoid(v)
        dz = dy[part][:, cols].to(F64) * p * (1 + v * (1 - p))
        for t in range(groups):
            mine = dz * (ids[part] == t)[:, None]
            want[t] += x[part].to(F64).t() @ mine
            wb[t] += mine.sum(0)
    eps = 2.0 ** -15 if dtype == torch.bfloat16 else 2.0 ** -16
    for got, exact in ((dw[:, :, cols], want), (db[:, cols], wb)):
        for t in range(groups):
            off, least = (got[t].to(F64) - exact[t]).norm(), (exact[t].to(dtype).to(F64) - exact[t]).norm()
            assert off <= 1.01 * least + eps * exact[t].norm(), (off / exact[t].norm()).item()
    del x, dy, z
    torch.cuda.empty_cache()
