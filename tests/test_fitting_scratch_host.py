"""Scratch of the grouped layers: room for what a call can use (no GPU: sizes only)."""
import ctypes

import pytest

import paper_2608_19041_amd as dp
from paper_2608_19041_amd import fitting as ft


def layer(n, k, m, groups, dtype=0):
    return ft._Grouped(dtype, groups, k, m, n, 256, None, 512, k, 1024)


def scratch(n, k, m, groups, dtype=0):
    l, lib, sizes = layer(n, k, m, groups, dtype), dp.library(), []
    for call in (lib.dpa4c_grouped_linear_work, lib.dpa4c_grouped_linear_backward_work):
        need = ctypes.c_int64(-1)
        assert call(ctypes.byref(l), ctypes.byref(need)) == 0
        sizes.append(need.value)
    return sizes


def up(x, by):
    return (x + by - 1) // by * by


def planes(n, depth, cols, groups, dtype):
    """Weights laid out for the groups that n rows can belong to, and the lists of tiles."""
    size = up(depth, 32) * up(cols, 128) * (4 if dtype == 0 else 2) + 4 * up(cols, 128)
    return min(n, groups) * size + 24 * (n // 64 + groups + 2) + 8 * groups + 4096


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,k,m,groups", [
    (1, 541, 384, 118), (108, 144, 192, 118), (108, 541, 384, 4096), (4000, 384, 384, 118),
    (20000, 384, 384, 4096), (31250, 384, 384, 4096), (31250, 541, 384, 118), (1000188, 541, 384, 118),
    (1000188, 5, 3, 4096)])
def test_scratch_is_what_rows_can_use(n, k, m, groups, dtype):
    forward, backward = scratch(n, k, m, groups, dtype)
    widened = n * 8 * 4 if k < 8 else 0
    assert forward <= planes(n, k, m, groups, dtype) + widened
    # dz; and sums of blocks, of 128 rows at the least, of groups of several
    dz = n * (up(m, 8) * 4 + 4)
    blocks = 2 * n // 128 + 1 if n > 128 else 0
    assert backward <= planes(n, m, k, groups, dtype) + widened + dz + blocks * (k + 1) * m * 4 + 8 * groups


def test_scratch_of_what_is_formed():
    lib, need, n, k, m = dp.library(), ctypes.c_int64(-1), 20000, 384, 256
    l = layer(n, k, m, 118)

    def of(*want):
        assert lib.dpa4c_grouped_linear_backward_work_of(ctypes.byref(l), *want, ctypes.byref(need)) == 0
        return need.value

    assert lib.dpa4c_grouped_linear_backward_work(ctypes.byref(l), ctypes.byref(need)) == 0
    assert need.value == of(1, 1, 1, 1)
    weights, dz = 118 * k * m * 4, n * m * 4
    assert of(1, 1, 0, 0) >= weights + dz
    assert of(0, 1, 0, 0) < weights + 8 * n + 2 ** 20          # no dz, no sums of blocks
    assert dz < of(1, 0, 0, 1) < dz + 2 ** 20                  # no weights, no sums of dW
    assert of(0, 0, 0, 1) < 2 ** 20 and of(1, 0, 0, 0) < 2 ** 10
    assert of(1, 0, 1, 0) < dz + 2 * n // 128 * k * m * 4 + 2 ** 20
    # a call takes what it needs, and no less
    some = of(0, 1, 0, 0)
    back = lib.dpa4c_grouped_linear_backward
    assert back(ctypes.byref(l), 256, m, None, 0, 0, 256, None, None, 256, some - 1, None) == dp.ERR_INVALID_ARG
    assert back(ctypes.byref(l), 256, m, 256, m, 0, 256, None, None, 256, some, None) == dp.ERR_INVALID_ARG
    assert lib.dpa4c_grouped_linear_backward_work_of(ctypes.byref(l), 1, 1, 1, 1, None) == dp.ERR_INVALID_ARG
    assert lib.dpa4c_grouped_linear_backward_work_of(None, 1, 1, 1, 1, ctypes.byref(need)) == dp.ERR_INVALID_ARG
