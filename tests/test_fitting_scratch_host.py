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
