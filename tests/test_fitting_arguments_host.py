"""Sizes that the library refuses and streams that the binding does (no GPU)."""
import ctypes
import types

import pytest
import torch

import paper_2608_19041_amd as dp
from paper_2608_19041_amd import fitting as ft


def test_sizes_beyond_32_bits():
    lib, need = dp.library(), ctypes.c_int64(-1)
    for shape in ((2 ** 32 + 8, 1), (3, 5, 2 ** 32 + 8)):
        stack = (ft._Stack * 1)(ft._Stack(256, 256, *ft._shape(torch.empty(shape, device="meta"))))
        assert lib.dpa4c_orthogonalize_work(1, stack, ctypes.byref(need)) == dp.ERR_INVALID_ARG
    stack = (ft._Stack * 1)(ft._Stack(256, 256, *ft._shape(torch.empty(2, 5, 6, device="meta"))))
    assert (stack[0].batch, stack[0].rows, stack[0].cols) == (2, 5, 6)
    for steps in (2 ** 32 + 5, -2 ** 32 + 5):
        how = ft._newton(steps, ft.MUON_COEFFICIENTS, 1e-7)
        assert lib.dpa4c_orthogonalize(0, 1, stack, ctypes.byref(how), 256, 1 << 40, None) == dp.ERR_INVALID_ARG


def test_rows_up_to_what_a_launch_takes():
    # 64 x 64 tiles below 2^24, as the header says: 2^29 rows and more of up to 64 columns
    lib, need = dp.library(), ctypes.c_int64(-1)
    for n, k, m, rc in ((2 ** 29, 8, 64, 0), (2 ** 30 - 2 ** 12, 5, 64, 0), (2 ** 30, 8, 8, dp.ERR_UNSUPPORTED),
                        (2 ** 29 - 2 ** 12, 65, 5, 0), (2 ** 29, 65, 8, dp.ERR_UNSUPPORTED)):
        layer = ft._Grouped(1, 3, k, m, n, 256, None, 512, k, 1024)
        assert lib.dpa4c_grouped_linear_work(ctypes.byref(layer), ctypes.byref(need)) == rc, n
        assert lib.dpa4c_grouped_linear_backward_work(ctypes.byref(layer), ctypes.byref(need)) == rc, n


def test_a_stream_of_another_device():
    stream = types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    with pytest.raises(ValueError, match="cuda:1"):
        ft._launch(torch.device("cuda", 0), stream)
