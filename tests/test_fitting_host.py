"""Argument checks of the fitting operators' C ABI (no GPU: nothing reaches a device)."""
import ctypes

import pytest

import paper_2608_19041_amd as dp
from paper_2608_19041_amd import fitting as ft

INVALID, UNSUPPORTED = dp.ERR_INVALID_ARG, dp.ERR_UNSUPPORTED


def layer(**change):
    args = dict(dtype=0, n_groups=3, k=5, n_out=7, n=10, group_ptr=256, order=None, x=512, ldx=5,
                weight=1024)
    args.update(change)
    return ft._Grouped(*[args[name] for name, _ in ft._Grouped._fields_])


def newton(**change):
    args = dict(steps=5, a=3.0, b=-4.0, c=2.0, eps=1e-7)
    args.update(change)
    return ft._Newton(*[args[name] for name, _ in ft._Newton._fields_])


@pytest.mark.parametrize("n,groups,rc", [(-1, 3, INVALID), (2 ** 31, 3, INVALID), (5, 0, INVALID),
                                         (5, 513, UNSUPPORTED), (5, 512, 0), (0, 1, 0)])
def test_group_rows_sizes(n, groups, rc):
    need = ctypes.c_int64(-1)
    assert dp.library().dpa4c_group_rows_work(n, groups, ctypes.byref(need)) == rc
    assert (need.value >= 0) == (rc == 0)
    if rc:
        assert dp.library().dpa4c_group_rows(256, n, groups, 256, 256, None, 0, None) == rc


@pytest.mark.parametrize("change", [dict(dtype=3), dict(dtype=-1), dict(n_groups=0), dict(k=0),
                                    dict(n_out=0), dict(k=65537), dict(n=-1), dict(n=2 ** 31),
                                    dict(group_ptr=None), dict(weight=None), dict(x=None),
                                    dict(ldx=4)])
def test_layer_refused(change):
    lib, l = dp.library(), layer(**change)
    big = 1 << 40
    assert lib.dpa4c_grouped_linear(ctypes.byref(l), None, 0, 0, 256, None, 256, big, None) == INVALID
    assert lib.dpa4c_grouped_linear_backward(ctypes.byref(l), 256, 7, None, 0, 0, 256, None, None,
                                             256, big, None) == INVALID
    assert lib.dpa4c_last_error()


def test_layer_call_refused():
    lib, l = dp.library(), layer()
    ref, big = ctypes.byref(l), 1 << 40
    assert lib.dpa4c_grouped_linear(None, None, 0, 0, 256, None, 256, big, None) == INVALID
    assert lib.dpa4c_grouped_linear(ref, None, 2, 0, 256, None, 256, big, None) == INVALID
    assert lib.dpa4c_grouped_linear(ref, None, 0, 1, 256, None, 256, big, None) == INVALID
    assert lib.dpa4c_grouped_linear(ref, None, 0, 0, None, None, 256, big, None) == INVALID
    back = lib.dpa4c_grouped_linear_backward
    assert back(ref, None, 7, None, 0, 0, 256, None, None, 256, big, None) == INVALID
    assert back(ref, 256, 6, None, 0, 0, 256, None, None, 256, big, None) == INVALID
    assert back(ref, 256, 7, 256, 6, 0, 256, None, None, 256, big, None) == INVALID
    l65 = layer(n_groups=4097)
    assert lib.dpa4c_grouped_linear(ctypes.byref(l65), None, 0, 0, 256, None, 256, big, None) == UNSUPPORTED


def test_scratch_is_checked():
    lib = dp.library()
    need = ctypes.c_int64()
    s = (ft._Stack * 1)(ft._Stack(256, 256, 2, 30, 20))
    assert lib.dpa4c_orthogonalize_work(1, s, ctypes.byref(need)) == 0 and need.value > 0
    how = newton()
    for work, size in ((None, need.value), (256, need.value - 1), (264, need.value)):
        assert lib.dpa4c_orthogonalize(0, 1, s, ctypes.byref(how), work, size, None) == INVALID


@pytest.mark.parametrize("change", [dict(steps=-1), dict(steps=101), dict(eps=0.0),
                                    dict(eps=float("nan")), dict(a=float("inf"))])
def test_newton_refused(change):
    lib, how = dp.library(), newton(**change)
    s = (ft._Stack * 1)(ft._Stack(256, 256, 2, 30, 20))
    assert lib.dpa4c_orthogonalize(0, 1, s, ctypes.byref(how), 256, 1 << 40, None) == INVALID


@pytest.mark.parametrize("stack", [(256, 256, 1, 0, 5), (256, 256, 1, 5, 65537), (256, 256, -1, 5, 5),
                                   (None, 256, 1, 5, 5), (256, None, 1, 5, 5),
                                   (256, 256, 1 << 40, 5, 5)])
def test_stacks_refused(stack):
    lib, how = dp.library(), newton()
    s = (ft._Stack * 1)(ft._Stack(*stack))
    assert lib.dpa4c_orthogonalize(0, 1, s, ctypes.byref(how), 256, 1 << 60, None) == INVALID
    many = (ft._Stack * 33)()
    assert lib.dpa4c_orthogonalize(0, 33, many, ctypes.byref(how), 256, 1 << 60, None) == INVALID
    assert lib.dpa4c_orthogonalize(3, 0, many, ctypes.byref(how), 256, 1 << 60, None) == INVALID


def test_update_refused():
    lib, how = dp.library(), newton()
    u = (ft._Update * 1)(ft._Update(256, 256, None, 1, 5, 5))
    call = lib.dpa4c_muon_step
    assert call(0, 1, u, ctypes.byref(how), 0.1, 0.9, 1, 0.0, 256, 1 << 40, None) == INVALID
    u[0].momentum_buf = 256
    assert call(0, 1, u, ctypes.byref(how), float("nan"), 0.9, 1, 0.0, 256, 1 << 40, None) == INVALID
    assert call(0, 1, u, None, 0.1, 0.9, 1, 0.0, 256, 1 << 40, None) == INVALID


@pytest.mark.parametrize("change,rc", [(dict(n=2 ** 31 - 1), UNSUPPORTED), (dict(n=2 ** 28), 0),
                                       (dict(n=2 ** 24, k=65536, ldx=65536), UNSUPPORTED),
                                       (dict(n_groups=4096, k=1, n_out=65536), UNSUPPORTED),
                                       (dict(n_groups=512, k=1, n_out=65536), 0)])
def test_layers_beyond_a_launch(change, rc):
    lib, l, need = dp.library(), layer(**change), ctypes.c_int64(-1)
    assert lib.dpa4c_grouped_linear_work(ctypes.byref(l), ctypes.byref(need)) == rc
    assert lib.dpa4c_grouped_linear_backward_work(ctypes.byref(l), ctypes.byref(need)) == rc
    if rc:
        big = 1 << 60
        assert lib.dpa4c_grouped_linear(ctypes.byref(l), None, 0, 0, 256, None, 256, big, None) == rc
        assert lib.dpa4c_grouped_linear_backward(ctypes.byref(l), 256, l.n_out, None, 0, 0, 256, 256, 256,
                                                 256, big, None) == rc


@pytest.mark.parametrize("batch,rows,cols,rc", [(2 ** 24, 1, 1, UNSUPPORTED), (2 ** 22, 1, 1, 0),
                                                (20, 65536, 65536, UNSUPPORTED), (1, 65536, 65536, 0)])
def test_matrices_beyond_a_launch(batch, rows, cols, rc):
    lib, need, how = dp.library(), ctypes.c_int64(-1), newton()
    s = (ft._Stack * 1)(ft._Stack(256, 256, batch, rows, cols))
    assert lib.dpa4c_orthogonalize_work(1, s, ctypes.byref(need)) == rc
    u = (ft._Update * 1)(ft._Update(256, 256, 256, batch, rows, cols))
    assert lib.dpa4c_muon_step_work(1, u, ctypes.byref(need)) == rc
    if rc:
        big = 1 << 60
        assert lib.dpa4c_orthogonalize(0, 1, s, ctypes.byref(how), 256, big, None) == rc
        assert lib.dpa4c_muon_step(0, 1, u, ctypes.byref(how), 0.1, 0.9, 1, 0.0, 256, big, None) == rc
