"""Argument checks of the residual block's operators (no GPU: nothing reaches a device), and the
generator's reference against published vectors."""
import ctypes

import numpy as np
import pytest
import torch

import block_reference as ref
import paper_2608_19041_amd as dp
from paper_2608_19041_amd import block as bl

INVALID, UNSUPPORTED = dp.ERR_INVALID_ARG, dp.ERR_UNSUPPORTED
REF = ctypes.byref


def make(struct, defaults, change):
    args = dict(defaults)
    args.update(change)
    return struct(*[args[name] for name, _ in struct._fields_])


def rows8(**change):
    return make(bl._Rows8, dict(format=0, k=100, n=10, values=4096, ld=112, scales=512, ld_scales=1), change)


def weights8(**change):
    return make(bl._Weights8, dict(n_groups=3, k=100, n_out=7, values=4096, turned=8192, scales=512), change)


def norm(**change):
    return make(bl._Norm, dict(dtype=0, n_groups=3, k=100, n=10, group_ptr=256, order=None, gain=512), change)


def layer(x=None, w=None, **change):
    return make(bl._Grouped8, dict(dtype=2, group_ptr=256, order=None, x=rows8(**(x or {})),
                                   w=weights8(**(w or {}))), change)


@pytest.mark.parametrize("change,rc", [
    (dict(format=2), INVALID), (dict(format=-1), INVALID), (dict(k=0), INVALID), (dict(k=65537), INVALID),
    (dict(n=-1), INVALID), (dict(n=2 ** 31), INVALID), (dict(values=None), INVALID), (dict(scales=None), INVALID),
    (dict(values=4104), INVALID), (dict(ld=104), INVALID), (dict(ld=96), INVALID), (dict(ld=0), INVALID),
    (dict(ld_scales=0), INVALID), (dict(n=2 ** 31 - 1, k=65536, ld=65536, ld_scales=512), UNSUPPORTED)])
def test_rows_refused(change, rc):
    lib, r = dp.library(), rows8(**change)
    assert lib.dpa4c_quantize_rows(0, 4096, 65536, REF(r), None) == rc
    assert lib.dpa4c_dequantize_rows(REF(r), 0, 4096, None) == rc
    same = {k: v for k, v in change.items() if k in ("k", "n")}
    y = lib.dpa4c_rms_norm(REF(norm(**same)), 4096, 65536, None, 0, 1e-6, None, REF(r), None, None, None)
    assert y == rc or (same and y in (INVALID, rc))
    assert lib.dpa4c_last_error()


def test_quantize_refused():
    lib, r = dp.library(), rows8()
    assert lib.dpa4c_quantize_rows(3, 4096, 100, REF(r), None) == INVALID
    assert lib.dpa4c_quantize_rows(0, None, 100, REF(r), None) == INVALID
    assert lib.dpa4c_quantize_rows(0, 4096, 99, REF(r), None) == INVALID
    assert lib.dpa4c_quantize_rows(0, 4096, 100, None, None) == INVALID
    assert lib.dpa4c_dequantize_rows(REF(r), 0, None, None) == INVALID
    assert lib.dpa4c_dequantize_rows(REF(r), -1, 4096, None) == INVALID
    # nothing is launched without rows
    assert lib.dpa4c_quantize_rows(0, None, 100, REF(rows8(n=0, values=None, scales=None)), None) == 0


@pytest.mark.parametrize("change,rc", [
    (dict(n_groups=0), INVALID), (dict(n_groups=4097), UNSUPPORTED), (dict(k=0), INVALID), (dict(n_out=0), INVALID),
    (dict(k=65537), INVALID), (dict(n_out=65537), INVALID), (dict(values=4100), INVALID), (dict(turned=4100), INVALID),
    (dict(scales=None), INVALID), (dict(n_groups=4096, k=65536, n_out=65536), UNSUPPORTED)])
def test_weights_refused(change, rc):
    lib, w = dp.library(), weights8(**change)
    assert lib.dpa4c_quantize_weights(0, 4096, REF(w), None) == rc
    assert lib.dpa4c_dequantize_weights(REF(w), 0, 4096, None) == rc


def test_weights_calls_refused():
    lib = dp.library()
    assert lib.dpa4c_quantize_weights(0, None, REF(weights8()), None) == INVALID
    assert lib.dpa4c_quantize_weights(5, 4096, REF(weights8()), None) == INVALID
    assert lib.dpa4c_quantize_weights(0, 4096, None, None) == INVALID
    assert lib.dpa4c_dequantize_weights(REF(weights8(values=None)), 0, 4096, None) == INVALID
    assert lib.dpa4c_dequantize_weights(REF(weights8()), 0, None, None) == INVALID


@pytest.mark.parametrize("change,rc", [
    (dict(dtype=3), INVALID), (dict(n_groups=0), INVALID), (dict(n_groups=4097), UNSUPPORTED), (dict(k=0), INVALID),
    (dict(k=65537), INVALID), (dict(n=-1), INVALID), (dict(n=2 ** 31), INVALID), (dict(gain=None), INVALID),
    (dict(group_ptr=None), INVALID), (dict(group_ptr=None, n_groups=1, order=256), INVALID)])
def test_norm_refused(change, rc):
    lib, l = dp.library(), norm(**change)
    assert lib.dpa4c_rms_norm(REF(l), 4096, 65536, None, 0, 1e-6, 4096, None, 4096, None, None) == rc
    assert lib.dpa4c_rms_norm_backward(REF(l), 4096, 65536, 4096, 65536, 4096, None, 0, 4096, None, None, 0,
                                       None) == rc


def test_norm_calls_refused():
    lib, l = dp.library(), norm()
    call, back = lib.dpa4c_rms_norm, lib.dpa4c_rms_norm_backward
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert call(REF(l), 4096, 100, None, 0, eps, 4096, None, 4096, None, None) == INVALID
    assert call(None, 4096, 100, None, 0, 1e-6, 4096, None, 4096, None, None) == INVALID
    assert call(REF(l), None, 100, None, 0, 1e-6, 4096, None, 4096, None, None) == INVALID
    assert call(REF(l), 4096, 99, None, 0, 1e-6, 4096, None, 4096, None, None) == INVALID
    assert call(REF(l), 4096, 100, 4096, 99, 1e-6, 4096, None, 4096, 4096, None) == INVALID
    assert call(REF(l), 4096, 100, 4096, 100, 1e-6, 4096, None, 4096, None, None) == INVALID   # no h
    assert call(REF(l), 4096, 100, None, 0, 1e-6, 4096, None, 4096, 4096, None) == INVALID     # no residual
    assert call(REF(l), 4096, 100, None, 0, 1e-6, None, None, 4096, None, None) == INVALID
    assert call(REF(l), 4096, 100, None, 0, 1e-6, 4096, REF(rows8()), 4096, None, None) == INVALID
    assert call(REF(l), 4096, 100, None, 0, 1e-6, None, REF(rows8(n=9)), 4096, None, None) == INVALID
    assert call(REF(l), 4096, 100, None, 0, 1e-6, None, REF(rows8(k=99)), 4096, None, None) == INVALID
    for bad in range(3):
        at = [4096] * 3
        at[bad] = None
        assert back(REF(l), at[0], 100, at[1], 100, at[2], None, 0, 4096, None, None, 0, None) == INVALID
    assert back(REF(l), 4096, 99, 4096, 100, 4096, None, 0, 4096, None, None, 0, None) == INVALID
    assert back(REF(l), 4096, 100, 4096, 99, 4096, None, 0, 4096, None, None, 0, None) == INVALID
    assert back(REF(l), 4096, 100, 4096, 100, 4096, 4096, 99, 4096, None, None, 0, None) == INVALID
    need = ctypes.c_int64(-1)
    assert lib.dpa4c_rms_norm_backward_work(REF(l), 0, REF(need)) == 0 and need.value == 0
    assert lib.dpa4c_rms_norm_backward_work(REF(l), 1, REF(need)) == 0 and need.value > 0
    assert lib.dpa4c_rms_norm_backward_work(REF(l), 1, None) == INVALID
    for work, size in ((None, need.value), (4096, need.value - 1), (4100, need.value)):
        assert back(REF(l), 4096, 100, 4096, 100, 4096, None, 0, 4096, 4096, work, size, None) == INVALID


@pytest.mark.parametrize("l,rc", [
    (layer(dtype=0), UNSUPPORTED), (layer(dtype=3), INVALID), (layer(group_ptr=None), INVALID),
    (layer(x=dict(k=99, ld=112)), INVALID), (layer(x=dict(values=None)), INVALID), (layer(x=dict(ld=104)), INVALID),
    (layer(w=dict(scales=None)), INVALID), (layer(w=dict(n_groups=4097)), UNSUPPORTED),
    (layer(x=dict(n=2 ** 31 - 1), w=dict(n_out=65536)), UNSUPPORTED)])
def test_layer_refused(l, rc):
    lib, big = dp.library(), 1 << 50
    assert lib.dpa4c_grouped_linear8(REF(l), None, 0, None, 0, 4096, None, 256, big, None) == rc
    assert lib.dpa4c_grouped_linear8_backward(REF(l), 0, 4096, 65536, None, 0, 4096, None, None, 256, big,
                                              None) == rc


def test_layer_calls_refused():
    lib, l, big = dp.library(), layer(), 1 << 50
    call, back = lib.dpa4c_grouped_linear8, lib.dpa4c_grouped_linear8_backward
    assert call(None, None, 0, None, 0, 4096, None, 256, big, None) == INVALID
    assert call(REF(l), None, 2, None, 0, 4096, None, 256, big, None) == INVALID
    assert call(REF(l), None, 0, None, 0, None, None, 256, big, None) == INVALID
    assert call(REF(l), None, 0, 4096, 6, 4096, None, 256, big, None) == INVALID
    assert call(REF(layer(w=dict(turned=None))), None, 0, None, 0, 4096, None, 256, big, None) == INVALID
    assert back(REF(l), 2, 4096, 7, None, 0, 4096, None, None, 256, big, None) == INVALID
    assert back(REF(l), 0, None, 7, None, 0, 4096, None, None, 256, big, None) == INVALID
    assert back(REF(l), 0, 4096, 6, None, 0, 4096, None, None, 256, big, None) == INVALID
    assert back(REF(l), 0, 4096, 7, 4096, 6, 4096, None, None, 256, big, None) == INVALID
    assert back(REF(layer(w=dict(values=None))), 0, 4096, 7, None, 0, 4096, None, None, 256, big, None) == INVALID
    assert back(REF(l), 0, 4096, 7, None, 0, 4096, None, None, None, 0, None) == INVALID   # scratch
    need = ctypes.c_int64(-1)
    assert lib.dpa4c_grouped_linear8_work(REF(l), None) == INVALID
    assert lib.dpa4c_grouped_linear8_backward_work(REF(l), 1, 1, 1, None) == INVALID
    sizes = []
    for want in ((1, 1, 1), (1, 0, 0), (0, 1, 1), (0, 0, 1)):
        assert lib.dpa4c_grouped_linear8_backward_work(REF(l), *want, REF(need)) == 0
        sizes.append(need.value)
    assert sizes[0] >= max(sizes[1:]) and sizes[3] <= sizes[2]


def test_scratch_of_every_size():
    """Sizes of all kinds of tiles, and the ends of the ranges, have a plan."""
    lib, need = dp.library(), ctypes.c_int64(0)
    for n in (0, 1, 30, 127, 4095, 4096, 100000, 2 ** 24):
        for groups in (1, 5, 600, 4096):
            for k in (1, 128, 640, 641, 1024, 1025, 65536):
                for m in (1, 7, 8, 384, 1025, 65536):
                    l = layer(x=dict(n=n, k=k, ld=65536, ld_scales=512), w=dict(n_groups=groups, k=k, n_out=m))
                    rc = lib.dpa4c_grouped_linear8_work(REF(l), REF(need))
                    assert rc in (0, UNSUPPORTED) and (rc or need.value >= 0)
                    assert lib.dpa4c_grouped_linear8_backward_work(REF(l), 1, 1, 1, REF(need)) == rc
                    assert rc == 0 or n * max(k, m) > 2 ** 29 or groups * k * m > 2 ** 28


def test_scratch_of_gradients_is_what_the_rows_can_use():
    """dz in 16 and in 8 bits with its scales, and the blocks' sums."""
    lib, need = dp.library(), ctypes.c_int64(0)
    for n, k, m, groups in ((108, 541, 384, 4096), (31250, 541, 384, 118), (1000188, 541, 384, 5)):
        l = layer(x=dict(n=n, k=k, ld=544, ld_scales=5), w=dict(n_groups=groups, k=k, n_out=m))
        assert lib.dpa4c_grouped_linear8_backward_work(REF(l), 1, 1, 1, REF(need)) == 0
        assert need.value < n * (3 * 384 + 3) + (1 << 20) + 4 * (k + 1) * m * (2 * n // 512 + 2)


@pytest.mark.parametrize("p", [-0.1, 1.1, float("nan")])
def test_dropout_refused(p):
    lib = dp.library()
    assert lib.dpa4c_dropout(0, 4096, 10, None, 0, 5, 10, p, 1, 0, None, 4096, None) == INVALID


def test_dropout_calls_refused():
    call = dp.library().dpa4c_dropout
    assert call(3, 4096, 10, None, 0, 5, 10, 0.5, 1, 0, None, 4096, None) == INVALID
    assert call(0, None, 10, None, 0, 5, 10, 0.5, 1, 0, None, 4096, None) == INVALID
    assert call(0, 4096, 10, None, 0, 5, 10, 0.5, 1, 0, None, None, None) == INVALID
    assert call(0, 4096, 9, None, 0, 5, 10, 0.5, 1, 0, None, 4096, None) == INVALID
    assert call(0, 4096, 10, 4096, 9, 5, 10, 0.5, 1, 0, None, 4096, None) == INVALID
    assert call(0, 4096, 10, None, 0, -1, 10, 0.5, 1, 0, None, 4096, None) == INVALID
    assert call(0, 4096, 10, None, 0, 5, 0, 0.5, 1, 0, None, 4096, None) == INVALID
    assert call(0, 4096, 10, None, 0, 2 ** 31 - 1, 65536, 0.5, 1, 0, None, 4096, None) == UNSUPPORTED
    assert call(0, None, 10, None, 0, 0, 10, 0.5, 1, 0, None, None, None) == 0


def test_binding_refuses_what_is_not_on_a_device():
    x = torch.zeros(4, 8)
    q = dp.Rows8(torch.zeros(4, 16, dtype=torch.uint8).view(torch.float8_e4m3fn),
                 torch.zeros(4, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu))
    for call in (lambda: dp.quantize_rows(x), lambda: dp.quantize_weights(x[None]), lambda: dp.rms_norm(x, x[0]),
                 lambda: dp.dropout(x, 0.1, 1), lambda: dp.dequantize(q), lambda: dp.dequantize(x),
                 lambda: dp.grouped_linear8(q, None, None), lambda: dp.grouped_linear8(x, None, None),
                 lambda: dp.grouped_linear8_backward(x, q, None, None), lambda: dp.quantize_rows(None),
                 lambda: dp.rms_norm(None, x), lambda: dp.dropout(x[0], 0.1, 1)):
        with pytest.raises(ValueError):
            call()


def test_reference_generator_gives_the_published_words():
    """The known answers that its authors publish for Philox4x32-10."""
    for c, k, want in (
            ((0,) * 4, (0,) * 2, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             "d16cfe09 94fdcceb 5001e420 24126ea1")):
        got = ref.philox(np.array(c, dtype=np.uint64), k)
        assert " ".join("%08x" % v for v in got) == want


def test_reference_rounds_as_torch_does():
    """Values in range: the reference's grid is torch's conversion of float32."""
    g = torch.Generator().manual_seed(1)
    for form in ("e4m3", "e5m2"):
        x = torch.randn(200, 128, generator=g) * torch.exp(3 * torch.randn(200, 1, generator=g))
        q, s = ref.quantize(x, form)
        assert torch.equal((x / s.float()).to(ref.F8[form]).to(torch.float64) * s, q)
        assert (x.abs().amax(1) <= ref.FORM[form][0] * s[:, 0]).all()
        assert (x.abs().amax(1) > ref.FORM[form][0] * s[:, 0] / 2).all()
