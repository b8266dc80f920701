"""What the residual block's operators refuse of tensors on a device, and calls that need no refusal (GPU)."""
import pytest
import torch

import paper_2608_19041_amd as dp

pytestmark = pytest.mark.gpu


def rows(n, k, dtype=torch.float32):
    return torch.randn(n, k, device="cuda").to(dtype)


def parts():
    ptr = torch.tensor([0, 4, 10], device="cuda")
    x8 = dp.quantize_rows(rows(10, 40))
    return ptr, x8, dp.quantize_weights(torch.randn(2, 40, 24, device="cuda"))


def refused(*calls):
    for call in calls:
        with pytest.raises((ValueError, dp.DPA4CError)):
            call()


def test_rows_of_wrong_types_and_shapes():
    x = rows(10, 40)
    gain, ptr = torch.ones(40, device="cuda"), torch.tensor([0, 10], device="cuda")
    refused(lambda: dp.quantize_rows(x.double()), lambda: dp.quantize_rows(x[0]), lambda: dp.quantize_rows(x.t()),
            lambda: dp.quantize_rows(x, "e3m4"), lambda: dp.quantize_rows(x.int()),
            lambda: dp.quantize_rows(torch.as_strided(x, (10, 40), (20, 1))),
            lambda: dp.quantize_rows(torch.zeros(10, 0, device="cuda")),
            lambda: dp.quantize_weights(x), lambda: dp.quantize_weights(x.view(2, 5, 40).transpose(1, 2)),
            lambda: dp.rms_norm(x, gain[:39]), lambda: dp.rms_norm(x, gain.bfloat16()), lambda: dp.rms_norm(x, gain[None]),
            lambda: dp.rms_norm(x, gain, ptr), lambda: dp.rms_norm(x, gain, eps=0.0), lambda: dp.rms_norm(x, gain, quantize="fp8"),
            lambda: dp.rms_norm(x, gain[None], ptr.int()), lambda: dp.rms_norm(x, gain[None], ptr[:1]),
            lambda: dp.rms_norm(x, gain[None, None], ptr), lambda: dp.rms_norm(x, gain, residual=x.half()),
            lambda: dp.rms_norm(x, gain[None], ptr, torch.zeros(9, dtype=torch.int32, device="cuda")),
            lambda: dp.rms_norm_backward(x, x, gain, torch.zeros(9, device="cuda")),
            lambda: dp.rms_norm_backward(x[:, :39], x, gain, torch.zeros(10, device="cuda")),
            lambda: dp.rms_norm_backward(x, x, gain, torch.zeros(10, device="cuda"), dh=x[:9]),
            lambda: dp.dropout(x, 1.5, 1), lambda: dp.dropout(x, 0.5, -1), lambda: dp.dropout(x, 0.5, 2 ** 64),
            lambda: dp.dropout(x, 0.5, 1, 2 ** 63), lambda: dp.dropout(x, 0.5, 1, torch.zeros(2, dtype=torch.int64, device="cuda")),
            lambda: dp.dropout(x, 0.5, 1, torch.tensor(1)), lambda: dp.dropout(x, 0.5, 1, residual=x[:, :39]))


def test_8_bit_rows_that_cannot_be_read():
    ptr, x8, w8 = parts()
    q, s = x8
    tight = torch.zeros(9 * 48 + 40, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    off = torch.zeros(10 * 48 + 8, dtype=torch.uint8, device="cuda")[8:].view(torch.float8_e4m3fn)

    def layer(values, scales=s):
        return lambda: dp.grouped_linear8(dp.Rows8(values, scales), w8, ptr)

    refused(layer(torch.as_strided(tight, (10, 40), (48, 1))),          # no room behind the last row
            layer(torch.as_strided(off, (10, 40), (48, 1))),            # starts at 8
            layer(torch.as_strided(tight, (10, 40), (40, 1))),          # 40 bytes apart
            layer(q.contiguous()[:, ::2]), layer(q.float()), layer(q[:9]), layer(q, s[:9]), layer(q, s.float()),
            layer(q, s[:1].expand(10, 1)), layer(q[0]))
    # one row, and none, need no distance
    assert dp.grouped_linear8(dp.Rows8(q[:1], s[:1]), w8, torch.tensor([0, 1, 1], device="cuda")).shape == (1, 24)


def test_layers_that_do_not_fit():
    ptr, x8, w8 = parts()
    dy = rows(10, 24, torch.bfloat16)
    forward = dp.quantize_weights(torch.randn(2, 40, 24, device="cuda"), backward=False)
    other = dp.quantize_weights(torch.randn(2, 41, 24, device="cuda"))
    refused(lambda: dp.grouped_linear8(x8, other, ptr), lambda: dp.grouped_linear8(x8, w8, ptr[:2]),
            lambda: dp.grouped_linear8(x8, w8, ptr, dtype=torch.float32),
            lambda: dp.grouped_linear8(x8, w8, ptr, activation="relu"),
            lambda: dp.grouped_linear8(x8, w8, ptr, bias=rows(2, 24)),
            lambda: dp.grouped_linear8(x8, w8, ptr, residual=rows(10, 23, torch.bfloat16)),
            lambda: dp.grouped_linear8(x8, w8._replace(turned=None), ptr),
            lambda: dp.grouped_linear8(x8, w8._replace(turned=w8.turned.contiguous()[:, :, :39]), ptr),
            lambda: dp.grouped_linear8(x8, w8._replace(scales=w8.scales[:1]), ptr),
            lambda: dp.grouped_linear8_backward(dy, x8, forward, ptr), lambda: dp.dequantize(forward),
            lambda: dp.grouped_linear8_backward(dy.float(), x8, w8, ptr),
            lambda: dp.grouped_linear8_backward(dy[:9], x8, w8, ptr),
            lambda: dp.grouped_linear8_backward(dy, x8, w8, ptr, preact=dy.half()),
            lambda: dp.grouped_linear8_backward(dy, x8, w8, ptr, format="fp8"))
    # gradients of the weights alone need no other layout, and rows no gradient at all
    dx, dw, db = dp.grouped_linear8_backward(dy, x8, forward, ptr, need=(False, True, True))
    assert dx is None and dw.shape == (2, 40, 24) and db.shape == (2, 24)
    assert dp.grouped_linear8_backward(dy, x8, w8, ptr, need=(False, False, False)) == (None, None, None)


def test_what_autograd_would_follow_is_refused():
    ptr, x8, w8 = parts()
    x = rows(10, 40)
    leaf = x.clone().requires_grad_()
    gain = torch.ones(2, 40, device="cuda")
    bias = torch.zeros(2, 24, device="cuda", dtype=torch.bfloat16).requires_grad_()
    _, s = dp.rms_norm(x, gain, ptr)
    calls = (lambda: dp.quantize_rows(leaf), lambda: dp.quantize_weights(leaf[None]), lambda: dp.rms_norm(leaf, gain, ptr),
             lambda: dp.rms_norm(x, gain, ptr, residual=leaf), lambda: dp.rms_norm(x, gain.clone().requires_grad_(), ptr),
             lambda: dp.rms_norm_backward(leaf, x, gain, s, ptr), lambda: dp.dropout(leaf, 0.5, 1),
             lambda: dp.dropout(x, 0.5, 1, residual=leaf), lambda: dp.grouped_linear8(x8, w8, ptr, bias=bias))
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
    with torch.no_grad():
        for call in calls:
            call()


def test_rows_in_any_order_and_entries_outside_it():
    """Entries of order outside [0, n) are passed over: their places give nothing, and all else is as it was."""
    n, k, m = 300, 70, 33
    x, dy = rows(n, k, torch.bfloat16), rows(n, m, torch.bfloat16)
    gain = torch.ones(3, k, device="cuda", dtype=torch.bfloat16)
    w8 = dp.quantize_weights(torch.randn(3, k, m, device="cuda"))
    ptr = torch.tensor([0, 100, 180, 290], device="cuda")
    order = torch.randperm(n, device="cuda").to(torch.int32)
    bad = order.clone()
    gone = [3, 120, 179, 289, 295]
    bad[gone] = torch.tensor([-1, n, 2 ** 31 - 1, -2 ** 31, n + 7], dtype=torch.int32, device="cuda")
    left = torch.ones(n, dtype=torch.bool, device="cuda")
    left[order[gone].long()] = False
    for many in (1, 40, 450):   # the kernels of few rows and of many
        xs, dys = x.repeat(many, 1), dy.repeat(many, 1)
        p = ptr * many
        at = torch.arange(many, device="cuda", dtype=torch.int32)[None] * n

        def spread(o):   # group by group, each row ``many`` times
            good = (o >= 0) & (o < n)
            outside = torch.where(o < 0, o, 2 ** 31 - 1 if many > 1 else o)   # of the longer order too
            return torch.where(good[:, None], o[:, None] + at, outside[:, None]).reshape(-1).contiguous()

        full, some = spread(order), spread(bad)
        keep = left.repeat(many)
        x8 = dp.quantize_rows(xs)
        y, z = (dp.grouped_linear8(x8, w8, p, o) for o in (full, some))
        assert torch.equal(y[keep], z[keep])
        (yn, sn), (zn, tn) = (dp.rms_norm(xs, gain, p, o) for o in (full, some))
        assert torch.equal(yn[keep], zn[keep]) and torch.equal(sn[keep], tn[keep])
        dx, dw, db = dp.grouped_linear8_backward(dys, x8, w8, p, some)
        clear = torch.where(keep[:, None], dys, 0)
        ex, ew, eb = dp.grouped_linear8_backward(clear, x8, w8, p, full)
        assert torch.equal(dx[keep], ex[keep]) and torch.equal(dw, ew) and torch.equal(db, eb)
        dn, dg = dp.rms_norm_backward(xs, xs, gain, sn, p, some)
        en, eg = dp.rms_norm_backward(torch.where(keep[:, None], xs, 0), xs, gain, sn, p, full)
        assert torch.equal(dn[keep], en[keep]) and torch.equal(dg, eg)


def test_numbers_that_are_no_integers():
    x = rows(10, 40)
    for call in (lambda: dp.dropout(x, 0.5, 1.5), lambda: dp.dropout(x, 0.5, 1, 0.5)):
        with pytest.raises(TypeError):
            call()


def test_8_bit_tensors_that_require_gradients():
    ptr, x8, w8 = parts()
    dy = rows(10, 24, torch.bfloat16)
    q = x8.values.detach().requires_grad_()
    w = w8.turned.detach().requires_grad_()
    x_wants, w_wants = dp.Rows8(q, x8.scales), dp.Weights8(w8.values, w, w8.scales)
    refused(lambda: dp.dequantize(x_wants), lambda: dp.grouped_linear8(x_wants, w8, ptr),
            lambda: dp.grouped_linear8(x8, w_wants, ptr), lambda: dp.grouped_linear8_backward(dy, x8, w_wants, ptr))
    with torch.no_grad():
        assert torch.equal(dp.grouped_linear8(x_wants, w_wants, ptr), dp.grouped_linear8(x8, w8, ptr))
