"""The fitting operators beside autograd: nothing is lost without a message (GPU)."""
import pytest
import torch

import paper_2608_19041_amd as dp

pytestmark = pytest.mark.gpu


@pytest.fixture
def layer():
    g = torch.Generator(device="cuda").manual_seed(0)
    n, k, groups = 50, 12, 3
    ids = torch.randint(0, groups, (n,), generator=g, device="cuda", dtype=torch.int32)
    x, w, b = (torch.randn(*s, generator=g, device="cuda") for s in ((n, k), (groups, k, k), (groups, k)))
    ptr, order = dp.group_rows(ids, groups)
    return x, w, b, ptr, order


def test_tensors_that_autograd_follows_are_refused(layer):
    x, w, b, ptr, order = layer

    def forward(x, w, b):
        return dp.grouped_linear(x, w, ptr, order, bias=b, activation="silu", preact=True)

    want = forward(x, w, b)
    y, z = want
    grads = dp.grouped_linear_backward(y, x, w, ptr, order, preact=z)
    follow = lambda t: t.clone().requires_grad_()
    bad = [lambda: forward(follow(x), w, b), lambda: forward(x, follow(w), b), lambda: forward(x, w, follow(b)),
           lambda: dp.grouped_linear_backward(follow(y), x, w, ptr, order, preact=z),
           lambda: dp.grouped_linear_backward(y, follow(x), w, ptr, order, preact=z),
           lambda: dp.grouped_linear_backward(y, x, follow(w), ptr, order, preact=z),
           lambda: dp.grouped_linear_backward(y, x, w, ptr, order, preact=follow(z)),
           lambda: dp.orthogonalize([w, follow(w)])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"case {i} was accepted")
        with torch.no_grad():
            call()
    with torch.no_grad():
        for a, c in zip(want, forward(follow(x), follow(w), follow(b))):
            assert torch.equal(a, c)
        for a, c in zip(grads, dp.grouped_linear_backward(y, x, follow(w), ptr, order, preact=z)):
            assert torch.equal(a, c)


def test_a_function_of_autograd_around_a_layer(layer):
    x, w, b, ptr, order = layer

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, z = dp.grouped_linear(x, w, ptr, order, bias=b, activation="silu", residual=True, preact=True)
            ctx.save_for_backward(x, w, z)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, z = ctx.saved_tensors
            return dp.grouped_linear_backward(dy.contiguous(), x, w, ptr, order, preact=z, residual=True)

    args = [t.clone().requires_grad_() for t in (x, w, b)]
    y = Layer.apply(*args)
    (y * y).sum().backward()
    y, z = dp.grouped_linear(x, w, ptr, order, bias=b, activation="silu", residual=True, preact=True)
    for p, want in zip(args, dp.grouped_linear_backward(2 * y, x, w, ptr, order, preact=z, residual=True)):
        assert torch.equal(p.grad, want)


def test_autograd_notices_an_update():
    w = torch.randn(4, 6, device="cuda", requires_grad=True)
    m = torch.zeros(4, 6, device="cuda")
    y = (w * w).sum()                       # keeps w for its backward pass
    kept = (m * w.detach().requires_grad_()).sum()
    dp.muon_step([w], [torch.randn(4, 6, device="cuda")], [m], lr=0.1)
    for loss in (y, kept):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    y = (w * w).sum()
    y.backward()
    assert torch.equal(w.grad, 2 * w.detach())
