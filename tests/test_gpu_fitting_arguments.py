"""Arguments that the fitting operators would answer wrongly are refused (GPU)."""
import pytest
import torch

import paper_2608_19041_amd as dp

pytestmark = pytest.mark.gpu


def test_sizes_beyond_32_bits():
    ids = torch.zeros(10, dtype=torch.int32, device="cuda")
    for groups in (2 ** 32 + 3, -2 ** 32 + 3):
        with pytest.raises(dp.DPA4CError):
            dp.group_rows(ids, groups)
    with pytest.raises(dp.DPA4CError):
        dp.orthogonalize([torch.randn(4, 4, device="cuda")], steps=2 ** 32 + 5)


def test_an_update_that_would_meet_itself():
    f = dict(device="cuda")
    w, v, g, m, p = (torch.randn(6, 4, **f) for _ in range(5))
    before = [t.clone() for t in (w, v, g, m, p)]
    for params, grads, momenta in (([w, w], [g, v], [m, p]),         # a tied weight listed twice
                                   ([w, v], [g, g], [m, m]),         # one momentum for two weights
                                   ([w], [g], [w]), ([w], [m], [m])):
        with pytest.raises(ValueError):
            dp.muon_step(params, grads, momenta, lr=0.1)
    for t, old in zip((w, v, g, m, p), before):
        assert torch.equal(t, old)
    # one gradient for two weights, and empty stacks, are no such thing
    none = torch.empty(0, 3, 3, **f)
    dp.muon_step([w, v, none, none], [g, g, none, none], [m, p, none, none], lr=0.1)
    alone = before[0].clone(), before[3].clone()
    dp.muon_step([alone[0]], [g], [alone[1]], lr=0.1)
    assert torch.equal(alone[0], w) and torch.equal(alone[1], m)


@pytest.mark.parametrize("k", [3, 8])
def test_more_rows_than_2_to_the_29(k):
    n, m, groups = 2 ** 29 + 77, 2, 2
    x = torch.empty(n, k, dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn(groups, k, m, device="cuda").bfloat16()
    ptr = torch.tensor([0, n // 3, n - 5], device="cuda")
    y = dp.grouped_linear(x, w, ptr)
    at = torch.cat([torch.arange(a - 60, a + 60) for a in (60, n // 3, 2 ** 29, n - 60)]).cuda()
    group = (at >= n // 3).long()
    want = (x[at].double()[:, :, None] * w.double()[group]).sum(1) * (at < n - 5)[:, None]
    # rounded once to 8 bits, and a sum of 8 in float32 whose terms are below 32
    assert ((y[at].double() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * 32 * 2.0 ** -24).all()
    _, dw, db = dp.grouped_linear_backward(y, x, w, ptr, need=(False, True, True))
    for t, (a, b) in enumerate(((0, n // 3), (n // 3, n - 5))):
        want, size = (torch.zeros(k + 1, m, dtype=torch.float64, device="cuda") for _ in range(2))
        for at in range(a, b, 2 ** 25):
            part = slice(at, min(b, at + 2 ** 25))
            for i in range(k + 1):
                for j in range(m):
                    term = y[part, j].double() * (x[part, i].double() if i < k else 1)
                    want[i, j] += term.sum()
                    size[i, j] += term.abs().sum()
        got = torch.cat([dw[t], db[t][None]]).double()
        # blocks of 8,192 rows in float32: 2^-14 of the sum of magnitudes at the most
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -14 * size).all()
        assert (want[:k].abs() > 2.0 ** -9 * size[:k]).any()
    del x, y
    torch.cuda.empty_cache()
