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
