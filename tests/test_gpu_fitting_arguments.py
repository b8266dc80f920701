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
