"""sifar_experts where few choices, long rows, values that are not finite and waits that run out meet its layouts."""
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests.test_experts import Moe

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T,k", [(1, 32), (4, 8), (5, 8), (8, 8)])
@pytest.mark.parametrize("H", [16, 64, 200])
def test_ctas_without_rows_in_clusters_that_share_columns(dtype, T, k, H):
    """Clusters are as large as choices of different experts would want; all tokens choose one, or none, so most of a cluster's CTAs are at their
    sums at once, when the one that adds them up may not have started yet."""
    m = Moe(T, H, 1000, 40, k, dtype=dtype, choice=[[7] * k] * T)
    first = m.check()
    for _ in range(30):
        m.out.fill_(9.0)
        assert torch.equal(first, m.run())
    assert not bool(Moe(T, H, 1000, 40, k, dtype=dtype, choice=[[-1] * k] * T).check().any())
