"""sifar_experts where few choices, long rows, values that are not finite and waits that run out meet its layouts."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests.test_experts import Moe

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


_WAITS = """
import sys, numpy as np, torch
sys.path.insert(0, %r)
from paper_2607_08973_b200 import binding as sf
from tests.test_experts import Moe
outs = []
for T, H, I, E, k in %r:
    m = Moe(T, H, I, E, k, seed=T)
    outs += [m.run().float().cpu().numpy() for _ in range(5)]
few = Moe(3, 64, 32, 4, 2)
few.check()                                                  # the GPU goes on as before
np.savez(sys.argv[1], *outs)
"""
_SHAPES = [(64, 1024, 256, 12, 3), (200, 512, 520, 40, 6), (256, 2048, 64, 4, 2), (33, 264, 72, 160, 8)]


@gpu
@pytest.mark.parametrize("polls", [0, 1, 3, 10, 30, 100, 300, 1000])
def test_a_wait_that_runs_out_gives_nan_and_nothing_wrong(polls, tmp_path):
    """Limits from none at all to more than any wait takes: every element is the right one or NaN, and the calls end."""
    path = str(tmp_path / "outs.npz")
    subprocess.run([sys.executable, "-c", _WAITS % (ROOT, _SHAPES), path], check=True, cwd=ROOT, env=dict(os.environ, SIFAR_EXPERTS_POLLS=str(polls)), timeout=300)
    got = np.load(path)
    short = 0
    for i, (T, H, I, E, k) in enumerate(_SHAPES):  # noqa: E741
        want = Moe(T, H, I, E, k, seed=T).run().float().cpu().numpy()
        assert np.isfinite(want).all()
        for n in range(5):
            out = got["arr_%d" % (5 * i + n)]
            nan = np.isnan(out)
            assert np.array_equal(out[~nan], want[~nan])
            short += int(nan.any())
    assert short == 5 * len(_SHAPES) if polls == 0 else True
