"""sifar_experts where few choices, long rows, values that are not finite and waits that run out meet its layouts."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref
from tests.decode_ref import DT
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


@gpu
@pytest.mark.parametrize("dtype,T,H,pad", [(sf.BF16, 4, 256, 0), (sf.BF16, 4, 250, 3), (sf.BF16, 40, 264, 3), (sf.BF16, 40, 250, 0), (sf.F32, 4, 255, 1), (sf.F32, 40, 256, 0), (sf.F32, 40, 255, 1)])
def test_what_the_kernels_in_front_write_is_seen(dtype, T, H, pad):
    """Tokens and weights that the kernels just before the call left, while the call's first kernel was started already."""
    m = Moe(T, H, 64, 6, 2, dtype=dtype, pad=pad)
    dt = m.x.dtype
    x0, gu0, dn0 = m.xd.clone(), m.gud.clone(), m.dnd.clone()
    want = [m.run()]
    m.xd.copy_(x0 * 2), m.gud.copy_(gu0 * 0.5), m.dnd.copy_(dn0 * -1)        # powers of two: the same products, the other sign
    torch.cuda.synchronize()
    want.append(m.run())
    assert torch.equal(want[0], -want[1])
    # residual and partials of the norm in front, whose h is the tokens
    zero, res = torch.zeros(T, H + pad, dtype=dt, device="cuda"), [x0 * s for s in (1, 2)]
    stream = torch.cuda.current_stream().cuda_stream
    outs = []
    for i in range(60):
        n = i % 2
        m.gud.copy_(gu0).mul_((1.0, 0.5)[n])
        m.dnd.copy_(dn0).mul_((1.0, -1.0)[n])
        a = sf.make_block_norm([zero.data_ptr()], rows=T, cols=H, dtype=dtype, residual=res[n].data_ptr(), h=m.xd.data_ptr(), ld_x=H + pad, ld_residual=H + pad, ld_h=H + pad)
        sf.sifar_block_norm(a, stream)
        sf.sifar_experts(m.args, stream)
        outs.append(m.out[:, :H].clone())
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out, want[i % 2])


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 3.4e38])
@pytest.mark.parametrize("T,H,I", [(1, 64, 48), (2, 64, 48), (4, 40, 700), (5, 64, 48), (8, 130, 75), (12, 130, 75), (12, 64, 48), (20, 130, 75), (40, 64, 48), (40, 130, 75)])
def test_weights_that_are_not_finite_reach_the_tokens_that_chose_them_alone(dtype, bad, T, H, I):  # noqa: E741
    """Expert 2 is token 0's alone; one element of its down weights, then of its gate weights, is not finite (or, 3.4e38, rounds to no finite
    bf16 value).  All other tokens, and of token 0 what the element does not reach, are the clean weights' sums."""
    E, col = 5, 3
    choice = [[2, 0, 7]] + [[0, 1, 9], [3, 4, -1], [-1, 5, 6], [4, 1, 3]] * T
    m = Moe(T, H, I, E, 3, dtype=dtype, choice=choice[:T], seed=T + H)
    want, err = dr.experts(ref.f64(m.x), m.idx, ref.f64(m.w), ref.f64(m.gu), ref.f64(m.dn), 0, False, dtype)
    dt = DT[dtype]
    keep = m.dnd.clone()
    m.dnd.view(E, H, I)[2, col, I - 1] = bad
    got = m.run()
    assert ref.outside(got[1:], want[1:], err[1:], dt) == ""
    others = [c for c in range(H) if c != col]
    assert ref.outside(got[:1, others], want[:1, others], err[:1, others], dt) == ""
    assert bad == 3.4e38 or not bool(got[0, col].isfinite())
    m.dnd.copy_(keep)
    m.gud.view(E, 2 * I, H)[2, I // 2, 1] = bad
    assert ref.outside(m.run()[1:], want[1:], err[1:], dt) == ""


def _sum_error(n: int) -> float:
    """Error of a sum of n binary32 products, relative to the sum of their sizes.  An instruction adds 16 products and the sum so far, each cut off
    by at most 2 U of the largest; after at most 8 instructions what they have is added to the row's sum, rounded; a few more adds at the
    end, and the products' own parts (2^-25)."""
    return (34 * min(8, -(-n // 16)) + -(-n // 128) + 16) * ref.U


@gpu
@pytest.mark.parametrize("T,H,I", [(40, 32768, 8), (40, 8, 32768), (256, 8, 16384), (33, 32767, 9), (40, 9, 32767), (4, 5700, 8), (4, 8, 32768), (31, 9, 32767), (16, 1000, 2000)])
def test_binary32_sums_of_long_rows(T, H, I):  # noqa: E741
    """All products are positive, so that what each add cuts off adds up; the gate is one product, the weight 1."""
    g = torch.Generator().manual_seed(H)
    m = Moe(T, H, I, 1, 1, dtype=sf.F32, choice=[[0]] * T, weights=[[1.0]] * T)
    draw = lambda *s: (torch.rand(*s, generator=g, dtype=torch.float64) + 0.5).float()  # noqa: E731
    m.x, m.gu, m.dn = draw(T, H), draw(1, 2 * I, H), draw(1, H, I)
    m.gu[:, :I, 1:] = 0.0
    m.xd.copy_(m.x), m.gud.copy_(m.gu.reshape(-1, H)), m.dnd.copy_(m.dn.reshape(-1, I))
    x, gu, dn = ref.f64(m.x), ref.f64(m.gu)[0], ref.f64(m.dn)[0]
    gate, up = x @ gu[:I].T, x @ gu[I:].T
    a = gate / (1.0 + torch.exp(-gate)) * up
    # the gate's one product (1.2 times through the activation, which is a few steps off itself), the sum
    ea = a * (1.2 * _sum_error(1) + 24 * ref.U + _sum_error(H))
    want = a @ dn.T
    assert ref.outside(m.run(), want, ea @ dn.T + _sum_error(I) * want, torch.float32) == ""
