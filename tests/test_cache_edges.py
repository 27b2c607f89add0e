"""The paged cache and its attention at the ends of what their calls allow."""
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import test_cache_append as append
from tests.decode_ref import DT

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_padding_among_tokens_that_follow_at_once(dtype, interleaved):
    """Whole pieces and many more CTAs than the GPU holds: every second token's CTA ends before its rows have come, and the next one takes
    its place in the SM's shared memory."""
    T, heads, kv, dim, page = 6000, 8, 8, 64, 16
    append._run(dtype=dtype, tokens=600, heads=heads, kv=kv, dim=dim, rotary=dim, seqs=20, interleaved=interleaved, pad=8,
                drop=[(i, ("padding", "no sequence")[i % 4 // 2]) for i in range(0, 600, 2)])
    dt = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn(T, (heads + 2 * kv) * dim, generator=g, device="cuda").to(dt)
    freq = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float().cuda()
    table = torch.randperm(-(-T // page), generator=g, device="cuda").to(torch.int32)[None].contiguous()
    at = torch.arange(T, dtype=torch.int32, device="cuda")
    real = torch.rand(T, generator=g, device="cuda") < 0.5
    seq = torch.zeros(T, dtype=torch.int32, device="cuda")

    def call(positions):
        q_out = torch.full((T, heads * dim), 5.0, dtype=dt, device="cuda")
        k, v = (torch.full((table.shape[1], page, kv, dim), 7.0, dtype=dt, device="cuda") for _ in range(2))
        p = lambda t: t.data_ptr()  # noqa: E731
        cols = rows.shape[1]
        a = sf.make_append(q=p(rows), k=p(rows[:, heads * dim:]), v=p(rows[:, (heads + kv) * dim:]), q_out=p(q_out), k_cache=p(k), v_cache=p(v), page_table=p(table),
                           sequence=p(seq), position=p(positions), inv_freq=p(freq), tokens=T, sequences=1, pages=table.shape[1], page_size=page, max_pages=table.shape[1],
                           heads=heads, kv_heads=kv, head_dim=dim, rotary_dim=dim, dtype=dtype, ld_q=cols, ld_k=cols, ld_v=cols, interleaved=interleaved)
        sf.sifar_cache_append(a, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        page_of = table[0].long()[at.long() // page]
        return q_out, k[page_of, at.long() % page], v[page_of, at.long() % page]
    every = call(at)
    some = call(torch.where(real, at, -1).to(torch.int32))
    for whole, part, fill in zip(every, some, (5.0, 7.0, 7.0)):
        assert torch.equal(part[real], whole[real]) and bool((part[~real] == fill).all())
