"""The paged cache and its attention at the ends of what their calls allow."""
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref
from tests import test_cache_append as append
from tests.decode_ref import DT, Cache

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


@gpu
@pytest.mark.parametrize("dtype,dim", [(sf.BF16, 64), (sf.BF16, 63), (sf.F32, 64)])
def test_a_page_table_that_the_kernel_in_front_wrote(dtype, dim):
    """Another table for every call, written on the stream just before it: append writes, and attention reads, the pages that it names then."""
    dt, S, page, pages = DT[dtype], 4, 16, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    p = lambda t: t.data_ptr()  # noqa: E731
    table, at = torch.zeros(S, 2, dtype=torch.int32, device="cuda"), torch.full((S,), 16, dtype=torch.int32, device="cuda")
    n = at + 1
    q, out = torch.randn(S, dim, generator=g, device="cuda").to(dt), torch.empty(S, dim, dtype=dt, device="cuda")
    k, v = (torch.zeros(pages, page, 1, dim, dtype=dt, device="cuda") for _ in range(2))
    v[:] = torch.arange(pages, device="cuda").to(dt)[:, None, None, None]
    cache = dict(k_cache=p(k), v_cache=p(v), page_table=p(table), pages=pages, page_size=page, max_pages=2, sequences=S, kv_heads=1, head_dim=dim, dtype=dtype)
    a = sf.make_attention(q=p(q), out=p(out), lengths=p(n), heads=1, scale=0.0, **cache)
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = p(ws), ws.numel()
    new = torch.full((S, dim), 2.0, dtype=dt, device="cuda")
    add = sf.make_append(k=p(new), v=p(new), position=p(at), tokens=S, heads=0, rotary_dim=0, **cache)
    tables = [torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[: 2 * S].view(S, 2).contiguous() for _ in range(40)]
    stream = torch.cuda.current_stream().cuda_stream
    outs, kept = [], []
    for t in tables:
        v[:] = torch.arange(pages, device="cuda").to(dt)[:, None, None, None]
        torch.add(t, 0, out=table)
        sf.sifar_cache_append(add, stream)
        sf.sifar_decode_attention(a, stream)
        outs.append(out.clone())
        kept.append(v[t[:, 1].long(), 0, 0].clone())
    torch.cuda.synchronize()
    for t, got, last in zip(tables, outs, kept):
        assert bool((last == 2.0).all())
        # the mean of 16 tokens of the first page and the new one: whole numbers below 64, the quotient a few roundings of binary32
        want = (16.0 * t[:, 0].double().cpu() + 2.0) / 17.0
        bound = {sf.BF16: 2.0 ** -8, sf.F32: 2.0 ** -24}[dtype] * want + 2.0 ** -16 * 64
        assert bool(((got.double().cpu() - want[:, None]).abs() <= bound[:, None]).all())


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("window", [1, 10, 36, 37, 64, 100, 2 ** 31 - 1])
def test_a_window_of_a_length_that_the_table_does_not_reach(dtype, window):
    """The window is that of the length: what the table does not hold is masked, and nothing before the window takes its place."""
    told = [101, 64, 65, 1000, 2 ** 31 - 1, 73, 0, -5]
    dt, heads, dim = DT[dtype], 4, 64
    c = Cache([64] * len(told), page=16, kv=2, dim=dim, dtype=dtype)
    q = torch.randn(len(told), heads * dim, generator=torch.Generator().manual_seed(1), dtype=torch.float64).to(dt).cuda()
    out, lse = torch.empty_like(q), torch.empty(len(told), heads, device="cuda")
    n = torch.tensor(told, dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), lengths=n.data_ptr(), heads=heads, window=window, **c.fields())
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    for s, length in enumerate(told):
        seen = slice(max(0, length - window), max(0, min(length, 64)))
        want, wl, err, el = dr.attention(ref.f64(q[s]).reshape(heads, dim), ref.f64(c.keys[s][seen]), ref.f64(c.values[s][seen]), a.scale, dtype)
        assert ref.outside(out[s].reshape(heads, dim), want, err, dt) == "", length
        got = lse[s].cpu().double()
        assert bool(((got == wl) | ((got - wl).abs() <= el)).all()), length


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("dim", [64, 256, 72])
@pytest.mark.parametrize("n", [3, 70, 3000])
def test_heads_without_a_score_give_zero_whatever_the_values_hold(dtype, dim, n):
    """Scores of -infinity alone, over one strip, several, several teams; values of NaN and infinity under them.  The second key head has a score."""
    dt = DT[dtype]
    c = Cache([n, n], page=16, kv=2, dim=dim, dtype=dtype)
    t = torch.arange(n)
    for s, fill in enumerate((float("nan"), float("inf"))):
        page, slot = c.table[s].long()[t // 16].cuda(), (t % 16).cuda()
        c.k[page, slot, 0, 0] = float("-inf")
        c.v[page, slot, 0] = fill
    q = (torch.rand(2, 4 * dim, device="cuda") + 0.5).to(dt)
    out, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    lengths = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), lengths=lengths.data_ptr(), heads=4, **c.fields())
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    out = out.reshape(2, 4, dim)
    assert bool((out[:, :2] == 0).all()) and bool((lse[:, :2] == float("-inf")).all())
    for s in range(2):
        want, _, err, _ = dr.attention(ref.f64(q[s]).reshape(4, dim)[2:], ref.f64(c.keys[s][:, 1:]), ref.f64(c.values[s][:, 1:]), a.scale, dtype)
        assert ref.outside(out[s, 2:], want, err, dt) == ""


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("n", [20, 3000])
def test_a_value_that_is_not_finite_stays_in_its_column(dtype, n):
    """NaN, and infinity under a weight that is not 0, reach their column of the heads that read them; binary32 keeps the infinity."""
    dt, dim = DT[dtype], 64
    c = Cache([n], page=16, kv=2, dim=dim, dtype=dtype)
    where = lambda t: (int(c.table[0, t // 16]), t % 16)  # noqa: E731
    c.v[(*where(7), 0, 5)], c.v[(*where(n - 1), 0, 9)] = float("inf"), float("nan")
    q = torch.randn(1, 4 * dim, generator=torch.Generator().manual_seed(2), dtype=torch.float64).to(dt).cuda()
    out = torch.empty_like(q)
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lengths=lengths.data_ptr(), heads=4, **c.fields())
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    out = out.reshape(4, dim)
    want, _, err, _ = dr.attention(ref.f64(q).reshape(4, dim), ref.f64(c.keys[0]), ref.f64(c.values[0]), a.scale, dtype)
    keep = [d for d in range(dim) if d not in (5, 9)]
    assert ref.outside(out[:, keep], want[:, keep], err[:, keep], dt) == "" and ref.outside(out[2:], want[2:], err[2:], dt) == ""
    assert bool(out[:2, 9].isnan().all()) and not bool(out[:2, 5].isfinite().any())
    if dtype == sf.F32:
        assert bool((out[:2, 5] == float("inf")).all())
