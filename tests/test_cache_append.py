"""sifar_cache_append against its formula in 64 bits, places and rows left as they were, and what it refuses."""
import math

import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref
from tests.decode_ref import DT, Cache

gpu = pytest.mark.gpu
A = [0x10000000 + (i << 24) for i in range(16)]


def _args(**over):
    d = dict(q=A[0], k=A[1], v=A[2], q_out=A[3], k_cache=A[4], v_cache=A[6], page_table=A[8], sequence=A[9], position=A[10], inv_freq=A[11],
             tokens=3, sequences=2, pages=5, page_size=4, max_pages=3, heads=4, kv_heads=2, head_dim=16, rotary_dim=16, dtype=sf.BF16)
    d.update(over)
    return sf.make_append(**d)


@pytest.mark.parametrize("over", [
    dict(dtype=2), dict(heads=-1), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=257), dict(rotary_dim=3), dict(rotary_dim=18), dict(rotary_dim=-2),
    dict(page_size=0), dict(page_size=1 << 31), dict(pages=1 << 31), dict(max_pages=1 << 30), dict(sequences=1 << 31), dict(tokens=1 << 31),
    dict(ld_page_table=2), dict(q=0), dict(q_out=0), dict(k=0), dict(v=0), dict(k_cache=0), dict(v_cache=0), dict(page_table=0), dict(position=0),
    dict(inv_freq=0), dict(heads=0), dict(ld_q=63), dict(ld_k=31), dict(q=A[0] + 1), dict(k_cache=A[4] + 1), dict(position=A[10] + 2),
    dict(q_out=A[1]), dict(q_out=A[0] + 2), dict(q_out=A[4]), dict(k=A[4] + 64), dict(v_cache=A[4]), dict(v_cache=A[4] + 30), dict(v_cache=A[4] - 32),
    dict(position=A[6]), dict(stride_token=32, stride_head=15, stride_page=128), dict(stride_token=31, stride_head=16, stride_page=128),
    dict(stride_token=32, stride_head=16, stride_page=127), dict(stride_token=16, stride_head=63, stride_page=128), dict(stride_page=1 << 50, stride_token=32, stride_head=16),
    dict(heads=1 << 16),
])
def test_append_refuses(over):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_cache_append(_args(**over))
    assert e.value.code == sf.ERR_INVALID and "sifar_cache_append" in str(e.value)


def test_no_tokens_is_a_call_without_work():
    assert sf.sifar_cache_append(_args(tokens=0, q=0, k=0, v=0, q_out=0, position=0)) == sf.OK


def test_no_argument_block_is_refused():
    assert sf.lib().sifar_cache_append(None, None) == sf.ERR_INVALID


def _run(*, dtype, tokens, heads, kv, dim, rotary, interleaved=False, page=16, layout="token", base=10000.0, pad=0, seqs=3, far=0, in_place=False,
         off=0, seed=0, with_sequence=True, drop=()):
    """One call; checks q_out, every place of the cache and what lies beside the rows."""
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    seqs = seqs if with_sequence else tokens
    n = [far + 5 * s + (-(-tokens // seqs)) for s in range(seqs)]
    pages = -(-(max(n) + 1) // page)
    # only the last pages of the table are there: the positions are far
    used = -(-(tokens + 5 * seqs) // page) + 2
    c = Cache([page * used] * seqs, page=page, kv=kv, dim=dim, dtype=dtype, layout=layout, fill=7.0, seed=seed, off=off)
    table = torch.full((seqs, max(pages, used)), -1, dtype=torch.int32)
    table[:, max(0, pages - used): max(0, pages - used) + used] = c.table[:, :used]
    table_dev = table.cuda()
    for raw in c.raw:
        raw.fill_(7.0)
    of = torch.arange(tokens) % seqs
    at = torch.tensor([n[s] - 1 - int((of[i + 1:] == s).sum()) for i, s in enumerate(of.tolist())], dtype=torch.int32)
    sequence = of.to(torch.int32)
    for i, kind in drop:
        if kind == "padding":
            at[i] = -1
        elif kind == "no sequence":
            sequence[i] = seqs
        elif kind == "negative sequence":
            sequence[i] = -1
        elif kind == "no page":
            at[i] = table.shape[1] * page
        elif kind == "far page":
            at[i] = 2 ** 31 - 1
    cols = (heads + 2 * kv) * dim
    wide = torch.randn(tokens, cols + pad, generator=g, dtype=torch.float64).to(dt)
    store = torch.full((tokens * (cols + pad) + 8 + off,), 3.0, dtype=dt, device="cuda")
    rows = store[off: off + tokens * (cols + pad)].view(tokens, cols + pad)
    rows.copy_(wide)
    freq = (base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))).float()
    q_out = rows[:, : heads * dim] if in_place else torch.full((tokens, heads * dim + pad), 5.0, dtype=dt, device="cuda")[:, : heads * dim]
    before = q_out.clone()
    seq_dev, at_dev, freq_dev = sequence.cuda(), at.cuda(), freq.cuda()
    f = c.fields() | dict(page_table=table_dev.data_ptr(), max_pages=table.shape[1])
    es = rows.element_size()
    a = sf.make_append(q=rows.data_ptr() if heads else 0, k=rows.data_ptr() + heads * dim * es, v=rows.data_ptr() + (heads + kv) * dim * es,
                       q_out=q_out.data_ptr() if heads else 0, sequence=seq_dev.data_ptr() if with_sequence else 0, position=at_dev.data_ptr(),
                       inv_freq=freq_dev.data_ptr(), tokens=tokens, heads=heads, ld_q=cols + pad, ld_k=cols + pad, ld_v=cols + pad,
                       ld_q_out=cols + pad if in_place else heads * dim + pad, rotary_dim=rotary, interleaved=interleaved, **f)
    assert sf.sifar_cache_append(a, torch.cuda.current_stream().cuda_stream) == sf.OK
    torch.cuda.synchronize()
    x = wide[:, :cols].to(torch.float64).reshape(tokens, -1, dim)
    turned, err = dr.turn(x[:, : heads + kv], at, freq, rotary, interleaved)
    if not with_sequence:
        sequence = torch.arange(tokens, dtype=torch.int32)
    real = (at >= 0) & (sequence >= 0) & (sequence < seqs)
    got_q = q_out.cpu().reshape(tokens, heads, dim)
    assert ref.outside(got_q[real], turned[real, :heads], err[real, :heads], dt) == ""
    assert torch.equal(q_out.cpu()[~real], before.cpu()[~real])
    # the cache: every place, those that nothing was written to among them
    want_k, want_v = torch.full(c.k.shape, 7.0, dtype=torch.float64), torch.full(c.k.shape, 7.0, dtype=torch.float64)
    err_k = torch.zeros(c.k.shape, dtype=torch.float64)
    for i in range(tokens):
        p = int(at[i])
        if not real[i] or p // page >= table.shape[1]:
            continue
        j = int(table[int(sequence[i]), p // page])
        if j >= 0:
            want_k[j, p % page], err_k[j, p % page], want_v[j, p % page] = turned[i, heads:], err[i, heads:], x[i, heads + kv:]
    assert int((want_k != 7.0).any(-1).any(-1).sum()) >= min(1, int(real.sum()) - len(drop))
    assert ref.outside(c.k, want_k, err_k, dt) == ""
    assert torch.equal(ref.f64(c.v), want_v)
    if layout == "wide":
        for raw in c.raw:
            assert bool((raw[off:].view(c.pages, page, kv, dim + 3)[..., dim:] == 7.0).all())
    assert bool((store[:off] == 3.0).all()) and bool((store[off + tokens * (cols + pad):] == 3.0).all())
    # inputs are as they were
    keep = slice(heads * dim, None) if in_place else slice(0, None)
    assert torch.equal(rows.cpu()[:, keep], wide[:, keep])


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("over", [
    dict(tokens=1, heads=32, kv=8, dim=128, rotary=128, seqs=1),
    dict(tokens=1, heads=32, kv=8, dim=128, rotary=128, seqs=1, interleaved=True),
    dict(tokens=37, heads=6, kv=2, dim=64, rotary=64, page=7, pad=8, layout="head"),
    dict(tokens=37, heads=6, kv=2, dim=64, rotary=32, page=7, interleaved=True, layout="both"),
    dict(tokens=9, heads=5, kv=5, dim=80, rotary=40, page=1, pad=8),
    dict(tokens=9, heads=5, kv=5, dim=80, rotary=44, page=3, pad=1),                        # halves that are no whole vectors
    dict(tokens=9, heads=3, kv=1, dim=33, rotary=32, pad=3, interleaved=True, layout="wide"),
    dict(tokens=9, heads=3, kv=1, dim=1, rotary=0),
    dict(tokens=5, heads=2, kv=2, dim=8, rotary=8, interleaved=True),
    dict(tokens=5, heads=2, kv=1, dim=256, rotary=256, layout="wide", off=1),
    dict(tokens=5, heads=4, kv=2, dim=64, rotary=0),
    dict(tokens=4, heads=0, kv=3, dim=64, rotary=64),
    dict(tokens=300, heads=8, kv=2, dim=64, rotary=64, seqs=40),
    dict(tokens=6, heads=4, kv=2, dim=64, rotary=64, with_sequence=False),
    dict(tokens=6, heads=4, kv=2, dim=64, rotary=64, in_place=True, pad=8),
    dict(tokens=6, heads=4, kv=2, dim=66, rotary=66, in_place=True, interleaved=True),
])
def test_append(dtype, over):
    _run(dtype=dtype, **over)


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_are_turned_as_exactly_as_near_ones(interleaved):
    _run(dtype=sf.F32, tokens=7, heads=2, kv=1, dim=128, rotary=128, base=1e6, far=1_000_000, interleaved=interleaved, page=64)


@gpu
@pytest.mark.parametrize("vec", [True, False])
def test_tokens_that_lead_nowhere_are_left_out(vec):
    _run(dtype=sf.BF16, tokens=12, heads=2, kv=2, dim=64 if vec else 63, rotary=64 if vec else 62, page=5,
         drop=[(0, "padding"), (3, "no sequence"), (4, "negative sequence"), (7, "no page"), (8, "far page"), (11, "padding")])


@gpu
def test_pages_out_of_the_pool_are_not_written():
    c = Cache([16, 16], page=16, kv=1, dim=64, fill=7.0)
    for raw in c.raw:
        raw.fill_(7.0)
    c.table_dev[0, 0], c.table_dev[1, 0] = c.pages, -5
    x = torch.randn(2, 64, device="cuda").to(torch.bfloat16)
    at = torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    a = sf.make_append(k=x.data_ptr(), v=x.data_ptr(), position=at.data_ptr(), tokens=2, heads=0, rotary_dim=0, **c.fields())
    sf.sifar_cache_append(a)
    torch.cuda.synchronize()
    assert all(bool((raw == 7.0).all()) for raw in c.raw)


@gpu
def test_places_beyond_32_bits():
    """A cache of 2^31 elements and more: the last page lies behind every 32-bit offset."""
    pages = (1 << 31) // (16 * 8 * 128) + 3
    k = torch.empty(pages, 16, 8, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    k[-1], v[-1], k[0], v[0] = 0, 0, 0, 0
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda")
    at = torch.tensor([15], dtype=torch.int32, device="cuda")
    x = torch.randn(1, 1024, device="cuda").to(torch.bfloat16)
    a = sf.make_append(k=x.data_ptr(), v=x.data_ptr(), k_cache=k.data_ptr(), v_cache=v.data_ptr(), page_table=table.data_ptr(), position=at.data_ptr(),
                       tokens=1, sequences=1, pages=pages, page_size=16, max_pages=1, heads=0, kv_heads=8, head_dim=128, rotary_dim=0, dtype=sf.BF16)
    sf.sifar_cache_append(a)
    torch.cuda.synchronize()
    assert torch.equal(k[-1, 15].reshape(-1), x[0]) and torch.equal(v[-1, 15].reshape(-1), x[0])
    assert not bool(k[0].any()) and not bool(v[0].any()) and not bool(k[-1, :15].any())
