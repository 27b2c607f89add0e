"""sifar_decode_attention against its formula in 64 bits, masked places, lengths and splits of every kind, and what it refuses."""
import math

import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref
from tests.decode_ref import DT, Cache

gpu = pytest.mark.gpu
A = [0x10000000 + (i << 26) for i in range(16)]


def _args(**over):
    d = dict(q=A[0], k_cache=A[1], v_cache=A[2], page_table=A[3], lengths=A[4], out=A[5], lse=A[6], workspace=A[7], workspace_bytes=1 << 26,
             sequences=2, pages=5, page_size=4, max_pages=3, heads=4, kv_heads=2, head_dim=16, dtype=sf.BF16)
    d.update(over)
    return sf.make_attention(**d)


@pytest.mark.parametrize("over", [
    dict(dtype=2), dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(head_dim=0, scale=1.0), dict(head_dim=257), dict(scale=math.inf), dict(scale=math.nan),
    dict(page_size=0), dict(pages=1 << 31), dict(max_pages=1 << 30), dict(sequences=1 << 31), dict(ld_page_table=2), dict(q=0), dict(k_cache=0), dict(v_cache=0),
    dict(page_table=0), dict(lengths=0), dict(out=0), dict(workspace=0), dict(workspace=A[7] + 8), dict(workspace_bytes=1024), dict(ld_q=63), dict(ld_out=63),
    dict(q=A[0] + 1), dict(lse=A[6] + 2), dict(out=A[0]), dict(out=A[1]), dict(lse=A[5]), dict(workspace=A[2]), dict(workspace=A[5]), dict(lse=A[4]),
    dict(stride_token=32, stride_head=15, stride_page=128), dict(stride_token=32, stride_head=16, stride_page=127),
])
def test_attention_refuses(over):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_decode_attention(_args(**over))
    assert e.value.code == sf.ERR_INVALID and "sifar_decode_attention" in str(e.value)


def test_no_sequences_is_a_call_without_work():
    assert sf.sifar_decode_attention(_args(sequences=0, q=0, lengths=0, out=0, lse=0, workspace=0)) == sf.OK


def test_no_argument_block_is_refused():
    assert sf.lib().sifar_decode_attention(None, None) == sf.ERR_INVALID and sf.lib().sifar_decode_attention_workspace(None) == 0


def test_the_workspace_is_a_pure_function_of_the_sizes():
    size = sf.sifar_decode_attention_workspace
    one = size(_args())
    assert 0 < one < 1 << 24
    # neither the number of sequences nor their room matters
    assert one == size(_args(sequences=1000)) == size(_args(max_pages=1 << 20)) == size(_args(lengths=0, q=0))
    assert size(_args(heads=3)) == 0 and size(_args(head_dim=300)) == 0


def _run(lengths, *, dtype=sf.BF16, heads=4, kv=2, dim=64, page=16, layout="token", window=0, pad=0, off=0, seed=0, scale=None, sharp=1.0, with_lse=True,
         told=None, fill=math.nan):
    """One call; `told`: the lengths that the call is given where they are not those of the cache."""
    dt = DT[dtype]
    c = Cache(lengths, page=page, kv=kv, dim=dim, dtype=dtype, layout=layout, seed=seed, off=off, fill=fill)
    g = torch.Generator().manual_seed(seed + 1)
    S, cols = len(lengths), heads * dim
    q = (torch.randn(S, cols + pad, generator=g, dtype=torch.float64) * sharp).to(dt)
    q_store = torch.empty(S * (cols + pad) + off, dtype=dt, device="cuda")
    q_dev = q_store[off:].view(S, cols + pad)
    q_dev.copy_(q)
    out_store = torch.full((S * (cols + pad) + 64 + off,), 9.0, dtype=dt, device="cuda")
    out = out_store[off: off + S * (cols + pad)].view(S, cols + pad)
    lse = torch.full((S * heads + 8,), 9.0, device="cuda")
    n = torch.tensor(told if told is not None else lengths, dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q_dev.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr() if with_lse else 0, lengths=n.data_ptr(), heads=heads, window=window,
                          ld_q=cols + pad, ld_out=cols + pad, scale=scale, **c.fields())
    size = sf.sifar_decode_attention_workspace(a)
    ws = torch.full((size + 64,), 0x7F, dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), size
    assert sf.sifar_decode_attention(a, torch.cuda.current_stream().cuda_stream) == sf.OK
    torch.cuda.synchronize()
    scale = a.scale
    for s, length in enumerate(lengths):
        lo = max(0, length - window) if window else 0
        rows = q[s, :cols].to(torch.float64).reshape(heads, dim)
        want, want_lse, err, err_lse = dr.attention(rows, ref.f64(c.keys[s][lo:]), ref.f64(c.values[s][lo:]), scale, dtype)
        why = ref.outside(out[s, :cols].reshape(heads, dim), want, err, dt)
        assert why == "", f"sequence {s} of length {length}: {why}"
        if with_lse:
            got = lse[s * heads: (s + 1) * heads].cpu().double()
            assert bool(((got == want_lse) | ((got - want_lse).abs() <= err_lse)).all()), (s, got, want_lse)
    if pad:
        assert bool((out[:, cols:] == 9.0).all())
    assert bool((out_store[:off] == 9.0).all()) and bool((out_store[off + S * (cols + pad):] == 9.0).all())
    assert bool((lse[S * heads if with_lse else 0:] == 9.0).all()) and bool((ws[size:] == 0x7F).all())
    return out.clone(), lse


LENGTHS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200]


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (8, 1, 128), (3, 3, 128), (16, 2, 128), (16, 1, 64), (10, 1, 256), (6, 1, 256), (20, 1, 128), (40, 2, 64),
                                          (2, 2, 80), (4, 4, 33), (12, 1, 1), (9, 1, 250), (17, 1, 24)])
def test_lengths_around_every_border(dtype, heads, kv, dim):
    _run(LENGTHS, dtype=dtype, heads=heads, kv=kv, dim=dim)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("layout,off,pad", [("token", 0, 0), ("head", 0, 8), ("both", 0, 5), ("wide", 0, 3), ("token", 1, 1), ("head", 8, 0)])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 1000])
def test_layouts_pages_and_odd_starts(dtype, layout, off, pad, page):
    _run([70, 0, 133, 1, 64], dtype=dtype, heads=6, kv=3, dim=72, page=page, layout=layout, off=off, pad=pad)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 199, 200, 201, 1 << 40])
def test_windows(dtype, window):
    _run(LENGTHS, dtype=dtype, window=window, heads=4, kv=1, dim=64, page=5)


@gpu
@pytest.mark.parametrize("dtype,dim", [(sf.BF16, 128), (sf.BF16, 64), (sf.BF16, 256), (sf.F32, 128), (sf.F32, 64)])
def test_one_long_sequence_over_all_ctas(dtype, dim):
    _run([30011], dtype=dtype, heads=4, kv=1, dim=dim, sharp=3.0)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_many_sequences_of_all_lengths(dtype):
    g = torch.Generator().manual_seed(5)
    lengths = (torch.rand(333, generator=g) ** 3 * 900).int().tolist()
    _run(lengths, dtype=dtype, heads=4, kv=2, dim=64, page=16)


@gpu
def test_more_items_than_ctas_and_tiles_that_cross_them():
    _run([65] * 700, heads=4, kv=4, dim=64, page=32)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_sharp_and_flat_scores(dtype):
    _run([500, 77], dtype=dtype, sharp=30.0, heads=8, kv=2, dim=128)          # one token takes nearly all
    _run([500, 77], dtype=dtype, scale=0.0, heads=8, kv=2, dim=128)           # the mean
    _run([500, 77], dtype=dtype, scale=-0.3, heads=8, kv=2, dim=128)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_without_lse(dtype):
    _run([100, 0, 900], dtype=dtype, with_lse=False)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf])
def test_masked_places_may_hold_anything(dtype, fill):
    _run([3, 70, 0, 129], dtype=dtype, fill=fill, window=60, page=16)


@gpu
def test_lengths_beyond_the_table_and_below_zero():
    _run([64, 0, 32], told=[1000, -3, 32], page=16)
    _run([64, 0, 64], told=[2 ** 31 - 1, -2 ** 31, 65], page=16)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_pages_that_are_not_there_are_masked(dtype):
    dt = DT[dtype]
    c = Cache([90, 48, 16], page=16, kv=1, dim=64, dtype=dtype)
    c.table_dev[0, 1], c.table_dev[0, 5] = -1, c.pages                       # tokens 16 .. 31 and 80 .. 89
    c.table_dev[2, 0] = 2 ** 31 - 1                                           # nothing is left of the last sequence
    q = torch.randn(3, 4 * 64, device="cuda").to(dt)
    out, lse = torch.empty_like(q), torch.empty(3, 4, device="cuda")
    n = torch.tensor([90, 48, 16], dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), lengths=n.data_ptr(), heads=4, **c.fields())
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    keep = [list(range(16)) + list(range(32, 80)), list(range(48)), []]
    for s in range(3):
        want, wl, err, el = dr.attention(ref.f64(q[s]).reshape(4, 64), ref.f64(c.keys[s][keep[s]]), ref.f64(c.values[s][keep[s]]), a.scale, dtype)
        assert ref.outside(out[s].reshape(4, 64), want, err, dt) == ""
        got = lse[s].cpu().double()
        assert bool(((got == wl) | ((got - wl).abs() <= el)).all())


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_scores_that_are_not_finite(dtype):
    """A key of -infinity under a positive query has no weight; a head that has nothing else gives 0; NaN stays in its head."""
    dt = DT[dtype]
    c = Cache([70, 3], page=16, kv=2, dim=64, dtype=dtype)
    page0 = int(c.table[0, 0])
    c.k[page0, 5, 0, 0] = -math.inf
    c.k[page0, 6, 1, 0] = math.nan
    for t in range(3):
        c.k[int(c.table[1, 0]), t, 0, 0] = -math.inf
    q = torch.rand(2, 4 * 64, device="cuda").to(dt) + 0.5
    out, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    n = torch.tensor([70, 3], dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), lengths=n.data_ptr(), heads=4, **c.fields())
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    out = out.reshape(2, 4, 64)
    rest = [t for t in range(70) if t != 5]
    want, _, err, _ = dr.attention(ref.f64(q[0]).reshape(4, 64), ref.f64(c.keys[0][rest]), ref.f64(c.values[0][rest]), a.scale, dtype)
    assert ref.outside(out[0, :2], want[:2], err[:2], dt) == ""
    assert bool(out[0, 2:].isnan().all()) and bool(lse[0, 2:].isnan().all())
    assert bool((out[1, :2] == 0).all()) and bool((lse[1, :2] == -math.inf).all()) and bool(out[1, 2:].isfinite().all())


@gpu
@pytest.mark.parametrize("n", [5, 70, 3000])
def test_nan_in_every_key_gives_nan(n):
    c = Cache([n, n], page=16, kv=1, dim=64)
    for t in range(n):
        c.k[int(c.table[0, t // 16]), t % 16, 0, 7] = math.nan
    q = torch.ones(2, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(2, 1, device="cuda")
    lengths = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lse=lse.data_ptr(), lengths=lengths.data_ptr(), heads=1, **c.fields())
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    assert bool(out[0].isnan().all()) and bool(lse[0].isnan().all()) and bool(out[1].isfinite().all()) and bool(lse[1].isfinite().all())


@gpu
@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 2), (3, 3)])
def test_few_strips_for_many_warps(heads, kv):
    """Shares of one strip and of the places between items: whole items in a warp, in a CTA, over CTAs, at the row's end."""
    for n in (1, 16, 17, 33, 48, 64, 65, 79, 81, 113, 160, 1000, 16 * 1183, 16 * 1184, 16 * 1185):
        _run([n], heads=heads, kv=kv, dim=64, seed=n)
    for lengths in ([16, 17], [1, 1, 1], [15, 64, 1], [33] * 5, [16 * 200, 1, 16 * 300], [1] * 700):
        _run(lengths, heads=heads, kv=kv, dim=64)


@gpu
def test_a_cache_beyond_32_bits():
    pages, n = (1 << 31) // (64 * 8 * 128) + 2, 100
    k = torch.zeros(pages, 64, 8, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, math.nan)
    last = [pages - 1, pages - 2]
    x = torch.randn(2, 128, 8, 128, device="cuda").to(torch.bfloat16)
    for i, p in enumerate(last):
        k[p], v[p] = x[0, i * 64: (i + 1) * 64], x[1, i * 64: (i + 1) * 64]
    table, length = torch.tensor([last], dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    q = torch.randn(1, 1024, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    a = sf.make_attention(q=q.data_ptr(), out=out.data_ptr(), lengths=length.data_ptr(), k_cache=k.data_ptr(), v_cache=v.data_ptr(), page_table=table.data_ptr(),
                          pages=pages, page_size=64, max_pages=2, sequences=1, heads=8, kv_heads=8, head_dim=128, dtype=sf.BF16)
    ws = torch.empty(sf.sifar_decode_attention_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_decode_attention(a)
    torch.cuda.synchronize()
    want, _, err, _ = dr.attention(ref.f64(q).reshape(8, 128), ref.f64(x[0, :n]), ref.f64(x[1, :n]), a.scale, sf.BF16)
    assert ref.outside(out.reshape(8, 128), want, err, torch.bfloat16) == ""


@gpu
def test_calls_repeat_bit_for_bit_whatever_the_workspace_held():
    first, _ = _run([4000, 3, 0, 700], heads=8, kv=2, dim=128)
    for _ in range(3):
        assert torch.equal(first, _run([4000, 3, 0, 700], heads=8, kv=2, dim=128)[0])
