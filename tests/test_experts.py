"""sifar_experts against its formula in 64 bits, choices of every kind, and what it refuses."""
import math

import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref
from tests.decode_ref import DT

gpu = pytest.mark.gpu
A = [0x10000000 + (i << 26) for i in range(16)]


def _args(**over):
    d = dict(x=A[0], indices=A[1], weights=A[2], gate_up=A[3], down=A[4], out=A[5], workspace=A[6], workspace_bytes=1 << 25, tokens=3, hidden=64, inter=32,
             experts=8, top_k=2, dtype=sf.BF16)
    d.update(over)
    return sf.make_experts(**d)


@pytest.mark.parametrize("over", [
    dict(dtype=2), dict(experts=0), dict(experts=sf.ROUTE_MAX_EXPERTS + 1), dict(top_k=0), dict(top_k=33), dict(activation=2), dict(activation=-1),
    dict(tokens=sf.EXPERTS_MAX_TOKENS + 1), dict(hidden=0), dict(hidden=sf.EXPERTS_MAX_COLS + 1), dict(inter=0), dict(inter=sf.EXPERTS_MAX_COLS + 1),
    dict(x=0), dict(indices=0), dict(weights=0), dict(gate_up=0), dict(down=0), dict(out=0), dict(workspace=0), dict(workspace=A[6] + 4), dict(workspace_bytes=64),
    dict(ld_x=63), dict(ld_gate_up=63), dict(ld_down=31), dict(ld_out=63), dict(x=A[0] + 1), dict(weights=A[2] + 2), dict(indices=A[1] + 1), dict(out=A[5] + 1),
    dict(out=A[0]), dict(out=A[3]), dict(out=A[4] + 64), dict(out=A[1]), dict(workspace=A[5]), dict(workspace=A[3]),
])
def test_experts_refuses(over):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_experts(_args(**over))
    assert e.value.code == sf.ERR_INVALID and "sifar_experts" in str(e.value)


def test_no_tokens_is_a_call_without_work():
    assert sf.sifar_experts(_args(tokens=0, x=0, indices=0, weights=0, out=0, workspace=0)) == sf.OK


def test_no_argument_block_is_refused():
    assert sf.lib().sifar_experts(None, None) == sf.ERR_INVALID and sf.lib().sifar_experts_workspace(None) == 0


def test_the_workspace_is_a_pure_function_of_the_sizes():
    size = sf.sifar_experts_workspace
    assert size(_args()) == size(_args(x=0, out=0, workspace=0)) > 0 and size(_args(tokens=0)) == 0
    assert size(_args(tokens=257)) == 0 and size(_args(inter=0)) == 0


class Moe:
    """A call on random weights; `choice`: tokens x k numbers of experts, or None for a random choice."""

    def __init__(self, T, H, I, E, k, *, dtype=sf.BF16, first=0, of=None, gelu=False, pad=0, off=0, wpad=0, choice=None, seed=0, weights=None):  # noqa: E741
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
        self.T, self.H, self.I, self.E, self.k, self.dtype, self.first, self.gelu, self.pad = T, H, I, E, k, dtype, first, gelu, pad
        of = of or E
        self.idx = torch.tensor(choice, dtype=torch.int32) if choice is not None else torch.stack([torch.randperm(of, generator=g)[:k] for _ in range(T)]).to(torch.int32)
        self.w = (torch.rand(T, k, generator=g) if weights is None else torch.as_tensor(weights, dtype=torch.float32)).clone()
        self.x = rnd(T, H).to(dt)
        self.gu, self.dn = (rnd(E, 2 * I, H) / H ** 0.5).to(dt), (rnd(E, H, I) / I ** 0.5).to(dt)

        def wide(t, cols, extra):                            # rows inside wider ones, from `off` elements on
            rows = t.reshape(-1, cols)
            store = torch.full((rows.shape[0] * (cols + extra) + off,), math.nan, dtype=dt, device="cuda")
            v = store[off:].view(rows.shape[0], cols + extra)
            v[:, :cols] = rows.cuda()
            return v
        self.xd, self.gud, self.dnd = wide(self.x, H, pad), wide(self.gu, H, wpad), wide(self.dn, I, wpad)
        self.out_store = torch.full((T * (H + pad) + off + 64,), 9.0, dtype=dt, device="cuda")
        self.out = self.out_store[off: off + T * (H + pad)].view(T, H + pad)
        self.off = off
        self.idxd, self.wd = self.idx.cuda(), self.w.cuda()
        self.args = sf.make_experts(x=self.xd.data_ptr(), indices=self.idxd.data_ptr(), weights=self.wd.data_ptr(), gate_up=self.gud.data_ptr(),
                                    down=self.dnd.data_ptr(), out=self.out.data_ptr(), tokens=T, hidden=H, inter=I, experts=E, first_expert=first, top_k=k,
                                    dtype=dtype, activation=sf.ACT_GELU if gelu else sf.ACT_SILU, ld_x=H + pad, ld_gate_up=H + wpad, ld_down=I + wpad,
                                    ld_out=H + pad)
        size = sf.sifar_experts_workspace(self.args)
        self.ws = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN, whatever is read as
        self.args.workspace, self.args.workspace_bytes = self.ws.data_ptr(), size

    def run(self):
        assert sf.sifar_experts(self.args, torch.cuda.current_stream().cuda_stream) == sf.OK
        torch.cuda.synchronize()
        return self.out[:, : self.H].clone()

    def check(self):
        got = self.run()
        want, err = dr.experts(ref.f64(self.x), self.idx, ref.f64(self.w), ref.f64(self.gu), ref.f64(self.dn), self.first, self.gelu, self.dtype)
        why = ref.outside(got, want, err, DT[self.dtype])
        assert why == "", why
        here = ((self.idx >= self.first) & (self.idx.long() < self.first + self.E)).any(1)
        assert not bool(got.cpu()[~here].any())
        assert bool((self.out[:, self.H:] == 9.0).all()) and bool((self.out_store[: self.off] == 9.0).all()) and bool((self.out_store[self.off + self.out.numel():] == 9.0).all())
        assert bool((self.ws[-64:] == 0xFF).all())
        return got


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 31, 33, 64, 65, 130, 256])
def test_tokens(dtype, T):
    Moe(T, 256, 64, 8, 2, dtype=dtype, seed=T).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [1, 6, 40])
@pytest.mark.parametrize("H,I", [(1, 1), (8, 8), (64, 16), (100, 36), (1001, 333), (33, 2000), (2048, 7), (520, 264), (4096, 24), (130, 70)])
def test_sizes(dtype, T, H, I):  # noqa: E741
    Moe(T, H, I, 5, 2, dtype=dtype, gelu=True, seed=H + I).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [3, 50])
@pytest.mark.parametrize("pad,wpad,off", [(8, 8, 0), (3, 0, 0), (0, 5, 0), (0, 0, 1), (1, 1, 3), (8, 8, 8)])
def test_strides_and_odd_starts(dtype, T, pad, wpad, off):
    Moe(T, 192, 72, 4, 2, dtype=dtype, pad=pad, wpad=wpad, off=off).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [5, 100])
def test_a_ranks_share_of_the_experts(dtype, T):
    m = Moe(T, 128, 48, 6, 4, dtype=dtype, first=10, of=24)
    m.check()
    # the shares of all ranks are the whole layer's
    assert bool(((m.idx < 10) | (m.idx >= 16)).any())


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [4, 8, 70, 200])
def test_one_expert_for_all_and_experts_for_none(dtype, T):
    Moe(T, 128, 64, 9, 1, dtype=dtype, choice=[[7]] * T).check()
    out = Moe(T, 128, 64, 9, 2, dtype=dtype, choice=[[9, -1]] * T).check()
    assert not bool(out.any())


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [3, 12])
def test_the_same_expert_twice_counts_with_both_weights(dtype, T):
    Moe(T, 128, 64, 6, 4, dtype=dtype, choice=[[2, 5, 2, (t % 6)] for t in range(T)]).check()
    Moe(T, 128, 64, 6, 3, dtype=dtype, choice=[[1, 1, 1]] * T).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [3, 12])
def test_choices_that_lead_nowhere_are_left_out(dtype, T):
    far = [-1, 6, 2 ** 31 - 1, -2 ** 31]
    m = Moe(T, 128, 64, 6, 4, dtype=dtype, choice=[[far[t % 4], t % 6, far[(t + 1) % 4], (t + 3) % 6] for t in range(T)])
    m.check()
    m = Moe(T, 128, 64, 6, 4, dtype=dtype, first=-(2 ** 31) + 1, choice=[[far[t % 4], t % 6, far[(t + 1) % 4], (t + 3) % 6] for t in range(T)])
    m.check()


@gpu
@pytest.mark.parametrize("T", [2, 20])
def test_weights_of_zero_negative_and_not_finite(T):
    m = Moe(T, 128, 64, 4, 2, choice=[[0, 1]] * T, weights=[[0.0, -2.5]] * T)
    m.check()
    w = torch.ones(T, 2)
    w[1, 0] = math.nan
    m = Moe(T, 128, 64, 4, 2, choice=[[0, 1]] * T, weights=w)
    out = m.run()
    assert bool(out[1].isnan().all()) and bool(out[[t for t in range(T) if t != 1]].isfinite().all())


@gpu
@pytest.mark.parametrize("T", [2, 20])
def test_a_token_that_is_not_finite_stays_in_its_row(T):
    m = Moe(T, 128, 64, 4, 2, choice=[[0, 1]] * T)
    want = m.run()
    m.xd[1, 3] = math.nan
    out = m.run()
    rest = [t for t in range(T) if t != 1]
    assert bool(out[1].isnan().all()) and torch.equal(out[rest], want[rest])


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_many_experts_and_many_choices(dtype):
    Moe(8, 64, 24, 1024, 32, dtype=dtype).check()
    Moe(256, 64, 24, 1024, 32, dtype=dtype).check()
    Moe(256, 64, 24, 3, 3, dtype=dtype).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [1, 8])
def test_rows_too_long_for_shared_memory(dtype, T):
    Moe(T, 32768, 16, 2, 1, dtype=dtype).check()
    Moe(T, 16, 32768, 2, 1, dtype=dtype).check()


@gpu
def test_weights_beyond_32_bits():
    """2^31 elements of gate and up rows and more: the last expert lies behind every 32-bit offset."""
    H, I, T = 4096, 8192, 2  # noqa: E741
    E = (1 << 31) // (2 * I * H) + 2
    gu = torch.zeros(E, 2 * I, H, dtype=torch.bfloat16, device="cuda")
    dn = torch.zeros(E, H, I, dtype=torch.bfloat16, device="cuda")
    gu[-1, 0, :8], gu[-1, I, :8], dn[-1, :, 0] = 1, 1, 1
    gu[0], dn[0] = math.nan, math.nan
    x = torch.ones(T, H, dtype=torch.bfloat16, device="cuda")
    idx, w = torch.full((T, 1), E - 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda")
    out = torch.empty_like(x)
    a = sf.make_experts(x=x.data_ptr(), indices=idx.data_ptr(), weights=w.data_ptr(), gate_up=gu.data_ptr(), down=dn.data_ptr(), out=out.data_ptr(), tokens=T,
                        hidden=H, inter=I, experts=E, top_k=1, dtype=sf.BF16)
    ws = torch.empty(sf.sifar_experts_workspace(a), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sf.sifar_experts(a)
    torch.cuda.synchronize()
    want = 64.0 / (1 + math.exp(-8.0))
    assert bool(((out.float() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -14)).all())


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [1, 8, 33])
def test_calls_repeat_bit_for_bit_whatever_the_workspace_held(dtype, T):
    m = Moe(T, 512, 136, 16, 4, dtype=dtype)
    first = m.run()
    for fill in (0, 0x7F, 0xFF):
        m.ws.fill_(fill)
        m.out.fill_(3.0)
        assert torch.equal(first, m.run())


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T,E,k", [(9, 4, 2), (16, 40, 3), (17, 4, 2), (20, 160, 4), (31, 40, 8), (32, 2, 2), (33, 40, 3), (100, 3, 3), (256, 200, 8)])
@pytest.mark.parametrize("H,I", [(95, 161), (520, 20), (200, 520), (64, 130)])
def test_more_tokens_of_sizes_that_are_not_whole_pieces(dtype, T, E, k, H, I):  # noqa: E741
    Moe(T, H, I, E, k, dtype=dtype, seed=T + H).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [12, 24, 60, 150])
@pytest.mark.parametrize("pad,off", [(8, 0), (1, 0), (0, 3), (5, 1)])
def test_only_the_tokens_rows_start_anywhere(dtype, T, pad, off):
    m = Moe(T, 264, 72, 12, 3, dtype=dtype, seed=T)
    store = torch.full((T * (264 + pad) + off,), math.nan, dtype=DT[dtype], device="cuda")
    x = store[off:].view(T, 264 + pad)
    x[:, :264] = m.x.cuda()
    m.args.x, m.args.ld_x = x.data_ptr(), 264 + pad
    m.check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [4, 12, 40, 200])
def test_all_tokens_of_few_units_choose_the_same(dtype, T):
    """A hot expert among others: more passes over few rows than columns of one pass."""
    Moe(T, 96, 40, 30, 3, dtype=dtype, choice=[[7, t % 30, (t * 7 + 1) % 30] for t in range(T)], seed=T).check()


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("T", [3, 20, 50])
def test_numbers_of_experts_at_the_ends_of_the_range(dtype, T):
    """A rank whose first expert is the last number that there is, and choices at the other end."""
    first, low = 2 ** 31 - 2, -2 ** 31
    m = Moe(T, 64, 24, 2, 3, dtype=dtype, first=first, choice=[[first + t % 2, low, [first, low, -1, 0][t % 4]] for t in range(T)], seed=T)
    m.check()


@gpu
@pytest.mark.parametrize("T", [5, 14, 40])
def test_binary32_values_of_every_size(T):
    """Values whose parts span the exponents: 2^-40 .. 2^40 in a token, and their products' sums."""
    m = Moe(T, 77, 33, 6, 2, dtype=sf.F32, seed=T)
    scale = torch.ldexp(torch.ones(77), torch.arange(77) % 9 * 10 - 40)
    m.x = (m.x * scale).float()
    m.xd[:, :77] = m.x.cuda()
    m.gu = (m.gu / scale).float()
    m.gud[:, :77] = m.gu.reshape(-1, 77).cuda()
    m.check()


@gpu
@pytest.mark.parametrize("T,H", [(8, 2912), (8, 2944), (16, 2848), (16, 2880), (32, 1408), (32, 1440)])
def test_the_longest_rows_that_a_few_tokens_keep_in_shared_memory(T, H):  # noqa: E741
    """binary32, next to both sides of what fits."""
    Moe(T, H, 24, 2, 2, dtype=sf.F32, seed=T).check()
