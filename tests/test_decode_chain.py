"""A decode step in which every operator reads what the one before it left: norm, cache, attention, its projection, the ranks' all-reduce and
norm, router, experts, the next all-reduce; and appends whose targets are filled with other values before each run."""
import importlib.util
import os

import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Chain:
    """P ranks' step for users with `lengths` cached tokens.  The projections are elementary: columns of the norm as they are for q, k and v, a
    rank's heads beside one another, once as they are and once negated and turned round, for the attention's partial."""

    def __init__(self, lengths, P=2, H=512, heads=4, kv=2, dim=64, E=8, k=3, inter=128, seed=0, page=16):
        g = torch.Generator().manual_seed(seed)
        bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
        zero = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        p = lambda t: t.data_ptr()  # noqa: E731
        S = len(lengths)
        self.P, self.S, self.H, self.heads, self.kv, self.dim, self.E, self.k, self.lengths = P, S, H, heads, kv, dim, E, k, lengths
        assert H == 2 * heads * dim and (heads + 2 * kv) * dim <= H
        self.caches = [dr.Cache(lengths, page=page, kv=kv, dim=dim, seed=seed + 10 + r, room=1, fill=0.0) for r in range(P)]
        self.before = [[raw.clone() for raw in c.raw] for c in self.caches]
        self.n = torch.tensor([n + 1 for n in lengths], dtype=torch.int32, device="cuda")
        self.position = (self.n - 1).contiguous()
        self.freq = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float().cuda()
        self.part, self.res, self.w = bf(S, H), bf(S, H), bf(H)
        self.h, self.y, self.h1, self.y1, self.h2, self.y2 = (zero(S, H) for _ in range(6))

        def norm(parts, res, h, y):
            return sf.make_block_norm([p(x) for x in parts], rows=S, cols=H, dtype=sf.BF16, residual=p(res), h=p(h), y=p(y), pre_norm=1, pre_weight=p(self.w))
        cols = (heads + 2 * kv) * dim
        self.qkv, self.attn = [zero(S, cols) for _ in range(P)], [zero(S, heads * dim) for _ in range(P)]
        self.projected, self.partial = [zero(S, H) for _ in range(P)], [zero(S, H) for _ in range(P)]
        self.first, self.middle, self.last = norm([self.part], self.res, self.h, self.y), norm(self.projected, self.h, self.h1, self.y1), norm(self.partial, self.h1, self.h2, self.y2)
        self.append, self.attend, self.experts, self.ws = [], [], [], []
        self.logits, self.indices, self.weights = torch.zeros(S, E, device="cuda"), torch.zeros(S, k, dtype=torch.int32, device="cuda"), torch.zeros(S, k, device="cuda")
        self.route = sf.make_route([p(self.logits)], tokens=S, experts=E, top_k=k, dtype=sf.F32, indices=p(self.indices), weights=p(self.weights), renormalize=1)
        mine = E // P
        self.gu = [(bf(mine, 2 * inter, H).float() / H ** 0.5).to(torch.bfloat16) for _ in range(P)]
        self.dn = [(bf(mine, H, inter).float() / inter ** 0.5).to(torch.bfloat16) for _ in range(P)]
        for r in range(P):
            f, q = self.caches[r].fields(), self.qkv[r]
            self.append.append(sf.make_append(q=p(q), k=p(q[:, heads * dim:]), v=p(q[:, (heads + kv) * dim:]), q_out=p(q), position=p(self.position), inv_freq=p(self.freq),
                                              tokens=S, heads=heads, rotary_dim=dim, ld_q=cols, ld_k=cols, ld_v=cols, ld_q_out=cols, **f))
            self.attend.append(self._room(sf.make_attention(q=p(q), out=p(self.attn[r]), lengths=p(self.n), heads=heads, ld_q=cols, **f), sf.sifar_decode_attention_workspace))
            self.experts.append(self._room(sf.make_experts(x=p(self.y1), indices=p(self.indices), weights=p(self.weights), gate_up=p(self.gu[r]), down=p(self.dn[r]),
                                                           out=p(self.partial[r]), tokens=S, hidden=H, inter=inter, experts=mine, first_expert=r * mine, top_k=k,
                                                           dtype=sf.BF16), sf.sifar_experts_workspace))

    def _room(self, a, size):
        self.ws.append(torch.full((size(a),), 0x7F, dtype=torch.uint8, device="cuda"))
        a.workspace, a.workspace_bytes = self.ws[-1].data_ptr(), self.ws[-1].numel()
        return a

    def project(self, r, to):
        half = self.H // 2
        to[:, :half].copy_(self.attn[r])
        torch.neg(self.attn[r].flip(1), out=to[:, half:])

    def attention(self):
        s = torch.cuda.current_stream().cuda_stream
        sf.sifar_block_norm(self.first, s)
        for r in range(self.P):
            self.qkv[r].copy_(self.y[:, : self.qkv[r].shape[1]])
            if r:
                self.qkv[r].neg_()
            sf.sifar_cache_append(self.append[r], s)
            sf.sifar_decode_attention(self.attend[r], s)

    def rest(self):
        s = torch.cuda.current_stream().cuda_stream
        self.logits.copy_(self.y1[:, : self.E])
        sf.sifar_route(self.route, s)
        for r in range(self.P):
            sf.sifar_experts(self.experts[r], s)
        sf.sifar_block_norm(self.last, s)

    def run(self):
        self.attention()
        for r in range(self.P):
            self.project(r, self.projected[r])
        sf.sifar_block_norm(self.middle, torch.cuda.current_stream().cuda_stream)
        self.rest()

    def outputs(self):
        return [self.h, self.y, self.h1, self.y1, self.h2, self.y2, self.indices, self.weights] + self.qkv + self.attn + self.projected + self.partial + [
            raw for c in self.caches for raw in c.raw]

    def snapshot(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()]

    def clear(self):
        """Everything that a step writes holds other values, the caches what they held before it."""
        for t in self.outputs()[: -2 * self.P]:
            t.fill_(3)
        for c, old in zip(self.caches, self.before):
            for raw, was in zip(c.raw, old):
                raw.copy_(was)
        for w in self.ws:
            w.fill_(0x7F)
        torch.cuda.synchronize()


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


LENGTHS = {5: [37, 0, 130, 16, 1], 24: [7 * i % 100 for i in range(24)], 40: [11 * i % 300 for i in range(40)]}


@gpu
@pytest.mark.parametrize("S", [5, 24, 40])
def test_a_step_whose_parts_feed_one_another(S):
    st = Chain(LENGTHS[S])
    st.run()
    torch.cuda.synchronize()
    y, cols = ref.f64(st.y), st.qkv[0].shape[1]
    for r in range(st.P):
        x = (y[:, :cols] * (-1) ** r).reshape(S, -1, st.dim)
        turned, err = dr.turn(x[:, : st.heads + st.kv], st.position.cpu(), st.freq.cpu(), st.dim, False)
        q = st.qkv[r][:, : st.heads * st.dim].reshape(S, st.heads, st.dim)
        assert ref.outside(q, turned[:, : st.heads], err[:, : st.heads], torch.bfloat16) == ""
        c = st.caches[r]
        for s, n in enumerate(st.lengths):
            t = torch.arange(n + 1)
            page, slot = c.table[s].long()[t // c.page].cuda(), (t % c.page).cuda()
            k, v = ref.f64(c.k[page, slot]), ref.f64(c.v[page, slot])
            assert ref.outside(k[n], turned[s, st.heads:], err[s, st.heads:], torch.bfloat16) == "" and torch.equal(v[n], x[s, st.heads + st.kv:])
            want, _, e, _ = dr.attention(ref.f64(q[s]), k, v, st.attend[r].scale, sf.BF16)
            assert ref.outside(st.attn[r][s].reshape(st.heads, st.dim), want, e, torch.bfloat16) == ""
    # the attention's partials are summed up with the residual, and what the experts read is their norm
    attn = [ref.f64(a) for a in st.attn]
    z = sum(torch.cat([a, -a.flip(1)], dim=1) for a in attn)
    h1 = ref.f64(st.h) + z
    assert ref.outside(st.h1, h1, 3 * ref.U * (ref.f64(st.h).abs() + sum(torch.cat([a.abs(), a.flip(1).abs()], dim=1) for a in attn)), torch.bfloat16) == ""
    want, err = ref.norm([torch.cat([a, -a.flip(1)], dim=1) for a in attn], ref.f64(st.h), None, None, ref.f64(st.w), post=0, pre=1, alpha=1.0, beta=1.0, eps=st.middle.eps,
                         offset=st.middle.weight_offset, span=0)
    assert ref.outside(st.y1, want["y"], err["y"], torch.bfloat16) == ""
    y1 = ref.f64(st.y1)
    idx, w = ref.route(ref.f64(st.logits), None, k=st.k, groups=1, top_groups=1, top2=False, sigmoid=False, renorm=True)
    assert torch.equal(st.logits, st.y1[:, : st.E].float()) and torch.equal(st.indices.cpu(), idx) and float((ref.f64(st.weights) - w).abs().max()) < 64 * ref.U
    for r in range(st.P):
        want, err = dr.experts(y1, st.indices.cpu(), ref.f64(st.weights), ref.f64(st.gu[r]), ref.f64(st.dn[r]), r * st.E // st.P, False, sf.BF16)
        assert ref.outside(st.partial[r], want, err, torch.bfloat16) == ""
    assert torch.equal(st.h2, (st.h1.float() + (st.partial[0].float() + st.partial[1].float())).to(torch.bfloat16))
    # a step from other values in every buffer gives the same bits
    first = st.snapshot()
    for _ in range(3):
        st.clear()
        assert not _same(first, st.snapshot())
        st.run()
        assert _same(first, st.snapshot())


@gpu
@pytest.mark.parametrize("S", [5, 24])
def test_the_attentions_partials_through_the_all_reduce(S):
    """The ranks' projections go into their buffers, the library's all-reduce sums them up, the norm and the experts read its result; the
    experts' partials go the same way."""
    st = Chain(LENGTHS[S])
    st.run()
    want = st.snapshot()
    st.clear()
    n = S * st.H
    z = [torch.zeros(S, st.H, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ctx = sf.sifar_create(st.P, n, sf.BF16)
    stream = torch.cuda.current_stream().cuda_stream
    try:
        st.attention()
        for r in range(st.P):
            st.project(r, st.projected[r])
            sf.sifar_pack(ctx, r, st.projected[r].data_ptr(), n, sf.DUALBUF, stream)
        sf.sifar_allreduce(ctx, None, z[0].data_ptr(), n, sf.DUALBUF, stream)
        sf.sifar_block_norm(sf.make_block_norm([z[0].data_ptr()], rows=S, cols=st.H, dtype=sf.BF16, residual=st.h.data_ptr(), h=st.h1.data_ptr(), y=st.y1.data_ptr(), pre_norm=1,
                                               pre_weight=st.w.data_ptr()), stream)
        st.logits.copy_(st.y1[:, : st.E])
        sf.sifar_route(st.route, stream)
        for r in range(st.P):
            st.experts[r].out, _ = sf.sifar_rank_buffer(ctx, r, sf.DUALBUF)
            sf.sifar_experts(st.experts[r], stream)
            sf.sifar_arrive(ctx, r, sf.DUALBUF, stream)
        sf.sifar_allreduce(ctx, None, z[1].data_ptr(), n, sf.DUALBUF, stream)
        torch.cuda.synchronize()
        assert sf.sifar_status(ctx) == 0
    finally:
        sf.sifar_destroy(ctx)
    total = (st.projected[0].float() + st.projected[1].float()).to(torch.bfloat16)
    assert torch.equal(z[0], total) and all(torch.equal(a, b) for a, b in zip(st.projected, want[8 + 2 * st.P: 8 + 3 * st.P]))
    assert torch.equal(st.h1, (st.h.float() + z[0].float()).to(torch.bfloat16))
    got = torch.zeros(S, st.H, dtype=torch.float64)
    bound = torch.zeros_like(got)
    for r in range(st.P):
        w, e = dr.experts(ref.f64(st.y1), st.indices.cpu(), ref.f64(st.weights), ref.f64(st.gu[r]), ref.f64(st.dn[r]), r * st.E // st.P, False, sf.BF16)
        got, bound = got + w, bound + e + 2.0 ** -8 * (w.abs() + e)            # each partial is rounded
    assert ref.outside(z[1], got, bound, torch.bfloat16) == ""


@gpu
@pytest.mark.parametrize("S", [5, 40])
def test_captured_steps_write_every_buffer_and_the_caches(S):
    sts = [Chain(LENGTHS[S], seed=s) for s in (1, 2)]
    want = []
    for st in sts:
        st.run()
        want.append(st.snapshot())
    graphs, streams = [], [torch.cuda.Stream() for _ in sts]
    for st in sts:
        st.clear()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    for st, w in zip(sts, want):                             # the capture itself ran nothing
        assert not any(torch.equal(raw, x) for raw, x in zip(st.outputs()[-2 * st.P:], w[-2 * st.P:]))
    for _ in range(3):
        for st in sts:
            st.clear()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        assert all(_same(w, st.snapshot()) for w, st in zip(want, sts))
    for _ in range(3):                                       # and without a graph, both at once
        for st in sts:
            st.clear()
        for st, s in zip(sts, streams):
            with torch.cuda.stream(s):
                sf.sifar_spin(500, s.cuda_stream)
                st.run()
        assert all(_same(w, st.snapshot()) for w, st in zip(want, sts))


@gpu
@pytest.mark.parametrize("name", ["append-1", "append-f32-ragged"])
def test_timed_appends_write_what_was_filled_with_other_values(name):
    """The append cases of perf/more_operators.py on a side stream and in a captured graph, their targets filled anew before each run."""
    spec = importlib.util.spec_from_file_location("timed_more_operators", os.path.join(ROOT, "perf", "more_operators.py"))
    cases = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(cases)
    cases.own = True
    state = cases.prepare(next(c for c in cases.listed() if c["name"] == name), 3)
    names = ("q_out", "k_cache", "v_cache")
    before = {n: state[n].clone() for n in names[1:]}

    def poison():
        state["q_out"].fill_(3.0)
        for n in names[1:]:
            state[n].copy_(before[n])
        torch.cuda.synchronize()
        return {n: state[n].clone() for n in names}
    blank = poison()
    cases.run(state)
    torch.cuda.synchronize()
    want = {n: state[n].clone() for n in names}
    assert not any(torch.equal(want[n], blank[n]) for n in names)
    padding = state["position"] < 0
    assert bool((want["q_out"][padding] == 3.0).all()) and not bool((want["q_out"][~padding] == 3.0).all(1).any())
    side = torch.cuda.Stream()
    poison()
    with torch.cuda.stream(side):
        sf.sifar_spin(2000, side.cuda_stream)
        cases.run(state)
    torch.cuda.synchronize()
    assert all(torch.equal(state[n], want[n]) for n in names)
    poison()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cases.run(state)
    torch.cuda.synchronize()
    assert all(torch.equal(state[n], blank[n]) for n in names)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(state[n], want[n]) for n in names)
