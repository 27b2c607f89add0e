"""A decode step as ranks run it between their all-reduces: norm, cache, attention, router, experts, and the all-reduce that sums them up;
in captured graphs, on other streams, without programmatic launches."""
import ctypes
import importlib.util
import os
import subprocess
import sys
import tempfile

import numpy as np
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import decode_ref as dr
from tests import ops_ref as ref

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_argument_blocks_lie_as_the_header_has_them(tmp_path):
    blocks = [sf.sifar_cache_append_args, sf.sifar_decode_attention_args, sf.sifar_experts_args]
    lines = "".join("P(sizeof(%s));" % b.__name__ + "".join("P(offsetof(%s, %s));" % (b.__name__, f) for f, _ in b._fields_) for b in blocks)
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include "sifar.h"\n#define P(x) printf("%zu\\n", (size_t)(x))\nint main(void) { ' + lines + " return 0; }\n")
    exe = tmp_path / "offsets"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for b in blocks:
        want += [ctypes.sizeof(b)] + [getattr(b, f).offset for f, _ in b._fields_]
    assert got == want


def test_the_header_and_the_binding_have_the_same_limits():
    text = open(os.path.join(ROOT, "include", "sifar.h")).read()
    for name in ("CACHE_MAX_HEAD_DIM", "EXPERTS_MAX_TOKENS", "EXPERTS_MAX_COLS", "ACT_SILU", "ACT_GELU"):
        assert f"SIFAR_{name} = {getattr(sf, name)}" in text


class Step:
    """P ranks' decode step for S users on fixed buffers: every rank has its heads and its experts."""

    def __init__(self, P=2, S=5, H=512, heads=4, kv=2, dim=64, E=8, k=3, inter=128, seed=0, lengths=None, page=16):
        g = torch.Generator().manual_seed(seed)
        bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
        p = lambda t: t.data_ptr()  # noqa: E731
        self.P, self.S, self.H, self.heads, self.kv, self.dim, self.E, self.k = P, S, H, heads, kv, dim, E, k
        # the cache before the step: `lengths` tokens, and room for one more
        self.lengths = lengths or [37, 0, 130, 16, 1][:S]
        self.caches = [dr.Cache(self.lengths, page=page, kv=kv, dim=dim, seed=seed + 10 + r, room=1, fill=0.0) for r in range(P)]
        self.n = torch.tensor([n + 1 for n in self.lengths], dtype=torch.int32, device="cuda")
        self.position = (self.n - 1).contiguous()
        self.freq = (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)).float().cuda()
        self.parts, self.res, self.w = [bf(S, H) for _ in range(P)], bf(S, H), bf(H)
        self.h, self.y = torch.zeros_like(self.res), torch.zeros_like(self.res)
        self.norm = sf.make_block_norm([p(x) for x in self.parts], rows=S, cols=H, dtype=sf.BF16, residual=p(self.res), h=p(self.h), y=p(self.y), pre_norm=1,
                                       pre_weight=p(self.w))
        cols = (heads + 2 * kv) * dim
        assert cols <= H
        self.qkv = [torch.zeros(S, cols, dtype=torch.bfloat16, device="cuda") for _ in range(P)]
        self.attn = [torch.zeros(S, heads * dim, dtype=torch.bfloat16, device="cuda") for _ in range(P)]
        self.lse = [torch.zeros(S, heads, device="cuda") for _ in range(P)]
        self.append, self.attend, self.ws = [], [], []
        for r in range(P):
            f = self.caches[r].fields()
            q = self.qkv[r]
            self.append.append(sf.make_append(q=p(q), k=p(q[:, heads * dim:]), v=p(q[:, (heads + kv) * dim:]), q_out=p(q), position=p(self.position), inv_freq=p(self.freq),
                                              tokens=S, heads=heads, rotary_dim=dim, ld_q=cols, ld_k=cols, ld_v=cols, ld_q_out=cols, **f))
            a = sf.make_attention(q=p(q), out=p(self.attn[r]), lse=p(self.lse[r]), lengths=p(self.n), heads=heads, ld_q=cols, **f)
            self.attend.append(self._room(a, sf.sifar_decode_attention_workspace(a)))
        # the router's logits are some of the normed values; a rank has E / P of the experts
        self.logits = torch.zeros(S, E, device="cuda")
        self.indices, self.weights = torch.zeros(S, k, dtype=torch.int32, device="cuda"), torch.zeros(S, k, device="cuda")
        self.route = sf.make_route([p(self.logits)], tokens=S, experts=E, top_k=k, dtype=sf.F32, indices=p(self.indices), weights=p(self.weights), renormalize=1)
        mine = E // P
        self.gu = [(bf(mine, 2 * inter, H).float() / H ** 0.5).to(torch.bfloat16) for _ in range(P)]
        self.dn = [(bf(mine, H, inter).float() / inter ** 0.5).to(torch.bfloat16) for _ in range(P)]
        self.partial = [torch.zeros(S, H, dtype=torch.bfloat16, device="cuda") for _ in range(P)]
        self.experts = []
        for r in range(P):
            a = sf.make_experts(x=p(self.y), indices=p(self.indices), weights=p(self.weights), gate_up=p(self.gu[r]), down=p(self.dn[r]), out=p(self.partial[r]), tokens=S,
                                hidden=H, inter=inter, experts=mine, first_expert=r * mine, top_k=k, dtype=sf.BF16)
            self.experts.append(self._room(a, sf.sifar_experts_workspace(a)))
        self.h2, self.y2 = torch.zeros_like(self.res), torch.zeros_like(self.res)
        self.last = sf.make_block_norm([p(x) for x in self.partial], rows=S, cols=H, dtype=sf.BF16, residual=p(self.h), h=p(self.h2), y=p(self.y2), pre_norm=1,
                                       pre_weight=p(self.w))

    def _room(self, a, size):
        self.ws.append(torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda"))
        a.workspace, a.workspace_bytes = self.ws[-1].data_ptr(), size
        return a

    def run(self):
        s = torch.cuda.current_stream().cuda_stream
        sf.sifar_block_norm(self.norm, s)
        for r in range(self.P):
            # a projection that takes columns as they are: no library product, whose workspace two graphs would share
            self.qkv[r].copy_(self.y[:, : self.qkv[r].shape[1]])
            sf.sifar_cache_append(self.append[r], s)
            sf.sifar_decode_attention(self.attend[r], s)
        self.logits.copy_(self.y[:, : self.E])
        sf.sifar_route(self.route, s)
        for r in range(self.P):
            sf.sifar_experts(self.experts[r], s)
        sf.sifar_block_norm(self.last, s)

    def outputs(self):
        out = [self.h, self.y, self.indices, self.weights, self.h2, self.y2] + self.qkv + self.attn + self.lse + self.partial
        return out + [raw for c in self.caches for raw in c.raw]

    def snapshot(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()]

    def clear(self):
        for t in [self.h, self.y, self.indices, self.weights, self.h2, self.y2] + self.qkv + self.attn + self.lse + self.partial:
            t.zero_()
        for w in self.ws:
            w.fill_(0x7F)


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@gpu
@pytest.mark.parametrize("S", [5, 24])
def test_a_step_of_two_ranks_against_the_formulas(S):
    """Every operator on what the one before it left, as it stands in memory."""
    st = Step(S=S, lengths=None if S == 5 else [7 * i % 100 for i in range(S)])
    st.run()
    torch.cuda.synchronize()
    y = ref.f64(st.y)
    cols = st.qkv[0].shape[1]
    for r in range(st.P):
        x = y[:, :cols].reshape(st.S, -1, st.dim)
        turned, err = dr.turn(x[:, : st.heads + st.kv], st.position.cpu(), st.freq.cpu(), st.dim, False)
        q = st.qkv[r][:, : st.heads * st.dim].reshape(st.S, st.heads, st.dim)
        assert ref.outside(q, turned[:, : st.heads], err[:, : st.heads], torch.bfloat16) == ""
        c = st.caches[r]
        for s, n in enumerate(st.lengths):
            t = torch.arange(n + 1)
            page, slot = c.table[s].long()[t // c.page], t % c.page
            k, v = ref.f64(c.k[page.cuda(), slot.cuda()]), ref.f64(c.v[page.cuda(), slot.cuda()])
            assert ref.outside(k[n], turned[s, st.heads:], err[s, st.heads:], torch.bfloat16) == "" and torch.equal(v[n], x[s, st.heads + st.kv:])
            assert torch.equal(k[:n], ref.f64(c.keys[s])) and torch.equal(v[:n], ref.f64(c.values[s]))
            want, lse, e, el = dr.attention(ref.f64(q[s]), k, v, st.attend[r].scale, sf.BF16)
            assert ref.outside(st.attn[r][s].reshape(st.heads, st.dim), want, e, torch.bfloat16) == ""
            assert bool(((ref.f64(st.lse[r][s]) - lse).abs() <= el).all())
    idx, w = ref.route(ref.f64(st.logits), None, k=st.k, groups=1, top_groups=1, top2=False, sigmoid=False, renorm=True)
    assert torch.equal(st.indices.cpu(), idx) and float((ref.f64(st.weights) - w).abs().max()) < 64 * ref.U
    whole, both = torch.zeros(st.S, st.H, dtype=torch.float64), torch.zeros(st.S, st.H, dtype=torch.float64)
    for r in range(st.P):
        want, err = dr.experts(y, st.indices.cpu(), ref.f64(st.weights), ref.f64(st.gu[r]), ref.f64(st.dn[r]), r * st.E // st.P, False, sf.BF16)
        assert ref.outside(st.partial[r], want, err, torch.bfloat16) == ""
        whole, both = whole + want, both + err + 2.0 ** -8 * want.abs()
    # the ranks' partials are the whole layer's, and the norm behind them takes them as an all-reduce does
    every, _ = dr.experts(y, st.indices.cpu(), ref.f64(st.weights), torch.cat([ref.f64(g) for g in st.gu]), torch.cat([ref.f64(d) for d in st.dn]), 0, False, sf.BF16)
    assert torch.allclose(every, whole, rtol=1e-12, atol=1e-12)
    assert torch.equal(st.h2, (st.h.float() + (st.partial[0].float() + st.partial[1].float())).to(torch.bfloat16))


@gpu
def test_experts_write_a_ranks_buffer_of_the_all_reduce():
    """The partial straight into the context's buffer, announced, reduced."""
    st = Step()
    st.run()
    torch.cuda.synchronize()
    n = st.S * st.H
    ctx = sf.sifar_create(st.P, n, sf.BF16)
    try:
        out = torch.zeros(st.S, st.H, dtype=torch.bfloat16, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        for r in range(st.P):
            st.experts[r].out, _ = sf.sifar_rank_buffer(ctx, r, sf.DUALBUF)
            sf.sifar_experts(st.experts[r], stream)
            sf.sifar_arrive(ctx, r, sf.DUALBUF, stream)
        sf.sifar_allreduce(ctx, None, out.data_ptr(), n, sf.DUALBUF, stream)
        torch.cuda.synchronize()
        assert sf.sifar_status(ctx) == 0
        assert torch.equal(out, (st.partial[0].float() + st.partial[1].float()).to(torch.bfloat16))
    finally:
        sf.sifar_destroy(ctx)


@gpu
@pytest.mark.parametrize("S", [5, 40])
def test_steps_repeat_bit_for_bit(S):
    st = Step(S=S, lengths=None if S == 5 else [11 * i % 300 for i in range(S)])
    st.run()
    first = st.snapshot()
    for _ in range(3):
        st.clear()
        st.run()
        assert _same(first, st.snapshot())


@gpu
@pytest.mark.parametrize("S", [5, 40])
def test_captured_steps_on_two_streams_with_workspaces_of_their_own(S):
    lengths = None if S == 5 else [11 * i % 300 for i in range(S)]
    sts = [Step(S=S, lengths=lengths, seed=s) for s in (1, 2)]
    want = []
    for st in sts:
        st.run()                                             # loads the kernels before the capture
        want.append(st.snapshot())
    graphs = []
    for st in sts:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in sts]
    for _ in range(3):
        for st in sts:
            st.clear()
        torch.cuda.synchronize()
        for _ in range(2):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        assert all(_same(w, st.snapshot()) for w, st in zip(want, sts))
    # a replay reads what its buffers hold then: other lengths, positions, choices
    for st in sts:
        for x in st.parts:
            x.mul_(-0.5)
        st.n.sub_(1).clamp_(min=1)
        st.position.copy_(st.n - 1)
    torch.cuda.synchronize()
    for g in graphs:
        g.replay()
    replayed = [st.snapshot() for st in sts]
    for st, got in zip(sts, replayed):
        st.clear()
        st.run()
        assert _same(got, st.snapshot())


@gpu
def test_two_graphs_that_share_workspaces_one_after_the_other():
    st = Step()
    st.run()
    want = st.snapshot()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    st.clear()
    for _ in range(5):
        for g in graphs:
            g.replay()
    assert _same(want, st.snapshot())


@gpu
def test_two_streams_at_once_without_a_graph():
    sts = [Step(S=24, lengths=[9 * i % 200 for i in range(24)], seed=s) for s in (3, 4)]
    want = []
    for st in sts:
        st.run()
        want.append(st.snapshot())
        st.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sts]
    for _ in range(10):
        for st, s in zip(sts, streams):
            with torch.cuda.stream(s):
                st.run()
    assert all(_same(w, st.snapshot()) for w, st in zip(want, sts))


@gpu
def test_an_argument_block_is_read_before_the_call_returns():
    st = Step()
    st.run()
    want = st.snapshot()
    st.clear()
    sf.sifar_block_norm(st.norm, 0)
    st.logits.copy_(st.y[:, : st.E])
    sf.sifar_route(st.route, 0)
    torch.cuda.synchronize()
    sf.sifar_spin(2000, 0)                                   # the calls wait behind this on the device
    for r in range(st.P):
        sf.sifar_experts(st.experts[r], 0)
        st.experts[r].out = st.experts[r].x = st.experts[r].workspace = st.experts[r].gate_up = 0
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(st.partial, want[6 + 3 * st.P: 6 + 4 * st.P]))


@gpu
@pytest.mark.parametrize("S", [5, 24])
def test_without_programmatic_launches(S):
    """SIFAR_PDL=0: the plain stream order gives the same bits."""
    lengths = "None" if S == 5 else "[9 * i % 200 for i in range(24)]"
    st = Step(S=S, lengths=eval(lengths), seed=9)
    st.run()
    want = np.concatenate([t.float().cpu().numpy().reshape(-1) for t in st.snapshot()])
    code = ("import sys, numpy as np, torch; sys.path.insert(0, %r)\n"
            "from tests.test_decode_step import Step\n"
            "st = Step(S=%d, lengths=%s, seed=9); st.run()\n"
            "np.save(sys.argv[1], np.concatenate([t.float().cpu().numpy().reshape(-1) for t in st.snapshot()]))\n") % (ROOT, S, lengths)
    with tempfile.TemporaryDirectory() as d:
        path = os.path.join(d, "out.npy")
        subprocess.run([sys.executable, "-c", code, path], check=True, cwd=ROOT, env=dict(os.environ, SIFAR_PDL="0"), timeout=300)
        assert np.array_equal(np.load(path), want)


@gpu
@pytest.mark.parametrize("name", ["append-1", "append-f32-ragged", "attend-1", "attend-f32-ragged", "experts-1", "experts-f32-ragged"])
def test_the_timed_calls_are_ordered_with_the_stream_that_they_are_made_on(name):
    """The cases of perf/more_operators.py under a side stream and in a captured graph."""
    spec = importlib.util.spec_from_file_location("timed_more_operators", os.path.join(ROOT, "perf", "more_operators.py"))
    cases = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(cases)
    cases.own = True
    state = cases.prepare(next(c for c in cases.listed() if c["name"] == name), 3)
    want = {n: t.clone() for n, t in cases.run(state).items()}
    torch.cuda.synchronize()
    outs = cases.run(state)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sf.sifar_spin(2000, side.cuda_stream)                # what comes before on the stream
        if not name.startswith("append"):                    # (a cache keeps what the call does not write)
            for t in outs.values():
                t.zero_()
        cases.run(state)
    torch.cuda.synchronize()
    assert all(torch.equal(t, want[n]) for n, t in outs.items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cases.run(state)
    if not name.startswith("append"):
        for t in outs.values():
            t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, want[n]) for n, t in outs.items())
