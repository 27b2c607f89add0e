"""The operators behind an all-reduce as a layer runs them: one after the other, beside the all-reduce itself, in captured
graphs, on other streams."""
import importlib.util
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import ops_ref as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Layer:
    """A block's norms and router with their gradients on fixed buffers: P ranks, T tokens, hidden size H, E experts."""

    def __init__(self, P=8, T=16, H=4096, E=128, k=8, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        self.P, self.T, self.H, self.E, self.k = P, T, H, E, k
        self.x, self.res = [bf(T, H) for _ in range(P)], bf(T, H)
        self.w1, self.w2, self.gate = bf(H), bf(H), bf(H)
        self.z, self.h, self.y = (torch.zeros_like(self.res) for _ in range(3))
        self.stats = torch.zeros(2, T, device="cuda")
        self.bias = 0.1 * torch.randn(E, generator=g, device="cuda")
        self.logits = torch.zeros(T, E, device="cuda")
        self.indices, self.weights = torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(T, k, device="cuda")
        self.dweights = torch.randn(T, k, generator=g, device="cuda")
        self.dlogits = torch.zeros(T, E, device="cuda")
        self.dy, self.dh = [bf(T, H) for _ in range(P)], bf(T, H)
        self.dx, self.dres = torch.zeros_like(self.res), torch.zeros_like(self.res)
        self.dw1, self.dw2, self.dgate = (torch.zeros(H, device="cuda") for _ in range(3))
        p = lambda t: t.data_ptr()  # noqa: E731
        self.fwd = sf.make_block_norm([p(x) for x in self.x], rows=T, cols=H, dtype=sf.BF16, residual=p(self.res), post_norm=1, pre_norm=1,
                                      post_weight=p(self.w1), pre_weight=p(self.w2), gate=p(self.gate), z=p(self.z), h=p(self.h), y=p(self.y),
                                      stats=p(self.stats), alpha=0.9)
        self.rt = sf.make_route([p(self.logits)], tokens=T, experts=E, top_k=k, dtype=sf.F32, bias=p(self.bias), indices=p(self.indices),
                                weights=p(self.weights), groups=8, top_groups=4, group_score=sf.GROUP_TOP2, score=sf.SCORE_SIGMOID, renormalize=1)
        self.rt_back = sf.make_route_grad([p(self.logits)], tokens=T, experts=E, top_k=k, dtype=sf.F32, indices=p(self.indices),
                                          dweights=p(self.dweights), dlogits=p(self.dlogits), score=sf.SCORE_SIGMOID, renormalize=1)
        self.back = sf.make_block_norm_grad([p(x) for x in self.dy], rows=T, cols=H, dtype=sf.BF16, dh=p(self.dh), h=p(self.h), z=p(self.z),
                                            stats=p(self.stats), post_weight=p(self.w1), gate=p(self.gate), pre_weight=p(self.w2), dx=p(self.dx),
                                            dresidual=p(self.dres), dpost_weight=p(self.dw1), dpre_weight=p(self.dw2), dgate=p(self.dgate),
                                            post_norm=1, pre_norm=1, alpha=0.9)
        size = sf.sifar_block_norm_backward_workspace(self.back)
        self.ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
        self.back.workspace, self.back.workspace_bytes = p(self.ws), size

    def run(self):
        """Forward, router, and back, on torch's current stream."""
        s = torch.cuda.current_stream().cuda_stream
        sf.sifar_block_norm(self.fwd, s)
        # a router that reads E of the normed values: no library product, whose workspace two graphs would share
        self.logits.copy_(self.y[:, :self.E])
        sf.sifar_route(self.rt, s)
        sf.sifar_route_backward(self.rt_back, s)
        # the router's gradient joins that of y as one more partial
        self.dy[-1][:, :self.E].copy_(self.dlogits)
        sf.sifar_block_norm_backward(self.back, s)

    def outputs(self):
        return [self.z, self.h, self.y, self.stats, self.indices, self.weights, self.dlogits, self.dx, self.dres, self.dw1, self.dw2, self.dgate]

    def snapshot(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()]

    def clear(self):
        for t in self.outputs():
            t.zero_()
        self.ws.fill_(0x7F)


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_layer_forward_and_back_against_the_formulas():
    L = Layer()
    L.run()
    torch.cuda.synchronize()
    f = ref.f64
    opt = dict(post=1, pre=1, alpha=0.9, beta=1.0, offset=0.0, span=0)
    gate = f(L.gate)[None]
    want, err = ref.norm([f(x) for x in L.x], f(L.res), f(L.w1), gate, f(L.w2), eps=1e-6, **opt)
    for n, t in (("z", L.z), ("h", L.h), ("y", L.y)):
        assert ref.outside(t, want[n], err[n], torch.bfloat16) == "", n
    idx, w = ref.route(f(L.logits), f(L.bias), k=L.k, groups=8, top_groups=4, top2=True, sigmoid=True, renorm=True)
    assert torch.equal(L.indices.cpu(), idx) and float((f(L.weights) - w).abs().max()) < 64 * ref.U
    dl, dl_err = ref.route_grad(f(L.logits), idx, f(L.dweights), sigmoid=True, renorm=True)
    assert ref.outside(L.dlogits, dl, dl_err, torch.float32) == ""
    got, err = ref.norm_grad([f(x) for x in L.dy], f(L.dh), f(L.h), f(L.z), f(L.stats[0]), f(L.stats[1]), f(L.w1), gate, f(L.w2), **opt)
    for n, t, dt in (("dx", L.dx, torch.bfloat16), ("dres", L.dres, torch.bfloat16), ("dw1", L.dw1, torch.float32), ("dw2", L.dw2, torch.float32)):
        assert ref.outside(t, got[n], err[n], dt) == "", n
    assert ref.outside(L.dgate[None], got["dgate"], err["dgate"], torch.float32) == ""


def test_the_all_reduce_of_a_context_and_the_norm_give_the_same_sum():
    """A decode step's two ways: speculative packs and reducer, then the norm of its result; or the norm on the partials."""
    L = Layer(P=8, T=2)
    n = L.T * L.H
    ctx = sf.sifar_create(L.P, n, sf.BF16)
    try:
        z = torch.zeros(L.T, L.H, dtype=torch.bfloat16, device="cuda")
        streams = [torch.cuda.Stream() for _ in range(L.P)]
        torch.cuda.synchronize()
        main = torch.cuda.Stream()
        for r in range(L.P):
            sf.sifar_pack(ctx, r, L.x[r].data_ptr(), n, sf.SPECULATIVE, streams[r].cuda_stream)
        sf.sifar_allreduce(ctx, None, z.data_ptr(), n, sf.SPECULATIVE, main.cuda_stream)
        h = torch.zeros_like(z)
        one = sf.make_block_norm([z.data_ptr()], rows=L.T, cols=L.H, dtype=sf.BF16, residual=L.res.data_ptr(), h=h.data_ptr())
        sf.sifar_block_norm(one, main.cuda_stream)          # behind the reducer on its stream
        sf.sifar_block_norm(L.fwd, main.cuda_stream)
        torch.cuda.synchronize()
        assert sf.sifar_status(ctx) == 0
        assert torch.equal(z, L.z)
        assert torch.equal(h, (L.res.float() + z.float()).to(torch.bfloat16))
    finally:
        sf.sifar_destroy(ctx)


def test_layers_in_a_row_on_one_residual_stream():
    """h written over the residual, layer after layer, against single calls with buffers of their own."""
    T, H, P = 5, 1000, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    parts, w, stream = [[rnd(T, H) for _ in range(P)] for _ in range(6)], rnd(H), rnd(T, H)
    want, y = stream.clone(), torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    for xs in parts:
        h = torch.empty_like(want)
        sf.sifar_block_norm(sf.make_block_norm([x.data_ptr() for x in xs], rows=T, cols=H, dtype=sf.BF16, residual=want.data_ptr(), h=h.data_ptr()))
        want = h
    for xs in parts:
        sf.sifar_block_norm(sf.make_block_norm([x.data_ptr() for x in xs], rows=T, cols=H, dtype=sf.BF16, residual=stream.data_ptr(),
                                               h=stream.data_ptr(), y=y.data_ptr(), pre_norm=1, pre_weight=w.data_ptr()))
    torch.cuda.synchronize()
    assert torch.equal(stream, want)


@pytest.mark.parametrize("T,H", [(16, 4096), (3, 4099), (200, 520), (40, 20000)])
def test_calls_repeat_bit_for_bit(T, H):
    L = Layer(P=3, T=T, H=H)
    L.run()
    first = L.snapshot()
    for _ in range(3):
        L.clear()
        L.run()
        assert _same(first, L.snapshot())


def test_captured_graphs_on_two_streams_with_workspaces_of_their_own():
    Ls = [Layer(P=2, T=300, H=1032, seed=s) for s in (1, 2)]
    want = []
    for L in Ls:
        L.run()                                              # loads the kernels before the capture
        want.append(L.snapshot())
    graphs = []
    for L in Ls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.run()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in Ls]
    for rep in range(3):
        for L in Ls:
            L.clear()
        torch.cuda.synchronize()
        for _ in range(2):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        assert all(_same(w, L.snapshot()) for w, L in zip(want, Ls))
    # a replay reads what its buffers hold then
    for L in Ls:
        for x in L.x:
            x.mul_(0.5)
    torch.cuda.synchronize()
    for g in graphs:
        g.replay()
    replayed = [L.snapshot() for L in Ls]
    for L, got in zip(Ls, replayed):
        L.clear()
        L.run()
        assert _same(got, L.snapshot())


def test_two_streams_at_once_without_a_graph():
    Ls = [Layer(P=4, T=64, H=2048, seed=s) for s in (3, 4)]
    want = []
    for L in Ls:
        L.run()
        want.append(L.snapshot())
        L.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in Ls]
    for _ in range(10):
        for L, s in zip(Ls, streams):
            with torch.cuda.stream(s):
                L.run()
    assert all(_same(w, L.snapshot()) for w, L in zip(want, Ls))


def test_an_argument_block_is_read_before_the_call_returns():
    L = Layer(P=2, T=8, H=512)
    sf.sifar_block_norm(L.fwd, 0)
    want = L.snapshot()
    L.clear()
    sf.sifar_spin(2000, 0)                                   # the call waits behind this on the device
    sf.sifar_block_norm(L.fwd, 0)
    L.fwd.h = L.fwd.y = L.fwd.z = 0
    L.fwd.rows = 0
    assert _same(want, L.snapshot())


def test_more_rows_than_a_grid_has_ctas_are_refused():
    """A size that no launch can have is told before it, and nothing is left behind."""
    x = torch.zeros(64, device="cuda")
    a = sf.make_block_norm([x.data_ptr()], rows=1 << 30, cols=32768, dtype=sf.F32, h=x.data_ptr() + (1 << 50), post_norm=1)
    with pytest.raises(sf.SifarError) as e:                  # more CTAs than a grid has
        sf.sifar_block_norm(a, 0)
    assert e.value.code == sf.ERR_INVALID
    torch.cuda.synchronize()


def test_without_programmatic_launches():
    """SIFAR_PDL=0: the plain stream order gives the same bits."""
    L = Layer(P=3, T=33, H=4104, seed=9)
    L.run()
    want = np.concatenate([t.float().cpu().numpy().reshape(-1) for t in L.snapshot()])
    code = ("import sys, numpy as np, torch; sys.path.insert(0, %r)\n"
            "from tests.test_layer_ops import Layer\n"
            "L = Layer(P=3, T=33, H=4104, seed=9); L.run()\n"
            "np.save(sys.argv[1], np.concatenate([t.float().cpu().numpy().reshape(-1) for t in L.snapshot()]))\n") % ROOT
    import tempfile
    with tempfile.TemporaryDirectory() as d:
        path = os.path.join(d, "out.npy")
        subprocess.run([sys.executable, "-c", code, path], check=True, cwd=ROOT, env=dict(os.environ, SIFAR_PDL="0"), timeout=300)
        assert np.array_equal(np.load(path), want)


@pytest.mark.parametrize("name", ["norm-1", "norm-grad-64", "route-1", "route-grad-64"])
def test_the_timed_calls_are_ordered_with_the_stream_that_they_are_made_on(name):
    """The cases of perf/operators.py under a side stream and in a captured graph: the kernels' form belongs to the current
    stream as the plain form does."""
    spec = importlib.util.spec_from_file_location("timed_operators", os.path.join(ROOT, "perf", "operators.py"))
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
        for t in outs.values():
            t.zero_()
        cases.run(state)
    torch.cuda.synchronize()
    assert all(torch.equal(t, want[n]) for n, t in outs.items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cases.run(state)
    for t in outs.values():
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, want[n]) for n, t in outs.items())
