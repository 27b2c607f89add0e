"""sifar_block_norm and its backward pass against their formulas in 64 bits, against differences, and what they refuse."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import ops_ref as ref

DT = {sf.BF16: torch.bfloat16, sf.F32: torch.float32}
gpu = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------------
# refusals: nothing of these reaches a device, the addresses are made up
# ---------------------------------------------------------------------------------------------------------------
A = [0x10000000 + (i << 24) for i in range(24)]      # far apart


def _forward_args(**over):
    d = dict(rows=4, cols=64, dtype=sf.BF16, residual=A[8], pre_norm=1, pre_weight=A[9], h=A[10], y=A[11])
    x = over.pop("x", A[:2])
    d.update(over)
    return sf.make_block_norm(x, **d)


def _backward_args(**over):
    d = dict(rows=4, cols=64, dtype=sf.BF16, dh=A[8], h=A[9], z=A[10], stats=A[11], post_norm=1, pre_norm=1, gate=A[12],
             dx=A[13], dresidual=A[14], dpost_weight=A[15], dpre_weight=A[16], dgate=A[17], workspace=A[18],
             workspace_bytes=1 << 20)
    dy = over.pop("dy", A[:2])
    d.update(over)
    return sf.make_block_norm_grad(dy, **d)


@pytest.mark.parametrize("over,words", [
    (dict(x=[]), "1 <= P <= 8"),
    (dict(dtype=2), "dtype"),
    (dict(cols=0), "cols must be"),
    (dict(cols=sf.NORM_MAX_COLS + 1), "cols must be"),
    (dict(rows=1 << 31), "rows less than"),
    (dict(eps=-1e-6), "eps"),
    (dict(eps=float("nan")), "eps"),
    (dict(alpha=float("inf")), "finite"),
    (dict(h=0, y=0), "no output"),
    (dict(pre_norm=0), "y needs pre_norm"),
    (dict(x=[A[0], 0]), "x[1] is NULL"),
    (dict(h=A[10] + 1), "not aligned"),
    (dict(ld_h=63), "row stride of h"),
    (dict(ld_x=1 << 50), "row stride of x"),
    (dict(h=A[11]), "overlaps"),
    (dict(h=A[0]), "overlaps"),
    (dict(h=A[8] + 2), "overlaps"),                       # in place only at the same address
    (dict(h=A[8], ld_h=128), "overlaps"),                 # ... and with the same stride
    (dict(y=A[9]), "overlaps"),
    (dict(stats=A[10] + 64), "overlaps"),
    (dict(y=A[10] + 126, ld_h=128, ld_y=128), "overlaps"),
])
def test_block_norm_refuses(over, words):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_block_norm(_forward_args(**over))
    assert e.value.code == sf.ERR_INVALID and words in str(e.value)


@pytest.mark.parametrize("over,words", [
    (dict(dtype=-1), "dtype"),
    (dict(dy=[]), "1 <= P <= 8"),
    (dict(cols=0), "cols must be"),
    (dict(beta=float("nan")), "finite"),
    (dict(dx=0, dresidual=0, dpost_weight=0, dpre_weight=0, dgate=0), "no output"),
    (dict(post_norm=0), "dpost_weight needs post_norm"),
    (dict(gate=0), "dgate a gate"),
    (dict(h=0), "h is needed"),
    (dict(z=0), "z with post_norm"),
    (dict(stats=0), "stats with a norm"),
    (dict(pre_norm=0, dpre_weight=0, dh=0), "dh without pre_norm"),
    (dict(workspace=0), "workspace"),
    (dict(workspace=A[18] + 4), "workspace"),
    (dict(workspace_bytes=16), "workspace"),
    (dict(dy=[A[0], 0]), "dy[1] is NULL"),
    (dict(dx=A[8]), "overlaps"),
    (dict(dresidual=A[8] + 2), "overlaps"),
    (dict(dpost_weight=A[16]), "overlaps"),
    (dict(workspace=A[17]), "overlaps"),
    (dict(ld_dx=2), "row stride of dx"),
])
def test_block_norm_backward_refuses(over, words):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_block_norm_backward(_backward_args(**over))
    assert e.value.code == sf.ERR_INVALID and words in str(e.value)


def test_no_rows_is_a_call_without_work():
    assert sf.sifar_block_norm(_forward_args(rows=0)) == sf.OK
    assert sf.sifar_block_norm_backward(_backward_args(rows=0, dpost_weight=0, dpre_weight=0, dgate=0)) == sf.OK


def test_more_than_eight_partials_are_refused_by_the_binding():
    with pytest.raises(sf.SifarError):
        sf.make_block_norm(A[:9], rows=1, cols=8, dtype=sf.BF16)


def test_the_workspace_is_a_pure_function_of_the_sizes():
    assert sf.sifar_block_norm_backward_workspace(_backward_args(dpost_weight=0, dpre_weight=0, dgate=0)) == 0
    one = sf.sifar_block_norm_backward_workspace(_backward_args(dpost_weight=0, dgate=0))
    assert 0 < one <= 4 * 64 * 4 and sf.sifar_block_norm_backward_workspace(_backward_args()) == 4 * one
    assert sf.sifar_block_norm_backward_workspace(_backward_args(cols=sf.NORM_MAX_COLS + 1)) == 0
    assert sf.sifar_block_norm_backward_workspace(_backward_args(rows=0)) == 0
    # it does not grow with the rows
    many = [sf.sifar_block_norm_backward_workspace(_backward_args(rows=r)) for r in (1 << 12, 1 << 20, (1 << 31) - 1)]
    assert many[0] == many[1] == many[2]


def test_the_argument_blocks_lie_as_the_header_has_them(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    blocks = [sf.sifar_block_norm_args, sf.sifar_block_norm_grad_args, sf.sifar_route_args, sf.sifar_route_grad_args]
    lines = "".join("P(sizeof(%s));" % b.__name__ + "".join("P(offsetof(%s, %s));" % (b.__name__, f) for f, _ in b._fields_) for b in blocks)
    src = tmp_path / "offsets.c"
    src.write_text('#include <stdio.h>\n#include "sifar.h"\n#define P(x) printf("%zu\\n", (size_t)(x))\nint main(void) { ' + lines + " return 0; }\n")
    exe = tmp_path / "offsets"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for b in blocks:
        want += [ctypes.sizeof(b)] + [getattr(b, f).offset for f, _ in b._fields_]
    assert got == want


# ---------------------------------------------------------------------------------------------------------------
# the formulas themselves: backward against differences of the forward, in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _inputs64(rows, cols, P, seed, gates):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    return dict(xs=[rnd(rows, cols) for _ in range(P)], res=rnd(rows, cols), w1=1 + 0.2 * rnd(cols),
                gate=rnd(gates, cols), w2=1 + 0.2 * rnd(cols)), rnd


@pytest.mark.parametrize("post,pre,gated,span", [(1, 1, True, 2), (1, 0, False, 0), (0, 1, True, 0), (0, 0, True, 3), (1, 1, False, 0)])
def test_gradient_formulas_against_differences(post, pre, gated, span):
    rows, cols, P = 5, 7, 3
    gates = -(-rows // span) if span else 1
    ins, rnd = _inputs64(rows, cols, P, 7 + post + 2 * pre, gates)
    if not gated:
        ins["gate"] = None
    opt = dict(post=post, pre=pre, alpha=0.8, beta=1.3, offset=0.5, span=span)
    dh, dys = rnd(rows, cols), [rnd(rows, cols) for _ in range(P)]

    def loss(d):
        o, _ = ref.norm(d["xs"], d["res"], d["w1"], d["gate"], d["w2"], eps=1e-6, **opt)
        return (o["h"] * dh).sum() + ((o["y"] * sum(dys)).sum() if pre else 0.0)

    o, _ = ref.norm(ins["xs"], ins["res"], ins["w1"], ins["gate"], ins["w2"], eps=1e-6, **opt)
    got, _ = ref.norm_grad(dys, dh, o["h"], o["z"], o["r1"], o["r2"], ins["w1"], ins["gate"], ins["w2"], **opt)
    pairs = [("xs", "dx"), ("res", "dres")] + [("w1", "dw1")] * post + [("w2", "dw2")] * pre + [("gate", "dgate")] * gated
    for name, grad in pairs:
        v = rnd(*(ins[name][1] if name == "xs" else ins[name]).shape)
        t = 1e-6
        def moved(s):
            d = dict(ins)
            d[name] = [x + (s * t * v if i == 1 else 0) for i, x in enumerate(ins["xs"])] if name == "xs" else ins[name] + s * t * v
            return d
        diff = (loss(moved(1)) - loss(moved(-1))) / (2 * t)
        # the third derivative times t^2, and the loss's own rounding over t
        assert abs(diff - (got[grad] * v).sum()) < 1e-7 * (1 + abs(diff)), name


# ---------------------------------------------------------------------------------------------------------------
# on the GPU
# ---------------------------------------------------------------------------------------------------------------
CANARY = 1024.0


class Wide:
    """rows x cols inside rows of `ld` elements with canaries around; `shift` elements off the allocation's start."""

    def __init__(self, rows, cols, pad, dtype, shift=0, values=None):
        self.ld = cols + pad
        self.all = torch.full((shift + rows * self.ld + 16,), CANARY, dtype=dtype, device="cuda")
        self.t = self.all[shift:shift + rows * self.ld].view(rows, self.ld)[:, :cols]
        self.rows, self.cols, self.shift = rows, cols, shift
        if values is not None:
            self.t.copy_(values)

    @property
    def ptr(self):
        return self.all.data_ptr() + self.shift * self.all.element_size()

    def clean(self):
        """Nothing written outside the columns."""
        x = self.all.clone()
        x[self.shift:self.shift + self.rows * self.ld].view(self.rows, self.ld)[:, :self.cols] = CANARY
        return bool((x == CANARY).all())


def _make(rows, cols, P, dtype, seed, pad=0, shift=0, gate="none", span=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    td = DT[dtype]
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    gates = 1 if gate == "channel" else -(-rows // span) if gate == "group" else 0
    d = dict(xs=[Wide(rows, cols, pad, td, shift, scale * rnd(rows, cols)) for _ in range(P)],
             res=Wide(rows, cols, pad, td, shift, scale * rnd(rows, cols)),
             w1=(0.5 + rnd(cols)).to(td).cuda(), w2=(0.5 + rnd(cols)).to(td).cuda(),
             gate=rnd(gates, cols).to(td).cuda() if gates else None)
    return d, rnd


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _run_forward(d, rows, cols, dtype, post, pre, span, alpha, beta, eps, offset, pad, shift, residual=True, weights=True,
                 stream=0):
    out = {n: Wide(rows, cols, pad, DT[dtype], shift) for n in "zhy"[:3 if pre else 2]}
    stats = torch.full((2 * rows + 3,), CANARY, device="cuda")
    a = sf.make_block_norm([x.ptr for x in d["xs"]], rows=rows, cols=cols, dtype=dtype,
                           residual=d["res"].ptr if residual else 0, post_norm=post, pre_norm=pre,
                           post_weight=_ptr(d["w1"]) if weights else 0, pre_weight=_ptr(d["w2"]) if weights else 0,
                           gate=_ptr(d["gate"]), z=out["z"].ptr, h=out["h"].ptr, y=out["y"].ptr if pre else 0,
                           stats=stats.data_ptr(), ld_x=cols + pad, ld_residual=cols + pad, ld_z=cols + pad,
                           ld_h=cols + pad, ld_y=cols + pad, rows_per_gate=span, alpha=alpha, beta=beta, eps=eps,
                           weight_offset=offset)
    torch.cuda.synchronize()
    sf.sifar_block_norm(a, stream)
    torch.cuda.synchronize()
    return out, stats, a


def _check_forward(d, out, stats, rows, dtype, post, pre, span, alpha, beta, eps, offset, residual=True, weights=True):
    want, err = ref.norm([ref.f64(x.t) for x in d["xs"]], ref.f64(d["res"].t) if residual else None,
                         ref.f64(d["w1"]) if weights else None, ref.f64(d["gate"]), ref.f64(d["w2"]) if weights else None,
                         post=post, pre=pre, alpha=alpha, beta=beta, eps=eps, offset=offset, span=span)
    for n, w in out.items():
        assert ref.outside(w.t, want[n], err[n], DT[dtype]) == "", n
        assert w.clean(), f"wrote outside the columns of {n}"
    for i, n in enumerate(("r1", "r2")):
        assert ref.outside(stats[i * rows:(i + 1) * rows], want[n], err[n], torch.float32) == "", n
    assert bool((stats[2 * rows:] == CANARY).all())
    return want


SHAPES = [
    # rows, cols, P, pad, shift: one token and one element, ends of vectors, warps, CTAs and clusters, odd strides
    (1, 1, 1, 0, 0), (3, 7, 2, 0, 0), (1, 8, 3, 0, 0), (5, 9, 8, 7, 0), (2, 255, 4, 0, 0), (2, 256, 5, 0, 0), (3, 257, 1, 0, 0),
    (1, 4096, 8, 0, 0), (2, 4095, 8, 1, 0), (2, 4096, 3, 8, 0), (3, 4097, 2, 0, 0), (1, 4104, 8, 24, 0), (2, 8192, 4, 0, 0),
    (2, 8191, 1, 0, 0), (1, 20001, 2, 0, 0), (1, 32768, 6, 0, 0), (2, 32767, 1, 9, 0), (4, 512, 8, 0, 3), (4, 100, 7, 4, 8),
    (700, 64, 1, 0, 0), (1300, 130, 2, 2, 0), (601, 300, 1, 0, 0), (2500, 33, 1, 0, 1),
    # more rows than SMs: 64 bytes of an array per thread
    (149, 5000, 2, 0, 0), (150, 4609, 1, 7, 0), (152, 8192, 4, 0, 0), (149, 10000, 3, 0, 0), (150, 16384, 1, 8, 0), (151, 16383, 2, 0, 0),
    # rows that start at every place of a 16-byte vector, on either side of the shortest that vectors may reach over
    (9, 24, 2, 1, 1), (17, 15, 3, 0, 0), (17, 16, 1, 1, 0), (19, 8, 2, 9, 5), (40, 4097, 3, 0, 0), (33, 1023, 8, 0, 7), (21, 130, 2, 4, 2), (12, 7, 4, 1, 0),
    (5, 9001, 2, 3, 5), (160, 9003, 2, 0, 1),
]


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_forward_at_the_ends_of_every_layout(i, dtype):
    rows, cols, P, pad, shift = SHAPES[i]
    post, pre = (1, 1) if i % 4 else (i // 4 % 2, 1)
    gate, span = [("none", 0), ("channel", 0), ("group", max(1, rows // 2))][i % 3]
    opt = dict(post=post, pre=pre, span=span, alpha=0.75, beta=1.5, eps=1e-5, offset=float(i % 2))
    d, _ = _make(rows, cols, P, dtype, i, pad, shift, gate, span)
    out, stats, _ = _run_forward(d, rows, cols, dtype, pad=pad, shift=shift, **opt)
    _check_forward(d, out, stats, rows, dtype, **opt)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("post,pre,residual,weights,gate", list(itertools.product((0, 1), (0, 1), (False, True), (False, True), ("none", "group"))))
def test_forward_every_part_may_be_left_out(dtype, post, pre, residual, weights, gate):
    rows, cols = 3, 136
    opt = dict(post=post, pre=pre, span=2, alpha=1.0, beta=-0.5, eps=1e-6, offset=1.0, residual=residual, weights=weights)
    d, _ = _make(rows, cols, 2, dtype, 5, gate=gate, span=2)
    out, stats, _ = _run_forward(d, rows, cols, dtype, pad=0, shift=0, **opt)
    _check_forward(d, out, stats, rows, dtype, **opt)


@gpu
@pytest.mark.parametrize("dtype,P,cols", [(sf.BF16, 8, 4099), (sf.F32, 5, 4096), (sf.BF16, 1, 640)])
def test_the_sum_is_that_of_the_all_reduce_bit_for_bit(oracle, dtype, P, cols):
    rows = 3
    d, _ = _make(rows, cols, P, dtype, 99)
    out, _, _ = _run_forward(d, rows, cols, dtype, 1, 1, 0, 1.0, 1.0, 1e-6, 0.0, 0, 0)
    bits = lambda t: t.contiguous().cpu().view(torch.int16).numpy().view(np.uint16) if dtype == sf.BF16 else t.contiguous().cpu().numpy()  # noqa: E731
    want = oracle.allreduce([bits(x.t).reshape(-1) for x in d["xs"]], dtype)
    got = bits(out["z"].t).reshape(-1)
    assert np.array_equal(got if dtype == sf.BF16 else got.view(np.uint32), want if dtype == sf.BF16 else want.view(np.uint32))


@gpu
def test_forward_in_place_and_columns_of_one_buffer():
    """h over the residual; z and y as neighbouring columns of one wide buffer."""
    rows, cols, P = 33, 200, 2
    d, _ = _make(rows, cols, P, sf.BF16, 3)
    opt = dict(post=1, pre=1, span=0, alpha=1.0, beta=1.0, eps=1e-6, offset=0.0)
    out, _, _ = _run_forward(d, rows, cols, sf.BF16, pad=0, shift=0, **opt)
    both = torch.zeros(rows, 2 * cols, dtype=torch.bfloat16, device="cuda")
    res = d["res"].t.clone()
    a = sf.make_block_norm([x.ptr for x in d["xs"]], rows=rows, cols=cols, dtype=sf.BF16, residual=res.data_ptr(),
                           h=res.data_ptr(), z=both.data_ptr(), y=both.data_ptr() + 2 * cols, ld_z=2 * cols, ld_y=2 * cols,
                           post_norm=1, pre_norm=1, post_weight=_ptr(d["w1"]), pre_weight=_ptr(d["w2"]))
    sf.sifar_block_norm(a, 0)
    torch.cuda.synchronize()
    assert torch.equal(res, out["h"].t) and torch.equal(both[:, :cols], out["z"].t) and torch.equal(both[:, cols:], out["y"].t)


@gpu
def test_forward_zeros_infinities_and_nan_stay_in_their_rows():
    rows, cols = 5, 300
    d, _ = _make(rows, cols, 2, sf.F32, 11)
    d["xs"][0].t[1] = 0
    d["xs"][1].t[1] = 0
    d["res"].t[1] = 0
    d["xs"][0].t[2, 7] = float("nan")
    d["xs"][1].t[3, 9] = float("inf")
    out, stats, _ = _run_forward(d, rows, cols, sf.F32, 1, 1, 0, 1.0, 1.0, 1e-6, 0.0, 0, 0)
    assert bool((out["h"].t[1] == 0).all()) and bool((out["y"].t[1] == 0).all())
    assert bool(torch.isnan(out["y"].t[2]).all()) and bool(torch.isnan(out["y"].t[3, 9]))
    assert abs(float(stats[1]) - 1e3) < 1e-3 * 2                 # 1 / sqrt(eps)
    for r in (0, 4):
        want, err = ref.norm([ref.f64(x.t)[r:r + 1] for x in d["xs"]], ref.f64(d["res"].t)[r:r + 1], ref.f64(d["w1"]), None,
                             ref.f64(d["w2"]), post=1, pre=1, alpha=1.0, beta=1.0, eps=1e-6, offset=0.0, span=0)
        assert ref.outside(out["y"].t[r:r + 1], want["y"], err["y"], torch.float32) == ""


@gpu
def test_forward_offsets_beyond_32_bits():
    """Rows 2^17 elements apart: the last ones lie more than 2^32 elements behind the first."""
    rows, cols, ld = 33000, 64, 1 << 17
    x = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    v = x.view(rows, ld)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=torch.Generator().manual_seed(1)))
    h = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    a = sf.make_block_norm([x.data_ptr()], rows=rows, cols=cols, dtype=sf.BF16, ld_x=ld, h=h.data_ptr(), post_norm=1)
    sf.sifar_block_norm(a, 0)
    torch.cuda.synchronize()
    at = torch.tensor([0, 1, 32766, 32767, 32768, 32769, 32999])
    want, err = ref.norm([ref.f64(v[at.cuda()])], None, None, None, None, post=1, pre=0, alpha=1.0, beta=1.0, eps=1e-6,
                         offset=0.0, span=0)
    assert ref.outside(h[at.cuda()], want["h"], err["h"], torch.bfloat16) == ""


def _run_backward(d, rnd, fwd, rows, cols, P, dtype, post, pre, span, alpha, beta, offset, pad, shift, with_dh=True, stream=0):
    td = DT[dtype]
    out, stats, _ = fwd
    dh = Wide(rows, cols, pad, td, shift, rnd(rows, cols)) if with_dh else None
    dys = [Wide(rows, cols, pad, td, shift, rnd(rows, cols)) for _ in range(P)] if pre else []
    gates = d["gate"].shape[0] if d["gate"] is not None else 0
    res = dict(dx=Wide(rows, cols, pad, td, shift), dres=Wide(rows, cols, pad, td, shift),
               dw1=torch.full((cols + 5,), CANARY, device="cuda") if post else None,
               dw2=torch.full((cols + 5,), CANARY, device="cuda") if pre else None,
               dgate=torch.full((gates * cols + 5,), CANARY, device="cuda") if gates else None)
    a = sf.make_block_norm_grad([x.ptr for x in dys], rows=rows, cols=cols, dtype=dtype, dh=dh.ptr if dh else 0,
                                h=out["h"].ptr, z=out["z"].ptr, stats=stats.data_ptr(), post_weight=_ptr(d["w1"]),
                                gate=_ptr(d["gate"]), pre_weight=_ptr(d["w2"]), dx=res["dx"].ptr, dresidual=res["dres"].ptr,
                                dpost_weight=_ptr(res["dw1"]), dpre_weight=_ptr(res["dw2"]), dgate=_ptr(res["dgate"]),
                                ld_dy=cols + pad, ld_dh=cols + pad, ld_h=cols + pad, ld_z=cols + pad, ld_dx=cols + pad,
                                ld_dresidual=cols + pad, rows_per_gate=span, alpha=alpha, beta=beta, weight_offset=offset,
                                post_norm=post, pre_norm=pre)
    size = sf.sifar_block_norm_backward_workspace(a)
    ws = torch.full((size + 64,), 0x7F, dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), size
    torch.cuda.synchronize()
    sf.sifar_block_norm_backward(a, stream)
    torch.cuda.synchronize()
    assert bool((ws[size:] == 0x7F).all()), "wrote behind the workspace"
    res["dh"], res["dys"], res["ws"], res["args"] = dh, dys, ws, a
    return res


def _check_backward(d, res, fwd, rows, cols, dtype, post, pre, span, alpha, beta, offset):
    out, stats, _ = fwd
    td = DT[dtype]
    dh = ref.f64(res["dh"].t) if res["dh"] else None
    want, err = ref.norm_grad([ref.f64(x.t) for x in res["dys"]], dh, ref.f64(out["h"].t), ref.f64(out["z"].t),
                              ref.f64(stats[:rows]), ref.f64(stats[rows:2 * rows]), ref.f64(d["w1"]), ref.f64(d["gate"]),
                              ref.f64(d["w2"]), post=post, pre=pre, alpha=alpha, beta=beta, offset=offset, span=span)
    for n in ("dx", "dres"):
        assert ref.outside(res[n].t, want[n], err[n], td) == "", n
        assert res[n].clean(), f"wrote outside the columns of {n}"
    for n in ("dw1", "dw2", "dgate"):
        if res[n] is not None:
            k = want[n].numel()
            assert ref.outside(res[n][:k].view(want[n].shape), want[n], err[n], torch.float32) == "", n
            assert bool((res[n][k:] == CANARY).all())
    return want, err


BACK = [
    # rows, cols, P, pad, shift, gate, span
    (1, 1, 1, 0, 0, "none", 0), (2, 7, 2, 0, 0, "channel", 0), (5, 9, 8, 7, 0, "group", 2), (3, 257, 1, 0, 0, "group", 1),
    (2, 4096, 8, 0, 0, "none", 0), (3, 4095, 3, 1, 0, "channel", 0), (2, 4097, 2, 0, 0, "group", 1), (2, 8192, 4, 8, 0, "channel", 0),
    (40, 20001, 1, 0, 0, "group", 7), (19, 32768, 2, 0, 0, "group", 3), (4, 512, 8, 0, 3, "group", 4), (149, 100, 1, 4, 8, "channel", 0),
    (1500, 64, 1, 0, 0, "group", 37), (2600, 33, 2, 0, 1, "group", 1), (3000, 130, 1, 2, 0, "group", 999), (601, 300, 5, 0, 0, "channel", 0),
    (9, 24, 2, 1, 1, "channel", 0), (17, 15, 3, 0, 0, "group", 5), (17, 16, 1, 1, 0, "none", 0), (19, 8, 2, 9, 5, "channel", 0),
    (40, 4097, 3, 0, 0, "group", 7), (33, 1023, 8, 0, 7, "channel", 0), (21, 130, 2, 4, 2, "none", 0), (200, 1001, 1, 0, 0, "group", 50),
    (5, 5001, 2, 3, 3, "group", 2), (90, 4097, 1, 0, 1, "channel", 0), (4, 12345, 8, 2, 0, "group", 3), (3, 8193, 2, 0, 6, "group", 100),
    (296, 1024, 2, 0, 0, "group", 2), (297, 1032, 1, 8, 0, "group", 5), (500, 4096, 1, 0, 0, "group", 250),
]


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("i", range(len(BACK)))
def test_backward_at_the_ends_of_every_layout(i, dtype):
    rows, cols, P, pad, shift, gate, span = BACK[i]
    post, pre = [(1, 1), (0, 1), (1, 0), (1, 1), (0, 0 if gate != "none" else 1)][i % 5]
    opt = dict(post=post, pre=pre, span=span, alpha=0.75, beta=1.5, offset=float(i % 2))
    d, rnd = _make(rows, cols, P, dtype, 100 + i, pad, shift, gate, span)
    fwd = _run_forward(d, rows, cols, dtype, pad=pad, shift=shift, eps=1e-5, **opt)
    res = _run_backward(d, rnd, fwd, rows, cols, P, dtype, pad=pad, shift=shift, with_dh=(i % 3 != 1) or not pre, **opt)
    _check_backward(d, res, fwd, rows, cols, dtype, **opt)


@gpu
@pytest.mark.parametrize("post,pre", [(1, 1), (0, 1), (1, 0)])
def test_backward_against_differences_of_the_formula(post, pre):
    """The kernel's gradients along a direction against the change of the loss in 64 bits."""
    rows, cols, P = 6, 72, 2
    opt = dict(post=post, pre=pre, span=2, alpha=0.8, beta=1.3, offset=1.0)
    d, rnd = _make(rows, cols, P, sf.F32, 21, gate="group", span=2)
    fwd = _run_forward(d, rows, cols, sf.F32, pad=0, shift=0, eps=1e-5, **opt)
    res = _run_backward(d, rnd, fwd, rows, cols, P, sf.F32, pad=0, shift=0, **opt)
    dh, dy = ref.f64(res["dh"].t), sum((ref.f64(x.t) for x in res["dys"]), torch.zeros(rows, cols, dtype=torch.float64))
    ins = dict(xs=[ref.f64(x.t) for x in d["xs"]], res=ref.f64(d["res"].t), w1=ref.f64(d["w1"]), gate=ref.f64(d["gate"]), w2=ref.f64(d["w2"]))

    def loss(e):
        o, _ = ref.norm(e["xs"], e["res"], e["w1"], e["gate"], e["w2"], eps=1e-5, **opt)
        return (o["h"] * dh).sum() + ((o["y"] * dy).sum() if pre else 0.0)

    t = 1e-6
    _, err = _check_backward(d, res, fwd, rows, cols, sf.F32, **opt)
    for name, grad in [("xs", "dx"), ("res", "dres"), ("gate", "dgate")] + [("w1", "dw1")] * post + [("w2", "dw2")] * pre:
        v = rnd(*(ins["xs"][0] if name == "xs" else ins[name]).shape).double()
        def at(s):
            e = dict(ins)
            e[name] = [ins["xs"][0] + s * t * v, ins["xs"][1]] if name == "xs" else ins[name] + s * t * v
            return e
        diff = float((loss(at(1)) - loss(at(-1))) / (2 * t))
        got = ref.f64(res[grad].t if name in ("xs", "res") else res[grad][:v.numel()]).reshape(v.shape)
        # the kernel's own bound along v; h, z and the statistics it was given are binary32 roundings of the formula's
        # (48 steps cover theirs: DEPTH / 2 + 6 of each statistic, one of h and z), and the difference quotient's error
        slack = float(((err[grad] + 2.0 ** -24 * (got.abs() + got.abs().mean()) * 48) * v.abs()).sum()) + 1e-6
        assert abs(diff - float((got * v).sum())) < slack, (name, diff, slack)


@gpu
def test_backward_of_no_rows_clears_the_sums_and_touches_nothing_else():
    cols = 40
    out = torch.full((3, cols), CANARY, device="cuda")
    x = torch.full((cols,), CANARY, dtype=torch.bfloat16, device="cuda")
    a = sf.make_block_norm_grad([x.data_ptr()], rows=0, cols=cols, dtype=sf.BF16, dh=x.data_ptr(), h=x.data_ptr(), z=x.data_ptr(),
                                stats=out[2].data_ptr(), dx=out[2].data_ptr() + 80, post_norm=1, pre_norm=1,
                                dpost_weight=out[0].data_ptr(), dpre_weight=out[1].data_ptr())
    sf.sifar_block_norm_backward(a, 0)
    torch.cuda.synchronize()
    assert bool((out[:2] == 0).all()) and bool((out[2] == CANARY).all())


@gpu
def test_backward_only_what_is_asked_for_and_in_place():
    """The gradient of the residual over dh; the sums over rows alone; the same bits as with everything asked for."""
    rows, cols, P = 301, 264, 2
    opt = dict(post=1, pre=1, span=50, alpha=0.75, beta=1.5, offset=0.0)
    d, rnd = _make(rows, cols, P, sf.BF16, 31, gate="group", span=50)
    fwd = _run_forward(d, rows, cols, sf.BF16, pad=0, shift=0, eps=1e-5, **opt)
    res = _run_backward(d, rnd, fwd, rows, cols, P, sf.BF16, pad=0, shift=0, **opt)
    keep = {n: res[n].t.clone() if n in ("dx", "dres") else res[n].clone() for n in ("dx", "dres", "dw1", "dw2", "dgate")}
    a = res["args"]
    a.dx = a.dresidual = a.dpost_weight = 0
    res["dw2"].zero_(); res["dgate"].zero_()
    sf.sifar_block_norm_backward(a, 0)
    torch.cuda.synchronize()
    assert torch.equal(res["dw2"][:cols], keep["dw2"][:cols]) and torch.equal(res["dgate"][:7 * cols], keep["dgate"][:7 * cols])
    a.dpre_weight = a.dgate = a.workspace = a.workspace_bytes = 0
    a.dresidual = a.dh
    sf.sifar_block_norm_backward(a, 0)
    torch.cuda.synchronize()
    assert torch.equal(res["dh"].t, keep["dres"])


@gpu
def test_backward_offsets_beyond_32_bits():
    """Rows 2^17 elements apart: the last ones lie more than 2^32 elements behind the first."""
    rows, cols, ld = 33000, 64, 1 << 17
    x = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    v = x.view(rows, ld)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=torch.Generator().manual_seed(2)))
    stats = 0.5 + torch.rand(2, rows, device="cuda")
    dx = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    a = sf.make_block_norm_grad([x.data_ptr()], rows=rows, cols=cols, dtype=sf.BF16, dh=x.data_ptr(), h=x.data_ptr(), stats=stats.data_ptr(),
                                dx=dx.data_ptr(), ld_dy=ld, ld_dh=ld, ld_h=ld, ld_dx=ld, pre_norm=1)
    sf.sifar_block_norm_backward(a)
    torch.cuda.synchronize()
    at = torch.tensor([0, 1, 16384, 32766, 32767, 32768, 32769, 32999]).cuda()
    t = ref.f64(v[at])
    want, err = ref.norm_grad([t], t, t, None, ref.f64(stats[0][at]), ref.f64(stats[1][at]), None, None, None, post=0, pre=1, alpha=1.0,
                              beta=1.0, offset=0.0, span=0)
    assert ref.outside(dx.view(rows, ld)[at, :cols], want["dx"], err["dx"], torch.bfloat16) == ""


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_a_gate_row_for_more_rows_than_there_are(dtype):
    rows, cols = 3, 40
    opt = dict(post=1, pre=1, span=1000, alpha=1.0, beta=0.5, offset=0.0)
    d, rnd = _make(rows, cols, 2, dtype, 77, gate="group", span=1000)
    fwd = _run_forward(d, rows, cols, dtype, pad=0, shift=0, eps=1e-6, **opt)
    _check_forward(d, fwd[0], fwd[1], rows, dtype, eps=1e-6, **opt)
    res = _run_backward(d, rnd, fwd, rows, cols, 2, dtype, pad=0, shift=0, **opt)
    _check_backward(d, res, fwd, rows, cols, dtype, **opt)


@gpu
@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
def test_backward_of_no_rows_clears_the_gradient_of_a_gate_of_all_rows(dtype, alone):
    """rows_per_gate = 0 is one gate row, whose gradient over no rows is 0; with one row per 5 there is no gate row."""
    cols = 1100
    x = torch.full((cols,), 2.0, dtype=DT[dtype], device="cuda")
    for span in (0, 5):
        out = torch.full((3, cols + 8), CANARY, device="cuda")
        a = sf.make_block_norm_grad([x.data_ptr()], rows=0, cols=cols, dtype=dtype, dh=x.data_ptr(), h=x.data_ptr(), z=x.data_ptr(),
                                    stats=x.data_ptr(), gate=x.data_ptr(), post_norm=1, pre_norm=1, rows_per_gate=span,
                                    dpost_weight=0 if alone else out[0].data_ptr(), dpre_weight=0 if alone else out[1].data_ptr(),
                                    dgate=out[2].data_ptr())
        sf.sifar_block_norm_backward(a, 0)
        torch.cuda.synchronize()
        assert bool((out[:2, :cols] == (CANARY if alone else 0)).all())
        assert bool((out[2, :cols] == (0 if span == 0 else CANARY)).all()), span
        assert bool((out[:, cols:] == CANARY).all())


def test_no_rows_need_no_row_arrays():
    """An empty tensor has the address 0: a rank without tokens passes those."""
    assert sf.sifar_block_norm(_forward_args(x=[0, 0], rows=0, residual=0, h=0, y=0)) == sf.OK
    none = dict(rows=0, dh=0, h=0, z=0, stats=0, dx=0, dresidual=0, dpost_weight=0, dpre_weight=0, workspace=0, workspace_bytes=0)
    assert sf.sifar_block_norm_backward(_backward_args(dy=[0, 0], dgate=0, **none)) == sf.OK
    assert sf.sifar_block_norm_backward(_backward_args(dy=[0, 0], gate=0, dgate=0, rows_per_gate=3, **none)) == sf.OK
    # what is wrong whatever the rows stays refused
    for over in (dict(x=[]), dict(dtype=7), dict(cols=0), dict(pre_norm=0), dict(eps=-1.0)):
        with pytest.raises(sf.SifarError):
            sf.sifar_block_norm(_forward_args(rows=0, **over))
    for over in (dict(dtype=7), dict(cols=0), dict(beta=float("inf")), dict(post_norm=0), dict(pre_norm=0)):
        with pytest.raises(sf.SifarError):
            sf.sifar_block_norm_backward(_backward_args(rows=0, **over))


@gpu
def test_backward_of_no_rows_without_row_arrays_clears_the_sums():
    cols = 260
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    out = torch.full((3, cols), CANARY, device="cuda")
    a = sf.make_block_norm_grad([0, 0], rows=0, cols=cols, dtype=sf.BF16, post_norm=1, pre_norm=1, post_weight=w.data_ptr(),
                                pre_weight=w.data_ptr(), gate=w.data_ptr(), dpost_weight=out[0].data_ptr(),
                                dpre_weight=out[1].data_ptr(), dgate=out[2].data_ptr())
    sf.sifar_block_norm_backward(a, 0)
    torch.cuda.synchronize()
    assert bool((out == 0).all())


@pytest.mark.parametrize("rows", [1 << 29, (1 << 31) - 1])
def test_statistics_of_2_to_the_29_rows_and_more_are_not_refused_for_their_length(rows):
    """The overlap is what stops these calls: nothing is launched, on any machine."""
    far = [(16 + i) << 40 for i in range(8)]
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_block_norm(_forward_args(x=[far[0]], rows=rows, cols=1, residual=0, y=0, h=far[1], stats=far[1] + 64))
    assert "overlaps" in str(e.value)
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_block_norm_backward(_backward_args(dy=[far[0]], rows=rows, cols=1, dh=0, h=far[1], z=far[2], stats=far[3], gate=0, dx=far[3] + 64,
                                                    dresidual=0, dpost_weight=0, dpre_weight=0, dgate=0))
    assert "overlaps" in str(e.value)


@gpu
def test_statistics_of_more_than_2_to_the_29_rows():
    rows = (1 << 29) + 5
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(rows, generator=g, device="cuda", dtype=torch.bfloat16)
    h, stats = torch.empty_like(x), torch.empty(2, rows, device="cuda")
    sf.sifar_block_norm(sf.make_block_norm([x.data_ptr()], rows=rows, cols=1, dtype=sf.BF16, h=h.data_ptr(), stats=stats.data_ptr(), post_norm=1,
                                           pre_norm=1, eps=0.25))
    at = torch.tensor([0, 1, (1 << 28) - 1, 1 << 28, (1 << 29) - 1, 1 << 29, rows - 1]).cuda()
    want, err = ref.norm([ref.f64(x[at])[:, None]], None, None, None, None, post=1, pre=1, alpha=1.0, beta=1.0, eps=0.25, offset=0.0, span=0)
    assert ref.outside(h[at][:, None], want["h"], err["h"], torch.bfloat16) == ""
    for i, n in enumerate(("r1", "r2")):
        assert ref.outside(stats[i][at], want[n], err[n], torch.float32) == "", n
    dx = torch.empty_like(x)
    sf.sifar_block_norm_backward(sf.make_block_norm_grad([x.data_ptr()], rows=rows, cols=1, dtype=sf.BF16, h=h.data_ptr(), z=x.data_ptr(),
                                                         stats=stats.data_ptr(), dx=dx.data_ptr(), post_norm=1, pre_norm=1))
    c = lambda t: ref.f64(t[at])[:, None]  # noqa: E731
    want, err = ref.norm_grad([c(x)], None, c(h), c(x), ref.f64(stats[0][at]), ref.f64(stats[1][at]), None, None, None, post=1, pre=1, alpha=1.0,
                              beta=1.0, offset=0.0, span=0)
    assert ref.outside(dx[at][:, None], want["dx"], err["dx"], torch.bfloat16) == ""


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("cols", [264, 300, 4104])
def test_an_infinite_weight_gives_the_formula_s_infinities(cols, dtype):
    """pre_weight[0] = inf: mean(a * n2) is infinite, and so is every column's D but the weight's own, where inf - inf is NaN,
    whether or not threads of the row have no columns."""
    rows = 4
    opt = dict(post=0, pre=1, span=0, alpha=1.0, beta=1.0, offset=0.0)
    d, rnd = _make(rows, cols, 2, dtype, 63)
    fwd = _run_forward(d, rows, cols, dtype, pad=0, shift=0, eps=1e-5, **opt)
    d["w2"][0] = float("inf")
    res = _run_backward(d, rnd, fwd, rows, cols, 2, dtype, pad=0, shift=0, **opt)
    want, _ = ref.norm_grad([ref.f64(x.t) for x in res["dys"]], ref.f64(res["dh"].t), ref.f64(fwd[0]["h"].t), None, ref.f64(fwd[1][:rows]),
                            ref.f64(fwd[1][rows:2 * rows]), None, None, ref.f64(d["w2"]), **opt)
    got, want = ref.f64(res["dres"].t), want["dres"]
    assert float(torch.isinf(want[:, 1:]).double().mean()) > 0.99 and bool(torch.isnan(want[:, 0]).all())
    # NaN as well where h is exactly 0
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=1.0), want.nan_to_num(nan=1.0))


# Rows that start on 16 bytes and take a cluster of two, four and eight CTAs, more of them than there are clusters at once (74,
# 33, 15): blocks hold several rows, and gate rows end inside them.
ALIGNED = [
    # rows, cols, P, post, pre, gate, span
    (160, 8192, 1, 1, 1, "group", 7), (160, 8192, 2, 0, 1, "group", 3), (150, 4104, 4, 1, 1, "channel", 0), (150, 4104, 4, 0, 1, "group", 50),
    (150, 4104, 1, 0, 1, "none", 0), (150, 4104, 2, 1, 1, "group", 1), (231, 4608, 3, 1, 1, "group", 11), (160, 5120, 8, 1, 1, "none", 0),
    (160, 5120, 3, 0, 1, "group", 2), (149, 4104, 8, 1, 0, "group", 4), (100, 16384, 2, 1, 1, "group", 6), (70, 12288, 1, 1, 1, "channel", 0),
    (70, 9000, 4, 1, 1, "group", 9), (50, 32768, 4, 1, 1, "group", 8), (40, 20000, 1, 0, 1, "channel", 0), (33, 32000, 2, 1, 1, "none", 0),
]


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("i", range(len(ALIGNED)))
def test_backward_of_aligned_rows_in_clusters(i, dtype):
    rows, cols, P, post, pre, gate, span = ALIGNED[i]
    opt = dict(post=post, pre=pre, span=span, alpha=0.75, beta=1.5, offset=float(i % 2))
    d, rnd = _make(rows, cols, P, dtype, 300 + i, 0, 0, gate, span)
    fwd = _run_forward(d, rows, cols, dtype, pad=0, shift=0, eps=1e-5, **opt)
    res = _run_backward(d, rnd, fwd, rows, cols, P, dtype, pad=0, shift=0, with_dh=i % 3 != 1 or not pre, **opt)
    _check_backward(d, res, fwd, rows, cols, dtype, **opt)


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("rows,cols,P", [(160, 8192, 2), (150, 4097, 3), (230, 4104, 1), (400, 1001, 2), (50, 20001, 1), (900, 100, 2)])
def test_the_gradient_of_the_residual_over_dh(rows, cols, P, dtype):
    """In place, where neighbouring rows' bytes are fetched ahead and where they are not: the bits of the call with a buffer of its own."""
    opt = dict(post=1, pre=1, span=7, alpha=0.75, beta=1.5, offset=0.0)
    d, rnd = _make(rows, cols, P, dtype, 41, gate="group", span=7)
    fwd = _run_forward(d, rows, cols, dtype, pad=0, shift=0, eps=1e-5, **opt)
    res = _run_backward(d, rnd, fwd, rows, cols, P, dtype, pad=0, shift=0, **opt)
    want, dx, dgate = res["dres"].t.clone(), res["dx"].t.clone(), res["dgate"].clone()
    a = res["args"]
    a.dresidual = a.dh
    sf.sifar_block_norm_backward(a, 0)
    torch.cuda.synchronize()
    assert torch.equal(res["dh"].t, want) and res["dh"].clean()
    assert torch.equal(res["dx"].t, dx) and torch.equal(res["dgate"], dgate)
