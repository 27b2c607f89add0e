"""sifar_route and its backward pass against their definitions in 64 bits, against differences, and what they refuse."""
import math

import pytest
import torch

from paper_2607_08973_b200 import binding as sf
from tests import ops_ref as ref

DT = {sf.BF16: torch.bfloat16, sf.F32: torch.float32}
gpu = pytest.mark.gpu
A = [0x10000000 + (i << 24) for i in range(16)]


def _args(**over):
    d = dict(tokens=3, experts=16, top_k=2, dtype=sf.BF16, bias=A[8], indices=A[9], weights=A[10], groups=4, top_groups=2)
    logits = over.pop("logits", A[:2])
    d.update(over)
    return sf.make_route(logits, **d)


def _grad_args(**over):
    d = dict(tokens=3, experts=16, top_k=2, dtype=sf.BF16, indices=A[9], dweights=A[10], dlogits=A[11])
    logits = over.pop("logits", A[:2])
    d.update(over)
    return sf.make_route_grad(logits, **d)


@pytest.mark.parametrize("over", [
    dict(logits=[]), dict(dtype=3), dict(experts=0), dict(experts=sf.ROUTE_MAX_EXPERTS + 1, groups=1, top_groups=1), dict(top_k=0),
    dict(top_k=17, groups=1, top_groups=1), dict(top_k=33, experts=64, groups=1, top_groups=1), dict(top_k=9), dict(groups=0), dict(groups=3),
    dict(groups=64, experts=64), dict(top_groups=0), dict(top_groups=5), dict(group_score=2), dict(score=2), dict(scale=math.inf),
    dict(tokens=1 << 31), dict(indices=0), dict(weights=0), dict(logits=[A[0], 0]), dict(weights=A[9]), dict(indices=A[0]), dict(weights=A[8]),
    dict(ld_logits=15), dict(logits=[A[0] + 1]), dict(weights=A[10] + 2),
])
def test_route_refuses(over):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_route(_args(**over))
    assert e.value.code == sf.ERR_INVALID and "sifar_route" in str(e.value)


@pytest.mark.parametrize("over", [
    dict(logits=[]), dict(dtype=3), dict(experts=0), dict(top_k=0), dict(top_k=17), dict(score=-1), dict(scale=math.nan), dict(indices=0),
    dict(dweights=0), dict(dlogits=0), dict(logits=[0]), dict(dlogits=A[0]), dict(dlogits=A[9]), dict(ld_dlogits=3), dict(dlogits=A[11] + 1),
])
def test_route_backward_refuses(over):
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_route_backward(_grad_args(**over))
    assert e.value.code == sf.ERR_INVALID and "sifar_route_backward" in str(e.value)


def test_no_tokens_is_a_call_without_work():
    assert sf.sifar_route(_args(tokens=0)) == sf.OK and sf.sifar_route_backward(_grad_args(tokens=0)) == sf.OK


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_formula_against_differences(sigmoid, renorm):
    g = torch.Generator().manual_seed(3)
    l = torch.randn(4, 9, generator=g, dtype=torch.float64) - 1.0
    dw = torch.randn(4, 3, generator=g, dtype=torch.float64)
    idx = torch.topk(l, 3, dim=1).indices
    got, _ = ref.route_grad(l, idx, dw, sigmoid=sigmoid, renorm=renorm, scale=1.7)
    s = lambda x: torch.sigmoid(x) if sigmoid else torch.softmax(x, 1)  # noqa: E731

    def loss(x):
        w = s(x).gather(1, idx)
        return (1.7 * dw * (w / w.sum(1, keepdim=True) if renorm else w)).sum()

    for _ in range(3):
        v, t = torch.randn(4, 9, generator=g, dtype=torch.float64), 1e-6
        assert abs((loss(l + t * v) - loss(l - t * v)) / (2 * t) - (got * v).sum()) < 1e-8


# ---------------------------------------------------------------------------------------------------------------
CANARY = 1024.0


def _rows(values, dtype, pad, shift=0):
    T, E = values.shape
    buf = torch.full((shift + T * (E + pad) + 8,), CANARY, dtype=DT[dtype], device="cuda")
    v = buf[shift:shift + T * (E + pad)].view(T, E + pad)[:, :E]
    v.copy_(values)
    return buf, v, buf.data_ptr() + shift * buf.element_size()


def _sum32(parts):
    acc = parts[0].float()
    for x in parts[1:]:
        acc = acc + x.float()
    return acc


def _go(parts, dtype, *, k, groups=1, top_groups=1, top2=False, sigmoid=False, renorm=False, bias=None, scale=1.0, pad=0, shift=0, stream=0):
    T, E = parts[0].shape
    ins = [_rows(p, dtype, pad, shift) for p in parts]
    idx = torch.full((T * k + 3,), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T * k + 3,), CANARY, device="cuda")
    b = None if bias is None else bias.float().cuda()
    a = sf.make_route([i[2] for i in ins], tokens=T, experts=E, top_k=k, dtype=dtype, bias=0 if b is None else b.data_ptr(),
                      indices=idx.data_ptr(), weights=w.data_ptr(), ld_logits=E + pad, scale=scale, groups=groups, top_groups=top_groups,
                      group_score=sf.GROUP_TOP2 if top2 else sf.GROUP_MAX, score=sf.SCORE_SIGMOID if sigmoid else sf.SCORE_SOFTMAX,
                      renormalize=renorm)
    torch.cuda.synchronize()
    sf.sifar_route(a, stream)
    torch.cuda.synchronize()
    assert bool((idx[T * k:] == -7).all()) and bool((w[T * k:] == CANARY).all()), "wrote behind the results"
    l = _sum32([i[1].cpu() for i in ins])
    return idx[:T * k].view(T, k).cpu(), w[:T * k].view(T, k).cpu(), l


def _check(parts, dtype, bias=None, **o):
    idx, w, l = _go(parts, dtype, bias=bias, **o)
    opt = {n: o.get(n, d) for n, d in dict(k=1, groups=1, top_groups=1, top2=False, sigmoid=False, renorm=False, scale=1.0).items()}
    want_i, want_w = ref.route(l.double(), None if bias is None else bias.float().double(), **opt)
    assert torch.equal(idx, want_i), f"{int((idx != want_i).any(1).sum())} tokens choose otherwise"
    # exp of a rounded argument (its magnitude times U), two steps of expf, the sums (each at most 45 adds of positive terms), a division, the scale
    fin = l.double().masked_fill(~torch.isfinite(l), 0.0)
    span = (fin.amax(1) - fin.amin(1)).clamp_min(fin.abs().amax(1))[:, None]
    tol = want_w.abs() * ref.U * (2 * span + 64) + 2.0 ** -148
    same = ((w.double() - want_w).abs() <= tol) | (torch.isnan(w) & torch.isnan(want_w))
    assert bool(same.all()), (w[~same][:4], want_w[~same][:4])
    return idx, w


CASES = [
    # T, E, k, groups, top_groups, P, pad
    (1, 1, 1, 1, 1, 1, 0), (2, 2, 2, 1, 1, 2, 1), (3, 31, 5, 1, 1, 3, 0), (5, 32, 32, 1, 1, 1, 0), (4, 33, 8, 3, 2, 1, 3), (7, 64, 6, 8, 3, 8, 0),
    (9, 65, 4, 5, 1, 2, 0), (6, 96, 6, 32, 4, 1, 7), (3, 128, 8, 1, 1, 8, 0), (5, 160, 10, 4, 4, 1, 0), (6, 256, 8, 8, 4, 1, 0), (4, 257, 3, 1, 1, 1, 0),
    (3, 512, 20, 16, 2, 4, 8), (2, 513, 1, 27, 26, 1, 0), (2, 1000, 32, 10, 1, 2, 0), (2, 1024, 7, 32, 31, 1, 0), (33, 12, 4, 12, 5, 1, 0),
]


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("sigmoid,renorm,biased,top2", [(False, True, False, False), (False, False, True, True), (True, True, True, True), (True, False, False, True),
                                                        (True, True, True, False), (False, True, True, False)])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_choices_and_weights(i, sigmoid, renorm, biased, top2, dtype):
    T, E, k, groups, top_groups, P, pad = CASES[i]
    g = torch.Generator().manual_seed(i)
    parts = [torch.randn(T, E, generator=g) for _ in range(P)]
    bias = 0.3 * torch.randn(E, generator=g) if biased else None
    _check(parts, dtype, bias, k=k, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, renorm=renorm, scale=2.5 if i % 2 else 1.0,
           pad=pad, shift=i % 2)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("groups,top_groups,top2", [(1, 1, False), (8, 3, False), (8, 3, True)])
def test_ties_go_to_the_lowest_index(sigmoid, biased, groups, top_groups, top2):
    g = torch.Generator().manual_seed(17)
    l = torch.randint(-1, 2, (64, 80), generator=g).float()
    bias = torch.randint(0, 2, (80,), generator=g).float() / 4 if biased else None
    _check([l], sf.F32, bias, k=9, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, renorm=True)
    _check([torch.zeros(3, 80)], sf.BF16, bias, k=9, groups=groups, top_groups=top_groups, top2=top2, sigmoid=sigmoid, renorm=False)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_values_that_binary32_would_confuse(sigmoid, biased, renorm):
    """Logits a few steps apart, saturated ones, and biases that bring unequal scores next to each other."""
    g = torch.Generator().manual_seed(5)
    l = torch.cat([12.0 + torch.randint(0, 6, (40, 96), generator=g) * 2.0 ** -20, 2.0 + torch.randint(0, 6, (40, 96), generator=g) * 2.0 ** -22,
                   -60.0 - torch.rand(8, 96, generator=g) * 60])
    bias = None
    if biased:
        s = torch.sigmoid(l[45].double()) if sigmoid else torch.softmax(l[45].double(), 0)
        bias = (0.5 - s).float()                       # the values of that token lie within a step of one another
    _check([l], sf.F32, bias, k=8, sigmoid=sigmoid, renorm=renorm)
    _check([l], sf.F32, bias, k=8, groups=8, top_groups=4, top2=True, sigmoid=sigmoid, renorm=renorm)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_closed_experts_infinities_and_nan(sigmoid, renorm, biased, groups):
    g = torch.Generator().manual_seed(8)
    E, inf, nan = 48, math.inf, math.nan
    l = torch.randn(9, E, generator=g)
    l[0] = -inf                                        # nothing is open
    l[1, 3:] = -inf                                    # fewer open than chosen
    l[2, ::2] = -inf
    l[3, 7] = nan
    l[4] = nan
    l[5] = torch.finfo(torch.float32).min              # the type's lowest value
    l[6, :40] = torch.finfo(torch.float32).min
    l[7, 5] = inf
    l[8, 11] = -inf
    bias = None
    if biased:
        bias = 0.2 * torch.randn(E, generator=g)
        bias[4], bias[30] = -inf, nan
    _check([l], sf.F32, bias, k=6, groups=groups, top_groups=max(1, groups // 2), top2=groups > 1, sigmoid=sigmoid, renorm=renorm)


@gpu
def test_many_tokens_and_wide_rows():
    """Choices of 70001 tokens, every one against a stable sort; rows that lie 2^17 elements apart beyond 32 bits."""
    g = torch.Generator(device="cuda").manual_seed(2)
    l = torch.randn(70001, 40, generator=g, device="cuda")
    idx, w, s = _go([l], sf.F32, k=4, renorm=True, pad=1)
    assert torch.equal(idx.long(), torch.sort(s, dim=1, descending=True, stable=True).indices[:, :4])
    assert bool(((w.double().sum(1) - 1).abs() < 8 * ref.U).all())
    T, E, ld = 33000, 16, 1 << 17
    x = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    v = x.view(T, ld)[:, :E]
    v.copy_(torch.randn(T, E, generator=g, device="cuda"))
    idx, w = torch.empty(T, 2, dtype=torch.int32, device="cuda"), torch.empty(T, 2, device="cuda")
    sf.sifar_route(sf.make_route([x.data_ptr()], tokens=T, experts=E, top_k=2, dtype=sf.BF16, indices=idx.data_ptr(), weights=w.data_ptr(), ld_logits=ld))
    torch.cuda.synchronize()
    assert torch.equal(idx.long(), torch.sort(v, dim=1, descending=True, stable=True).indices[:, :2])
    dw, out = torch.randn(T, 2, generator=g, device="cuda"), torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    sf.sifar_route_backward(sf.make_route_grad([x.data_ptr()], tokens=T, experts=E, top_k=2, dtype=sf.BF16, indices=idx.data_ptr(),
                                               dweights=dw.data_ptr(), dlogits=out.data_ptr(), ld_logits=ld, ld_dlogits=ld))
    torch.cuda.synchronize()
    at = torch.tensor([0, 16384, 32767, 32768, 32769, 32999]).cuda()
    want, err = ref.route_grad(ref.f64(v[at]), idx[at].cpu(), ref.f64(dw[at]), sigmoid=False, renorm=False)
    assert ref.outside(out.view(T, ld)[at, :E], want, err, torch.bfloat16) == ""


def _grad(parts, idx, dw, dtype, *, sigmoid, renorm, scale=1.0, pad=0, shift=0):
    T, E = parts[0].shape
    ins = [_rows(p, dtype, pad, shift) for p in parts]
    out = _rows(torch.full((T, E), 3.0), dtype, pad, shift)
    i, d = idx.to(torch.int32).contiguous().cuda(), dw.float().contiguous().cuda()
    a = sf.make_route_grad([x[2] for x in ins], tokens=T, experts=E, top_k=idx.shape[1], dtype=dtype, indices=i.data_ptr(), dweights=d.data_ptr(),
                           dlogits=out[2], ld_logits=E + pad, ld_dlogits=E + pad, scale=scale,
                           score=sf.SCORE_SIGMOID if sigmoid else sf.SCORE_SOFTMAX, renormalize=renorm)
    torch.cuda.synchronize()
    sf.sifar_route_backward(a)
    torch.cuda.synchronize()
    rest = out[0].clone()
    rest[shift:shift + T * (E + pad)].view(T, E + pad)[:, :E] = CANARY
    assert bool((rest == CANARY).all()), "wrote outside the experts"
    return out[1].cpu(), _sum32([x[1].cpu() for x in ins])


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_backward(i, sigmoid, renorm, dtype):
    T, E, k, _, _, P, pad = CASES[i]
    g = torch.Generator().manual_seed(50 + i)
    parts = [torch.randn(T, E, generator=g) for _ in range(P)]
    l = _sum32([p.to(DT[dtype]) for p in parts])
    idx = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :k]
    dw = torch.randn(T, k, generator=g)
    got, l = _grad(parts, idx, dw, dtype, sigmoid=sigmoid, renorm=renorm, scale=1.5, pad=pad, shift=i % 2)
    want, err = ref.route_grad(l.double(), idx, dw.double(), sigmoid=sigmoid, renorm=renorm, scale=1.5)
    assert ref.outside(got, want, err, DT[dtype]) == ""


@gpu
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_backward_of_dropped_repeated_and_closed_choices(sigmoid, renorm):
    g = torch.Generator().manual_seed(4)
    l = torch.randn(6, 40, generator=g)
    l[2, 5:] = -math.inf
    l[3] = -math.inf
    l[5] = -110.0 - torch.rand(40, generator=g) * 20        # scores that are 0 in binary32
    idx = torch.tensor([[3, 39, 0, 11], [3, 3, 8, 3], [1, 2, 20, 30], [0, 1, 2, 3], [-1, 40, 7, 2 ** 30], [4, 9, 14, 19]])
    dw = torch.randn(6, 4, generator=g)
    got, l = _grad([l], idx, dw, sf.F32, sigmoid=sigmoid, renorm=renorm)
    want, err = ref.route_grad(l.double(), idx, dw.double(), sigmoid=sigmoid, renorm=renorm)
    assert ref.outside(got, want, err + 2.0 ** -140, torch.float32) == ""


@gpu
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_backward_against_differences_of_the_forward_kernel_s_definition(sigmoid, renorm):
    g = torch.Generator().manual_seed(14)
    parts = [torch.randn(5, 24, generator=g) for _ in range(2)]
    idx, _, l = _go(parts, sf.F32, k=4, sigmoid=sigmoid, renorm=renorm, scale=2.0)
    dw = torch.randn(5, 4, generator=g)
    got, _ = _grad(parts, idx, dw, sf.F32, sigmoid=sigmoid, renorm=renorm, scale=2.0)
    _, err = ref.route_grad(l.double(), idx, dw.double(), sigmoid=sigmoid, renorm=renorm, scale=2.0)
    loss = lambda x: (ref.route(x, None, k=4, groups=1, top_groups=1, top2=False, sigmoid=sigmoid, renorm=renorm, scale=2.0)[1] * dw.double()).sum()  # noqa: E731
    v, t = torch.randn(5, 24, generator=g, dtype=torch.float64), 1e-7
    diff = (loss(l.double() + t * v) - loss(l.double() - t * v)) / (2 * t)
    assert abs(float(diff - (got.double() * v).sum())) < float(((err + ref.U * got.abs()) * v.abs()).sum()) + 1e-7


@gpu
@pytest.mark.parametrize("dtype", [sf.BF16, sf.F32])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("shift", [0.0, -30.0, 20.0])
def test_the_only_choice_renormalised_has_a_gradient_of_exactly_zero(sigmoid, shift, dtype):
    """Its weight is the scale whatever its logit is: w = s / s = 1, w * (d - d * w) = 0, without a rounding."""
    g = torch.Generator().manual_seed(23)
    parts = [torch.randn(301, 70, generator=g) + shift for _ in range(2)]
    l = _sum32([p.to(DT[dtype]) for p in parts])
    idx = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :1]
    got, _ = _grad(parts, idx, torch.randn(301, 1, generator=g), dtype, sigmoid=sigmoid, renorm=True, scale=1.5, pad=1)
    assert bool((got == 0).all())


@gpu
@pytest.mark.parametrize("sigmoid", [False, True])
def test_weights_are_quotients_rounded_once(sigmoid):
    """Where numerator and sum are exact in binary32 the weight is their quotient rounded once: of k equal logits 1 / k, of
    a single choice 1, of E equal experts without renormalising 1 / E."""
    one = torch.ones((), dtype=torch.float32)
    for k in range(1, 33):
        _, w, _ = _go([torch.zeros(2, 40)], sf.F32, k=k, sigmoid=sigmoid, renorm=True)
        assert bool((w == one / k).all()), k
    g = torch.Generator().manual_seed(31)
    _, w, _ = _go([4.0 * torch.randn(500, 40, generator=g)], sf.F32, k=1, sigmoid=sigmoid, renorm=True, scale=1.25)
    assert bool((w == 1.25).all())
    if not sigmoid:
        for E in [*range(1, 70), 100, 187, 255, 257, 511, 771, 1023]:
            _, w, _ = _go([torch.full((2, E), -3.0)], sf.BF16, k=1, sigmoid=False, renorm=False)
            assert bool((w == one / E).all()), E


@pytest.mark.parametrize("tokens,top_k", [(1 << 26, 16), ((1 << 31) - 1, 16), ((1 << 30) + 7, 1)])
def test_lists_of_2_to_the_30_results_and_more_are_not_refused_for_their_length(tokens, top_k):
    """The overlap is what stops these calls: nothing is launched, on any machine."""
    far = [(16 + i) << 40 for i in range(4)]
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_route(_args(logits=[far[0]], tokens=tokens, experts=16, top_k=top_k, groups=1, top_groups=1, bias=0, indices=far[1], weights=far[1] + 64))
    assert "overlaps" in str(e.value)
    with pytest.raises(sf.SifarError) as e:
        sf.sifar_route_backward(_grad_args(logits=[far[0]], tokens=tokens, experts=16, top_k=top_k, indices=far[1], dweights=far[2], dlogits=far[2] + 64))
    assert "overlaps" in str(e.value)
    with pytest.raises(sf.SifarError) as e:                  # the stride of rows has its limit
        sf.sifar_route(_args(logits=[far[0]], ld_logits=1 << 30, indices=far[1], weights=far[2]))
    assert "row stride of logits" in str(e.value)


@gpu
def test_more_than_2_to_the_30_results():
    T, E, k = (1 << 25) + 3, 32, 32
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(T, E, generator=g, device="cuda", dtype=torch.bfloat16)
    idx, w = torch.full((T, k), -7, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    a = sf.make_route([x.data_ptr()], tokens=T, experts=E, top_k=k, dtype=sf.BF16, indices=idx.data_ptr(), weights=w.data_ptr(), renormalize=1)
    sf.sifar_route(a)
    at = torch.tensor([0, 1, (1 << 24) - 1, 1 << 24, (1 << 25) - 1, 1 << 25, T - 1]).cuda()
    assert torch.equal(idx[at].long(), torch.sort(x[at], dim=1, descending=True, stable=True).indices)
    assert bool(((w.sum(1) - 1).abs() < 64 * ref.U).all())
    dw, out = torch.randn(T, k, generator=g, device="cuda"), torch.empty_like(x)
    b = sf.make_route_grad([x.data_ptr()], tokens=T, experts=E, top_k=k, dtype=sf.BF16, indices=idx.data_ptr(), dweights=dw.data_ptr(),
                           dlogits=out.data_ptr(), renormalize=1)
    sf.sifar_route_backward(b)
    want, err = ref.route_grad(ref.f64(x[at]), idx[at].cpu(), ref.f64(dw[at]), sigmoid=False, renorm=True)
    assert ref.outside(out[at], want, err, torch.bfloat16) == ""
