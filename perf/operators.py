"""The operators around an all-reduce of a transformer layer, as cases that can be timed and compared.

* ``norm``        what a layer does with the P partial sums of a block: their sum, the norm behind the block, its gate,
                  the scaled residual and the norm before the next block (``sifar_block_norm``);
* ``norm-grad``   its backward pass; the gradient of the normed rows comes as P partials again
                  (``sifar_block_norm_backward``);
* ``route``       the choice of experts from P partial router logits (``sifar_route``);
* ``route-grad``  its backward pass (``sifar_route_backward``).

Hidden size 4096, up to 8192 tokens (the 64 MiB per rank of the payload sweep) and two to eight ranks are this
repository's own; odd sizes, wider row strides and both types are among the cases.

In their plain form the operators are elementary torch operations in binary32; the routing scores that a bias or a
group's sum may put next to a border are compared in binary64.
"""
from __future__ import annotations

from functools import reduce

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_ELEM = {"bf16": 2, "f32": 4}
_EPS = 1e-6
_LARGEST_BYTES = 11 * 8192 * 4096 * 2           # what the largest listed case moves


def listed() -> list[dict]:
    norm = {"cols": 4096, "dtype": "bf16", "post": False, "pre": True, "gate": "none", "span": 0, "pad": 0,
            "save": False, "alpha": 1.0, "beta": 1.0, "offset": 0.0}
    return [
        # decode, one token: attention's partials of eight ranks, residual, norm before the next block
        {"name": "norm-1", "op": "norm", "P": 8, "rows": 1, **norm},
        # the largest decode batch of the mixture-of-experts shape, a norm on either side of the block, scaled residual
        {"name": "norm-64-both", "op": "norm", "P": 8, "rows": 64, **norm, "post": True, "alpha": 0.5, "offset": 1.0},
        # prefill of 8192 tokens on eight ranks, both norms and a gate per channel (a learned layer scale)
        {"name": "norm-8192-gated", "op": "norm", "P": 8, "rows": 8192, **norm, "post": True, "gate": "channel"},
        # a training step in binary32: odd sizes, rows inside wider ones, a gate row for every 59 tokens, all saved
        {"name": "norm-f32-ragged", "op": "norm", "P": 3, "rows": 1003, **norm, "cols": 4099, "dtype": "f32",
         "post": True, "gate": "group", "span": 59, "pad": 5, "save": True, "beta": 0.7},
        # the backward pass of a small micro-batch, partial gradients of eight ranks
        {"name": "norm-grad-64", "op": "norm-grad", "P": 8, "rows": 64, **norm, "beta": 0.5},
        # ... of 8192 tokens in sequences of 2048 that each have a gate row of their own
        {"name": "norm-grad-8192-gated", "op": "norm-grad", "P": 2, "rows": 8192, **norm, "post": True,
         "gate": "group", "span": 2048},
        # ... of the odd training step
        {"name": "norm-grad-f32-ragged", "op": "norm-grad", "P": 3, "rows": 1003, **norm, "cols": 4099,
         "dtype": "f32", "post": True, "gate": "group", "span": 59, "pad": 5, "beta": 0.7},
        # decode, one token: 8 of 128 experts, their softmax renormalised
        {"name": "route-1", "op": "route", "P": 1, "tokens": 1, "experts": 128, "k": 8, "groups": 1, "top_groups": 1,
         "group_score": "max", "score": "softmax", "bias": False, "renorm": True, "dtype": "bf16", "pad": 0},
        # prefill: sigmoid scores with a bias for balance, the best 4 of 8 groups by the sum of two, 8 of 256 experts
        {"name": "route-8192-groups", "op": "route", "P": 1, "tokens": 8192, "experts": 256, "k": 8, "groups": 8,
         "top_groups": 4, "group_score": "top2", "score": "sigmoid", "bias": True, "renorm": True, "dtype": "f32",
         "pad": 0},
        # a router whose input is split over eight ranks, odd counts, plain softmax weights
        {"name": "route-ragged", "op": "route", "P": 8, "tokens": 1237, "experts": 61, "k": 5, "groups": 1,
         "top_groups": 1, "group_score": "max", "score": "softmax", "bias": False, "renorm": False, "dtype": "bf16",
         "pad": 3},
        # the backward pass of a small micro-batch
        {"name": "route-grad-64", "op": "route-grad", "P": 1, "tokens": 64, "experts": 128, "k": 8, "groups": 1,
         "top_groups": 1, "group_score": "max", "score": "softmax", "bias": False, "renorm": False, "dtype": "bf16",
         "pad": 0},
        # ... of the grouped prefill shape
        {"name": "route-grad-8192", "op": "route-grad", "P": 1, "tokens": 8192, "experts": 256, "k": 8, "groups": 8,
         "top_groups": 4, "group_score": "top2", "score": "sigmoid", "bias": True, "renorm": True, "dtype": "f32",
         "pad": 0},
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    """Log-uniform on [lo, hi]; half of them odd, half multiples of 64 where there is room for one."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    v = v - v % 64 if rng.random() < 0.5 and v >= 64 else v | 1
    return max(lo, min(hi, v))


def draw(rng) -> dict:
    op = rng.choice(["norm", "norm", "norm-grad", "norm-grad", "route", "route", "route-grad"])
    P = rng.choice([1, 2, 4, 8, rng.randint(1, 8)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 40)])
    if op.startswith("norm"):
        cols = _log_int(rng, 64, 16384)
        rows = _log_int(rng, 1, max(1, min(8192, _LARGEST_BYTES // ((P + 6) * cols * _ELEM[dtype]))))
        post = rng.random() < 0.5
        return {"op": op, "P": P, "rows": rows, "cols": cols, "dtype": dtype, "post": post,
                "pre": not post or rng.random() < 0.8, "gate": rng.choice(["none", "channel", "group"]),
                "span": _log_int(rng, 1, max(1, rows)), "pad": pad, "save": rng.random() < 0.5,
                "alpha": rng.choice([1.0, 0.5, 1.25]), "beta": rng.choice([1.0, 0.7]),
                "offset": rng.choice([0.0, 1.0])}
    groups = rng.choice([1, 1, 2, 4, 8])
    per_group = max(2, _log_int(rng, 8, 512) // groups)
    top_groups = rng.randint(1, groups)
    return {"op": op, "P": P, "tokens": _log_int(rng, 1, 8192), "experts": groups * per_group,
            "k": min(rng.randint(1, 10), top_groups * per_group), "groups": groups, "top_groups": top_groups,
            "group_score": rng.choice(["max", "top2"]), "score": rng.choice(["softmax", "sigmoid"]),
            "bias": rng.random() < 0.5, "renorm": rng.random() < 0.6, "dtype": dtype, "pad": pad}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _rows(g, rows: int, cols: int, pad: int, dtype, outliers: bool = False, scale: float = 1.0) -> torch.Tensor:
    """N(0, scale^2) rows inside rows that are `pad` elements wider; one element in a hundred an outlier if asked."""
    t = torch.randn(rows, cols + pad, generator=g, device="cuda") * scale
    if outliers:
        t *= 1.0 + 99.0 * (torch.rand(rows, cols + pad, generator=g, device="cuda") < 0.01)
    return t.to(dtype)[:, :cols]


def _gate_rows(case: dict) -> int:
    return -(-case["rows"] // case["span"]) if case["gate"] == "group" else 1


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, pad = _TORCH[case["dtype"]], case["pad"]
    s = dict(case=case)
    if case["op"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        weight = lambda n: (1.0 - case["offset"] + 0.1 * torch.randn(n, cols, generator=g, device="cuda")).to(dt)  # noqa: E731
        s["x"] = [_rows(g, rows, cols, pad, dt) for _ in range(case["P"])]
        s["res"] = _rows(g, rows, cols, pad, dt, outliers=True)
        s["w1"] = weight(1)[0] if case["post"] else None
        s["w2"] = weight(1)[0] if case["pre"] else None
        s["gate"] = (0.5 * torch.randn(_gate_rows(case), cols, generator=g, device="cuda")).to(dt) \
            if case["gate"] != "none" else None
        wide = lambda: torch.empty(rows, cols + pad, dtype=dt, device="cuda")[:, :cols]  # noqa: E731
        if case["op"] == "norm":
            s["z"] = wide() if case["save"] else None
            s["h"] = wide()
            s["y"] = wide() if case["pre"] else None
            s["stats"] = torch.empty(2, rows, device="cuda") if case["save"] else None
        else:
            # what the forward pass saved, and the gradients that come back: of h from its other uses, of y as partials
            z, h, _, r1, r2 = _forward(s)
            s["saved"] = {"z": wide().copy_(z), "h": wide().copy_(h), "stats": torch.stack([r1, r2])}
            s["dh"] = _rows(g, rows, cols, pad, dt)
            s["dy"] = [_rows(g, rows, cols, pad, dt) for _ in range(case["P"])] if case["pre"] else []
            s["dx"], s["dres"] = wide(), wide()
            s["dw1"] = torch.empty(cols, device="cuda") if case["post"] else None
            s["dw2"] = torch.empty(cols, device="cuda") if case["pre"] else None
            s["dgate"] = torch.empty(_gate_rows(case), cols, device="cuda") if s["gate"] is not None else None
            del s["x"], s["res"]
    else:
        T, E, k = case["tokens"], case["experts"], case["k"]
        s["logits"] = [_rows(g, T, E, pad, dt, scale=(2.0 / case["P"]) ** 0.5) for _ in range(case["P"])]
        s["bias"] = 0.1 * torch.randn(E, generator=g, device="cuda") if case["bias"] else None
        if case["op"] == "route":
            s["indices"] = torch.empty(T, k, dtype=torch.int32, device="cuda")
            s["weights"] = torch.empty(T, k, device="cuda")
        else:
            s["indices"] = _choose(s).to(torch.int32)
            s["dweights"] = torch.randn(T, k, generator=g, device="cuda")
            s["dlogits"] = torch.empty(T, E + pad, dtype=dt, device="cuda")[:, :E]
    if own:
        _plan(s)
    return s


def _plan(s: dict) -> None:
    """The argument block that a program fills once per layer and passes with every call."""
    from paper_2607_08973_b200 import binding as sf
    c = s["case"]
    s["device"] = torch.cuda.current_device()
    dtype = sf.BF16 if c["dtype"] == "bf16" else sf.F32
    ptr = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    if c["op"].startswith("norm"):
        ld = c["cols"] + c["pad"]
        shape = dict(rows=c["rows"], cols=c["cols"], dtype=dtype, post_norm=c["post"], pre_norm=c["pre"],
                     post_weight=ptr(s["w1"]), gate=ptr(s["gate"]), pre_weight=ptr(s["w2"]),
                     rows_per_gate=c["span"] if c["gate"] == "group" else 0, alpha=c["alpha"], beta=c["beta"],
                     weight_offset=c["offset"])
        if c["op"] == "norm":
            a = sf.make_block_norm([ptr(x) for x in s["x"]], residual=ptr(s["res"]), z=ptr(s["z"]), h=ptr(s["h"]),
                                   y=ptr(s["y"]), stats=ptr(s["stats"]), eps=_EPS, ld_x=ld, ld_residual=ld, ld_z=ld,
                                   ld_h=ld, ld_y=ld, **shape)
            s["call"], s["args"] = sf.sifar_block_norm, a
        else:
            a = sf.make_block_norm_grad([ptr(x) for x in s["dy"]], dh=ptr(s["dh"]), z=ptr(s["saved"]["z"]),
                                        h=ptr(s["saved"]["h"]), stats=ptr(s["saved"]["stats"]), dx=ptr(s["dx"]),
                                        dresidual=ptr(s["dres"]), dpost_weight=ptr(s["dw1"]), dgate=ptr(s["dgate"]),
                                        dpre_weight=ptr(s["dw2"]), ld_dy=ld, ld_dh=ld, ld_z=ld, ld_h=ld, ld_dx=ld,
                                        ld_dresidual=ld, **shape)
            size = sf.sifar_block_norm_backward_workspace(a)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
            a.workspace, a.workspace_bytes = ptr(s["workspace"]), size
            s["call"], s["args"] = sf.sifar_block_norm_backward, a
        return
    ld = c["experts"] + c["pad"]
    shape = dict(tokens=c["tokens"], experts=c["experts"], top_k=c["k"], dtype=dtype, ld_logits=ld,
                 score=sf.SCORE_SOFTMAX if c["score"] == "softmax" else sf.SCORE_SIGMOID, renormalize=c["renorm"])
    logits = [ptr(x) for x in s["logits"]]
    if c["op"] == "route":
        s["args"] = sf.make_route(logits, bias=ptr(s["bias"]), indices=ptr(s["indices"]), weights=ptr(s["weights"]),
                                  groups=c["groups"], top_groups=c["top_groups"],
                                  group_score=sf.GROUP_MAX if c["group_score"] == "max" else sf.GROUP_TOP2, **shape)
        s["call"] = sf.sifar_route
    else:
        s["args"] = sf.make_route_grad(logits, indices=ptr(s["indices"]), dweights=ptr(s["dweights"]),
                                       dlogits=ptr(s["dlogits"]), ld_dlogits=ld, **shape)
        s["call"] = sf.sifar_route_backward


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _sum(partials) -> torch.Tensor:
    """Rank-order sum in binary32."""
    return reduce(lambda acc, x: acc + x.float(), partials[1:], partials[0].float())


def _rrms(t: torch.Tensor) -> torch.Tensor:
    return 1.0 / torch.sqrt((t * t).mean(dim=1) + _EPS)


def _scaled(w, offset: float):
    return w.float() + offset if w is not None else 1.0


def _gate(s: dict):
    """The gate of every row (or of all), 1 where there is none."""
    c, g = s["case"], s["gate"]
    if g is None:
        return 1.0
    g = g.float()
    return g.repeat_interleave(c["span"], dim=0)[: c["rows"]] if c["gate"] == "group" else g


def _forward(s: dict):
    c = s["case"]
    z = _sum(s["x"])
    r1 = _rrms(z)
    u = z * r1[:, None] * _scaled(s["w1"], c["offset"]) if c["post"] else z
    h = c["alpha"] * s["res"].float() + c["beta"] * _gate(s) * u
    r2 = _rrms(h)
    y = h * r2[:, None] * _scaled(s["w2"], c["offset"]) if c["pre"] else None
    return z, h, y, r1, r2


def _norm_outputs(c: dict, z, h, y, r1, r2, cast) -> dict:
    out = {"h": cast(h)}
    if c["pre"]:
        out["y"] = cast(y)
    if c["save"]:
        out["z"] = cast(z)
        out["stats"] = torch.stack([r1 if c["post"] else torch.ones_like(r1), r2 if c["pre"] else torch.ones_like(r2)])
    return out


def _by_gate(t: torch.Tensor, c: dict) -> torch.Tensor:
    """Sum over the rows that share a gate row."""
    if c["gate"] == "channel":
        return t.sum(dim=0, keepdim=True)
    n, rows, cols = _gate_rows(c), c["rows"], c["cols"]
    full = torch.zeros(n * c["span"], cols, dtype=t.dtype, device=t.device)
    full[:rows] = t
    return full.view(n, c["span"], cols).sum(dim=1)


def _backward(s: dict):
    c, saved = s["case"], s["saved"]
    D = s["dh"].float()
    dw1 = dw2 = dgate = None
    if c["pre"]:
        G, hh = _sum(s["dy"]), saved["h"].float() * saved["stats"][1][:, None]
        dw2 = (G * hh).sum(dim=0)
        a = G * _scaled(s["w2"], c["offset"])
        D = D + saved["stats"][1][:, None] * (a - hh * (a * hh).mean(dim=1, keepdim=True))
    dres = c["alpha"] * D
    zh = saved["z"].float() * saved["stats"][0][:, None] if c["post"] else saved["z"].float()
    if s["gate"] is not None:
        dgate = _by_gate(c["beta"] * D * zh * _scaled(s["w1"], c["offset"]), c)
    dx = c["beta"] * _gate(s) * D
    if c["post"]:
        dw1 = (dx * zh).sum(dim=0)
        b = dx * _scaled(s["w1"], c["offset"])
        dx = saved["stats"][0][:, None] * (b - zh * (b * zh).mean(dim=1, keepdim=True))
    return dx, dres, dw1, dw2, dgate


def _lowest(v: torch.Tensor) -> torch.Tensor:
    """NaN counts as the lowest value."""
    return torch.where(torch.isnan(v), torch.full_like(v, float("-inf")), v)


def _scores64(l: torch.Tensor, kind: str) -> torch.Tensor:
    l = l.double()
    if kind == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    e = torch.exp(l - l.amax(dim=1, keepdim=True))
    return e / e.sum(dim=1, keepdim=True)


def _choose(s: dict) -> torch.Tensor:
    """The chosen experts of every token, best first, ties to the lowest index.  Scores only grow with the logits, so
    without a bias the logits themselves are compared."""
    c = s["case"]
    l = _sum(s["logits"])
    value = None
    if c["bias"] or (c["groups"] > 1 and c["group_score"] == "top2"):
        value = _scores64(l, c["score"])
        value = _lowest(value + s["bias"].double() if c["bias"] else value)
    key = value if c["bias"] else _lowest(l)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    if c["groups"] > 1:
        per = c["experts"] // c["groups"]
        if c["group_score"] == "max":
            score = key.view(-1, c["groups"], per).amax(dim=2)
        else:
            score = _lowest(value.view(-1, c["groups"], per).topk(min(2, per), dim=2).values.sum(dim=2))
        best = torch.sort(score, dim=1, descending=True, stable=True).indices[:, : c["top_groups"]]
        closed = torch.ones(score.shape, dtype=torch.bool, device=l.device).scatter_(1, best, False)
        closed = closed.gather(1, order // per)
        order = order.gather(1, torch.sort(closed.int(), dim=1, stable=True).indices)
    return order[:, : c["k"]]


def _route(s: dict):
    c = s["case"]
    l, chosen = _sum(s["logits"]), _choose(s)
    if c["score"] == "sigmoid":
        w = 1.0 / (1.0 + torch.exp(-l.gather(1, chosen)))
    elif c["renorm"]:
        w = l.gather(1, chosen)
        w = torch.exp(w - w.amax(dim=1, keepdim=True))
    else:
        e = torch.exp(l - l.amax(dim=1, keepdim=True))
        w = (e / e.sum(dim=1, keepdim=True)).gather(1, chosen)
    return chosen, w / w.sum(dim=1, keepdim=True) if c["renorm"] else w


def _route_backward(s: dict) -> torch.Tensor:
    c, chosen, dw = s["case"], s["indices"].long(), s["dweights"]
    l = _sum(s["logits"])
    lc = l.gather(1, chosen)
    if c["score"] == "softmax" and not c["renorm"]:
        e = torch.exp(l - l.amax(dim=1, keepdim=True))
        p = e / e.sum(dim=1, keepdim=True)
        return p * (torch.zeros_like(l).scatter(1, chosen, dw) - (dw * p.gather(1, chosen)).sum(dim=1, keepdim=True))
    if c["score"] == "softmax":
        e = torch.exp(lc - lc.amax(dim=1, keepdim=True))
        w = e / e.sum(dim=1, keepdim=True)
        d = w * (dw - (dw * w).sum(dim=1, keepdim=True))
    else:
        sc, rest = 1.0 / (1.0 + torch.exp(-lc)), 1.0 / (1.0 + torch.exp(lc))
        d = dw
        if c["renorm"]:
            total = sc.sum(dim=1, keepdim=True)
            d = (dw - (dw * sc).sum(dim=1, keepdim=True) / total) / total
        d = d * sc * rest
    return torch.zeros_like(l).scatter(1, chosen, d)


def run(s: dict):
    c = s["case"]
    if own:
        # on torch's current stream, as the plain form; torch.cuda.current_stream() makes an object each time (4 us)
        s["call"](s["args"], torch._C._cuda_getCurrentRawStream(s["device"]))
        if c["op"] == "norm":
            return {n: s[n] for n in ("h", "y", "z", "stats") if s[n] is not None}
        if c["op"] == "norm-grad":
            return {n: s[n] for n in ("dx", "dres", "dw1", "dw2", "dgate") if s[n] is not None}
        return {"indices": s["indices"], "weights": s["weights"]} if c["op"] == "route" else {"dlogits": s["dlogits"]}
    dt = _TORCH[c["dtype"]]
    if c["op"] == "norm":
        return _norm_outputs(c, *_forward(s), lambda t: t.to(dt))
    if c["op"] == "norm-grad":
        dx, dres, dw1, dw2, dgate = _backward(s)
        out = {"dx": dx.to(dt), "dres": dres.to(dt), "dw1": dw1, "dw2": dw2, "dgate": dgate}
        return {n: t for n, t in out.items() if t is not None}
    if c["op"] == "route":
        chosen, w = _route(s)
        return {"indices": chosen.to(torch.int32), "weights": w}
    return {"dlogits": _route_backward(s).to(dt)}


def work(case: dict) -> dict:
    P = case["P"]
    es = _ELEM[case["dtype"]]
    if case["op"].startswith("norm"):
        n, cols, post, pre = case["rows"] * case["cols"], case["cols"], case["post"], case["pre"]
        gates = _gate_rows(case) * cols if case["gate"] != "none" else 0
        weights = (post + pre) * cols + gates
        if case["op"] == "norm":
            save = case["save"]
            return {"bytes": es * ((P + 2 + pre + save) * n + weights) + (8 * case["rows"] if save else 0),
                    "flops": n * (P - 1 + 4 + 5 * post + 4 * pre)}
        # reads dh, h and the partials of dy behind a norm, z where the gate or the norm needs it; writes dx and dres
        reads = 1 + (1 + P) * pre + (1 if post or gates else 0)
        return {"bytes": es * ((reads + 2) * n + weights) + 4 * weights + 4 * (post + pre) * case["rows"],
                "flops": n * (4 + (P + 9) * pre + 9 * post + (3 if gates else 0))}
    T, E, k = case["tokens"], case["experts"], case["k"]
    if case["op"] == "route":
        return {"bytes": T * (P * E * es + 8 * k) + (4 * E if case["bias"] else 0), "flops": T * E * (P + 4)}
    # behind a softmax over all experts every logit counts; otherwise the chosen ones alone are read
    read = P * es * (E if case["score"] == "softmax" and not case["renorm"] else k)
    return {"bytes": T * (read + E * es + 8 * k), "flops": T * (E + 8 * k)}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case: dict, seed: int):
    s = prepare(case, seed)
    d = lambda t: t.to(torch.float64)  # noqa: E731
    if case["op"].startswith("norm"):
        rows, cols, alpha, beta, off = case["rows"], case["cols"], case["alpha"], case["beta"], case["offset"]
        gate = torch.ones(1, cols, dtype=torch.float64, device="cuda") if s["gate"] is None else d(s["gate"])
        of_row = torch.arange(rows, device="cuda") // case["span"] if case["gate"] == "group" \
            else torch.zeros(rows, dtype=torch.long, device="cuda")
        w1 = d(s["w1"]) + off if case["post"] else torch.ones(cols, dtype=torch.float64, device="cuda")
        w2 = d(s["w2"]) + off if case["pre"] else w1
        if case["op"] == "norm":
            z = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
            for x in s["x"]:
                z += d(x)
            r1 = (z.square().sum(1) / cols + _EPS).rsqrt()
            h = alpha * d(s["res"]) + beta * gate[of_row] * (z * r1.unsqueeze(1) * w1 if case["post"] else z)
            r2 = (h.square().sum(1) / cols + _EPS).rsqrt()
            return _norm_outputs(case, z, h, h * r2.unsqueeze(1) * w2, r1, r2, d)
        # the gradients by the chain rule, one product at a time
        stats = d(s["saved"]["stats"])
        D = d(s["dh"])
        out = {}
        if case["pre"]:
            hh = d(s["saved"]["h"]) * stats[1].unsqueeze(1)
            G = torch.zeros_like(D)
            for x in s["dy"]:
                G += d(x)
            out["dw2"] = torch.einsum("rc,rc->c", G, hh)
            along = torch.einsum("rc,rc->r", G * w2, hh) / cols
            D = D + (G * w2 - along.unsqueeze(1) * hh) * stats[1].unsqueeze(1)
        out["dres"] = D * alpha
        z = d(s["saved"]["z"])
        zh = z * stats[0].unsqueeze(1) if case["post"] else z
        if s["gate"] is not None:
            out["dgate"] = torch.zeros_like(gate).index_add_(0, of_row, D * beta * (zh * w1 if case["post"] else zh))
        du = D * beta * gate[of_row]
        if case["post"]:
            out["dw1"] = torch.einsum("rc,rc->c", du, zh)
            along = torch.einsum("rc,rc->r", du * w1, zh) / cols
            du = (du * w1 - along.unsqueeze(1) * zh) * stats[0].unsqueeze(1)
        out["dx"] = du
        return {n: out[n] for n in ("dx", "dres", "dw1", "dw2", "dgate") if n in out}
    # the sum over ranks is binary32 in rank order by definition; everything behind it in 64 bits
    l = torch.zeros(case["tokens"], case["experts"], device="cuda")
    for i, x in enumerate(s["logits"]):
        l = x.float() if i == 0 else l + x.float()
    l64 = d(l)
    score = torch.sigmoid(l64) if case["score"] == "sigmoid" else torch.softmax(l64, dim=1)
    if case["op"] == "route":
        value = score + d(s["bias"]) if case["bias"] else l64
        if case["groups"] > 1:
            # one group after the other is opened, always the best one that is left
            T, n = case["tokens"], case["groups"]
            of = (score + d(s["bias"]) if case["bias"] else score).reshape(T, n, -1)
            top = of.sort(dim=2, descending=True).values
            rank = top[:, :, :2].sum(2) if case["group_score"] == "top2" else value.reshape(T, n, -1).amax(2)
            open_ = torch.zeros(T, n, dtype=torch.bool, device="cuda")
            for _ in range(case["top_groups"]):
                open_[torch.arange(T, device="cuda"), rank.masked_fill(open_, -float("inf")).argmax(1)] = True
            value = value.masked_fill(~open_.repeat_interleave(case["experts"] // n, dim=1), -float("inf"))
        chosen = value.sort(dim=1, descending=True, stable=True).indices[:, : case["k"]]
        w = score.gather(1, chosen)
        return {"indices": None, "weights": w / w.sum(1, keepdim=True) if case["renorm"] else w}
    # the gradient of sum(dweights * weights) through the score's own derivative
    chosen, dw = s["indices"].long(), d(s["dweights"])
    w = score.gather(1, chosen)
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        dw = (dw - (dw * w).sum(1, keepdim=True) / total) / total
    ds = torch.zeros_like(l64).scatter_(1, chosen, dw)
    if case["score"] == "sigmoid":
        return {"dlogits": ds * score * torch.sigmoid(-l64)}
    return {"dlogits": score * (ds - (ds * score).sum(1, keepdim=True))}
