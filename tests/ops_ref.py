"""The operators behind an all-reduce from their formulas, in 64 bits on the CPU, with bounds on what binary32 may lose.

Inputs are float64 tensors that hold the values of the bf16 or fp32 inputs.  U is half a step of binary32 relative to
a value; DEPTH the longest chain of adds behind a sum over a row in the kernels (8 items of a thread, 5 shuffles, 16
warps, 8 CTAs) plus the products' own roundings.
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
DEPTH = 40
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64)


def gate_of_rows(gate, rows: int, span: int):
    """Row i of the result is the gate row of row i."""
    if gate is None:
        return None
    return gate[torch.arange(rows) // (span or max(rows, 1))]


def norm(xs, res, w1, gate, w2, *, post, pre, alpha, beta, eps, offset, span):
    """z, h, y, r1, r2 and the binary32 errors of h, y, r1, r2 (before the outputs are rounded)."""
    rows, cols = xs[0].shape
    one = torch.ones(cols, dtype=torch.float64)
    z = sum(xs[1:], xs[0])
    ez = (len(xs) - 1) * U * sum((x.abs() for x in xs[1:]), xs[0].abs())
    f1 = (w1 + offset) if w1 is not None else one
    f2 = (w2 + offset) if w2 is not None else one
    g = gate_of_rows(gate, rows, span)
    g = torch.ones(rows, 1, dtype=torch.float64) if g is None else g
    length = lambda t: t.square().sum(1).sqrt()  # noqa: E731
    r1, er1 = torch.ones(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    u, eu = z, ez
    if post:
        r1 = 1.0 / (z.square().mean(1) + eps).sqrt()
        # half of the sum's relative error, the division, the add of eps, two steps of the reciprocal root
        er1 = r1 * (length(ez) / length(z).clamp_min(1e-300) + (DEPTH / 2 + 6) * U)
        u = z * r1[:, None] * f1
        eu = ez * (r1[:, None] * f1).abs() + u.abs() * ((er1 / r1)[:, None] + 4 * U)
    b = 0.0 if res is None else alpha * res
    h = b + beta * g * u
    eh = (beta * g).abs() * (eu + 4 * U * u.abs()) + U * (abs(b) + (beta * g * u).abs())
    r2, er2, y, ey = torch.ones(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64), None, None
    if pre:
        r2 = 1.0 / (h.square().mean(1) + eps).sqrt()
        er2 = r2 * (length(eh) / length(h).clamp_min(1e-300) + (DEPTH / 2 + 6) * U)
        y = h * r2[:, None] * f2
        ey = eh * (r2[:, None] * f2).abs() + y.abs() * ((er2 / r2)[:, None] + 4 * U)
    return {"z": z, "h": h, "y": y, "r1": r1, "r2": r2}, {"z": ez, "h": eh, "y": ey, "r1": er1, "r2": er2}


def norm_grad(dys, dh, h, z, r1, r2, w1, gate, w2, *, post, pre, alpha, beta, offset, span):
    """dx, dres, dw1, dw2, dgate and their binary32 errors (before the outputs are rounded)."""
    rows, cols = (h if h is not None else dh).shape
    one = torch.ones(cols, dtype=torch.float64)
    f1 = (w1 + offset) if w1 is not None else one
    f2 = (w2 + offset) if w2 is not None else one
    out, err = {}, {}
    D = torch.zeros(rows, cols, dtype=torch.float64) if dh is None else dh
    eD = torch.zeros_like(D)
    if pre:
        G = sum(dys[1:], dys[0])
        eG = (len(dys) - 1) * U * sum((x.abs() for x in dys[1:]), dys[0].abs())
        n2 = h * r2[:, None]
        a = G * f2
        ea = eG * f2.abs() + 3 * U * a.abs()
        m = (a * n2).mean(1, keepdim=True)
        em = (ea * n2.abs() + (DEPTH + 8) * U * (a * n2).abs()).mean(1, keepdim=True) + 2 * U * m.abs()
        out["dw2"] = (G * n2).sum(0)
        err["dw2"] = (eG * n2.abs() + (rows + 40) * U * (G * n2).abs()).sum(0)
        eD = r2[:, None] * (ea + n2.abs() * em + 4 * U * (a.abs() + (n2 * m).abs())) + 2 * U * D.abs()
        t, et = D + r2[:, None] * a, r2[:, None] * (ea + 3 * U * a.abs()) + U * (D + r2[:, None] * a).abs()
        m2, em2, n2sum = r2[:, None] * m, r2[:, None] * em + 2 * U * (r2[:, None] * m).abs(), n2
        D = D + r2[:, None] * (a - n2 * m)
    else:
        t, et, m2, em2, n2sum = D, 0.0 * D, torch.zeros(rows, 1, dtype=torch.float64), torch.zeros(rows, 1, dtype=torch.float64), 0.0 * D
    eD = eD + U * D.abs()
    out["dres"], err["dres"] = alpha * D, abs(alpha) * eD + U * (alpha * D).abs()
    g = gate_of_rows(gate, rows, span)
    n1 = None if z is None else z * r1[:, None] if post else z
    if gate is not None and z is not None:
        u = n1 * f1 if post else n1
        terms, eterms = beta * D * u, abs(beta) * (eD * u.abs() + (rows + 48) * U * (D * u).abs())
        of_row = torch.arange(rows) // (span or max(rows, 1))
        out["dgate"] = torch.zeros(gate.shape, dtype=torch.float64).index_add_(0, of_row, terms)
        err["dgate"] = torch.zeros(gate.shape, dtype=torch.float64).index_add_(0, of_row, eterms)
    d = beta * D if g is None else beta * g * D
    ed = (abs(beta) * eD if g is None else (beta * g).abs() * eD) + 3 * U * d.abs()
    if post:
        out["dw1"] = (d * n1).sum(0)
        err["dw1"] = (ed * n1.abs() + (rows + 40) * U * (d * n1).abs()).sum(0)
        b = d * f1
        eb = ed * f1.abs() + 3 * U * b.abs()
        m = (b * n1).mean(1, keepdim=True)
        # the kernel takes this sum as that of (b n1 with t = dh + r2 a for D) - r2 m2 * that of (b n1 with n2 for D), so
        # that both sums of a row need one pass: each term has three products and the sum's DEPTH, t and m2 their own error
        fn = (beta if g is None else beta * g) * f1 * n1
        em = (fn.abs() * et + (DEPTH + 8) * U * (fn * t).abs()).mean(1, keepdim=True)
        em = em + m2.abs() * ((DEPTH + 8) * U * (fn * n2sum).abs()).mean(1, keepdim=True)
        em = em + em2 * (fn * n2sum).abs().mean(1, keepdim=True)
        em = em + 3 * U * ((fn * t).abs().mean(1, keepdim=True) + (m2 * fn * n2sum).abs().mean(1, keepdim=True))
        ed = r1[:, None] * (eb + n1.abs() * em + 5 * U * (b.abs() + (n1 * m).abs()))
        d = r1[:, None] * (b - n1 * m)
    out["dx"], err["dx"] = d, ed
    return out, err


def outside(got, want, err, dtype) -> str:
    """Empty where every element lies within its bound: the binary32 error and half a step of the stored type."""
    got = f64(got)
    bound = err + HALF[dtype] * (want.abs() + err) + 1e-37
    bad = ~((got - want).abs() <= bound)
    if not bool(bad.any()):
        return ""
    i = int(((got - want).abs() / bound).nan_to_num(nan=math.inf).argmax())
    return (f"{int(bad.sum())} of {bad.numel()} outside, worst at {i}: got {got.reshape(-1)[i]!r} want "
            f"{want.reshape(-1)[i]!r} bound {bound.expand_as(want).reshape(-1)[i]!r}")


# ---------------------------------------------------------------------------------------------------------------
def _lowest(v: float) -> float:
    return -math.inf if v != v else v


def _sigmoid(x: float) -> float:
    if x != x:
        return x
    return 1.0 / (1.0 + math.exp(-x)) if x > -700 else (math.exp(x) if x > -745 else 0.0)


def route(l, bias, *, k, groups, top_groups, top2, sigmoid, renorm, scale=1.0):
    """indices and weights, token by token; l are the binary32 rank-order sums as float64."""
    T, E = l.shape
    idx, wts = torch.zeros(T, k, dtype=torch.int32), torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        row = l[t].tolist()
        top = math.nan if any(x != x for x in row) else max(row)
        if sigmoid:
            s = [_sigmoid(x) for x in row]
        elif top == -math.inf:
            s = [0.0] * E
        elif not math.isfinite(top):
            s = [math.nan if x == top or top != top else 0.0 for x in row]
            s = [math.nan] * E
        else:
            e = [math.exp(x - top) for x in row]
            total = math.fsum(e)
            s = [x / total for x in e]
        v = [_lowest(a + (bias[i].item() if bias is not None else 0.0)) for i, a in enumerate(s)]
        key = v if bias is not None else [_lowest(x) for x in row]
        cand = range(E)
        if groups > 1:
            per = E // groups
            def value(g):
                run = v if top2 else key
                run = sorted(run[g * per:(g + 1) * per], reverse=True)
                return _lowest(sum(run[:2])) if top2 else run[0]
            best = sorted(range(groups), key=lambda g: (-value(g), g))[:top_groups]
            cand = [e for e in range(E) if e // per in best]
        chosen = sorted(cand, key=lambda e: (-key[e], e))[:k]
        w = [s[e] for e in chosen]
        if renorm:
            m = math.nan if any(row[e] != row[e] for e in chosen) else max(row[e] for e in chosen)
            if m == -math.inf:
                w = [0.0] * k
            elif m != m or (m == math.inf and not sigmoid):
                w = [math.nan] * k
            else:
                # the ratio of the s, without the factor that they share
                w = [math.exp(row[e] - m) if not sigmoid else s[e] if m >= 0 else
                     math.exp(row[e] - m) / (1.0 + math.exp(row[e])) for e in chosen]
                total = math.fsum(w)
                w = [x / total for x in w]
        idx[t] = torch.tensor(chosen, dtype=torch.int32)
        wts[t] = torch.tensor([scale * x for x in w], dtype=torch.float64)
    return idx, wts


def route_grad(l, idx, dw, *, sigmoid, renorm, scale=1.0):
    """d l of sum(dw * weights) and a bound of its binary32 error; indices outside the experts have no part."""
    T, E = l.shape
    out, err = torch.zeros(T, E, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    for t in range(T):
        on = [(int(e), scale * float(d)) for e, d in zip(idx[t], dw[t]) if 0 <= int(e) < E]
        row = l[t].tolist()
        if renorm and on:
            m = max(row[e] for e, _ in on)
            if m == -math.inf:
                continue
            s = [math.exp(row[e] - m) if not sigmoid or m < 0 else 1.0 for e, _ in on]
            if sigmoid:
                s = [a / (1.0 + math.exp(row[e])) if m < 0 else _sigmoid(row[e]) for a, (e, _) in zip(s, on)]
            total = math.fsum(s)
            w = [a / total for a in s]
            mean = math.fsum(a * d for a, (_, d) in zip(w, on))
            size = math.fsum(a * abs(d) for a, (_, d) in zip(w, on))
            span = max((m - row[e] for e, _ in on if row[e] > -math.inf), default=0.0)
            for a, (e, d) in zip(w, on):
                rest = _sigmoid(-row[e]) if sigmoid else 1.0
                out[t, e] += a * (d - mean) * rest
                err[t, e] += a * (abs(d) + size) * rest * U * (4 * span + 2 * abs(row[e] if sigmoid and math.isfinite(row[e]) else 0.0) + 80)
        elif sigmoid:
            for e, d in on:
                x = d * _sigmoid(row[e]) * _sigmoid(-row[e])
                out[t, e] += x
                err[t, e] += abs(x) * U * (2 * abs(row[e] if math.isfinite(row[e]) else 0.0) + 40)
        else:
            m = max(row)
            if m == -math.inf:
                continue
            p = [math.exp(x - m) for x in row]
            total = math.fsum(p)
            p = [x / total for x in p]
            mean = math.fsum(p[e] * d for e, d in on)
            size = math.fsum(p[e] * abs(d) for e, d in on)
            span = m - min(x for x in row if x > -math.inf)
            ds = [0.0] * E
            mag = [size] * E
            for e, d in on:
                ds[e] += d
                mag[e] += abs(d)
            for e in range(E):
                out[t, e] = p[e] * (ds[e] - mean)
                err[t, e] = p[e] * mag[e] * U * (4 * span + 80)
    return out, err
