"""What runs between two all-reduces of a decode step, from its formulas in 64 bits on the CPU, with bounds on what the kernels may
lose, and caches whose pages lie in any order.

Inputs are float64 tensors that hold the values of the bf16 or fp32 inputs.  U is half a step of binary32 relative to a value.
"""
from __future__ import annotations

import math

import torch

from paper_2607_08973_b200 import binding as sf
from tests.ops_ref import U, f64

DT = {sf.BF16: torch.bfloat16, sf.F32: torch.float32}


class Cache:
    """Keys and values of `lengths` tokens on shuffled pages; all other places, and spare pages, hold `fill`."""

    def __init__(self, lengths, *, page=16, kv=2, dim=64, dtype=sf.BF16, layout="token", fill=math.nan, seed=0, spare=2, scale=1.0,
                 off=0, room=0):
        g = torch.Generator().manual_seed(seed)
        self.page, self.kv, self.dim, self.dtype, self.lengths = page, kv, dim, dtype, list(lengths)
        need = [-(-n // page) + room for n in self.lengths]
        self.pages, self.width = sum(need) + spare, max(1, max(need, default=1))
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = torch.full((len(need), self.width), -1, dtype=torch.int32)
        for s, n in enumerate(need):
            for i in range(n):
                self.table[s, i] = order.pop()
        shapes = {"token": (page, kv, dim), "head": (kv, page, dim), "both": (page, kv, 2 * dim), "wide": (page, kv, dim + 3)}
        inner = shapes[layout]
        count = 1 if layout == "both" else 2
        raw = [torch.full((self.pages * math.prod(inner) + off,), fill, dtype=torch.float64).to(DT[dtype]) for _ in range(count)]
        self.raw = [t.cuda() for t in raw]
        flat = [t[off:].view(self.pages, *inner) for t in self.raw]
        if layout == "both":
            self.k, self.v = flat[0][..., :dim], flat[0][..., dim:]
        elif layout == "head":
            self.k, self.v = flat[0].transpose(1, 2), flat[1].transpose(1, 2)
        else:
            self.k, self.v = flat[0][..., :dim], flat[1][..., :dim]
        self.keys, self.values = [], []
        for s, n in enumerate(self.lengths):
            k, v = ((torch.randn(n, kv, dim, generator=g, dtype=torch.float64) * scale).to(DT[dtype]) for _ in range(2))
            self.keys.append(k)
            self.values.append(v)
            self._put(s, k, v)
        self.table_dev = self.table.cuda()

    def _put(self, s, k, v):
        n = len(k)
        if n:
            t = torch.arange(n)
            page, slot = self.table[s].long()[t // self.page].cuda(), (t % self.page).cuda()
            self.k[page, slot], self.v[page, slot] = k.cuda(), v.cuda()

    def fields(self) -> dict:
        return dict(k_cache=self.k.data_ptr(), v_cache=self.v.data_ptr(), page_table=self.table_dev.data_ptr(), pages=self.pages,
                    page_size=self.page, max_pages=self.width, stride_page=self.k.stride(0), stride_token=self.k.stride(1),
                    stride_head=self.k.stride(2), sequences=len(self.lengths), kv_heads=self.kv, head_dim=self.dim, dtype=self.dtype)


def attention(q, k, v, scale: float, dtype):
    """out, lse of one sequence and their errors.  q: heads x dim, k, v: visible tokens x kv_heads x dim."""
    heads, dim = q.shape
    n, kv = k.shape[0], k.shape[1]
    if n == 0:
        return torch.zeros(heads, dim, dtype=torch.float64), torch.full((heads,), -math.inf, dtype=torch.float64), torch.zeros(heads, dim, dtype=torch.float64), torch.zeros(heads, dtype=torch.float64)
    q3 = q.reshape(kv, heads // kv, dim)
    x = scale * torch.einsum("hgd,thd->hgt", q3, k)
    # a sum of dim products, each add off by at most 2 U of what was added so far (the matrix instructions cut); then the scale's product
    ex = abs(scale) * 2 * (dim + 2) * U * torch.einsum("hgd,thd->hgt", q3.abs(), k.abs()) + 2 * U * x.abs()
    top = x.amax(2, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(2, keepdim=True)
    p = p / total
    out = torch.einsum("hgt,thd->hgd", p, v)
    # a probability: the scores' errors (its own and the maximum's), exp2 of x log2(e): the product's, the difference's and two
    # steps of its own, and again for each time that the maximum moved (at most once per strip; their exponents add up to at most
    # the same range), the sum's error
    rel = ex + ex.amax(2, keepdim=True) + (8 + 4 * (x - top).abs() + 2 * x.abs()) * U
    mean = (p * rel).sum(2, keepdim=True) + (n / 8 + 64) * U
    size = torch.einsum("hgt,thd->hgd", p, v.abs())
    err = torch.einsum("hgt,thd->hgd", p * rel, v.abs()) + (mean + 2 * (n / 8 + 64) * U) * size
    if dtype == sf.BF16:
        err = err + 2.0 ** -16 * size                        # two bf16 roundings of a probability, 2^-8 each
    lse = (top + torch.log(total)).reshape(heads)
    elog = mean.reshape(heads) + 8 * U * (lse.abs() + 1) + 2 * U * top.abs().reshape(heads)
    return out.reshape(heads, dim), lse, err.reshape(heads, dim), elog


def turn(x, positions, inv_freq, rotary: int, interleaved: bool):
    """x: tokens x heads x dim turned by the tokens' positions, and its error in binary32."""
    out, err = x.clone(), torch.zeros_like(x)
    half = rotary // 2
    if half:
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = (positions.double()[:, None] * f64(inv_freq)[None])[:, None]
        c, s = torch.cos(angle), torch.sin(angle)
        p, q = x[..., a], x[..., b]
        out[..., a], out[..., b] = p * c - q * s, p * s + q * c
        # cosine and sine: the angle over pi rounded once (pi U), two steps of their own; two products and an add; positions
        # below 2^31 lose at most 2^-22 of a turn's 2^-53 steps each
        size = p.abs() + q.abs()
        e = size * ((math.pi + 4 + 3) * U + positions.abs().double()[:, None, None] * 2.0 ** -50)
        err[..., a], err[..., b] = e, e
    return out, err


def _act(g, gelu: bool):
    return 0.5 * g * (1.0 + torch.erf(g * 0.5 ** 0.5)) if gelu else g / (1.0 + torch.exp(-g))


def experts(x, idx, w, gate_up, down, first: int, gelu: bool, dtype):
    """out and its error.  gate_up: experts x 2 inter x hidden, down: experts x hidden x inter."""
    T, H = x.shape
    E, I2, _ = gate_up.shape
    I = I2 // 2  # noqa: E741
    out, err = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for e in range(E):
        share = (w * (idx == e + first)).sum(1)
        t = (idx == e + first).any(1).nonzero()[:, 0]
        if not len(t):
            continue
        gu = x[t] @ gate_up[e].T
        # a sum of `hidden` products: adds off by 2 U of what was added so far (the matrix instructions cut)
        eg = 2 * (H + 8) * U * (x[t].abs() @ gate_up[e].abs().T)
        g, u = gu[:, :I], gu[:, I:]
        s = share[t][:, None]
        a = s * _act(g, gelu) * u
        # both activations change by at most 1.2 times what their argument does; exp, erf and the quotient a few steps
        ea = s.abs() * (1.2 * eg[:, :I] * (u.abs() + eg[:, I:]) + _act(g, gelu).abs() * eg[:, I:]) + (16 + 2 * g.abs()) * U * (s * g * u).abs()
        ew = 32 * U * (w.abs() * (idx == e + first)).sum(1)[t][:, None] * (_act(g, gelu) * u).abs()
        ea = ea + ew
        if dtype == sf.BF16:
            ea = ea + 2.0 ** -16 * a.abs()                   # two bf16 roundings, 2^-8 each
        out.index_add_(0, t, a @ down[e].T)
        err.index_add_(0, t, ea @ down[e].abs().T + 2 * (2 * I + E + 16) * U * (a.abs() @ down[e].abs().T))
    return out, err
