"""The operators between two all-reduces of a decode step, as cases that can be timed and compared.

* ``append``   queries and keys turned by their positions, keys and values written to a paged cache
  (``sifar_cache_append``);
* ``attend``   attention of one new token per sequence over that cache (``sifar_decode_attention``);
* ``experts``  the products of the chosen experts for a few tokens: one rank's partial of the layer's second all-reduce
  (``sifar_experts``).

Hidden size 4096, 8 of 128 experts and up to 64 tokens of a decode batch are this repository's own; both types, odd sizes,
pages that end anywhere, wider strides, empty sequences and padding tokens are among the cases.  Which tokens, lengths
and experts a case has is part of the case (its ``mix``); the values come from the seed.

In their plain form the operators are elementary torch operations in binary32, the angles in binary64.
"""
from __future__ import annotations

import random

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_ELEM = {"bf16": 2, "f32": 4}
_LARGEST_CACHE = 2 * 131072 * 8 * 2 * 128 * 2         # bytes of keys and values of the largest listed attention


def listed() -> list[dict]:
    heads = {"heads": 32, "kv_heads": 8, "dim": 128, "dtype": "bf16", "layout": "token", "pad": 0, "mix": 1}
    turn = {"rotary": 128, "interleaved": False, "base": 500000.0}
    moe = {"hidden": 4096, "inter": 768, "experts": 128, "first": 0, "of": 128, "k": 8, "dtype": "bf16", "pad": 0, "act": "silu",
           "mix": 1}
    return [
        # decode, one token: its query, key and value out of one fused projection
        {"name": "append-1", "op": "append", "tokens": 1, "sequences": 1, "context": 2048, "page": 16, **heads, **turn},
        # prefill of 8192 tokens in four sequences at far positions, pages of 64
        {"name": "append-8192", "op": "append", "tokens": 8192, "sequences": 4, "context": 131072, "page": 64, **heads, **turn},
        # binary32, five heads of 80 of which 40 turn pairwise, pages of 7, some tokens padding
        {"name": "append-f32-ragged", "op": "append", "tokens": 1003, "sequences": 9, "context": 900, "page": 7, **heads,
         "heads": 10, "kv_heads": 5, "dim": 80, "dtype": "f32", "layout": "head", "pad": 5, "rotary": 40, "interleaved": True,
         "base": 10000.0},
        # decode, one user at 2000 tokens
        {"name": "attend-1", "op": "attend", "sequences": 1, "context": 2000, "ragged": False, "window": 0, "page": 16, **heads},
        # a decode batch of 64 users between nothing and 8192 tokens
        {"name": "attend-64", "op": "attend", "sequences": 64, "context": 8192, "ragged": True, "window": 0, "page": 16, **heads},
        # two users with 131072 tokens, pages of 64 by heads
        {"name": "attend-long", "op": "attend", "sequences": 2, "context": 131072, "ragged": False, "window": 0, "page": 64, **heads,
         "layout": "head"},
        # sixteen queries to a key head of 256, the last 1000 tokens of each user alone
        {"name": "attend-window", "op": "attend", "sequences": 48, "context": 6001, "ragged": True, "window": 1000, "page": 32, **heads,
         "kv_heads": 2, "dim": 256},
        # binary32, heads of 80, pages of 7
        {"name": "attend-f32-ragged", "op": "attend", "sequences": 37, "context": 1777, "ragged": True, "window": 0, "page": 7, **heads,
         "heads": 15, "kv_heads": 5, "dim": 80, "dtype": "f32", "pad": 5},
        # decode, one token: 8 of 128 experts
        {"name": "experts-1", "op": "experts", "tokens": 1, **moe},
        # the largest decode batch, nearly every expert is chosen
        {"name": "experts-64", "op": "experts", "tokens": 64, **moe},
        # a rank's quarter of the experts, 256 tokens of speculative decoding
        {"name": "experts-256-quarter", "op": "experts", "tokens": 256, **moe, "experts": 32, "first": 64},
        # binary32, odd sizes, 3 of 7 experts
        {"name": "experts-f32-ragged", "op": "experts", "tokens": 13, **moe, "hidden": 1001, "inter": 333, "experts": 7, "of": 7, "k": 3,
         "dtype": "f32", "pad": 3, "act": "gelu"},
    ]


def _log_int(rng, lo: int, hi: int, step: int = 8, odd: float = 0.5) -> int:
    """Log-uniform on [lo, hi]; a share of them odd, the others multiples of `step` where there is room for one."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    v = v - v % step if rng.random() >= odd and v >= step else v | 1
    return max(lo, min(hi, v))


def draw(rng) -> dict:
    op = rng.choice(["append", "attend", "attend", "attend", "experts", "experts", "experts"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    c = {"op": op, "dtype": dtype, "pad": rng.choice([0, 0, 8, rng.randint(1, 40)]), "mix": rng.randint(2, 1 << 20)}
    if op == "experts":
        of = rng.choice([8, 64, 128, rng.randint(2, 160)])
        experts = rng.choice([of, of, max(1, of // 4), rng.randint(1, of)])
        tokens = _log_int(rng, 1, 256)
        hidden = _log_int(rng, 64, 4096, 64, 0.25)
        # the plain form of many tokens runs every expert over all of them
        most = 256 * 32 * 768 * 4096
        inter = _log_int(rng, 16, max(17, min(2048, most // (hidden * max(experts * tokens, experts * 64)))), 16, 0.25)
        c |= {"tokens": tokens, "hidden": hidden, "inter": inter, "experts": experts, "first": rng.randint(0, of - experts),
              "of": of, "k": rng.randint(1, min(of, 10)), "act": rng.choice(["silu", "silu", "gelu"])}
        if not any(c["first"] <= e < c["first"] + experts for row in _chosen(c) for e in row):
            c |= {"experts": of, "first": 0}            # a rank that no token goes to has nothing to time
        return c
    dim = rng.choice([64, 128, 128, 128, 256, _log_int(rng, 16, 256)])
    kv = rng.choice([1, 2, 4, 8, rng.randint(1, 9)])
    c |= {"heads": kv * rng.choice([1, 2, 4, 8, rng.randint(1, 20)]), "kv_heads": kv, "dim": dim, "page": rng.choice([16, 32, 64, rng.randint(1, 128)]),
          "layout": rng.choice(["token", "token", "head"])}
    if op == "append":
        tokens = _log_int(rng, 1, max(2, min(8192, 8192 * 48 * 128 * 2 // ((c["heads"] + 2 * kv) * dim * _ELEM[dtype]))))
        return c | {"tokens": tokens, "sequences": min(tokens, _log_int(rng, 1, 64)), "context": _log_int(rng, 64, 131072), "base": rng.choice([1e4, 5e5, 1e6]),
                    "rotary": rng.choice([dim - dim % 2, dim - dim % 2, 2 * rng.randint(0, dim // 2)]), "interleaved": rng.random() < 0.4}
    sequences = _log_int(rng, 1, 256)
    return c | {"sequences": sequences, "ragged": rng.random() < 0.7, "window": rng.choice([0, 0, 0, _log_int(rng, 1, 4096)]),
                "context": _log_int(rng, 1, max(1, min(131072, _LARGEST_CACHE // (4 * sequences * kv * 2 * dim * _ELEM[dtype]))))}


# ---------------------------------------------------------------------------------------------------------------
# what a case's tokens are
# ---------------------------------------------------------------------------------------------------------------
def _lengths(c: dict) -> list[int]:
    """Tokens of each sequence: all `context`, or log-uniform below it with an empty one, one of a single token and a full one."""
    if not c["ragged"]:
        return [c["context"]] * c["sequences"]
    rng = random.Random(c["mix"])
    n = [int(round((c["context"] + 1.0) ** rng.random() * (0.5 if rng.random() < 0.5 else 1.0))) for _ in range(c["sequences"])]
    n[0] = c["context"]
    if len(n) > 4:
        n[1], n[2] = 0, 1
    return [max(0, min(c["context"], v)) for v in n]


def _visible(c: dict) -> int:
    return sum(min(n, c["window"] or n) for n in _lengths(c))


def _new_tokens(c: dict) -> tuple[list[int], list[int]]:
    """Sequence and position of each new token: equal runs of consecutive positions that end at the context; every tenth token
    of a padded case is padding, at position -1."""
    T, S = c["tokens"], c["sequences"]
    of = [i * S // T for i in range(T)]
    rng = random.Random(c["mix"])
    runs = [of.count(s) for s in range(S)]
    starts = [max(0, c["context"] - n - rng.randint(0, min(40, max(0, c["context"] - n)))) for n in runs]
    at, positions = list(starts), []
    for i, s in enumerate(of):
        positions.append(at[s] if not c["pad"] or i % 10 != 9 else -1)
        at[s] += 1
    return of, positions


def _chosen(c: dict) -> list[list[int]]:
    """The experts of each token, some liked better than others."""
    rng = random.Random(c["mix"])
    liked = [rng.random() for _ in range(c["of"])]
    return [sorted(range(c["of"]), key=lambda e: -(liked[e] * 0.5 + rng.random()))[: c["k"]] for _ in range(c["tokens"])]


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _rows(g, rows: int, cols: int, pad: int, dtype, scale: float = 1.0) -> torch.Tensor:
    """N(0, scale^2) rows inside rows that are `pad` elements wider."""
    return (torch.randn(rows, cols + pad, generator=g, device="cuda") * scale).to(dtype)[:, :cols]


def _cache(g, c: dict, pages: int) -> torch.Tensor:
    """pages x page x kv_heads x dim, whatever order it lies in; bf16 pages are made in their own type, which is quick."""
    shape = (pages, c["page"], c["kv_heads"], c["dim"]) if c["layout"] == "token" else (pages, c["kv_heads"], c["page"], c["dim"])
    t = torch.empty(shape, dtype=_TORCH[c["dtype"]], device="cuda").normal_(generator=g)
    return t if c["layout"] == "token" else t.transpose(1, 2)


def _table(g, pages_of: list[int], width: int) -> tuple[torch.Tensor, int]:
    """A page table whose pages lie in no order in a pool with a few spare ones; -1 where a sequence has no page."""
    total = sum(pages_of)
    pool = total + 3
    ids = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    n = torch.tensor(pages_of, device="cuda")
    first = torch.cumsum(n, 0) - n
    col = torch.arange(width, device="cuda")[None]
    at = (first[:, None] + col).clamp_(max=pool - 1)
    return torch.where(col < n[:, None], ids[at], -1).to(torch.int32).contiguous(), pool


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, dt, pad = case, _TORCH[case["dtype"]], case["pad"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = dict(case=case)
    if c["op"] == "append":
        T, nq, nk = c["tokens"], c["heads"] * c["dim"], c["kv_heads"] * c["dim"]
        of, positions = _new_tokens(c)
        s["sequence"], s["position"] = ints(of), ints(positions)
        # the pages of the new tokens alone: nothing reads what lies before them
        width = -(-(max(c["context"], max(positions) + 1)) // c["page"])
        low, high = {}, {}
        for p, o in zip(positions, of):
            if p >= 0:
                low[o], high[o] = min(low.get(o, p), p), max(high.get(o, p), p)
        first = [low.get(q, 0) // c["page"] for q in range(c["sequences"])]
        pages_of = [high[q] // c["page"] + 1 - first[q] if q in high else 0 for q in range(c["sequences"])]
        packed, pool = _table(g, pages_of, max(1, max(pages_of)))
        table = torch.full((c["sequences"], width), -1, dtype=torch.int32, device="cuda")
        for q in range(c["sequences"]):
            table[q, first[q]: first[q] + pages_of[q]] = packed[q, : pages_of[q]]
        s["table"] = table
        s["qkv"] = _rows(g, T, nq + 2 * nk, pad, dt)
        s["q_out"] = torch.zeros(T, nq, dtype=dt, device="cuda")
        s["inv_freq"] = (c["base"] ** (-torch.arange(0, c["rotary"], 2, dtype=torch.float64, device="cuda") / max(1, c["rotary"]))).float()
        s["k_cache"], s["v_cache"] = _cache(g, c, pool), _cache(g, c, pool)
    elif c["op"] == "attend":
        lengths = _lengths(c)
        pages_of = [-(-n // c["page"]) for n in lengths]
        s["table"], pool = _table(g, pages_of, max(1, max(pages_of)))
        s["lengths"] = ints(lengths)
        s["k_cache"], s["v_cache"] = _cache(g, c, pool), _cache(g, c, pool)
        s["q"] = _rows(g, c["sequences"], c["heads"] * c["dim"], pad, dt, 2.0)
        s["scale"] = c["dim"] ** -0.5
        s["out"] = torch.empty(c["sequences"], c["heads"] * c["dim"], dtype=dt, device="cuda")
        s["lse"] = torch.empty(c["sequences"], c["heads"], device="cuda")
    else:
        T, H, I, E = c["tokens"], c["hidden"], c["inter"], c["experts"]  # noqa: E741
        weight = lambda rows, cols: torch.empty(rows, cols, dtype=dt, device="cuda").normal_(0.0, cols ** -0.5, generator=g)  # noqa: E731
        s["gate_up"], s["down"] = weight(E * 2 * I, H), weight(E * H, I)
        s["x"] = _rows(g, T, H, pad, dt)
        s["indices"] = ints(_chosen(c))
        s["weights"] = torch.softmax(torch.randn(T, c["k"], generator=g, device="cuda"), dim=1)
        s["out"] = torch.empty(T, H + pad, dtype=dt, device="cuda")[:, :H]
    if own:
        _plan(s)
    return s


def _plan(s: dict) -> None:
    """The argument block that a program fills once per layer and passes with every call."""
    from paper_2607_08973_b200 import binding as sf
    c = s["case"]
    s["device"] = torch.cuda.current_device()
    dtype = sf.BF16 if c["dtype"] == "bf16" else sf.F32
    ptr = lambda t: t.data_ptr()  # noqa: E731
    if c["op"] == "experts":
        a = sf.make_experts(x=ptr(s["x"]), indices=ptr(s["indices"]), weights=ptr(s["weights"]), gate_up=ptr(s["gate_up"]),
                            down=ptr(s["down"]), out=ptr(s["out"]), tokens=c["tokens"], hidden=c["hidden"], inter=c["inter"],
                            experts=c["experts"], first_expert=c["first"], top_k=c["k"], dtype=dtype,
                            activation=sf.ACT_SILU if c["act"] == "silu" else sf.ACT_GELU, ld_x=s["x"].stride(0),
                            ld_out=s["out"].stride(0))
        s["call"], size = sf.sifar_experts, sf.sifar_experts_workspace(a)
    else:
        k, page = s["k_cache"], c["page"]
        cache = dict(k_cache=ptr(k), v_cache=ptr(s["v_cache"]), page_table=ptr(s["table"]), pages=k.shape[0], page_size=page,
                     max_pages=s["table"].shape[1], stride_page=k.stride(0), stride_token=k.stride(1), stride_head=k.stride(2),
                     sequences=c["sequences"], heads=c["heads"], kv_heads=c["kv_heads"], head_dim=c["dim"], dtype=dtype)
        if c["op"] == "append":
            nq, nk, ld = c["heads"] * c["dim"], c["kv_heads"] * c["dim"], s["qkv"].stride(0)
            q = s["qkv"]
            a = sf.make_append(q=ptr(q), k=ptr(q[:, nq:]), v=ptr(q[:, nq + nk:]), q_out=ptr(s["q_out"]), sequence=ptr(s["sequence"]),
                               position=ptr(s["position"]), inv_freq=ptr(s["inv_freq"]), tokens=c["tokens"], ld_q=ld, ld_k=ld, ld_v=ld,
                               rotary_dim=c["rotary"], interleaved=c["interleaved"], **cache)
            s["call"], size = sf.sifar_cache_append, 0
        else:
            a = sf.make_attention(q=ptr(s["q"]), out=ptr(s["out"]), lse=ptr(s["lse"]), lengths=ptr(s["lengths"]), scale=s["scale"],
                                  window=c["window"], ld_q=s["q"].stride(0), **cache)
            s["call"], size = sf.sifar_decode_attention, sf.sifar_decode_attention_workspace(a)
    if size:
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = ptr(s["workspace"]), size
    s["args"] = a


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _turn(x: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor, c: dict) -> torch.Tensor:
    """x: tokens x heads x dim in binary32; cos, sin: tokens x 1 x rotary / 2."""
    r = c["rotary"]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2: r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, x[..., r:]), dim=-1)


def _append(s: dict) -> dict:
    c, dt = s["case"], _TORCH[s["case"]["dtype"]]
    nq, nk = c["heads"] * c["dim"], c["kv_heads"] * c["dim"]
    q, k, v = s["qkv"].split((nq, nk, nk), dim=1)
    angle = (s["position"].double()[:, None] * s["inv_freq"].double()[None])[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    at = (s["position"] >= 0).nonzero()[:, 0]            # what is not padding
    q_out = _turn(q.float().unflatten(1, (-1, c["dim"])), cos, sin, c).to(dt).flatten(1)
    s["q_out"][at] = q_out[at]
    k = _turn(k.float().unflatten(1, (-1, c["dim"])), cos, sin, c).to(dt)
    page = s["table"][s["sequence"][at].long(), (s["position"][at] // c["page"]).long()].long()
    slot = (s["position"][at] % c["page"]).long()
    s["k_cache"][page, slot] = k[at]
    s["v_cache"][page, slot] = v.unflatten(1, (-1, c["dim"]))[at]
    return {"q_out": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend(s: dict) -> dict:
    c, dt = s["case"], _TORCH[s["case"]["dtype"]]
    n = s["lengths"].long()[:, None]
    first = (n - c["window"]).clamp_(min=0) if c["window"] else torch.zeros_like(n)
    most = min(c["context"], c["window"] or c["context"])
    j = first + torch.arange(most, device="cuda")[None]
    seen = j < n
    page = s["table"].gather(1, (j // c["page"]).clamp_(max=s["table"].shape[1] - 1)).long()
    page, slot = torch.where(seen, page, 0), torch.where(seen, j % c["page"], 0)
    k, v = s["k_cache"][page, slot].float(), s["v_cache"][page, slot].float()      # sequences x tokens x kv_heads x dim
    q = s["q"].float().reshape(c["sequences"], c["kv_heads"], -1, c["dim"])
    x = torch.einsum("shgd,sthd->shgt", q, k) * s["scale"]
    x = torch.where(seen[:, None, None], x, float("-inf"))
    top = x.amax(dim=3, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(dim=3, keepdim=True)
    out = torch.einsum("shgt,sthd->shgd", p, v) / torch.where(total == 0.0, 1.0, total)
    return {"out": out.to(dt).reshape(c["sequences"], -1), "lse": (top + torch.log(total)).reshape(c["sequences"], -1)}


def _act(g: torch.Tensor, kind: str) -> torch.Tensor:
    return g / (1.0 + torch.exp(-g)) if kind == "silu" else 0.5 * g * (1.0 + torch.erf(g * 0.5 ** 0.5))


def _experts(s: dict) -> dict:
    c, dt = s["case"], _TORCH[s["case"]["dtype"]]
    T, H, I, E = c["tokens"], c["hidden"], c["inter"], c["experts"]  # noqa: E741
    local = s["indices"].long() - c["first"]
    here = (local >= 0) & (local < E)
    w, local = torch.where(here, s["weights"], 0.0), local.clamp(0, E - 1)
    x, gate_up, down = s["x"].float(), s["gate_up"].view(E, 2 * I, H), s["down"].view(E, H, I)
    if T * c["k"] <= E:                                   # the chosen experts' weights alone
        gu = torch.einsum("tkih,th->tki", gate_up[local].float(), x)
        a = _act(gu[..., :I], c["act"]) * gu[..., I:] * w[..., None]
        return {"out": torch.einsum("tkhi,tki->th", down[local].float(), a).to(dt)}
    gu = torch.einsum("eih,th->tei", gate_up.float(), x)  # every expert, and 0 as the weight of those not chosen
    share = torch.zeros(T, E, device="cuda").scatter_add_(1, local, w)
    a = _act(gu[..., :I], c["act"]) * gu[..., I:] * share[..., None]
    return {"out": torch.einsum("ehi,tei->th", down.float(), a).to(dt)}


def run(s: dict):
    op = s["case"]["op"]
    if own:
        # on torch's current stream, as the plain form; torch.cuda.current_stream() makes an object each time (4 us)
        s["call"](s["args"], torch._C._cuda_getCurrentRawStream(s["device"]))
        return {n: s[n] for n in {"append": ("q_out", "k_cache", "v_cache"), "attend": ("out", "lse"), "experts": ("out",)}[op]}
    return _append(s) if op == "append" else _attend(s) if op == "attend" else _experts(s)


def work(case: dict) -> dict:
    c, es = case, _ELEM[case["dtype"]]
    if c["op"] == "append":
        T = sum(p >= 0 for p in _new_tokens(c)[1])
        n = T * (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        return {"bytes": 2 * es * n + 12 * T, "flops": 3 * T * (c["heads"] + c["kv_heads"]) * c["rotary"]}
    if c["op"] == "attend":
        n, rows = _visible(c), c["sequences"] * c["heads"]
        return {"bytes": es * (2 * n * c["kv_heads"] * c["dim"] + 2 * rows * c["dim"]) + 4 * (rows + n // c["page"]),
                "flops": 4 * n * c["heads"] * c["dim"]}
    here = [[e for e in row if c["first"] <= e < c["first"] + c["experts"]] for row in _chosen(c)]
    slots, active = sum(len(r) for r in here), len({e for r in here for e in r})
    return {"bytes": es * (3 * active * c["inter"] * c["hidden"] + 2 * c["tokens"] * c["hidden"]) + 8 * c["tokens"] * c["k"],
            "flops": 6 * slots * c["inter"] * c["hidden"]}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case: dict, seed: int):
    s = prepare(case, seed)
    c, d = case, lambda t: t.to(torch.float64)
    if c["op"] == "append":
        half, D = c["rotary"] // 2, c["dim"]
        # each pair is a complex number, turned by exp(i angle)
        pairs = torch.arange(2 * half, device="cuda").reshape((half, 2) if c["interleaved"] else (2, half))
        re, im = (pairs[:, 0], pairs[:, 1]) if c["interleaved"] else (pairs[0], pairs[1])
        spin = torch.polar(torch.ones(c["tokens"], half, dtype=torch.float64, device="cuda"),
                           torch.outer(d(s["position"]), d(s["inv_freq"])))
        rows = d(s["qkv"]).reshape(c["tokens"], -1, D)
        turned = rows[:, : c["heads"] + c["kv_heads"]].clone()
        z = torch.complex(turned[..., re], turned[..., im]) * spin[:, None]
        turned[..., re], turned[..., im] = z.real, z.imag
        out = {"q_out": d(s["q_out"]), "k_cache": d(s["k_cache"]), "v_cache": d(s["v_cache"])}
        keep = s["position"] >= 0
        out["q_out"][keep] = turned[keep, : c["heads"]].reshape(-1, c["heads"] * D)
        flat = s["table"].long().gather(1, torch.arange(s["table"].shape[1], device="cuda").expand_as(s["table"]))
        where = flat[s["sequence"].long()[keep], s["position"].long()[keep] // c["page"]] * c["page"] + s["position"].long()[keep] % c["page"]
        for name, rows in (("k_cache", turned[keep, c["heads"]:]), ("v_cache", rows[keep, c["heads"] + c["kv_heads"]:])):
            t = out[name].reshape(-1, c["kv_heads"], D)
            t[where] = rows
            out[name] = t.reshape(s[name].shape)
        return out
    if c["op"] == "attend":
        outs, lses = [], []
        group = c["heads"] // c["kv_heads"]
        for q, n in enumerate(_lengths(c)):
            j = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device="cuda")
            page, slot = s["table"][q].long()[j // c["page"]], j % c["page"]
            for h in range(c["kv_heads"]):
                k, v = d(s["k_cache"][page, slot, h]), d(s["v_cache"][page, slot, h])
                rows = d(s["q"][q, h * group * c["dim"]: (h + 1) * group * c["dim"]]).reshape(group, c["dim"])
                x = rows @ k.T * s["scale"]
                if n == 0:
                    outs.append(torch.zeros_like(rows))
                    lses.append(torch.full((group,), -float("inf"), dtype=torch.float64, device="cuda"))
                    continue
                outs.append(torch.softmax(x, dim=1) @ v)
                lses.append(torch.logsumexp(x, dim=1))
        return {"out": torch.cat(outs).reshape(c["sequences"], -1), "lse": torch.cat(lses).reshape(c["sequences"], -1)}
    # expert by expert, as the layer is defined
    I, H = c["inter"], c["hidden"]  # noqa: E741
    x, out = d(s["x"]), torch.zeros(c["tokens"], c["hidden"], dtype=torch.float64, device="cuda")
    for e in range(c["experts"]):
        t, j = (s["indices"] == e + c["first"]).nonzero(as_tuple=True)
        if len(t):
            gu = x[t] @ d(s["gate_up"][e * 2 * I: (e + 1) * 2 * I]).T
            g = gu[:, :I]
            a = (torch.nn.functional.silu(g) if c["act"] == "silu" else torch.nn.functional.gelu(g)) * gu[:, I:]
            out.index_add_(0, t, (a @ d(s["down"][e * H: (e + 1) * H]).T) * d(s["weights"][t, j])[:, None])
    return {"out": out}
