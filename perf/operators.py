"""Timed cases of the operators whose rows choose their weights.

Four operators of int8 inference with many experts or many adapters:
  route     scores of experts -> the chosen ids, their weights, and the slots in
            order of expert
  grouped   the experts' int8 products on the rows that chose them
  combine   the weighted sum of a token's slots
  adapters  a shared int8 projection with low-rank adapters of many requests

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges,
``prepare`` makes a case's device tensors, ``run`` is one call (the library's
where ``own`` is true, else the same in elementary torch operations), ``work``
the bytes and operations that call cannot do without, and ``exact`` the result
from the definition in float64.
"""
from __future__ import annotations

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ES = {"f32": 4, "bf16": 2, "f16": 2}


def _named(name, c):
    if name:
        c["name"] = name
    return c


def _route(name, tokens, experts, top_k, dtype, score, groups=1, top_groups=1, group_best=1,
           bias=False, renorm=True, scale=1.0, masked=False):
    return _named(name, {"op": "route", "tokens": tokens, "experts": experts, "top_k": top_k,
                         "dtype": dtype, "score": score, "groups": groups,
                         "top_groups": top_groups, "group_best": group_best, "bias": bias,
                         "renorm": renorm, "scale": scale, "masked": masked})


def _grouped(name, tokens, top_k, experts, n, k, dtype, scatter):
    return _named(name, {"op": "grouped", "tokens": tokens, "top_k": top_k, "experts": experts,
                         "n": n, "k": k, "dtype": dtype, "scatter": scatter})


def _combine(name, tokens, top_k, n, dtype, base):
    return _named(name, {"op": "combine", "tokens": tokens, "top_k": top_k, "n": n,
                         "dtype": dtype, "base": base})


def _adapters(name, rows, n, k, requests, adapters, rank, dtype, weights, plain_share):
    return _named(name, {"op": "adapters", "rows": rows, "n": n, "k": k, "requests": requests,
                         "adapters": adapters, "rank": rank, "dtype": dtype, "weights": weights,
                         "plain_share": plain_share})


def listed():
    return [
        # The router of one decode step of eight sequences: latency alone.
        _route("route_8x64", 8, 64, 8, "f32", "softmax"),
        # A prompt of 4096 tokens: sigmoid scores, a bias that balances the
        # load, the best 4 of 8 groups, 8 of 256 experts.
        _route("route_4096x256_groups", 4096, 256, 8, "f32", "sigmoid", groups=8, top_groups=4,
               group_best=2, bias=True, scale=2.5),
        # The largest batch of tokens, logits as a bf16 projection leaves them,
        # experts that a token may not take and padded tokens that take none.
        _route("route_16384x128_masked", 16384, 128, 8, "bf16", "softmax", masked=True),
        # One decode step of eight sequences through the experts' first
        # product: every chosen expert's weights are read for a row or two.
        _grouped("experts_decode_8of64_1024x2048", 8, 8, 64, 1024, 2048, "bf16", False),
        # 512 tokens through the second product: about 64 rows an expert, the
        # results written back to the tokens' slots.
        _grouped("experts_512tok_2048x1024", 512, 8, 64, 2048, 1024, "bf16", True),
        # A long prompt through the first product: bound by the matrix cores.
        _grouped("experts_4096tok_4096x2048", 4096, 8, 64, 4096, 2048, "bf16", False),
        # Few experts of odd sizes (pruned layers), rows at any byte address.
        _grouped("experts_ragged_777tok_1111x1777", 777, 2, 13, 1111, 1777, "f32", True),
        # One decode step's slots added up beside the shared expert's output.
        _combine("combine_16x8x4096", 16, 8, 4096, "bf16", True),
        # The same for a long prompt: one pass over the slots.
        _combine("combine_4096x8x4096", 4096, 8, 4096, "bf16", True),
        # One decode step of 16 requests, an adapter each, beside an attention
        # projection of a 7B-class decoder.
        _adapters("adapters_decode_16x4096x4096", 16, 4096, 4096, 16, 16, 16, "bf16", "bf16",
                  0.0),
        # Prompts of nine requests in one batch, some of them without adapter.
        _adapters("adapters_2048x4096x4096_r64", 2048, 4096, 4096, 9, 6, 64, "f16", "f16", 0.25),
        # A large batch through an MLP projection of the same decoder.
        _adapters("adapters_8192x11008x4096_r16", 8192, 11008, 4096, 40, 24, 16, "bf16", "bf16",
                  0.1),
    ]


# No drawn case has more than these (the largest listed ones do more).
_MAX_MACS = 5.0e10
_MAX_BYTES = 2.5e8


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi, step):
    """A size over the logarithm of the range: a multiple of step, or any."""
    v = _log(rng, lo, hi)
    return max(lo, v // step * step) if rng.random() < 0.65 else v


def draw(rng):
    op = rng.choice(["route", "grouped", "grouped", "combine", "adapters", "adapters"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log(rng, 2 if groups > 1 else 4, 512 // groups)
        top_groups = rng.randint(1, groups)
        top_k = rng.randint(1, max(1, min(16, experts * top_groups // groups)))
        tokens = max(1, min(_log(rng, 1, 16384), int(_MAX_BYTES / 8 / experts)))
        return _route(None, tokens, experts, top_k, rng.choice(["f32", "bf16", "f16"]),
                      rng.choice(["softmax", "sigmoid"]), groups, top_groups,
                      rng.choice([1, 2]), rng.random() < 0.5, rng.random() < 0.7,
                      rng.choice([1.0, 2.5]), rng.random() < 0.3)
    if op == "combine":
        top_k = rng.randint(1, 10)
        n = _size(rng, 64, 8192, 64)
        tokens = max(1, min(_log(rng, 1, 4096), int(_MAX_BYTES / (2 * n * top_k))))
        return _combine(None, tokens, top_k, n, rng.choice(["bf16", "f16", "f32"]),
                        rng.random() < 0.5)
    n, k = _size(rng, 128, 5000, 64), _size(rng, 128, 5000, 64)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "grouped":
        experts = max(2, min(_log(rng, 2, 128), int(_MAX_BYTES / (n * k))))
        top_k = rng.randint(1, min(8, experts))
        tokens = max(1, min(_log(rng, 1, 4096), int(_MAX_MACS / (float(n) * k * top_k))))
        return _grouped(None, tokens, top_k, experts, n, k, dtype, rng.random() < 0.5)
    rows = max(1, min(_log(rng, 1, 8192), int(_MAX_MACS / (float(n) * k))))
    requests = min(rows, _log(rng, 1, 64))
    adapters = rng.randint(1, min(32, requests))
    return _adapters(None, rows, n, k, requests, adapters,
                     rng.choice([4, 8, 16, 16, 24, 32, 64, 128]), dtype,
                     rng.choice(["bf16", "f16"]), rng.choice([0.0, 0.2]))


# ---- inputs -------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _ints(g, *shape):
    """int8 values as a symmetric quantisation leaves them."""
    return torch.empty(shape, dtype=torch.int8, device="cuda").random_(-127, 128, generator=g)


def _logits(g, case):
    # a router's logits: some experts are liked more by every token
    x = _randn(g, case["tokens"], case["experts"]) * 1.5 + _randn(g, case["experts"]) * 0.5
    return x


def _prepare_route(case, g):
    T, E = case["tokens"], case["experts"]
    logits = _logits(g, case)
    if case["masked"]:
        logits = logits.masked_fill(_rand(g, T, E) < 0.1, float("-inf"))
        logits = logits.masked_fill(_rand(g, T, 1) < 0.05, float("-inf"))  # padded tokens
    bias = _randn(g, E) * 0.1 if case["bias"] else None
    return {"logits": logits.to(_DT[case["dtype"]]), "bias": bias}


def _prepare_grouped(case, g):
    T, K, E, n, k = (case[x] for x in ("tokens", "top_k", "experts", "n", "k"))
    like = _randn(g, T, E) + 0.3 * _randn(g, E)
    ids = like.topk(K, dim=1).indices.flatten()
    by_expert, order = ids.sort(stable=True)
    counts = torch.bincount(by_expert, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    rows = T * K
    return {"A": _ints(g, rows if case["scatter"] else T, k), "B": _ints(g, E, k, n),
            "scale_a": 0.005 + 0.01 * _rand(g, rows if case["scatter"] else T),
            "scale_b": 0.001 + 0.002 * _rand(g, E, n),
            "offsets": offsets, "order": order.int(), "most": int(counts.max()),
            "out": torch.zeros(rows, n, dtype=_DT[case["dtype"]], device="cuda")}


def _prepare_combine(case, g):
    T, K, n = case["tokens"], case["top_k"], case["n"]
    dt = _DT[case["dtype"]]
    w = _rand(g, T, K)
    return {"Z": _randn(g, T * K, n).to(dt), "weights": w / w.sum(1, keepdim=True),
            "ids": torch.where(_rand(g, T, K) < 0.03, -1, 1).int(),
            "base": _randn(g, T, n).to(dt) if case["base"] else None,
            "out": torch.zeros(T, n, dtype=dt, device="cuda")}


def _prepare_adapters(case, g):
    m, n, k, N, r = (case[x] for x in ("rows", "n", "k", "adapters", "rank"))
    R = case["requests"]
    wt = _DT[case["weights"]]
    # ragged requests, one after the other in the batch; a request's rows share
    # its adapter
    cuts = torch.cat([torch.zeros(1, device="cuda"), _rand(g, R - 1).sort().values]) * m
    request = torch.searchsorted(cuts, torch.arange(m, device="cuda") + 0.5) - 1
    if R == m:
        request = torch.arange(m, device="cuda")
    which = torch.empty(R, dtype=torch.int64, device="cuda").random_(0, N, generator=g)
    if R == N:
        which = torch.rand(R, generator=g, device="cuda").argsort()
    which = torch.where(_rand(g, R) < case["plain_share"], -1, which)
    return {"A": _ints(g, m, k), "B": _ints(g, k, n),
            "scale_a": 0.005 + 0.01 * _rand(g, m), "scale_b": 0.001 + 0.002 * _rand(g, n),
            "ids": which[request].int(), "down": (_randn(g, N, r, k) * k ** -0.5).to(wt),
            "up": (_randn(g, N, n, r) * 0.3 * r ** -0.5).to(wt),
            "scaling": 0.5 + _rand(g, N),
            "out": torch.zeros(m, n, dtype=_DT[case["dtype"]], device="cuda")}


def prepare(case, seed):
    make = {"route": _prepare_route, "grouped": _prepare_grouped, "combine": _prepare_combine,
            "adapters": _prepare_adapters}[case["op"]]
    return {"case": dict(case), **make(case, _gen(seed))}


# ---- the library's calls --------------------------------------------------------

def _own(state):
    import paper_2302_07594_amd as ig
    c = state["case"]
    if c["op"] == "route":
        return ig.route(state["logits"], c["top_k"], bias=state["bias"], groups=c["groups"],
                        top_groups=c["top_groups"], group_best=c["group_best"],
                        score=c["score"], renormalise=c["renorm"], scale=c["scale"])
    if c["op"] == "grouped":
        return ig.grouped_i8(state["A"], state["B"], state["offsets"], state["order"],
                             scale_a=state["scale_a"], scale_b=state["scale_b"],
                             slots=0 if c["scatter"] else c["top_k"], scatter=c["scatter"],
                             out=state["out"])
    if c["op"] == "combine":
        return ig.combine(state["Z"], state["weights"], ids=state["ids"], base=state["base"],
                          out=state["out"])
    return ig.adapters_i8(state["A"], state["B"], state["ids"], state["down"], state["up"],
                          scale_a=state["scale_a"], scale_b=state["scale_b"],
                          scaling=state["scaling"], out=state["out"])


# ---- the plain forms -------------------------------------------------------------

def _plain_route(state):
    c = state["case"]
    T, E, K, G = c["tokens"], c["experts"], c["top_k"], c["groups"]
    # in 64 bits: an expert next to the border of the chosen ones must not change
    # sides
    x = state["logits"].double()
    if c["score"] == "softmax":
        top = x.max(dim=1, keepdim=True).values
        e = torch.exp(x - torch.where(top.isinf(), 0.0, top))
        total = e.sum(dim=1, keepdim=True)
        s = e / torch.where(total > 0, total, 1.0)
    else:
        s = 1.0 / (1.0 + torch.exp(-x))
    key = s if state["bias"] is None else s + state["bias"].double()
    key = key.masked_fill(x == float("-inf"), float("-inf"))
    if G > 1:
        by = key.view(T, G, E // G).sort(dim=2, descending=True).values[:, :, :c["group_best"]]
        score = by[:, :, 0]
        if by.shape[2] > 1:
            score = score + torch.where(by[:, :, 1].isinf(), 0.0, by[:, :, 1])
        best = score.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        kept = torch.zeros(T, G, dtype=torch.bool, device=x.device).scatter_(1, best, True)
        key = key.masked_fill(~kept.repeat_interleave(E // G, dim=1), float("-inf"))
    by, ids = key.sort(dim=1, descending=True, stable=True)
    ids, some = ids[:, :K], by[:, :K] > float("-inf")
    w = s.gather(1, ids) * some
    if c["renorm"]:
        total = w.sum(dim=1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    w = (w * c["scale"]).float()
    ids = torch.where(some, ids, -1).int()
    expert, order = torch.where(some, ids, E).flatten().sort(stable=True)
    offsets = torch.searchsorted(expert, torch.arange(E + 1, device=x.device)).int()
    order = torch.where(expert < E, order, -1).int()
    return ids, w, offsets, order


def _plain_grouped(state):
    c = state["case"]
    E, K, k, n = c["experts"], c["top_k"], c["k"], c["n"]
    order = state["order"].long()
    at = torch.arange(order.numel(), device="cuda")
    expert = torch.searchsorted(state["offsets"], at.int(), right=True) - 1
    place = at - state["offsets"][expert]
    src = at if c["scatter"] else order // K
    x = torch.zeros(E, state["most"], k, device="cuda")
    x[expert, place] = state["A"].float()[src]
    y = torch.bmm(x, state["B"].float())[expert, place]
    y = y * state["scale_a"][src][:, None] * state["scale_b"][expert]
    if not c["scatter"]:
        return y.to(_DT[c["dtype"]])
    out = torch.empty_like(y)
    out[order] = y
    return out.to(_DT[c["dtype"]])


def _plain_combine(state):
    c = state["case"]
    T, K, n = c["tokens"], c["top_k"], c["n"]
    w = torch.where(state["ids"] >= 0, state["weights"], 0.0)
    y = (state["Z"].float().view(T, K, n) * w[:, :, None]).sum(dim=1)
    if state["base"] is not None:
        y = y + state["base"].float()
    return y.to(_DT[c["dtype"]])


def _plain_adapters(state):
    c = state["case"]
    n, k, N, r = c["n"], c["k"], c["adapters"], c["rank"]
    x = state["A"].float() * state["scale_a"][:, None]
    y = (state["A"].float() @ state["B"].float()) * state["scale_a"][:, None] * state["scale_b"]
    # all adapters side by side; a row keeps its own one's part
    u = (x @ state["down"].float().view(N * r, k).t()).view(-1, N, r)
    mine = state["ids"][:, None] == torch.arange(N, device="cuda")
    u = (u * (mine * state["scaling"])[:, :, None]).view(-1, N * r)
    y = y + u @ state["up"].float().permute(0, 2, 1).reshape(N * r, n)
    return y.to(_DT[c["dtype"]])


def run(state):
    if own:
        return _own(state)
    plain = {"route": _plain_route, "grouped": _plain_grouped, "combine": _plain_combine,
             "adapters": _plain_adapters}[state["case"]["op"]]
    return plain(state)


# ---- what a call cannot do without ------------------------------------------------

def work(case):
    es = _ES[case["dtype"]]
    if case["op"] == "route":
        T, E, K = case["tokens"], case["experts"], case["top_k"]
        return {"bytes": T * E * es + (4 * E if case["bias"] else 0) + 12 * T * K + 4 * (E + 1),
                "flops": T * E * 4}
    if case["op"] == "combine":
        T, K, n = case["tokens"], case["top_k"], case["n"]
        return {"bytes": T * n * es * (K + 1 + (1 if case["base"] else 0)) + 8 * T * K,
                "flops": 2 * T * K * n}
    n, k = case["n"], case["k"]
    if case["op"] == "grouped":
        T, K, E = case["tokens"], case["top_k"], case["experts"]
        rows = T * K
        used = E * (1.0 - (1.0 - K / E) ** T)  # experts that some token chose, on average
        return {"bytes": int((rows if case["scatter"] else T) * (k + 4) + used * n * (k + 4) +
                             rows * (n * es + 4)),
                "flops": 2 * rows * n * k}
    m, N, r = case["rows"], case["adapters"], case["rank"]
    return {"bytes": m * (k + 8) + n * (k + 4) + N * r * (k + n) * 2 + m * n * es,
            "flops": 2 * m * n * k + 2 * m * r * (n + k)}


# ---- from the definition, in float64 -----------------------------------------------

def _exact_route(case, state):
    import numpy as np
    T, E, K, G = case["tokens"], case["experts"], case["top_k"], case["groups"]
    size = E // G
    x = state["logits"].double().cpu().numpy()
    bias = None if state["bias"] is None else state["bias"].double().cpu().numpy()
    ids = np.full((T, K), -1, np.int32)
    w = np.zeros((T, K))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        if case["score"] == "softmax":
            e = np.exp(x - np.max(np.where(np.isinf(x), -1e300, x), axis=1)[:, None])
            total = e.sum(1, keepdims=True)
            s = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
        else:
            s = 1.0 / (1.0 + np.exp(-x))
    s = np.where(np.isinf(x), 0.0, s)
    key = np.where(np.isinf(x), -np.inf, s if bias is None else s + bias)
    if G > 1:
        g = -np.sort(-key.reshape(T, G, size), axis=2)
        total = g[:, :, 0].copy()
        if case["group_best"] == 2 and size > 1:
            total += np.where(np.isinf(g[:, :, 1]), 0.0, g[:, :, 1])
        best = np.argsort(-total, axis=1, kind="stable")[:, :case["top_groups"]]
        keep = np.zeros((T, G), bool)
        np.put_along_axis(keep, best, True, axis=1)
        key = np.where(np.repeat(keep, size, axis=1), key, -np.inf)
    best = np.argsort(-key, axis=1, kind="stable")[:, :K]
    ok = np.take_along_axis(key, best, axis=1) > -np.inf
    ids[ok] = best[ok]
    w[ok] = np.take_along_axis(s, best, axis=1)[ok]
    if case["renorm"]:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    flat = ids.ravel()
    slots = [np.flatnonzero(flat == e) for e in range(E)]
    offsets = np.concatenate([[0], np.cumsum([len(v) for v in slots])]).astype(np.int32)
    order = np.full(T * K, -1, np.int32)
    order[:offsets[-1]] = np.concatenate(slots)
    return ids, w * case["scale"], offsets, order


def _exact_grouped(case, state):
    cuts = state["offsets"].tolist()
    order = state["order"].long()
    out = torch.zeros(order.numel(), case["n"], dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        lo, hi = cuts[e], cuts[e + 1]
        if lo == hi:
            continue
        slot = order[lo:hi]
        src = torch.arange(lo, hi, device="cuda") if case["scatter"] else \
            torch.div(slot, case["top_k"], rounding_mode="floor")
        y = state["A"][src].double() @ state["B"][e].double()
        y = y * state["scale_a"][src].double()[:, None] * state["scale_b"][e].double()[None, :]
        out[slot if case["scatter"] else slice(lo, hi)] = y
    return out


def _exact_combine(case, state):
    T, K = case["tokens"], case["top_k"]
    out = torch.zeros(T, case["n"], dtype=torch.float64, device="cuda") \
        if state["base"] is None else state["base"].double()
    for j in range(K):
        used = (state["ids"][:, j] >= 0)[:, None]
        z = state["Z"][j::K].double() * state["weights"][:, j:j + 1].double()
        out = torch.where(used, out + z, out)
    return out


def _exact_adapters(case, state):
    sa = state["scale_a"].double()[:, None]
    a = state["A"].double()
    out = (a @ state["B"].double()) * sa * state["scale_b"].double()[None, :]
    for which in state["ids"].unique().tolist():
        if which < 0:
            continue
        rows = (state["ids"] == which).nonzero().flatten()
        u = (a[rows] @ state["down"][which].double().t()) * sa[rows]
        out[rows] += (u @ state["up"][which].double().t()) * state["scaling"][which].double()
    return out


def exact(case, seed):
    f = {"route": _exact_route, "grouped": _exact_grouped, "combine": _exact_combine,
         "adapters": _exact_adapters}[case["op"]]
    got = f(case, prepare(case, seed))
    return tuple(got) if isinstance(got, tuple) else got
