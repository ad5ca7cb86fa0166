"""Operators of a sparse layer with 4-bit experts, as timed cases: the router and the plan that puts tokens in the order of their experts, the
experts' products up (gate and up with the activation) and down (joined by the router's weights), and the norms before and after a block
with its gate and residual scale.

`kind` says which operator a case takes:
  route    scores of the experts, the choice of k of them, their weights; the plan of the products
  up       h = silu(G_e x) * (U_e x) for every pair of a token and one of its experts, in the order of the experts
  down     y = sum over a token's experts of weight * (W_e h)
  norm     r' = r + scale * gate * norm(y), and the norm of r'

Experts' weights are DialectFP4 (blocks of 32 along the contraction), and x and h are quantized to it within the products, block by block, as
everywhere in this library.  The plain forms take the values that the weights' codes stand for.
"""
import math

import torch

own = False

# half-unit magnitudes of the 16 dialects (value = 0.5 u)
BOOK = [
    [0, 1, 2, 3, 4, 6, 12, 15], [0, 1, 2, 3, 4, 6, 10, 15], [0, 1, 2, 3, 4, 6, 11, 14], [0, 1, 2, 3, 4, 6, 9, 14],
    [0, 1, 2, 3, 4, 6, 10, 13], [0, 1, 2, 3, 4, 6, 8, 13], [0, 1, 2, 3, 4, 6, 9, 12], [0, 1, 2, 3, 4, 6, 8, 12],
    [0, 1, 2, 3, 4, 6, 9, 11], [0, 1, 2, 3, 4, 6, 8, 11], [0, 1, 2, 3, 4, 6, 8, 10], [0, 1, 2, 3, 4, 6, 7, 10],
    [0, 1, 2, 3, 4, 6, 8, 9], [0, 1, 2, 3, 4, 6, 7, 9], [0, 1, 2, 3, 4, 6, 7, 8], [0, 1, 2, 3, 4, 5, 6, 8],
]
BITS = 4.5                                  # of a weight: code, and a dialect and an exponent byte for 32


def _route(tokens, experts, k, **more):
    return dict(dict(kind="route", tokens=tokens, experts=experts, k=k, score="softmax", bias=False, groups=1, kept=1, best=1, renormalize=True, scale=1.0,
                     half=False), **more)


def _up(tokens, experts, k, dim, inner, **more):
    return dict(dict(kind="up", tokens=tokens, experts=experts, k=k, dim=dim, inner=inner), **more)


def _down(tokens, experts, k, dim, inner, **more):
    return dict(dict(kind="down", tokens=tokens, experts=experts, k=k, dim=dim, inner=inner), **more)


def _norm(tokens, dim, **more):
    return dict(dict(kind="norm", tokens=tokens, dim=dim, post=True, gate="none", scale=1.0, wide=False), **more)


def listed():
    return [
        # one token: latency alone
        _route(1, 128, 8, name="route_1_token"),
        # an odd batch, sigmoid scores with a bias for balance, the best 3 of 8 groups by their two largest
        _route(777, 160, 6, score="sigmoid", bias=True, groups=8, kept=3, best=2, scale=2.5, name="route_groups"),
        # prompts of 16384 tokens
        _route(16384, 256, 8, half=True, name="route_prompt"),
        # one token through 8 of 128 experts: the weights' way from memory, and latency
        _up(1, 128, 8, 2048, 1024, name="up_1_token"),
        # an odd batch, odd numbers of blocks, more experts than fit the tokens evenly
        _up(333, 40, 5, 1440, 736, name="up_ragged"),
        # 64 sequences' tokens through 2 of 8 large experts: all weights are read for a few rows each
        _up(64, 8, 2, 4096, 14336, name="up_batch"),
        # a prompt of 4096 tokens through 8 of 64 experts
        _up(4096, 64, 8, 2048, 1024, name="up_prompt"),
        _down(1, 128, 8, 2048, 1024, name="down_1_token"),
        _down(333, 40, 5, 1440, 736, name="down_ragged"),
        _down(4096, 64, 8, 2048, 1024, name="down_prompt"),
        # an odd batch of odd rows, gates by token, the residual in f32
        _norm(333, 1448, gate="token", scale=0.7, wide=True, name="norm_ragged"),
        # a prompt of 8192 tokens
        _norm(8192, 4096, name="norm_prompt"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["route", "up", "up", "down", "down", "norm"])
    if kind == "norm":
        dim = 8 * spread(8, 2048)
        return _norm(min(spread(1, 16384), 8192 * 4096 // dim), dim, post=rng.random() < 0.7, gate=rng.choice(["none", "all", "token"]), scale=rng.choice([1.0, 0.5]),
                     wide=rng.random() < 0.3)
    experts = rng.choice([8, 16, 40, 64, 96, 128, 160, 256])
    k = rng.choice([1, 2, 4, 5, 6, 8])
    if kind == "route":
        groups = rng.choice([1, 1, 4, 8])
        kept = rng.randint(-(-groups // 2), groups)
        size = experts // groups
        return _route(min(spread(1, 16384), 16384 * 256 // experts), experts, min(k, kept * size), score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups,
                      kept=kept, best=1 if size < 2 else rng.choice([1, 2]), renormalize=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]), half=rng.random() < 0.5)
    dim = 32 * spread(4, 160)
    inner = 32 * min(spread(2, 448), 8 * 4096 * 448 // (experts * dim))
    tokens = min(spread(1, 4096), 4096 * 8 * 2048 * 1024 // (k * dim * inner))
    return (_up if kind == "up" else _down)(max(1, tokens), experts, k, dim, inner)


def work(case):
    t = case["tokens"]
    if case["kind"] == "norm":
        each = t * case["dim"]
        return {"bytes": each * (2 + 2 * (4 if case["wide"] else 2) + 2 + (2 if case["gate"] == "token" else 0)), "flops": 12 * each}
    e, k = case["experts"], case["k"]
    if case["kind"] == "route":
        return {"bytes": t * e * (2 if case["half"] else 4) + 16 * t * k, "flops": 10 * t * e}
    active = e * (1.0 - (1.0 - k / e) ** t)                                # experts that a token goes to, were all alike
    one = case["dim"] * case["inner"]
    parts = 2 if case["kind"] == "up" else 1
    return {"bytes": int(parts * active * one * BITS / 8) + 2 * t * case["dim"] + 2 * t * k * case["inner"], "flops": 2 * parts * t * k * one}


# ---- DialectFP4 -------------------------------------------------------------------------------------------------------------

def _tables(device):
    """For a 5-bit magnitude t (quarter units): the index of the nearest half-unit value of every dialect, halfway up, and the vote of every
    pair of dialects (+1: in the even one's range, -1: in the odd one's)."""
    book, t = torch.tensor(BOOK), torch.arange(32)
    index = (t[None, :, None] >= (book[:, None, :-1] + book[:, None, 1:])).sum(-1)                  # [16, 32]
    both = torch.cat([book[0::2], book[1::2]], 1).sort(1).values                                      # [8, 16]
    at = t[None, :, None] >= (both[:, None, :-1] + both[:, None, 1:])
    nearest = torch.gather(both, 1, at.sum(-1))
    even = (nearest[:, :, None] == book[0::2, None, :]).any(-1).int()
    odd = (nearest[:, :, None] == book[1::2, None, :]).any(-1).int()
    return index.to(device), (even - odd).to(device), book.float().to(device)


def _code(x, tables):
    """index and sign of the elements, dialect and exponent of the blocks, of x [..., 32] float32."""
    index, vote, _ = tables
    size = x.abs()
    top = size.amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, -127)
    t = torch.floor(torch.ldexp(size, 2 - e)).to(torch.int32)
    pair = 15 - torch.div(t.amax(-1, keepdim=True) + 1, 2, rounding_mode="floor").clamp(8, 15)
    dialect = 2 * pair + (vote[pair, t].sum(-1, keepdim=True) < 0)
    return index[dialect, t], torch.signbit(x), dialect, e


def _values(i, sign, dialect, e, tables):
    v = torch.ldexp(tables[2][dialect, i], e - 1)
    return torch.where(sign, -v, v)


def _stands_for(x, tables):
    """The DialectFP4 values of x [rows, K], float32."""
    return _values(*_code(x.float().unflatten(-1, (-1, 32)), tables), tables).flatten(-2)


# ---- plain forms ------------------------------------------------------------------------------------------------------------

def _best(score, k):
    """The k largest of the last dimension, equal ones by index."""
    return torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :k]


def _plain_route(s):
    c = s["case"]
    x = s["logits"].double()                                                  # (choices lie next to each other)
    if c["score"] == "softmax":
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
    else:
        p = 1.0 / (1.0 + torch.exp(-x))
    choice = p + s["bias"].double() if c["bias"] else p
    if c["groups"] > 1:
        by_group = choice.unflatten(-1, (c["groups"], -1))
        total = torch.sort(by_group, dim=-1, descending=True).values[..., :c["best"]].sum(-1)
        stays = torch.zeros_like(total, dtype=torch.bool).scatter_(-1, _best(total, c["kept"]), True)
        choice = torch.where(stays[..., None], by_group, -math.inf).flatten(-2)
    ids = _best(choice, c["k"])
    w = torch.gather(p, -1, ids)
    if c["renormalize"]:
        w = w / w.sum(-1, keepdim=True)
    flat = ids.flatten()
    order = torch.sort(flat, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    offsets = (flat[None, :] < torch.arange(c["experts"] + 1, device=flat.device)[:, None]).sum(-1)
    return ids.int(), (w * c["scale"]).float(), offsets.int(), order.int(), place.int()


def _plain_up(s):
    c, at = s["case"], s["offsets"]
    x = _stands_for(s["x"], s["tables"])
    h = torch.empty((c["tokens"] * c["k"], c["inner"]), dtype=torch.bfloat16, device=x.device)
    for e in range(c["experts"]):
        if at[e + 1] > at[e]:
            rows = x[s["order"][at[e]:at[e + 1]] // c["k"]]
            g, u = rows @ s["gate"][e].T, rows @ s["up"][e].T
            h[at[e]:at[e + 1]] = (g / (1.0 + torch.exp(-g)) * u).to(torch.bfloat16)
    return h


def _plain_down(s):
    c, at = s["case"], s["offsets"]
    h = _stands_for(s["h"], s["tables"])
    y = torch.empty((c["tokens"] * c["k"], c["dim"]), device=h.device)
    for e in range(c["experts"]):
        if at[e + 1] > at[e]:
            y[s["order"][at[e]:at[e + 1]]] = h[at[e]:at[e + 1]] @ s["down"][e].T
    return (y.unflatten(0, (-1, c["k"])) * s["weights"][..., None]).sum(1).to(torch.bfloat16)


def _plain_norm(s):
    z = s["y"].float()
    if s["post"] is not None:
        z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + s["eps"]) * s["post"]
    if s["gate"] is not None:
        z = z * s["gate"].float()
    r = s["residual"].float() + s["case"]["scale"] * z
    n = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + s["eps"]) * s["weight"]
    return r.to(s["residual"].dtype), n.to(torch.bfloat16)


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _normal(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * std


def _with_outliers(g, rows, dim, factor=20.0):
    """bf16 [rows, dim], N(0, 1) with one channel of 200 that stands out for every row."""
    x = _normal(g, rows, dim)
    x[:, torch.randperm(dim, generator=g, device="cuda")[:-(-dim // 200)]] *= factor
    return x.to(torch.bfloat16)


def _inputs(case, seed):
    """The inputs of a case but for the experts' weights, as the plain forms and `exact` take them; the generator."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case, "eps": 1e-6}
    t = case["tokens"]
    if case["kind"] == "norm":
        dim = case["dim"]
        s["y"], s["residual"] = _with_outliers(g, t, dim), _normal(g, t, dim, std=3.0).to(torch.float32 if case["wide"] else torch.bfloat16)
        s["post"], s["weight"] = 1.0 + _normal(g, dim, std=0.2) if case["post"] else None, 1.0 + _normal(g, dim, std=0.2)
        s["gate"] = None if case["gate"] == "none" else _normal(g, *((dim,) if case["gate"] == "all" else (t, dim)), std=0.5).to(torch.bfloat16)
        return s, g
    # some experts are more popular than others
    logits = _normal(g, t, case["experts"], std=1.5) + _normal(g, case["experts"], std=0.7)
    if case["kind"] == "route":
        s["logits"] = logits.to(torch.bfloat16) if case["half"] else logits
        s["bias"] = _normal(g, case["experts"], std=0.05) if case["bias"] else None
        return s, g
    s["ids"] = _best(logits, case["k"]).int().contiguous()
    flat = s["ids"].flatten()
    s["order"] = torch.sort(flat, stable=True).indices
    s["offsets"] = [0] + torch.bincount(flat.long(), minlength=case["experts"]).cumsum(0).tolist()
    if case["kind"] == "up":
        s["x"] = _with_outliers(g, t, case["dim"])
    else:
        a = _normal(g, t * case["k"], case["inner"])
        s["h"] = (a / (1.0 + torch.exp(-a)) * _normal(g, t * case["k"], case["inner"])).to(torch.bfloat16)
        w = torch.rand(t, case["k"], generator=g, device="cuda") + 0.05
        s["weights"] = w / w.sum(-1, keepdim=True)
    return s, g


def _weights(case, g, rows, K, tables):
    """An expert's DialectFP4 weights after the other: (codes, dialects, exponent bytes) [rows, ...]."""
    for _ in range(case["experts"]):
        i, sign, dialect, e = _code(_normal(g, rows, K, std=0.02).to(torch.bfloat16).float().unflatten(-1, (-1, 32)), tables)
        code = (i + 8 * sign).to(torch.uint8).flatten(-2)
        yield code[:, 0::2] | code[:, 1::2] << 4, dialect.squeeze(-1).to(torch.uint8), (e + 127).squeeze(-1).to(torch.uint8)


def _stand_for(weights, tables):
    """The values of one expert's weights, float32."""
    codes, dialect, exponent = weights
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, 32)).int()
    return _values(code & 7, code >= 8, dialect.int()[..., None], exponent.int()[..., None] - 127, tables).flatten(-2)


def _parts(case):
    """The experts' matrices of a case: name, rows, contraction."""
    return [("gate", case["inner"], case["dim"]), ("up", case["inner"], case["dim"])] if case["kind"] == "up" else [("down", case["dim"], case["inner"])]


def prepare(case, seed):
    """Inputs; experts' weights (as the library lays them out, or the values that they stand for); the plan of the router's choice."""
    s, g = _inputs(case, seed)
    if case["kind"] in ("route", "norm"):
        return s
    tables = _tables("cuda")
    if own:
        from paper_2501_01144_amd import dfp4
        q = []
        for _, rows, K in _parts(case):
            codes, dialect, exponent = (torch.cat(x) for x in zip(*_weights(case, g, rows, K, tables)))
            q.append(dfp4.QTensor(codes, dialect, exponent, rows * case["experts"], K))
        s["experts"] = dfp4.expert_weights(q[0], case["experts"], up=q[1] if len(q) > 1 else None)
        s["plan"] = dfp4.expert_plan(s["ids"], case["experts"])
    else:
        s["tables"] = tables
        for name, rows, K in _parts(case):
            s[name] = torch.empty((case["experts"], rows, K), device="cuda")
            for e, w in enumerate(_weights(case, g, rows, K, tables)):
                s[name][e] = _stand_for(w, tables)
    return s


def run(s):
    c = s["case"]
    if own:
        from paper_2501_01144_amd import dfp4
        if c["kind"] == "route":
            ids, weights = dfp4.route(s["logits"], c["k"], score=c["score"], bias=s["bias"], groups=c["groups"], kept=c["kept"], best=c["best"],
                                      renormalize=c["renormalize"], scale=c["scale"])
            plan = dfp4.expert_plan(ids, c["experts"])
            return ids, weights, plan.offsets, plan.order, plan.place
        if c["kind"] == "up":
            return dfp4.experts_up(s["x"], s["plan"], s["experts"])
        if c["kind"] == "down":
            return dfp4.experts_down(s["h"], s["plan"], s["experts"], s["weights"])
        return dfp4.add_norm(s["y"], s["residual"], s["weight"], post_weight=s["post"], gate=s["gate"], scale=c["scale"], eps=s["eps"])
    return {"route": _plain_route, "up": _plain_up, "down": _plain_down, "norm": _plain_norm}[c["kind"]](s)


# ---- in 64 bits, from the definitions -----------------------------------------------------------------------------------------

def _exact_blocks(x):
    """The quantizer of blocks x [..., 32] in real arithmetic."""
    rows = torch.tensor(BOOK, dtype=torch.float64, device="cuda") / 2
    # a dialect's own value (the one that the other of its pair lacks) and the cell that it has among the values of both
    cells = []
    for d in range(16):
        mine = sorted(set(BOOK[d]) - set(BOOK[d ^ 1]))[0]
        both = sorted(set(BOOK[d]) | set(BOOK[d ^ 1]))
        i = both.index(mine)
        cells.append(((both[i - 1] + mine) / 4, (mine + both[i + 1]) / 4))
    cells = torch.tensor(cells, dtype=torch.float64, device="cuda")
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2)
    size = x.abs() / unit
    peak = (torch.floor(2 * size.amax(-1, keepdim=True) + 0.5) / 2).clamp(4.0, 7.5)
    even = (2 * (15 - 2 * peak)).long()
    count = [((size >= cells[even + o][..., 0]) & (size < cells[even + o][..., 1])).sum(-1, keepdim=True) for o in (0, 1)]
    row = rows[(even + (count[1] > count[0])).squeeze(-1)]                       # [..., 8]
    found = row[..., :1].expand_as(size).clone()
    for j in range(1, 8):
        v = row[..., j:j + 1]
        found = torch.where((v - size).abs() <= (found - size).abs(), v.expand_as(size), found)
    return torch.sign(x) * found * unit


def _exact_weights(weights):
    """The values of one expert's codes, 64 bits."""
    codes, dialect, exponent = weights
    rows = torch.tensor(BOOK, dtype=torch.float64, device="cuda") / 2
    both = torch.stack([torch.remainder(codes, 16), torch.div(codes, 16, rounding_mode="floor")], -1).reshape(codes.shape[0], -1, 32).long()
    size = torch.gather(rows[dialect.long()], -1, both % 8) * torch.exp2(exponent.double() - 127)[..., None]
    return (size * (1 - 2 * (both // 8))).reshape(codes.shape[0], -1)


def exact(case, seed):
    s, g = _inputs(case, seed)
    if case["kind"] == "norm":
        z = s["y"].double()
        if s["post"] is not None:
            z = z / (z.square().sum(-1, keepdim=True) / case["dim"] + s["eps"]).sqrt() * s["post"].double()
        if s["gate"] is not None:
            z = z * s["gate"].double()
        r = s["residual"].double() + case["scale"] * z
        return r, r / (r.square().sum(-1, keepdim=True) / case["dim"] + s["eps"]).sqrt() * s["weight"].double()
    if case["kind"] == "route":
        x = s["logits"].double()
        p = torch.softmax(x, -1) if case["score"] == "softmax" else torch.sigmoid(x)
        c = p + s["bias"].double() if case["bias"] else p.clone()
        if case["groups"] > 1:
            size = case["experts"] // case["groups"]
            total = torch.stack([c[:, i * size:(i + 1) * size].topk(case["best"], -1).values.sum(-1) for i in range(case["groups"])], -1)
            for _ in range(case["groups"] - case["kept"]):                     # the worst group goes, of equal ones the last
                worst = case["groups"] - 1 - total.flip(-1).argmin(-1)
                total[torch.arange(case["tokens"], device="cuda"), worst] = math.inf
            c = torch.where((total == math.inf).repeat_interleave(size, -1), -math.inf, c)
        ids = []
        for _ in range(case["k"]):                                             # the largest, of equal ones the first
            ids.append(c.argmax(-1))
            c[torch.arange(case["tokens"], device="cuda"), ids[-1]] = -math.inf
        ids = torch.stack(ids, -1)
        w = p.gather(-1, ids)
        if case["renormalize"]:
            w = w / w.sum(-1, keepdim=True)
        flat = ids.flatten().tolist()
        order = sorted(range(len(flat)), key=lambda i: (flat[i], i))
        place, counts = [0] * len(flat), [0] * (case["experts"] + 1)
        for at, i in enumerate(order):
            place[i] = at
            counts[flat[i] + 1] += 1
        for e in range(case["experts"]):
            counts[e + 1] += counts[e]
        whole = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        return ids.int(), w * case["scale"], whole(counts), whole(order), whole(place)
    tables = _tables("cuda")
    lists = [list(_weights(case, g, rows, K, tables)) for _, rows, K in _parts(case)]
    if case["kind"] == "up":
        x = _exact_blocks(s["x"].reshape(case["tokens"], -1, 32)).flatten(-2)
        h = []
        for e in range(case["experts"]):
            rows = x[torch.nonzero(s["ids"] == e)[:, 0]]
            a, b = rows @ _exact_weights(lists[0][e]).T, rows @ _exact_weights(lists[1][e]).T
            h.append(a * torch.sigmoid(a) * b)
        return torch.cat(h)
    h = _exact_blocks(s["h"].reshape(s["h"].shape[0], -1, 32)).flatten(-2)
    y, taken = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device="cuda"), 0
    for e in range(case["experts"]):
        token, j = torch.nonzero(s["ids"] == e).unbind(-1)
        y[token] += s["weights"][token, j].double()[:, None] * (h[taken:taken + len(token)] @ _exact_weights(lists[0][e]).T)
        taken += len(token)
    return y
