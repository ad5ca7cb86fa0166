"""Operators of a sparse layer: the router, the plan of the experts' products, the products, the norms around a block, each against a
plain implementation in float64 (the quantizer: the oracle)."""
import ctypes
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import dfp4_oracle as O
from paper_2501_01144_amd import dfp4, synth

HALF = torch.finfo(torch.bfloat16).eps / 2          # a rounding to bf16, relative to the value
gpu = pytest.mark.gpu


# ---- refusals: no device is touched ----------------------------------------------------------------------------------------

def test_route_refuses():
    lib, vp = dfp4.load(), ctypes.c_void_p

    def route(logits=16, dtype=0, ld=64, tokens=4, experts=64, k=8, score=0, bias=0, groups=1, kept=1, best=1, ids=16, weights=16):
        return lib.dfp4_route(vp(logits), dtype, ld, tokens, experts, k, score, vp(bias), groups, kept, best, 1, 1.0, vp(ids), vp(weights), vp(0))
    assert (route(dtype=2), route(dtype=-1)) == (-4, -4)
    for bad in (dict(tokens=-1), dict(experts=0), dict(experts=1025, ld=1025), dict(k=0), dict(k=33), dict(experts=4, k=5), dict(ld=63), dict(score=2), dict(groups=0),
                dict(groups=3), dict(groups=4, kept=5), dict(groups=8, kept=0), dict(groups=16, kept=1, k=5), dict(best=0), dict(best=3), dict(groups=64, kept=64, best=2),
                dict(experts=1024, ld=1024, groups=128, kept=128), dict(tokens=(1 << 25) + 1)):
        assert route(**bad) == -2, bad
    assert (route(logits=0), route(ids=0), route(weights=0)) == (-1,) * 3
    assert (route(logits=18), route(logits=17, dtype=1), route(bias=2), route(ids=6), route(weights=10)) == (-3,) * 5
    assert route(tokens=0, logits=0, ids=0, weights=0) == 0


def test_plan_refuses():
    lib, vp = dfp4.load(), ctypes.c_void_p
    plan = lambda ids=16, data=16, tokens=4, k=2, experts=8: lib.dfp4_expert_plan(vp(ids), dfp4._CPlan(data, tokens, k, experts), vp(0))  # noqa: E731
    for bad in (dict(tokens=-1), dict(k=0), dict(k=33), dict(experts=0), dict(experts=1025), dict(tokens=1 << 27)):
        assert plan(**bad) == -2, bad
        assert lib.dfp4_expert_plan_bytes(*(dict(dict(tokens=4, k=2, experts=8), **bad)[n] for n in ("tokens", "k", "experts"))) == 0
    assert (plan(ids=0), plan(data=0), plan(ids=2), plan(data=8)) == (-1, -1, -3, -3)
    assert lib.dfp4_expert_plan_bytes(0, 2, 8) >= 4 * 9 and lib.dfp4_expert_plan_bytes(100, 2, 8) >= 4 * (9 + 400)


def _weights_c(packed=256, experts=8, rows=64, K=64, gated=1):
    return dfp4._CExperts(packed, experts, rows, K, gated)


def test_expert_weights_refuse():
    lib, vp = dfp4.load(), ctypes.c_void_p
    t = lambda codes=256, dialect=256, exponent=256, rows=512, K=64: dfp4._CTensor(codes, dialect, exponent, rows, K)  # noqa: E731
    call = lambda gate, up, w: lib.dfp4_expert_weights(gate, up, w, vp(0))  # noqa: E731
    for bad in (dict(experts=0), dict(experts=2000), dict(rows=0), dict(rows=12), dict(rows=(1 << 19) + 8), dict(K=0), dict(K=48), dict(experts=1024, rows=1 << 18)):
        assert call(t(), t(), _weights_c(**bad)) == -2, bad
        w = _weights_c(**bad)
        assert lib.dfp4_expert_weights_bytes(w.experts, w.rows, w.K, w.gated) == 0
    assert (call(t(rows=256), t(), _weights_c()), call(t(), t(K=32), _weights_c()), call(t(K=32), t(), _weights_c())) == (-2,) * 3
    assert (call(t(codes=0), t(), _weights_c()), call(t(), t(dialect=0), _weights_c()), call(t(), t(exponent=0), _weights_c()), call(t(), t(), _weights_c(packed=0))) == (-1,) * 4
    assert (call(t(), t(), _weights_c(packed=128)), call(t(codes=2), t(), _weights_c())) == (-3, -3)
    assert lib.dfp4_expert_weights_bytes(8, 64, 64, 0) > 8 * 64 * 64 * 0.78


def test_products_refuse():
    lib, vp = dfp4.load(), ctypes.c_void_p
    P = lambda data=16, tokens=4, k=2, experts=8: dfp4._CPlan(data, tokens, k, experts)  # noqa: E731

    def up(x=16, ld=64, plan=P(), w=_weights_c(), h=16, ws=256, n=1 << 30):
        return lib.dfp4_experts_up(vp(x), ld, plan, w, vp(h), vp(ws), n, vp(0))

    def down(h=16, ld=64, plan=P(), w=_weights_c(gated=0), weights=16, y=16, dtype=1, ws=256, n=1 << 30):
        return lib.dfp4_experts_down(vp(h), ld, plan, w, vp(weights), vp(y), dtype, vp(ws), n, vp(0))
    for f, gated in ((up, 1), (down, 0)):
        assert f(w=_weights_c(gated=1 - gated)) == -2
        for bad in (dict(ld=56), dict(plan=P(experts=9)), dict(plan=P(tokens=-1)), dict(plan=P(k=0)), dict(w=_weights_c(gated=gated, K=40)), dict(w=_weights_c(gated=gated, rows=4))):
            assert f(**bad) == -2, bad
        assert (f(plan=P(data=0)), f(w=_weights_c(gated=gated, packed=0))) == (-1, -1)
        assert (f(ld=68), f(plan=P(data=8)), f(w=_weights_c(gated=gated, packed=64)), f(ws=128)) == (-3,) * 4
        need = lib.dfp4_experts_workspace_bytes(P(), _weights_c(gated=gated))
        assert need > 0 and f(n=need - 1) == -5 and f(ws=0, n=0) == -5
        assert f(plan=P(tokens=0)) == 0 and lib.dfp4_experts_workspace_bytes(P(tokens=0), _weights_c(gated=gated)) == 0
    assert lib.dfp4_experts_workspace_bytes(P(experts=9), _weights_c()) == 0
    # more tiles than a launch holds
    big = dict(plan=P(tokens=1 << 26, k=2, experts=8), w=_weights_c(rows=1 << 14))
    assert up(**big) == -2 and lib.dfp4_experts_workspace_bytes(*big.values()) == 0
    assert (up(x=0), up(h=0), up(x=8), up(h=8)) == (-1, -1, -3, -3)
    assert (down(h=0), down(y=0), down(weights=0), down(h=8), down(y=24), down(weights=2), down(dtype=3)) == (-1, -1, -1, -3, -3, -3, -4)


def test_add_norm_refuses():
    lib, vp = dfp4.load(), ctypes.c_void_p

    def call(y=16, yl=64, r=16, rl=64, dtype=1, gate=0, gl=0, tokens=2, dim=64, post=0, weight=16, ro=16, normed=16):
        return lib.dfp4_add_norm(vp(y), yl, vp(r), rl, dtype, vp(gate), gl, tokens, dim, vp(post), vp(weight), 1.0, 1e-6, vp(ro), vp(normed), vp(0))
    for bad in (dict(tokens=-1), dict(dim=0), dict(dim=60), dict(dim=16392, yl=16392, rl=16392), dict(yl=56), dict(rl=32), dict(gate=16, gl=8)):
        assert call(**bad) == -2, bad
    assert call(dtype=2) == -4
    assert (call(y=0), call(r=0), call(weight=0), call(ro=0), call(normed=0)) == (-1,) * 5
    assert (call(y=8), call(r=8), call(gate=8), call(ro=8), call(normed=8), call(weight=18), call(post=2), call(yl=68), call(rl=68), call(gate=16, gl=68)) == (-3,) * 10
    assert call(tokens=0, y=0, r=0) == 0


# ---- plain implementations -------------------------------------------------------------------------------------------------

def plain_route(logits, k, score="softmax", bias=None, groups=1, kept=1, best=1, renormalize=True, scale=1.0):
    """float64 scores; ids by (largest choice, lowest index).  Without a bias a choice is the score's, which orders strictly as the logit does
    (-infinity: 0), where float64 rounds scores of different logits to one; only sums of two scores need the scores themselves."""
    x = np.asarray(logits, np.float64)
    x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
    ids, weights = [], []
    for row in x:
        if score == "softmax":
            s = np.zeros_like(row) if np.all(row == -np.inf) else np.exp(row - row.max())
            s = s / s.sum() if s.sum() > 0 else s
        else:
            s = 1 / (1 + np.exp(-row))
        c = row if bias is None and (groups == 1 or best == 1) else s + (0 if bias is None else np.asarray(bias, np.float64))
        if groups > 1:
            g = np.sort(c.reshape(groups, -1), 1)[:, ::-1][:, :best].sum(1)
            stay = sorted(range(groups), key=lambda i: (-g[i], i))[:kept]
            c = np.where(np.isin(np.arange(len(row)) // (len(row) // groups), stay), c, -np.inf)
        i = sorted(range(len(row)), key=lambda e: (-c[e], e))[:k]
        w = s[i]
        if renormalize:
            w = w / w.sum() if w.sum() > 0 else np.zeros_like(w)
        ids.append(i)
        weights.append(w * scale)
    return np.array(ids), np.array(weights)


def plain_plan(ids, experts):
    flat = [int(i) for i in np.asarray(ids).reshape(-1)]
    rows = sorted((i for i in range(len(flat)) if 0 <= flat[i] < experts), key=lambda i: (flat[i], i))
    place = [-1] * len(flat)
    for r, i in enumerate(rows):
        place[i] = r
    offsets = [sum(1 for i in rows if flat[i] < e) for e in range(experts + 1)]
    return offsets, rows + [-1] * (len(flat) - len(rows)), place


def quantized(x):
    return O.dfp4_dequantize(*O.dfp4_quantize(synth.to_f64(x)))


class Layer:
    """Random experts: the library's handle and the values."""

    def __init__(self, experts, rows, K, gated, seed=0):
        g = torch.Generator().manual_seed(seed)
        w = [(torch.randn(experts * rows, K, generator=g) * 0.05).bfloat16() for _ in range(2 if gated else 1)]
        q = [dfp4.quantize(x.cuda()) for x in w]
        self.handle = dfp4.expert_weights(q[0], experts, up=q[1] if gated else None)
        self.values = [quantized(x).reshape(experts, rows, K) for x in w]


def ids_of(tokens, k, experts, seed=0, absent=0.0, twice=False, only=None):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(experts, generator=g)[:k] for _ in range(tokens)]).int() if tokens else torch.zeros(0, k, dtype=torch.int32)
    if only is not None:
        ids = torch.randint(0, only, (tokens, k), generator=g).int()
    if twice and k > 1:
        ids[:, 1] = ids[:, 0]
    gone = torch.rand(tokens, k, generator=g) < absent
    return torch.where(gone, torch.where(torch.rand(tokens, k, generator=g) < 0.5, -1, experts).int(), ids)


def check_up(x, ids, layer, experts, h):
    """h against float64, within the products' 1e-5 sum |x||w|, fp32 arithmetic of the activation and one rounding."""
    xq = quantized(x)
    offsets, order, _ = plain_plan(ids, experts)
    k = ids.shape[1]
    h = h.float().cpu().double().numpy()
    for e in range(experts):
        rows = np.array(order[offsets[e]:offsets[e + 1]], dtype=int) // k
        if not len(rows):
            continue
        a = xq[rows]
        g, u = (a @ w[e].T for w in layer.values)
        dg, du = (1e-5 * np.abs(a) @ np.abs(w[e]).T for w in layer.values)
        s = g / (1 + np.exp(-g))
        # |silu'| <= 1.1; silu and the product in fp32: exp to 2^-20 (its argument's rounding, |g| up to 16, among it), three operations
        want, tol = s * u, 1.1 * dg * (np.abs(u) + du) + np.abs(s) * du
        tol = (tol + 2.0 ** -19 * np.abs(want)) * (1 + HALF) + HALF * np.abs(want) + 1e-38
        got = h[offsets[e]:offsets[e + 1]]
        assert (np.abs(got - want) <= tol).all(), (e, float((np.abs(got - want) / tol).max()))


def check_down(h, ids, layer, experts, weights, y):
    hq = quantized(h)
    offsets, order, _ = plain_plan(ids, experts)
    tokens, k = ids.shape
    w = synth.to_f64(weights)
    dim = layer.values[0].shape[1]
    want, size, tol = np.zeros((tokens, dim)), np.zeros((tokens, dim)), np.zeros((tokens, dim))
    for e in range(experts):
        for r in range(offsets[e], offsets[e + 1]):
            t, j = order[r] // k, order[r] % k
            v = hq[r] @ layer.values[0][e].T
            want[t] += w[t, j] * v
            size[t] += np.abs(w[t, j] * v)
            tol[t] += np.abs(w[t, j]) * (1e-5 * np.abs(hq[r]) @ np.abs(layer.values[0][e]).T)
    # rows' products are held in no fewer bits than bf16 (half a step each), the sum in fp32
    half = HALF if y.dtype == torch.bfloat16 else 2.0 ** -24
    tol = (tol + (2.0 ** -23 * (k + 1) + (HALF if y.dtype == torch.bfloat16 else 0.0)) * size) * (1 + half) + half * np.abs(want) + 1e-38
    got = y.float().cpu().double().numpy()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


# ---- router and plan ---------------------------------------------------------------------------------------------------------

ROUTES = [
    (1, 128, 8, {}), (5, 8, 2, dict(renormalize=False)), (3, 1, 1, {}), (67, 160, 6, dict(score="sigmoid", bias=True, groups=8, kept=3, best=2, scale=2.5)),
    (33, 64, 32, dict(bias=True)), (130, 256, 8, dict(score="sigmoid")), (9, 300, 7, dict(groups=4, kept=1, best=1)), (4, 1024, 32, dict(score="sigmoid", bias=True, groups=64, kept=5, best=2)),
    (12, 66, 3, dict(groups=33, kept=2, best=2, bias=True)), (2, 512, 1, dict(groups=64, kept=1)), (6, 64, 5, dict(groups=64, kept=5)),
]


@gpu
@pytest.mark.parametrize("tokens,experts,k,more", ROUTES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_route(tokens, experts, k, more, dtype):
    g = torch.Generator().manual_seed(tokens + experts)
    wide = (torch.randn(tokens, experts + 3, generator=g) * 2).to(dtype)             # (bf16: many equal logits)
    logits, more = wide[:, 1:experts + 1], dict(more)
    if more.pop("bias", False):
        more["bias"] = torch.randn(experts, generator=g) * 0.1
    ids, weights = dfp4.route(wide.cuda()[:, 1:experts + 1], k, **{n: v.cuda() if n == "bias" else v for n, v in more.items()})
    want, w = plain_route(logits.float().numpy(), k, **more)
    assert ids.dtype == torch.int32 and np.array_equal(ids.cpu().numpy(), want)
    got = weights.cpu().double().numpy()
    # 64-bit arithmetic (far below 2^-40) and one rounding to fp32
    assert (np.abs(got - w) <= (2.0 ** -24 + 2.0 ** -40) * np.abs(w)).all()


@gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_of_masked_infinite_and_equal_logits(score):
    inf, nan = float("inf"), float("nan")
    rows = [[0.0] * 8, [-inf] * 8, [nan] * 8, [1.0, -inf, 3.0, -inf, -inf, -inf, -inf, -inf], [inf, 0.0, inf, 1.0, -inf, nan, 2.0, 2.0], [-inf, nan, 5.0, 5.0, 5.0, 5.0, 5.0, 5.0],
            [-3.4e38] * 7 + [-inf], [3.4e38, 3.4e38] + [0.0] * 6, [torch.finfo(torch.float32).min] * 4 + [-1e30] * 4]
    for more in ({}, dict(groups=4, kept=2, best=2), dict(bias=torch.tensor([0.0, 0, 0, 0.5, 0, 0, 0, 0.25]))):
        ids, weights = dfp4.route(torch.tensor(rows).cuda(), 4, score=score, **{n: v.cuda() if n == "bias" else v for n, v in more.items()})
        with np.errstate(all="ignore"):
            want, w = plain_route(np.array(rows), 4, score=score, **more)
        assert np.array_equal(ids.cpu().numpy(), want)
        got = weights.cpu().double().numpy()
        assert np.isfinite(got).all() and (np.abs(got - w) <= (2.0 ** -24 + 2.0 ** -40) * np.abs(w) + 2.0 ** -149).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts,k", [(8, 8), (16, 3), (100, 16), (256, 9), (300, 17)])
def test_route_of_few_values(dtype, experts, k):
    # zeros of both signs, equal numbers, infinities and NaN, in every position
    g = torch.Generator().manual_seed(experts)
    values = torch.tensor([0.0, -0.0, 1.0, -1.0, float("inf"), float("-inf"), float("nan"), 3.3895e38, -3.3895e38, 1e-40])
    logits = values[torch.randint(0, len(values), (50, experts), generator=g)].to(dtype)
    logits[:25][logits[:25].isinf()] = 0.5
    for more in ({}, dict(score="sigmoid"), dict(renormalize=False), dict(groups=4, kept=3) if experts % 4 == 0 and 3 * experts >= 4 * k else {}):
        ids, weights = dfp4.route(logits.cuda(), k, **more)
        with np.errstate(all="ignore"):
            want, w = plain_route(logits.float().numpy(), k, **more)
        assert np.array_equal(ids.cpu().numpy(), want)
        got = weights.cpu().double().numpy()
        assert (np.abs(got - w) <= (2.0 ** -24 + 2.0 ** -40) * np.abs(w) + 2.0 ** -149).all()


PLANS = [(1, 8, 128, {}), (1, 1, 1, {}), (0, 2, 4, {}), (37, 3, 5, {}), (300, 4, 9, dict(absent=0.3)), (50, 2, 4, dict(absent=1.0)), (1025, 8, 64, {}), (64, 6, 8, dict(twice=True)),
         (700, 1, 1024, {}), (200, 32, 40, {}), (5000, 8, 16, dict(only=2)), (129, 2, 300, dict(absent=0.1, twice=True)), (3000, 7, 33, {}),
         (4096, 1, 7, {}), (4097, 1, 7, dict(only=1)), (9000, 8, 12, dict(only=3, absent=0.01))]


@gpu
@pytest.mark.parametrize("tokens,k,experts,more", PLANS)
def test_plan(tokens, k, experts, more):
    ids = ids_of(tokens, k, experts, seed=tokens, **more)
    for _ in range(2):
        plan = dfp4.expert_plan(ids.cuda(), experts)
        offsets, order, place = plain_plan(ids, experts)
        assert plan.offsets.tolist() == offsets and plan.order.tolist() == order and plan.place.tolist() == place


# ---- products ----------------------------------------------------------------------------------------------------------------

PRODUCTS = [                                  # tokens, k, experts, K, rows
    (1, 1, 1, 32, 8, {}), (1, 8, 16, 256, 96, {}), (3, 2, 4, 96, 40, {}), (33, 1, 2, 64, 72, {}), (65, 4, 9, 160, 128, dict(absent=0.3)), (40, 2, 4, 1056, 264, dict(twice=True)),
    (7, 3, 40, 2080, 56, {}), (130, 2, 3, 544, 300 // 8 * 8, {}), (20, 2, 4, 64, 64, dict(absent=1.0)), (300, 2, 4, 128, 64, dict(only=1)), (257, 4, 8, 96, 520, {}),
    (1100, 2, 2, 224, 136, {}), (600, 5, 20, 64, 256, dict(absent=0.5)),
    (100, 1, 8, 2176, 40, dict(only=1)), (40, 2, 6, 4192, 48, {}), (70, 3, 12, 4128, 24, dict(only=3, absent=0.2)), (4, 3, 5, 4256, 104, dict(twice=True)),
    (2, 32, 64, 96, 1000, dict(absent=0.4)), (260, 1, 10, 64, 1032, {}), (16, 1, 8, 8224, 16, {}), (3, 2, 4, 14336, 32, {}), (90, 2, 1024, 128, 8, {}),
    (40, 2, 3, 64, 2056, {}), (700, 1, 2, 32, 4104, dict(absent=0.1)),
]


@gpu
@pytest.mark.parametrize("tokens,k,experts,K,rows,more", PRODUCTS)
def test_up(tokens, k, experts, K, rows, more):
    layer = Layer(experts, rows, K, True, seed=tokens)
    x = torch.randn(tokens, K, generator=torch.Generator().manual_seed(K))
    x[:, 5] *= 20
    x = x.bfloat16()
    ids = ids_of(tokens, k, experts, seed=rows, **more)
    plan = dfp4.expert_plan(ids.cuda(), experts)
    h = dfp4.experts_up(x.cuda(), plan, layer.handle)
    check_up(x, ids, layer, experts, h)
    # into buffers of the caller's, from rows with a stride; what is behind the last row stays
    wide = torch.zeros(tokens, K + 24, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:K + 8] = x.cuda()
    out = torch.full_like(h, 7.0)
    ws = torch.full((int(dfp4.load().dfp4_experts_workspace_bytes(plan.c(), layer.handle.c())),), 0xff, dtype=torch.uint8, device="cuda")
    dfp4.experts_up(wide[:, 8:K + 8], plan, layer.handle, out=out, workspace=ws)
    n = int(plan.offsets[-1])
    assert torch.equal(out[:n], h[:n]) and (out[n:] == 7.0).all()


@gpu
@pytest.mark.parametrize("tokens,k,experts,K,rows,more", PRODUCTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_down(tokens, k, experts, K, rows, more, dtype):
    layer = Layer(experts, rows, K, False, seed=tokens)
    g = torch.Generator().manual_seed(K)
    h = (torch.randn(tokens * k, K, generator=g) * torch.rand(tokens * k, 1, generator=g)).bfloat16()
    ids = ids_of(tokens, k, experts, seed=rows, **more)
    weights = torch.rand(tokens, k, generator=g)
    plan = dfp4.expert_plan(ids.cuda(), experts)
    n = int(plan.offsets[-1])
    mine = h.cuda()
    mine[n:] = float("nan")                          # (rows behind the last are not read)
    mine[n::2] = float("-inf")
    y = dfp4.experts_down(mine, plan, layer.handle, weights.cuda(), dtype=dtype)
    check_down(h, ids, layer, experts, weights, y)
    wide = torch.full((tokens * k, K + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = mine
    out = torch.full_like(y, 7.0)
    ws = torch.full((int(dfp4.load().dfp4_experts_workspace_bytes(plan.c(), layer.handle.c())),), 0xff, dtype=torch.uint8, device="cuda")
    dfp4.experts_down(wide[:, :K], plan, layer.handle, weights.cuda(), out=out, workspace=ws)
    assert torch.equal(out, y)


@gpu
@pytest.mark.parametrize("tokens,k,experts,K,absent", [(2100, 4, 5, 4000, 0.0), (1500, 3, 4, 8224, 0.3), (4200, 8, 7, 1056, 0.0)])
def test_up_of_tokens_quantized_once(tokens, k, experts, K, absent):
    """Long rows of several experts (tokens * k * K from 2^25 on): the rows of a token are alike, and those of its neighbours in a smaller call."""
    layer = Layer(experts, 40, K, True, seed=K)
    x = torch.randn(tokens, K, generator=torch.Generator().manual_seed(1)).bfloat16()
    ids = ids_of(tokens, min(k, experts), experts, seed=2, absent=absent)
    k = ids.shape[1]
    plan = dfp4.expert_plan(ids.cuda(), experts)
    wide = torch.zeros(tokens, K + 8, dtype=torch.bfloat16, device="cuda")
    wide[:, :K] = x.cuda()
    h = dfp4.experts_up(wide[:, :K], plan, layer.handle)
    assert torch.equal(h[:int(plan.offsets[-1])], dfp4.experts_up(x.cuda(), plan, layer.handle)[:int(plan.offsets[-1])])
    # a few tokens from everywhere against the plain form
    some = torch.linspace(0, tokens - 1, 33).long()
    few = dfp4.expert_plan(ids[some].contiguous().cuda(), experts)
    rows = plan.place.cpu().view(tokens, k)[some].flatten()
    mine = torch.zeros(33 * k, 40, dtype=torch.bfloat16)
    there = rows >= 0
    mine[few.place.cpu()[there].long()] = h.cpu()[rows[there].long()]
    check_up(x[some], ids[some], layer, experts, mine)


@gpu
@pytest.mark.parametrize("tokens", [2, 40, 400])
@pytest.mark.parametrize("span", [12, 30])
def test_products_of_uneven_blocks(tokens, span):
    """Blocks whose scales lie up to 2^60 apart in a product, by every way."""
    K, rows, experts, k = 1312, 48, 4, 2
    g = torch.Generator().manual_seed(span)
    uneven = lambda n: (torch.randn(n, K // 32, 32, generator=g) * torch.exp2(torch.randint(-span, 1, (n, K // 32, 1), generator=g).float())).view(n, K).bfloat16()  # noqa: E731
    up, down = Layer(experts, rows, K, True), Layer(experts, rows, K, False)
    for layer in (up, down):
        w = [uneven(experts * rows) for _ in layer.values]
        q = [dfp4.quantize(x.cuda()) for x in w]
        layer.handle = dfp4.expert_weights(q[0], experts, up=q[1] if len(q) > 1 else None)
        layer.values = [quantized(x).reshape(experts, rows, K) for x in w]
    ids, x, h = ids_of(tokens, k, experts, seed=1), uneven(tokens), uneven(tokens * k)
    plan, weights = dfp4.expert_plan(ids.cuda(), experts), torch.rand(tokens, k, generator=g)
    check_up(x, ids, up, experts, dfp4.experts_up(x.cuda(), plan, up.handle))
    for dtype in (torch.bfloat16, torch.float32):
        check_down(h, ids, down, experts, weights, dfp4.experts_down(h.cuda(), plan, down.handle, weights.cuda(), dtype=dtype))


@gpu
@pytest.mark.parametrize("tokens", [1, 40, 200])
def test_up_of_far_gates(tokens):
    """silu where exp(-g) leaves fp32 and its product with u does not: results down to the least normal number.  g and u are single products of
    numbers of a few bits, so exact."""
    experts, rows, K = 2, 256, 64
    g, u = torch.linspace(-160.0, 100.0, experts * rows), 2.0 ** (torch.arange(experts * rows) % 101)
    w = [torch.zeros(experts * rows, K) for _ in range(2)]
    w[0][:, 0], w[1][:, 32] = g, u
    w = [t.bfloat16() for t in w]
    q = [dfp4.quantize(t.cuda()) for t in w]
    handle, (gate, up) = dfp4.expert_weights(q[0], experts, up=q[1]), (quantized(t).reshape(experts, rows, K) for t in w)
    x = torch.zeros(tokens, K)
    x[:, 0], x[:, 32] = 1.0, 1.0
    ids = (torch.arange(tokens) % experts).int()[:, None].contiguous()
    plan = dfp4.expert_plan(ids.cuda(), experts)
    h = dfp4.experts_up(x.bfloat16().cuda(), plan, handle).float().cpu().double().numpy()
    offsets, _, _ = plain_plan(ids, experts)
    for e in range(experts):
        a, b = gate[e][:, 0], up[e][:, 32]
        want = a / (1 + np.exp(-a)) * b
        # exp's argument is off by 2^-23 of itself at most (its factor's rounding and its own), which is 2^-23 |g| of the result; a few operations in
        # fp32; one rounding to bf16; numbers below the least normal one may be zero
        tol = (2.0 ** -23 * np.abs(a) + 2.0 ** -20) * np.abs(want) * (1 + HALF) + HALF * np.abs(want) + 2.0 ** -126
        got = h[offsets[e]:offsets[e + 1]]
        assert (np.abs(got - want) <= tol).all(), (e, a[(np.abs(got - want) > tol).any(0)])


@gpu
def test_products_of_no_tokens():
    up, down = Layer(4, 64, 64, True), Layer(4, 64, 64, False)
    plan = dfp4.expert_plan(torch.zeros(0, 2, dtype=torch.int32, device="cuda"), 4)
    assert plan.offsets.tolist() == [0] * 5
    h = dfp4.experts_up(torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda"), plan, up.handle)
    y = dfp4.experts_down(h, plan, down.handle, torch.zeros(0, 2, device="cuda"))
    assert h.shape == (0, 64) and y.shape == (0, 64)


# ---- every way of the products -----------------------------------------------------------------------------------------------

# tokens, k, experts, K, rows, absent; the way: rows a workgroup takes, waves that share K, how rows are quantized (0 within, 1 before, 2 once a token).
# Blocks of 32 rows have up to 32 quads of K (4096 elements) in LDS at a time, those of more rows 16
UP_WAYS = [
    (9, 2, 8, 96, 104, 0.2, (32, 1, 0)), (4, 2, 3, 416, 8240, 0.0, (32, 2, 0)), (16, 2, 2, 800, 8736, 0.1, (32, 2, 1)), (7, 1, 2, 288, 48, 0.0, (32, 4, 0)),
    (30, 1, 1, 480, 72, 0.0, (32, 4, 1)), (27, 1, 2, 2112, 4472, 0.1, (32, 4, 1)), (5, 2, 3, 544, 40, 0.3, (32, 8, 0)), (23, 1, 1, 576, 56, 0.1, (32, 8, 1)),
    (4, 1, 2, 4320, 4128, 0.0, (32, 4, 0)), (2, 1, 1, 4320, 4128, 0.0, (32, 8, 0)), (11, 1, 1, 2144, 4112, 0.0, (32, 8, 1)), (3, 2, 4, 1056, 136, 0.2, (32, 16, 0)), (1, 8, 9, 4128, 40, 0.4, (32, 16, 0)),
    (19, 1, 2, 8224, 24, 0.1, (32, 16, 1)),
    (70, 2, 20, 96, 104, 0.2, (64, 1, 0)), (100, 2, 6, 384, 72, 0.1, (64, 1, 1)), (242, 1, 33, 416, 464, 0.0, (64, 2, 0)), (327, 2, 33, 672, 480, 0.1, (64, 2, 1)),
    (17, 4, 8, 416, 40, 0.2, (64, 4, 0)), (60, 1, 2, 448, 72, 0.0, (64, 4, 1)), (205, 2, 33, 2144, 232, 0.1, (64, 4, 1)), (33, 1, 2, 576, 24, 0.0, (64, 8, 0)),
    (66, 1, 2, 992, 40, 0.1, (64, 8, 1)), (36, 2, 33, 4320, 144, 0.2, (64, 8, 0)), (17, 4, 5, 2080, 848, 0.1, (64, 8, 1)), (20, 4, 8, 1088, 56, 0.2, (64, 16, 0)),
    (23, 2, 5, 1344, 40, 0.0, (64, 16, 1)), (19, 2, 16, 4832, 24, 0.2, (64, 16, 0)), (60, 2, 5, 4256, 72, 0.1, (64, 16, 1)),
    (300, 2, 4, 288, 72, 0.1, (128, 1, 1)), (1500, 3, 4, 7488, 40, 0.1, (128, 1, 2)), (2100, 2, 2, 1056, 904, 0.1, (256, 1, 1)), (2100, 2, 2, 1024, 904, 0.0, (256, 1, 1)),
    (4200, 7, 7, 2048, 136, 0.1, (256, 1, 2)), (4200, 7, 8, 1184, 136, 0.0, (256, 1, 2)),
]
DOWN_WAYS = [
    (5, 3, 8, 1056, 72, 0.3, (1, 16, 0)), (1, 8, 16, 2080, 264, 0.5, (1, 16, 0)),
    (31, 1, 1, 32, 648, 0.0, (32, 1, 0)), (4, 2, 3, 416, 11048, 0.1, (32, 2, 0)), (10, 3, 3, 1376, 11448, 0.0, (32, 2, 1)), (25, 1, 1, 416, 1016, 0.0, (32, 4, 0)),
    (27, 1, 1, 480, 1392, 0.1, (32, 4, 1)), (26, 1, 2, 2240, 8208, 0.0, (32, 4, 1)), (15, 1, 1, 544, 1192, 0.0, (32, 8, 0)), (29, 1, 1, 576, 712, 0.2, (32, 8, 1)),
    (6, 2, 5, 4160, 1776, 0.2, (32, 8, 0)), (11, 1, 1, 2144, 9128, 0.0, (32, 8, 1)), (28, 1, 3, 1056, 688, 0.1, (32, 16, 0)), (1, 8, 16, 8224, 72, 0.4, (32, 16, 0)),
    (19, 1, 2, 1376, 952, 0.0, (32, 16, 1)), (31, 1, 1, 4320, 232, 0.1, (32, 16, 1)),
    (258, 1, 8, 32, 40, 0.0, (64, 1, 0)), (266, 2, 16, 384, 40, 0.2, (64, 1, 1)), (58, 3, 33, 416, 920, 0.1, (64, 2, 0)), (139, 4, 33, 736, 920, 0.1, (64, 2, 1)),
    (117, 1, 5, 448, 136, 0.0, (64, 4, 0)), (191, 2, 12, 448, 72, 0.1, (64, 4, 1)), (264, 1, 24, 2112, 672, 0.0, (64, 4, 1)), (317, 1, 16, 576, 56, 0.1, (64, 8, 0)),
    (276, 1, 12, 608, 40, 0.0, (64, 8, 1)), (41, 2, 33, 4288, 272, 0.1, (64, 8, 0)), (255, 2, 33, 2144, 232, 0.1, (64, 8, 1)), (67, 1, 8, 1056, 288, 0.0, (64, 16, 0)),
    (322, 1, 33, 1440, 40, 0.1, (64, 16, 1)), (82, 2, 5, 2592, 72, 0.2, (64, 16, 1)),
    (300, 2, 4, 288, 64, 0.1, (128, 1, 1)), (700, 3, 5, 1056, 1032, 0.2, (128, 1, 1)), (2100, 2, 2, 1056, 1800, 0.1, (256, 1, 1)), (2100, 2, 2, 224, 1800, 0.0, (256, 1, 1)),
]


def way_of(tokens, k, experts, K, rows, gated):
    way = (ctypes.c_int32 * 3)()
    rc = dfp4.load().dfp4_experts_way(dfp4._CPlan(16, tokens, k, experts), dfp4._CExperts(256, experts, rows, K, gated), way)
    return rc, tuple(way)


def test_the_way_of_a_product():
    """Without a device, as on one of 256 compute units."""
    for gated, ways in ((1, UP_WAYS), (0, DOWN_WAYS)):
        for *sizes, _, way in ways:
            assert way_of(*sizes, gated) == (0, way), (gated, sizes)
        seen = {w for *_, w in ways}
        assert seen >= {(rows, waves, q) for rows in (32, 64) for waves in (2, 4, 8, 16) for q in (0, 1)} | {(64, 1, 0), (64, 1, 1), (32, 1, 0), (128, 1, 1), (256, 1, 1)}
    assert {(128, 1, 2), (256, 1, 2)} <= {w for *_, w in UP_WAYS} and (1, 16, 0) in {w for *_, w in DOWN_WAYS}
    assert [way_of(*s, 1)[0] for s in ((0, 2, 8, 64, 64), (4, 0, 8, 64, 64), (4, 2, 8, 48, 64), (4, 2, 8, 64, 4), (1 << 26, 2, 8, 64, 1 << 14))] == [-2] * 5
    lib = dfp4.load()
    assert lib.dfp4_experts_way(dfp4._CPlan(16, 4, 2, 8), dfp4._CExperts(256, 8, 64, 64, 1), None) == -1
    assert lib.dfp4_experts_way(dfp4._CPlan(16, 4, 2, 9), dfp4._CExperts(256, 8, 64, 64, 1), None) == -2


class UnevenLayer:
    """Experts whose blocks' sizes lie up to 2^4 apart, and rows alike; values from the dequantizer (exact), in float64 on the device."""

    def __init__(self, experts, rows, K, gated):
        self.g = torch.Generator(device="cuda").manual_seed(K + rows)
        self.values, q = [], []
        for _ in range(2 if gated else 1):
            q.append(dfp4.quantize(self.uneven(experts * rows, K)))
            self.values.append(dfp4.dequantize(q[-1], dtype=torch.float32).double().view(experts, rows, K))
        self.handle = dfp4.expert_weights(q[0], experts, up=q[1] if gated else None)

    def uneven(self, n, K):
        blocks = torch.randn(n, K // 32, 32, generator=self.g, device="cuda")
        return (blocks * torch.exp2(torch.randint(-4, 1, (n, K // 32, 1), generator=self.g, device="cuda").float())).view(n, K).bfloat16()


def quantized_on_device(x):
    return dfp4.dequantize(dfp4.quantize(x), dtype=torch.float32).double()


@gpu
@pytest.mark.parametrize("tokens,k,experts,K,rows,absent,way", UP_WAYS)
def test_up_by_every_way(tokens, k, experts, K, rows, absent, way):
    layer = UnevenLayer(experts, rows, K, True)
    x, ids = layer.uneven(tokens, K), ids_of(tokens, k, experts, seed=rows, absent=absent)
    plan = dfp4.expert_plan(ids.cuda(), experts)
    assert dfp4.experts_way(plan, layer.handle) == way
    out = torch.full((tokens * k, rows), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((int(dfp4.load().dfp4_experts_workspace_bytes(plan.c(), layer.handle.c())),), 0xff, dtype=torch.uint8, device="cuda")
    h = dfp4.experts_up(x, plan, layer.handle, out=out, workspace=ws)
    offsets, order, _ = plain_plan(ids, experts)
    xq = quantized_on_device(x)
    for e in range(experts):
        lo, hi = offsets[e], offsets[e + 1]
        if hi == lo:
            continue
        a = xq[torch.tensor(order[lo:hi], device="cuda") // k]
        g, u = (a @ w[e].T for w in layer.values)
        dg, du = (1e-5 * (a.abs() @ w[e].abs().T) for w in layer.values)
        s = g / (1 + torch.exp(-g))
        # as check_up: |silu'| <= 1.1, fp32 arithmetic of silu, one rounding
        want, tol = s * u, 1.1 * dg * (u.abs() + du) + s.abs() * du
        tol = (tol + (2.0 ** -19 + 2.0 ** -23 * g.abs()) * want.abs()) * (1 + HALF) + HALF * want.abs() + 1e-38
        off = (h[lo:hi].double() - want).abs() / tol
        assert (off <= 1).all(), (e, float(off.max()))
    assert (h[offsets[-1]:] == 7.0).all()


@gpu
@pytest.mark.parametrize("tokens,k,experts,K,rows,absent,way", DOWN_WAYS)
def test_down_by_every_way(tokens, k, experts, K, rows, absent, way):
    layer = UnevenLayer(experts, rows, K, False)
    ids, weights = ids_of(tokens, k, experts, seed=rows, absent=absent), torch.rand(tokens, k, generator=layer.g, device="cuda") - 0.5
    plan = dfp4.expert_plan(ids.cuda(), experts)
    assert dfp4.experts_way(plan, layer.handle) == way
    h = layer.uneven(tokens * k, K)
    offsets, order, _ = plain_plan(ids, experts)
    hq = quantized_on_device(h)
    h[offsets[-1]:] = float("nan")                   # (rows behind the last are not read)
    h[offsets[-1]::2] = float("inf")
    shape = (tokens, rows)
    want, size, tol = (torch.zeros(shape, dtype=torch.float64, device="cuda") for _ in range(3))
    for e in range(experts):
        lo, hi = offsets[e], offsets[e + 1]
        if hi == lo:
            continue
        pairs, a = torch.tensor(order[lo:hi], device="cuda"), hq[lo:hi]
        w = weights.double().flatten()[pairs, None]
        v = w * (a @ layer.values[0][e].T)
        want.index_add_(0, pairs // k, v)
        size.index_add_(0, pairs // k, v.abs())
        tol.index_add_(0, pairs // k, 1e-5 * w.abs() * (a.abs() @ layer.values[0][e].abs().T))
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full(shape, 7.0, dtype=dtype, device="cuda")
        ws = torch.full((int(dfp4.load().dfp4_experts_workspace_bytes(plan.c(), layer.handle.c())),), 0xff, dtype=torch.uint8, device="cuda")
        y = dfp4.experts_down(h, plan, layer.handle, weights, out=out, workspace=ws)
        # k products and additions in fp32, one rounding, y's own
        half = HALF if dtype == torch.bfloat16 else 2.0 ** -24
        off = (y.double() - want).abs() / ((tol + 2.0 ** -23 * (k + 1) * size) * (1 + half) + half * want.abs() + 1e-38)
        assert (off <= 1).all(), (dtype, float(off.max()))
        assert torch.equal(y, dfp4.experts_down(h, plan, layer.handle, weights, dtype=dtype))


# ---- norms -------------------------------------------------------------------------------------------------------------------

def check_norm(y, residual, weight, post, gate, scale, eps, r_got, n_got):
    y, r0, w = synth.to_f64(y), synth.to_f64(residual), synth.to_f64(weight)
    z = y
    if post is not None:
        z = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps) * synth.to_f64(post)
    if gate is not None:
        z = z * synth.to_f64(gate)
    z = scale * z
    r = r0 + z
    rms = np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    n = r / rms * w
    # sums of up to 16384 squares, at most 2^7 additions deep in fp32: 2^-17 of a sum, half of that of its root; a few operations more
    f32 = 2.0 ** -17
    e_r = f32 * np.abs(z) + 2.0 ** -23 * (np.abs(r) + np.abs(z))
    half = HALF if r_got.dtype == torch.bfloat16 else 2.0 ** -24
    got = r_got.float().cpu().double().numpy()
    tol = e_r * (1 + half) + half * np.abs(r) + 1e-38
    assert (np.abs(got - r) <= tol).all(), float((np.abs(got - r) / tol).max())
    got = n_got.float().cpu().double().numpy()
    tol = (e_r / rms * np.abs(w) + np.abs(n) * (f32 + np.sqrt((e_r * e_r).mean(-1, keepdims=True)) / rms)) * (1 + HALF) + HALF * np.abs(n) + 1e-38
    assert (np.abs(got - n) <= tol).all(), float((np.abs(got - n) / tol).max())


@gpu
@pytest.mark.parametrize("tokens,dim", [(1, 8), (3, 512), (5, 520), (2, 2048), (7, 2056), (3, 4096), (2, 4104), (1, 8192), (2, 16384), (3, 16376), (1029, 64), (513, 1448)])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("post,gate", [(True, "token"), (False, None), (True, "all"), (False, "token")])
def test_add_norm(tokens, dim, wide, post, gate):
    g = torch.Generator().manual_seed(tokens + dim)
    y, r = torch.randn(tokens, dim + 8, generator=g).bfloat16(), torch.randn(tokens, dim + 16, generator=g) * 3
    y[:, 3] *= 50
    r = r if wide else r.bfloat16()
    w, p = 1 + 0.2 * torch.randn(dim, generator=g), 1 + 0.2 * torch.randn(dim, generator=g) if post else None
    gt = None if gate is None else torch.randn(dim, generator=g).bfloat16() if gate == "all" else torch.randn(tokens, dim, generator=g).bfloat16()
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    yc, rc = y.cuda()[:, :dim], r.cuda()[:, 8:dim + 8]
    got = dfp4.add_norm(yc, rc, w.cuda(), post_weight=dev(p), gate=dev(gt), scale=0.7, eps=1e-5)
    check_norm(y[:, :dim], r[:, 8:dim + 8], w, p, gt, 0.7, 1e-5, *got)
    # in place
    y2, r2 = yc.contiguous(), rc.contiguous()
    same = dfp4.add_norm(y2, r2, w.cuda(), post_weight=dev(p), gate=dev(gt), scale=0.7, eps=1e-5, out=(r2, y2))
    assert same[0] is r2 and torch.equal(r2, got[0]) and torch.equal(y2, got[1])


@gpu
@pytest.mark.parametrize("size", [2.0 ** -70, 2.0 ** 70, 2.0 ** 100])
@pytest.mark.parametrize("dim", [64, 4096])
def test_add_norm_of_numbers_whose_squares_leave_fp32(size, dim):
    g = torch.Generator().manual_seed(1)
    y, r = (torch.randn(3, dim, generator=g) * size).bfloat16(), torch.randn(3, dim, generator=g)
    w = torch.ones(dim)
    got = dfp4.add_norm(y.cuda(), r.cuda(), w.cuda(), post_weight=w.cuda(), eps=0.0)
    check_norm(y, r, w, w, None, 1.0, 0.0, *got)
    r = r * size
    got = dfp4.add_norm(y.cuda(), r.cuda(), w.cuda(), eps=0.0)
    check_norm(y, r, w, None, None, 1.0, 0.0, *got)


@gpu
@pytest.mark.parametrize("dim", [4104, 8192, 16384])
@pytest.mark.parametrize("wide", [False, True])
def test_add_norm_of_rows_near_the_largest_number(dim, wide):
    """Up to dim numbers of 2^127 and more: their squares, scaled, still have a sum in fp32."""
    g = torch.Generator().manual_seed(dim)
    sign = lambda: torch.randint(0, 2, (3, dim), generator=g).float() * 2 - 1  # noqa: E731
    big, w = sign() * torch.linspace(1.7e38, 3.3e38, dim), 1 + 0.2 * torch.randn(dim, generator=g)
    y, r = big.bfloat16(), (big if wide else big.bfloat16())
    small = torch.randn(3, dim, generator=g)
    got = dfp4.add_norm(y.cuda(), (small if wide else small.bfloat16()).cuda(), w.cuda(), post_weight=w.cuda())         # the norm before
    check_norm(y, small if wide else small.bfloat16(), w, w, None, 1.0, 1e-6, *got)
    got = dfp4.add_norm(small.bfloat16().cuda(), r.cuda(), w.cuda())                                                    # the norm after
    check_norm(small.bfloat16(), r, w, None, None, 1.0, 1e-6, *got)


# ---- together ----------------------------------------------------------------------------------------------------------------

@gpu
def test_the_example_runs():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "sparse_layer.py")
    spec = importlib.util.spec_from_file_location("sparse_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    off, _ = module.run(tokens=40, hidden=256, inner=96, experts=8, k=2, steps=4)
    # bf16 results: HALF of every element at most, twice where rows are rounded before they are added; fp32 sums besides
    assert off <= 2 * HALF + 2.0 ** -12


@gpu
def test_calls_from_python_refuse():
    layer = Layer(4, 64, 64, True)
    x, ids = torch.zeros(6, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    plan = dfp4.expert_plan(ids, 4)
    for bad in (lambda: dfp4.expert_plan(ids.long(), 4), lambda: dfp4.expert_plan(ids[:, ::2], 4), lambda: dfp4.experts_up(x[:5], plan, layer.handle),
                lambda: dfp4.experts_up(x.float(), plan, layer.handle), lambda: dfp4.experts_up(x[:, :32], plan, layer.handle), lambda: dfp4.route(x[0].float(), 2),
                lambda: dfp4.route(x.half(), 2), lambda: dfp4.route(x, 2, bias=x[0]), lambda: dfp4.route(x, 2, score="other"),
                lambda: dfp4.add_norm(x, x[:, :32], torch.ones(64, device="cuda")), lambda: dfp4.add_norm(x, x, torch.ones(32, device="cuda")),
                lambda: dfp4.add_norm(x, x, torch.ones(64, device="cuda"), gate=x[:3]), lambda: dfp4.expert_weights(dfp4.empty_qtensor(10, 64, x.device), 4),
                lambda: dfp4.experts_down(x, plan, layer.handle, torch.zeros(6, 2, device="cuda"))):
        with pytest.raises(AssertionError):
            bad()
    h = torch.zeros(12, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: dfp4.experts_down(h, plan, layer.handle, torch.zeros(6, 2, device="cuda")), lambda: dfp4.experts_up(x, dfp4.expert_plan(ids, 5), layer.handle),
                lambda: dfp4.route(x.float(), 65), lambda: dfp4.route(x.float(), 0), lambda: dfp4.route(x.float(), 1 << 40), lambda: dfp4.route(x.float(), -3), lambda: dfp4.expert_plan(ids, 2000), lambda: dfp4.route(x.float(), 4, groups=5),
                lambda: dfp4.add_norm(x[:, 4:], x[:, 4:], torch.ones(60, device="cuda")), lambda: dfp4.expert_weights(dfp4.empty_qtensor(16, 64, x.device, mx=True), 4)):
        with pytest.raises(dfp4.Dfp4Error):
            bad()


@gpu
@pytest.mark.parametrize("tokens", [1, 16, 700])
def test_a_layer_eager_on_another_stream_and_in_a_graph(tokens):
    """norm -> router -> plan -> experts -> norm, as a program runs them; every replay against eager calls."""
    dim, inner, experts, k = 256, 160, 12, 3
    up, down = Layer(experts, inner, dim, True, 1), Layer(experts, dim, inner, False, 2)
    g = torch.Generator().manual_seed(3)
    wr, w = torch.randn(experts, dim, generator=g).cuda() * 0.1, (1 + 0.1 * torch.randn(dim, generator=g)).cuda()
    batches = [(torch.randn(tokens, dim, generator=g).bfloat16().cuda(), torch.randn(tokens, dim, generator=g).cuda()) for _ in range(3)]

    def layer(y, r):
        r, x = dfp4.add_norm(y, r, w, post_weight=w)
        ids, weights = dfp4.route((x.float()[:, None, :] * wr).sum(-1), k)
        plan = dfp4.expert_plan(ids, experts)
        h = dfp4.experts_up(x, plan, up.handle)
        return (x, ids, weights, h) + tuple(dfp4.add_norm(dfp4.experts_down(h, plan, down.handle, weights), r, w))

    want = [layer(*b) for b in batches]
    for (y, r), (x, ids, weights, h, *_) in zip(batches, want):
        check_up(x.cpu(), ids.cpu(), up, experts, h)
        plan = dfp4.expert_plan(ids, experts)
        check_down(h.cpu(), ids.cpu(), down, experts, weights.cpu(), dfp4.experts_down(h, plan, down.handle, weights))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = [layer(*b) for b in batches]
    torch.cuda.current_stream().wait_stream(other)
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    static = [t.clone() for t in batches[0]]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = layer(*static)
    for turn in (0, 1, 2, 1, 0):
        for t, b in zip(static, batches[turn]):
            t.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[turn])), turn
        layer(*batches[(turn + 1) % 3])


def check_down_to_its_rounding(h, ids, layer, experts, weights, y):
    """y against float64: rows' products within 1e-5 sum |h||w|, k products and additions in fp32 (2^-24 each), and one rounding, y's own."""
    hq = quantized(h)
    offsets, order, _ = plain_plan(ids, experts)
    tokens, k = ids.shape
    dim = layer.values[0].shape[1]
    want, size, tol = np.zeros((tokens, dim)), np.zeros((tokens, dim)), np.zeros((tokens, dim))
    for e in range(experts):
        pairs, a = np.array(order[offsets[e]:offsets[e + 1]], dtype=int), hq[offsets[e]:offsets[e + 1]]
        if not len(pairs):
            continue
        w = synth.to_f64(weights).reshape(-1)[pairs][:, None]
        v = w * (a @ layer.values[0][e].T)
        np.add.at(want, pairs // k, v)
        np.add.at(size, pairs // k, np.abs(v))
        np.add.at(tol, pairs // k, 1e-5 * np.abs(w) * (np.abs(a) @ np.abs(layer.values[0][e]).T))
    half = HALF if y.dtype == torch.bfloat16 else 2.0 ** -24
    tol = (tol + 2.0 ** -23 * (k + 1) * size) * (1 + half) + half * np.abs(want) + 1e-38
    got = y.float().cpu().double().numpy()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())


@gpu
@pytest.mark.parametrize("tokens,k,experts,K,rows", [(300, 2, 4, 128, 64), (333, 5, 12, 224, 264), (1030, 2, 2, 96, 1800), (64, 2, 8, 128, 2056), (5, 3, 8, 96, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_down_rounds_once(tokens, k, experts, K, rows, dtype):
    """Weights of both signs, so that the experts' results cancel in part: what is rounded before their sum shows."""
    layer = Layer(experts, rows, K, False, seed=tokens)
    g = torch.Generator().manual_seed(K)
    h, weights = torch.randn(tokens * k, K, generator=g).bfloat16(), torch.rand(tokens, k, generator=g) - 0.5
    ids = ids_of(tokens, k, experts, seed=rows)
    plan = dfp4.expert_plan(ids.cuda(), experts)
    check_down_to_its_rounding(h, ids, layer, experts, weights, dfp4.experts_down(h.cuda(), plan, layer.handle, weights.cuda(), dtype=dtype))
