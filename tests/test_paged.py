"""Serving operators over the paged 4-bit cache: norms and rotation, the cache written and read back, attention over it, each
against a plain implementation in float64 (the quantizer: the oracle)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import dfp4_oracle as O
from paper_2501_01144_amd import dfp4, kvcache, synth

DIMS = [64, 96, 128, 192, 256]
HALF = torch.finfo(torch.bfloat16).eps / 2          # a rounding to bf16, relative to the value


# ---- refusals: no device is touched ----------------------------------------------------------------------------------------

def _cache(pages=256, residual=256, n_pages=4, page_tokens=32, n_slots=2, kv_heads=2, head_dim=64):
    return dfp4._CCache(pages, residual, n_pages, page_tokens, n_slots, kv_heads, head_dim)


def _batch(cu=256, lengths=256, table=256, slots=256, batch=2, table_width=2, tokens=4, max_new=0, max_length=0):
    return dfp4._CBatch(cu, lengths, table, slots, batch, table_width, tokens, max_new, max_length)


BAD = [
    (dict(head_dim=80), {}, -2), (dict(head_dim=0), {}, -2), (dict(page_tokens=48), {}, -2), (dict(page_tokens=0), {}, -2), (dict(kv_heads=0), {}, -2),
    (dict(n_pages=-1), {}, -2), (dict(n_slots=-1), {}, -2), (dict(n_pages=1 << 31), {}, -2), ({}, dict(batch=-1), -2), ({}, dict(tokens=-1), -2),
    ({}, dict(table_width=1 << 26), -2), ({}, dict(max_new=-1), -2), ({}, dict(max_length=-5), -2), ({}, dict(batch=1 << 30), -2),
    (dict(pages=0), {}, -1), (dict(residual=0), {}, -1), ({}, dict(cu=0), -1), ({}, dict(lengths=0), -1), ({}, dict(table=0), -1), ({}, dict(slots=0), -1),
    (dict(pages=128), {}, -3), (dict(residual=8), {}, -3), ({}, dict(table=2), -3),
]


@pytest.mark.parametrize("cache,batch,rc", BAD)
def test_calls_refuse_bad_caches_and_batches(cache, batch, rc):
    lib, c, b, vp = dfp4.load(), _cache(**cache), _batch(**batch), ctypes.c_void_p
    assert lib.dfp4_paged_write(vp(16), 128, 64, vp(16), 128, 64, c, b, vp(0)) == rc
    assert lib.dfp4_paged_read(c, b, vp(16), vp(16), 1, vp(0)) == rc
    assert lib.dfp4_paged_attention(vp(16), 256, 64, 4, c, b, 1.0, 0.0, 0, vp(0), vp(16), 256, 64, vp(0), vp(16), 1 << 30, vp(0)) == rc


def test_calls_refuse_bad_arguments():
    lib, vp = dfp4.load(), ctypes.c_void_p
    c, b = _cache(), _batch()
    write = lambda k=16, ks=128, kh=64, v=16, vs=128, vh=64: lib.dfp4_paged_write(vp(k), ks, kh, vp(v), vs, vh, c, b, vp(0))  # noqa: E731
    assert (write(k=0), write(v=0), write(k=8), write(ks=4), write(kh=63), write(vs=132), write(vh=4)) == (-1, -1, -3, -3, -3, -3, -3)
    read = lambda k=16, v=16, t=1: lib.dfp4_paged_read(c, b, vp(k), vp(v), t, vp(0))  # noqa: E731
    assert (read(k=0), read(v=0), read(k=24), read(t=2)) == (-1, -1, -3, -4)

    def attend(q=16, qs=256, qh=64, heads=4, softcap=0.0, window=0, slopes=0, out=16, os=256, oh=64, lse=0, ws=16, n=1 << 30, b=b):
        return lib.dfp4_paged_attention(vp(q), qs, qh, heads, c, b, 1.0, softcap, window, vp(slopes), vp(out), os, oh, vp(lse), vp(ws), n, vp(0))
    assert (attend(heads=3), attend(heads=0), attend(heads=-2), attend(window=-1), attend(softcap=-1.0), attend(softcap=float("nan")), attend(softcap=float("inf"))) == (-2,) * 7
    assert (attend(q=0), attend(out=0), attend(q=20), attend(qs=12), attend(oh=2), attend(slopes=2), attend(lse=1), attend(ws=8)) == (-1, -1) + (-3,) * 6
    # a long context is split between workgroups, and that takes a workspace
    long = _batch(table_width=1 << 12)
    need = lib.dfp4_paged_attention_workspace_bytes(c, long, 4, 0)
    assert need > 0 and attend(b=long, ws=0, n=0) == -5 and attend(b=long, n=need - 1) == -5
    assert lib.dfp4_paged_attention_workspace_bytes(c, _batch(table_width=4), 4, 0) == 0
    # nothing to do
    assert attend(b=_batch(tokens=0)) == 0 and attend(b=_batch(batch=0)) == 0
    assert lib.dfp4_paged_write(vp(0), 0, 0, vp(0), 0, 0, c, _batch(tokens=0), vp(0)) == 0

    def rope(q=16, qs=256, qh=64, heads=2, k=16, ks=64, kh=64, kv=1, tokens=4, dim=64, pos=16, freq=16, rotary=64, qo=16, ko=16, w=0):
        return lib.dfp4_norm_rope(vp(q), qs, qh, heads, vp(k), ks, kh, kv, tokens, dim, vp(w), vp(0), 1e-6, vp(pos), vp(freq), rotary, 0, vp(qo), vp(ko), vp(0))
    assert (rope(dim=80), rope(dim=288), rope(dim=0), rope(rotary=8), rope(rotary=96), rope(rotary=-16), rope(tokens=-1), rope(heads=-1)) == (-2,) * 8
    assert (rope(q=0), rope(k=0), rope(pos=0), rope(freq=0), rope(qo=0), rope(ko=0)) == (-1,) * 6
    assert (rope(q=8), rope(qs=100), rope(kh=4), rope(qo=24), rope(w=2)) == (-3,) * 5
    assert rope(tokens=0) == 0 and rope(heads=0, kv=0) == 0


def test_cell_bytes():
    # 4 bits an element, a scale and a dialect a block of 32, rounded up for the lanes that read them
    for dim in DIMS:
        assert 32 * dim <= dfp4.paged_cell_bytes(dim) - 3 * dim / 2 * 2 <= 32 * dim + 32 * 8
    assert [dfp4.paged_cell_bytes(d) for d in (0, 32, 80, 160, 512, -64)] == [0] * 6
    assert dfp4.paged_cell_bytes(128) == 4480


# ---- plain implementations -------------------------------------------------------------------------------------------------

def _quantized(x):
    """x bf16 [rows, K]: the values of its 4-bit form, float64."""
    return O.dfp4_dequantize(*O.dfp4_quantize(synth.to_f64(x))) if x.numel() else synth.to_f64(x)


def _keys(k):
    return _quantized(k.reshape(-1, k.shape[-1])).reshape(k.shape)


def _values(v, length):
    """v bf16 [length, heads, dim]: whole chunks of 32 tokens in 4 bits, the rest as it is."""
    out = synth.to_f64(v).copy()
    whole = length // 32 * 32
    if whole:
        t = v[:whole].permute(1, 2, 0).reshape(-1, whole)
        out[:whole] = _quantized(t).reshape(v.shape[1], v.shape[2], whole).transpose(2, 0, 1)
    return out


class Sequences:
    """Sequences of random keys and values in a cache of pages in random order, brought there in steps."""

    def __init__(self, lengths, dim, kv_heads, page, seed=0, spare=3, poison=True, width=None, factor=6.0):
        self.g = torch.Generator().manual_seed(seed)
        self.lengths, self.dim, self.kv_heads, self.page = list(lengths), dim, kv_heads, page
        n = len(lengths)
        self.width = width or max(1, -(-max(lengths + [1]) // page))
        n_pages = n * self.width + spare
        self.cache = kvcache.PagedCache(n_pages, page, kv_heads, dim, n + 2, torch.device("cuda"))
        if poison:                      # what nobody wrote may be anything
            self.cache.pages.fill_(0xff)
            self.cache.residual.fill_(float("nan"))
        self.table = torch.randperm(n_pages, generator=self.g)[:n * self.width].view(n, self.width).int()
        self.slots = torch.randperm(n + 2, generator=self.g)[:n].int()
        self.k, self.v = [], []
        for L in lengths:
            k, v = torch.randn(L, kv_heads, dim, generator=self.g), torch.randn(L, kv_heads, dim, generator=self.g)
            k[..., 3] *= factor
            v[..., 5] *= factor
            self.k.append(k.bfloat16())
            self.v.append(v.bfloat16())

    def batch(self, new, lengths=None, **hints):
        cu = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        lengths = torch.tensor(self.lengths if lengths is None else lengths, dtype=torch.int32)
        return kvcache.PagedBatch(cu.cuda(), lengths.cuda(), self.table.cuda(), self.slots.cuda(), tokens=int(sum(new)), **hints)

    def write(self, new, after, **hints):
        k, v = (torch.cat([x[b][after[b] - new[b]:after[b]] for b in range(len(new))]).cuda() for x in (self.k, self.v))
        dfp4.paged_write(k, v, self.cache, self.batch(new, after, **hints))

    def fill(self):
        self.write(self.lengths, self.lengths, max_new=max(self.lengths))
        return self

    def stands_for(self):
        return [_keys(k) for k in self.k], [_values(v, len(v)) for v in self.v]


def _attention(s, q, new, scale, softcap=0.0, window=0, slopes=None):
    """out, lse, and for the tolerance: sum p |v|, the largest sum |q| |k| of a row's keys, each [tokens, heads(, dim)]."""
    ks, vs = s.stands_for()
    q = synth.to_f64(q)
    heads, group = q.shape[1], q.shape[1] // s.kv_heads
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    size, dot = np.zeros(q.shape), np.zeros(q.shape[:2])
    row = 0
    for b, n in enumerate(new):
        L = s.lengths[b]
        for i in range(n):
            p = L - n + i
            lo = max(0, p - window + 1) if window else 0
            for h in range(heads if p >= 0 else 0):
                k, v = ks[b][lo:p + 1, h // group], vs[b][lo:p + 1, h // group]
                z = scale * (k @ q[row, h])
                if softcap:
                    z = softcap * np.tanh(z / softcap)
                if slopes is not None:
                    z = z - float(slopes[h]) * (p - np.arange(lo, p + 1))
                w = np.exp(z - z.max())
                lse[row, h] = z.max() + math.log(w.sum())
                w /= w.sum()
                out[row, h], size[row, h], dot[row, h] = w @ v, w @ np.abs(v), (np.abs(k) @ np.abs(q[row, h])).max() * abs(scale)
            row += 1
    return out, lse, size, dot


def _check_attention(got, lse, want):
    """A probability is off by 2^-8 of itself at most (a bf16), the instruction's sums by 2^-12 of sum |a| |b|
    (it aligns products to the largest), a score by that of its own sum; the result is rounded to bf16."""
    out, wlse, size, dot = want
    score = 2.0 ** -12 * dot
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(got).all()
    tol = HALF * np.abs(out) + (2.0 ** -8 + 2.0 ** -12 + 2 * score[..., None]) * size + 1e-30
    assert (np.abs(got - out) <= tol).all(), float((np.abs(got - out) / tol).max())
    none = np.isneginf(wlse)
    assert np.array_equal(np.isneginf(lse), none) and (got[none] == 0).all()
    assert (np.abs(lse - wlse)[~none] <= (score + 2.0 ** -20 * (1 + np.abs(wlse)))[~none]).all()
    norm = np.linalg.norm(out)
    if norm:
        assert np.linalg.norm(got - out) <= HALF * norm * 1.1


def _attend(s, new, heads, seed=1, softcap=0.0, window=0, slopes=None, scale=None, **hints):
    q = torch.randn(sum(new), heads, s.dim, generator=torch.Generator().manual_seed(seed))
    q[..., 7] *= 3
    q = q.bfloat16()
    scale = s.dim ** -0.5 if scale is None else scale
    got, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch(new, **hints), scale=scale, softcap=softcap, window=window,
                                    slopes=None if slopes is None else slopes.cuda(), return_lse=True)
    torch.cuda.synchronize()
    _check_attention(got, lse, _attention(s, q, new, scale, softcap, window, slopes))
    return q, got, lse


# ---- the cache ---------------------------------------------------------------------------------------------------------------

def _check_read(s, new, lengths, dtype, **hints):
    k, v = dfp4.paged_read(s.cache, s.batch(new, lengths, **hints), dtype=dtype)
    torch.cuda.synchronize()
    row = 0
    for b, n in enumerate(new):
        if n:
            L = lengths[b]
            assert np.array_equal(k[row:row + n].double().cpu().numpy(), _keys(s.k[b][:L])[L - n:]), b
            assert np.array_equal(v[row:row + n].double().cpu().numpy(), _values(s.v[b][:L], L)[L - n:]), b
        row += n


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("page,kv_heads,lengths", [(32, 1, [1, 31, 32, 33]), (64, 3, [200, 1, 64, 95]), (96, 2, [97, 300])])
def test_cache_holds_what_the_quantizer_makes(dim, page, kv_heads, lengths):
    s = Sequences(lengths, dim, kv_heads, page, seed=dim).fill()
    _check_read(s, lengths, lengths, torch.bfloat16)
    _check_read(s, [min(L, 5) for L in lengths], lengths, torch.float32, max_new=5)


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [[1] * 70, [31, 1, 1, 31, 33, 5], [40, 64, 7, 20], [5, 100, 3, 3, 61]])
def test_cache_grows_in_steps(steps):
    """Steps that start and end anywhere in a chunk, begin and end in the same one, or span several."""
    s = Sequences([sum(steps), sum(steps) - 9], 64, 2, 64, seed=len(steps))
    at = [0, 0]
    for n in steps:
        new = [n, max(0, min(n, s.lengths[1] - at[1]))]
        at = [at[0] + n, at[1] + new[1]]
        s.write(new, at)
        _check_read(s, at, at, torch.bfloat16)


@pytest.mark.gpu
def test_cache_from_strided_rows():
    s = Sequences([77, 50], 128, 2, 64, seed=5)
    joint = torch.randn(127, 3 + 2 + 2, 128, generator=s.g).bfloat16().cuda()         # queries, keys and values of a token in a row
    k, v = joint[:, 3:5], joint[:, 5:]
    s.k, s.v = ([x[:77].cpu().contiguous(), x[77:].cpu().contiguous()] for x in (k, v))
    dfp4.paged_write(k, v, s.cache, s.batch([77, 50]))
    _check_read(s, [77, 50], [77, 50], torch.bfloat16)
    by_head = torch.empty(2, 127, 128, dtype=torch.bfloat16, device="cuda").copy_(k.transpose(0, 1))
    s.cache.pages.fill_(0xff)
    dfp4.paged_write(by_head.transpose(0, 1), v, s.cache, s.batch([77, 50], max_new=1))
    _check_read(s, [77, 50], [77, 50], torch.float32, max_new=1)


@pytest.mark.gpu
def test_cache_beyond_four_gigabytes():
    s = Sequences([70], 128, 1, 32, seed=3)
    n_pages = (5 << 30) // dfp4.paged_cell_bytes(128)
    s.cache = kvcache.PagedCache(n_pages, 32, 1, 128, 3, torch.device("cuda"))
    s.table = torch.tensor([[n_pages - 1, n_pages - 5, n_pages // 2 + 1]], dtype=torch.int32)
    s.fill()
    _check_read(s, [70], [70], torch.bfloat16)
    _attend(s, [3], 4)
    assert int(s.cache.pages[:n_pages // 2].max()) == 0


@pytest.mark.gpu
def test_pages_and_slots_out_of_range_are_absent():
    s = Sequences([100, 70, 40], 64, 2, 32, seed=8)
    for bad in (-1, s.cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        s.table[0, 1] = bad                               # tokens 32 .. 63 of sequence 0
        s.slots[1] = bad                                  # the incomplete chunk's values of sequence 1: tokens 64 .. 69
        before = s.cache.pages.clone()
        s.fill()
        k, v = dfp4.paged_read(s.cache, s.batch(s.lengths))
        out, lse = dfp4.paged_attention(torch.ones(3, 2, 64, dtype=torch.bfloat16, device="cuda"), s.cache, s.batch([1, 1, 1]), return_lse=True)
        torch.cuda.synchronize()
        used = set(int(x) for row, L in zip(s.table, s.lengths) for x in row[:-(-L // 32)] if 0 <= int(x) < s.cache.n_pages)
        others = [x for x in range(s.cache.n_pages) if x not in used]
        assert torch.equal(s.cache.pages[others], before[others])
        k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
        want_k, want_v = s.stands_for()
        want_k[0][32:64], want_v[0][32:64], want_v[1][64:] = 0, 0, 0
        assert np.array_equal(k, np.concatenate(want_k)) and np.array_equal(v, np.concatenate(want_v))
        seen = [np.r_[0:32, 64:100], np.r_[0:64], np.r_[0:40]]
        for b in range(3):
            z = want_k[b][seen[b]].sum(-1) / 8
            w = np.exp(z - z.max(0))
            w /= w.sum(0)
            want = np.einsum("th,thd->hd", w, want_v[b][seen[b]])
            assert np.abs(out[b].double().cpu().numpy() - want).max() <= 2.0 ** -6 * np.abs(want).max()
            # a score: 64 products of at most 2^-12 of their sizes
            assert np.abs(lse[b].double().cpu().numpy() - (z.max(0) + np.log(np.exp(z - z.max(0)).sum(0)))).max() <= 2.0 ** -12 * 64


@pytest.mark.gpu
def test_lengths_and_token_ranges_out_of_range():
    """Lengths beyond the table, below zero, and shorter than their new tokens; ranges beyond the rows."""
    s = Sequences([64, 64, 64], 64, 1, 32, seed=4, poison=False).fill()
    b = s.batch([2, 2, 2], [10 ** 9, -7, 1])
    q = torch.randn(6, 1, 64, generator=s.g).bfloat16().cuda()
    out, lse = dfp4.paged_attention(q, s.cache, b, return_lse=True)
    k, v = dfp4.paged_read(s.cache, b)
    torch.cuda.synchronize()
    assert (out[2:5] == 0).all() and torch.isneginf(lse[2:5]).all() and torch.isfinite(lse[[0, 1, 5]]).all()
    assert (k[2:5] == 0).all() and (v[2:5] == 0).all()
    assert np.array_equal(k[:2].double().cpu().numpy(), _keys(s.k[0])[62:])
    for cu in ([-5, 3, 2, 10 ** 6], [0, 100, 100, 100], [4, 2, 0, -1]):
        b.cu_tokens.copy_(torch.tensor(cu, dtype=torch.int32))
        dfp4.paged_attention(q, s.cache, b)
        dfp4.paged_read(s.cache, b)
        torch.cuda.synchronize()


# ---- attention -----------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("page,kv_heads,heads,lengths,new", [
    (32, 1, 1, [1], [1]),
    (64, 2, 8, [1, 31, 32, 33, 128, 129, 700], [1] * 7),
    (32, 2, 2, [5, 160, 161, 40], [5, 3, 2, 40]),
    (96, 1, 5, [333, 200, 64], [7, 0, 33]),
    (128, 3, 48, [257], [2]),
])
def test_attention(dim, page, kv_heads, heads, lengths, new):
    s = Sequences(lengths, dim, kv_heads, page, seed=dim + heads).fill()
    _attend(s, new, heads, max_new=max(new))


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("options", [
    dict(softcap=5.0), dict(window=1), dict(window=33), dict(window=64, softcap=20.0), dict(slopes=True), dict(slopes=True, window=100, softcap=30.0), dict(scale=0.5),
    dict(scale=0.0), dict(scale=-0.3)])
def test_attention_options(dim, options):
    s = Sequences([300, 45, 129], dim, 2, 64, seed=dim).fill()
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = torch.tensor([0.5, 0.25, 0.0, 0.03125, 0.1, 2.0])
    _attend(s, [9, 45, 1], 6, **options)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_rows_without_keys(dim):
    """More new tokens than the sequence is long: those before position 0 see nothing."""
    s = Sequences([3, 0, 40, 1], dim, 2, 32, seed=dim)
    s.lengths[1] = 0
    new = [8, 4, 50, 1]
    s.write([3, 0, 40, 1], s.lengths)
    _attend(s, new, 4)
    _attend(s, new, 4, window=2)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128, 192])
@pytest.mark.parametrize("new", [1, 5, 70])
def test_attention_of_long_contexts_is_split(dim, new):
    s = Sequences([9000, 2049, 515], dim, 1, 64, seed=new).fill()
    c, b = s.cache.c, s.batch([new] * 3, max_new=new).c(3 * new)
    assert dfp4.load().dfp4_paged_attention_workspace_bytes(c, b, 4, 0) > 0
    q, got, lse = _attend(s, [new] * 3, 4, max_new=new)
    # the same bits again, and with a workspace of the caller's that holds anything
    ws = torch.full((dfp4.load().dfp4_paged_attention_workspace_bytes(c, b, 4, 0),), 0xff, dtype=torch.uint8, device="cuda")
    again, lse2 = dfp4.paged_attention(q.cuda(), s.cache, s.batch([new] * 3, max_new=new), return_lse=True, workspace=ws)
    assert torch.equal(again.view(torch.int16), got.view(torch.int16)) and torch.equal(lse2, lse)
    with pytest.raises(dfp4.Dfp4Error, match="workspace"):
        dfp4.paged_attention(q.cuda(), s.cache, s.batch([new] * 3, max_new=new), workspace=ws[:-16])


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("options", [dict(), dict(window=100), dict(softcap=5.0, slopes=True), dict(scale=-0.2), dict(scale=0.0, window=33)])
def test_attention_of_many_rows(dim, options):
    """Enough rows for the kernel that expands keys once for 256 of them (2400 rows of each KV head, a table wide enough)."""
    s = Sequences([600, 33, 431, 20, 64], dim, 2, 64, seed=dim, width=40).fill()
    options = dict(options)
    if options.get("slopes"):
        options["slopes"] = torch.tensor([0.5, 0.25, 0.0, 0.03125, 0.1, 2.0, 1.0, 0.01])
    _attend(s, [90, 33, 3, 0, 64], 8, max_new=600, **options)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_attention_of_many_rows_split_and_without_keys(dim):
    """The same where the keys are split, rows come before position 0, and pages or slots are missing: against 16 rows a workgroup."""
    s = Sequences([3000, 40, 0, 777], dim, 1, 32, seed=dim, width=1024).fill()
    new = [70, 90, 5, 64]
    q, got, lse = _attend(s, new, 8, max_new=90)
    assert dfp4.load().dfp4_paged_attention_workspace_bytes(s.cache.c, s.batch(new, max_new=90).c(sum(new)), 8, 0) > 0
    s.table[0, 5], s.table[0, 90], s.table[3, 0], s.slots[3] = -1, 10 ** 6, s.cache.n_pages, -1
    many, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch(new, max_new=90), return_lse=True)
    few, lse2 = dfp4.paged_attention(q.cuda(), s.cache, s.batch(new, max_new=1), return_lse=True)
    torch.cuda.synchronize()
    assert torch.isfinite(many).all() and torch.equal(torch.isneginf(lse), torch.isneginf(lse2))
    # both are within 2^-8 sum p |v| (and a rounding) of the same values
    assert float((many.float() - few.float()).norm() / few.float().norm()) <= 2 * HALF
    assert float((lse - lse2)[~torch.isneginf(lse)].abs().max()) <= 2.0 ** -10
    assert (many[70:70 + 50] == 0).all() and not torch.equal(many[:70], got[:70])


@pytest.mark.gpu
@pytest.mark.parametrize("hints", [dict(), dict(max_new=1), dict(max_new=1000), dict(max_length=1), dict(max_length=10 ** 6), dict(max_new=2, max_length=400)])
def test_attention_does_not_depend_on_the_hints(hints):
    s = Sequences([1500, 300, 700], 128, 2, 32, seed=2).fill()
    _attend(s, [40, 3, 17], 4, **hints)


@pytest.mark.gpu
def test_attention_of_extreme_values():
    """Queries and keys from tiny to huge, scores that leave one key, values far above and below 1."""
    for q_size, k_size, v_size, scale in [(1e-30, 1.0, 1.0, 1.0), (1e18, 1e18, 1.0, 1e-36), (1.0, 1e-25, 1e30, 1.0), (30.0, 30.0, 1e-30, 1.0), (1.0, 1.0, 1e-36, 1.0)]:
        s = Sequences([150], 64, 1, 32, seed=9, factor=1.0)
        s.k, s.v = [(s.k[0].double() * k_size).bfloat16()], [(s.v[0].double() * v_size).bfloat16()]
        s.fill()
        q = (torch.randn(2, 2, 64, generator=s.g).double() * q_size).bfloat16()
        got, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch([2]), scale=scale, return_lse=True)
        want = _attention(s, q, [2], scale)
        _check_attention(got, lse, (want[0], want[1], want[2] + 1e-38, want[3]))


@pytest.mark.gpu
def test_attention_into_strided_rows_on_another_stream():
    s = Sequences([140, 35], 128, 2, 64, seed=6).fill()
    joint = torch.randn(36, 4 + 2, 128, generator=s.g).bfloat16()
    q = joint[:, :4].contiguous()
    into = torch.full((36, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    dense = joint.cuda()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got, lse = dfp4.paged_attention(dense[:, :4], s.cache, s.batch([1, 35]), out=into[:, 2:6], return_lse=True)
    stream.synchronize()
    _check_attention(got, lse, _attention(s, q, [1, 35], 128 ** -0.5))
    assert (into[:, :2] == 7).all() and (into[:, 6:] == 7).all()


@pytest.mark.gpu
def test_a_step_in_a_graph():
    """Norms, write and attention of one token a sequence, captured once; lengths and pages are device memory, so that every replay
    is the next token."""
    n, dim, kv, heads = 3, 128, 2, 8
    s = Sequences([100, 62, 2100], dim, kv, 64, seed=11)
    grown = [L - 8 for L in s.lengths]
    s.write(grown, grown)
    raw = torch.randn(8, n, heads + kv, dim, generator=s.g).bfloat16().cuda()
    freq = (1.0 / 10000.0 ** (torch.arange(0, dim, 2).double() / dim)).float().cuda()
    weight = torch.ones(dim, device="cuda")
    x, v, pos = raw[0].clone(), s.v[0][:n].cuda().clone(), torch.zeros(n, dtype=torch.int32, device="cuda")
    b = s.batch([1] * n, grown, max_new=1)

    def step():
        q, k = dfp4.norm_rope(x[:, :heads], x[:, heads:], pos, freq, weight, weight)
        dfp4.paged_write(k, v, s.cache, b)
        return k, dfp4.paged_attention(q, s.cache, b, return_lse=True)
    # (captured without a run before it: what a run would write is written by the first replay)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        k, (out, lse) = step()
    for i in range(8):
        at = [L + i + 1 for L in grown]
        new_v = torch.stack([s.v[j][at[j] - 1] for j in range(n)])
        x.copy_(raw[i])
        v.copy_(new_v.cuda())
        b.lengths.copy_(torch.tensor(at, dtype=torch.int32))
        pos.copy_(b.lengths - 1)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = out.clone(), lse.clone()
        for j in range(n):
            s.k[j][at[j] - 1] = k[j].cpu()
        q, _ = dfp4.norm_rope(x[:, :heads], x[:, heads:], pos, freq, weight, weight)
        eager, eager_lse = dfp4.paged_attention(q, s.cache, s.batch([1] * n, at, max_new=1), return_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), eager.view(torch.int16)) and torch.equal(got_lse, eager_lse), i
    _check_attention(got, got_lse, _attention(s, q.cpu(), [1] * n, dim ** -0.5))


# ---- norms and rotation ----------------------------------------------------------------------------------------------------------

def _rope(x, w, pos, freq, interleaved, eps):
    y = synth.to_f64(x)
    if w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * w.double().numpy()
    half = len(freq)
    angle = pos.double().numpy()[:, None, None] * freq.double().numpy()
    c, s = np.cos(angle), np.sin(angle)
    out, size = y.copy(), np.abs(y)
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    out[..., i], out[..., j] = y[..., i] * c - y[..., j] * s, y[..., j] * c + y[..., i] * s
    size[..., i] = size[..., j] = np.abs(y[..., i]) + np.abs(y[..., j])
    return out, size


@pytest.mark.gpu
@pytest.mark.parametrize("dim,rotary", [(32, 32), (64, 64), (64, 32), (96, 96), (96, 16), (128, 128), (128, 0), (160, 80), (192, 192), (256, 256), (256, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv_heads,norm", [(1, 32, 8, True), (37, 3, 1, True), (5, 17, 17, False), (3, 6, 0, True)])
def test_norm_rope(dim, rotary, interleaved, tokens, heads, kv_heads, norm):
    g = torch.Generator().manual_seed(dim + rotary)
    x = (torch.randn(tokens, heads + kv_heads, dim, generator=g) * torch.exp(2 * torch.randn(tokens, 1, 1, generator=g))).bfloat16()
    pos = torch.randint(0, 1 << 20, (tokens,), generator=g).int()
    freq = (1.0 / 500000.0 ** (torch.arange(0, rotary, 2).double() / max(rotary, 1))).float()
    wq, wk = ((1 + 0.3 * torch.randn(dim, generator=g)) if norm else None for _ in range(2))
    d = x.cuda()
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    q, k = dfp4.norm_rope(d[:, :heads], d[:, heads:] if kv_heads else None, pos.cuda(), freq.cuda(), cuda(wq), cuda(wk), eps=1e-5, interleaved=interleaved)
    torch.cuda.synchronize()
    for got, part, w in ((q, x[:, :heads], wq), (k, x[:, heads:], wk)):
        if got is None:
            continue
        want, size = _rope(part, w, pos, freq, interleaved, 1e-5)
        # a rounding to bf16; before it some twenty roundings to fp32
        assert (np.abs(got.double().cpu().numpy() - want) <= HALF * np.abs(want) + 20 * 2.0 ** -24 * size).all()


@pytest.mark.gpu
def test_norm_rope_in_place_and_zeros():
    x, y = torch.randn(4, 6, 128).bfloat16().cuda(), torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    pos, freq, w = torch.arange(4, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda"), torch.ones(128, device="cuda")
    q, k = dfp4.norm_rope(x, y, pos, freq, w, w)
    q2, k2 = dfp4.norm_rope(x, y, pos, freq, w, w, out=(x, y))
    torch.cuda.synchronize()
    assert q2.data_ptr() == x.data_ptr() and torch.equal(q2.view(torch.int16), q.view(torch.int16)) and (k2 == 0).all()


@pytest.mark.gpu
def test_the_layer_of_the_example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    off, _ = example.run(prompts=(40, 31, 1), tokens=5)
    assert off <= HALF


# ---- scores with caps of any size -----------------------------------------------------------------------------------------------

def _few_or_many_rows(dim, many):
    """Sequences, new tokens, heads and hints of a call with few rows, or with enough for the kernel that takes 256 rows a workgroup."""
    if many:
        s, new, hints = Sequences([600, 33, 431, 20, 64], dim, 2, 64, seed=dim, width=40).fill(), [90, 33, 3, 0, 64], dict(max_new=190)
        assert dfp4.paged_attention_rows(s.cache, s.batch(new, **hints), sum(new), 8) == 256
        return s, new, 8, hints
    return Sequences([300, 45, 129], dim, 2, 64, seed=dim).fill(), [9, 45, 1], 6, dict(max_new=45)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,many", [(64, False), (128, False), (256, False), (64, True), (96, True), (128, True)])
def test_caps_far_above_the_scores_leave_them_alone(dim, many):
    s, new, heads, hints = _few_or_many_rows(dim, many)
    scale = dim ** -0.5
    q, _, plain = _attend(s, new, heads, **hints)
    want = _attention(s, q, new, scale)
    seen = ~np.isneginf(want[1])
    for cap in (1e3, 1e6, 1e10, 1e30):
        _, _, lse = _attend(s, new, heads, softcap=cap, **hints)
        shift = (lse - plain).double().cpu().numpy()[seen]
        want_shift = (_attention(s, q, new, scale, softcap=cap)[1] - want[1])[seen]
        # both calls have the same scores: a cap changes one by what it should and 2^-18 of it (at most `dot`); two results of 2^-20
        tol = 2.0 ** -18 * want[3][seen] + 2 * 2.0 ** -20 * (1 + np.abs(want[1][seen]))
        assert (np.abs(shift - want_shift) <= tol).all(), (cap, float((np.abs(shift - want_shift) / tol).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("dim,many", [(128, False), (128, True)])
@pytest.mark.parametrize("cap", [1e-39, 1e-30, 0.01, 1.0, 300.0])
def test_caps_near_and_below_the_scores(dim, many, cap):
    s, new, heads, hints = _few_or_many_rows(dim, many)
    _attend(s, new, heads, softcap=cap, **hints)
    s.k[0][:] = 0                                    # scores of zero
    s.fill()
    _attend(s, new, heads, softcap=cap, scale=4.0, **hints)


# ---- batches whose tensors change -----------------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_read_takes_the_tokens_that_a_batch_has_now():
    s = Sequences([70, 40], 64, 2, 32, seed=21).fill()
    b = s.batch([3, 2])
    b = kvcache.PagedBatch(b.cu_tokens, b.lengths, b.table, b.slots)
    for new in ([3, 2], [70, 40], [1, 0], [0, 0], [5, 33]):
        b.cu_tokens.copy_(torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32))
        k, v = dfp4.paged_read(s.cache, b)
        assert b.tokens == len(k) == len(v) == sum(new)
        want_k, want_v = ([x[i][len(x[i]) - n:] for i, n in enumerate(new)] for x in s.stands_for())
        assert np.array_equal(k.double().cpu().numpy(), np.concatenate(want_k)) and np.array_equal(v.double().cpu().numpy(), np.concatenate(want_v))


# ---- positions far beyond any cache that fits ------------------------------------------------------------------------------------

def test_the_page_of_a_chunk(tmp_path):
    """chunk / chunks of a page for every size of a page, around every power of two and every border of a page near it."""
    import os
    import subprocess
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_01144_amd", "csrc")
    (tmp_path / "t.cpp").write_text(r"""
#include <cstdio>
#include <initializer_list>
#include "page_of.h"
int main() {
    for (uint32_t n = 1; n <= 1u << 15; ++n) {
        const dfp4::PageDivision by = dfp4::page_division(n);
        for (int bit = 0; bit < 31; ++bit)
            for (int64_t near : {(int64_t)1 << bit, ((int64_t)1 << bit) / n * n, ((((int64_t)1 << bit) / n) + 1) * n})
                for (int64_t chunk = near - 2; chunk <= near + 2; ++chunk)
                    if (chunk >= 0 && chunk < (int64_t)1 << 31 && dfp4::page_of(by, (int)chunk) != (int)(chunk / n)) {
                        std::printf("%lld / %u: %d\n", (long long)chunk, n, dfp4::page_of(by, (int)chunk));
                        return 1;
                    }
    }
    return 0;
}
""")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", csrc, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    done = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout


@pytest.mark.gpu
@pytest.mark.parametrize("page", [32, 64, 96])
def test_positions_beyond_two_to_the_29(page):
    """The last 102 tokens of a sequence whose earlier pages are not there."""
    s = Sequences([102], 64, 2, page, seed=page)
    first = -(-(1 << 29) // page) + 3                    # pages before them
    table = torch.full((1, first + s.width), -1, dtype=torch.int32)
    table[:, first:] = s.table
    s.table = table
    at = first * page + 102
    dfp4.paged_write(s.k[0].cuda(), s.v[0].cuda(), s.cache, s.batch([102], [at]))
    k, v = dfp4.paged_read(s.cache, s.batch([102], [at]))
    torch.cuda.synchronize()
    assert np.array_equal(k.double().cpu().numpy(), _keys(s.k[0])) and np.array_equal(v.double().cpu().numpy(), _values(s.v[0], 102))
    q = torch.randn(3, 4, 64, generator=s.g).bfloat16()
    got, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch([3], [at], max_new=3), window=90, return_lse=True)
    _check_attention(got, lse, _attention(s, q, [3], 64 ** -0.5, window=90))


# ---- arguments of the Python calls -----------------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_workspaces_are_memory_of_the_device():
    s = Sequences([2049], 64, 1, 64, seed=31).fill()
    need = dfp4.load().dfp4_paged_attention_workspace_bytes(s.cache.c, s.batch([1], max_new=1).c(1), 4, 0)
    q = torch.randn(1, 4, 64, generator=s.g).bfloat16().cuda()
    for bad in (torch.empty(need, dtype=torch.uint8), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            dfp4.paged_attention(q, s.cache, s.batch([1], max_new=1), workspace=bad)
    # of any type: its bytes count
    ws = torch.empty(-(-need // 4), dtype=torch.float32, device="cuda")
    assert torch.equal(dfp4.paged_attention(q, s.cache, s.batch([1], max_new=1), workspace=ws), dfp4.paged_attention(q, s.cache, s.batch([1], max_new=1)))


@pytest.mark.gpu
def test_norm_rope_without_a_rotation():
    x, w = torch.randn(5, 4, 64).bfloat16().cuda(), torch.rand(64, device="cuda")
    q, k = dfp4.norm_rope(x, None, None, None, w)
    want, size = _rope(x.cpu(), w.cpu(), torch.zeros(5), torch.zeros(0), False, 1e-6)
    assert k is None and (np.abs(q.double().cpu().numpy() - want) <= HALF * np.abs(want) + 20 * 2.0 ** -24 * size).all()
    into = torch.empty_like(x)
    q2, k2 = dfp4.norm_rope(x, None, None, None, w, out=(into, None))
    assert q2 is into and k2 is None and torch.equal(q2, q)
    with pytest.raises(dfp4.Dfp4Error):                  # a rotation by what?
        dfp4.norm_rope(x, None, None, torch.ones(32, device="cuda"), w, out=(into, None))


@pytest.mark.gpu
def test_the_stride_of_a_single_token_or_head_does_not_matter():
    s = Sequences([40], 64, 1, 32, seed=33)
    s.write([39], [39])
    one = lambda x: torch.as_strided(x.cuda(), (1, 1, 64), (3, 5, 1))  # noqa: E731
    dfp4.paged_write(one(s.k[0][39]), one(s.v[0][39]), s.cache, s.batch([1], [40]))
    _check_read(s, [40], [40], torch.bfloat16)
    q = torch.randn(1, 1, 64, generator=s.g).bfloat16()
    freq, pos = torch.ones(32, device="cuda"), torch.tensor([7], dtype=torch.int32, device="cuda")
    assert torch.equal(dfp4.norm_rope(one(q), one(q), pos, freq)[1], dfp4.norm_rope(q.cuda(), None, pos, freq)[0])
    into = torch.empty(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(dfp4.norm_rope(one(q), None, pos, freq, out=(into, None))[0], dfp4.norm_rope(q.cuda(), None, pos, freq)[0])
    want = dfp4.paged_attention(q.cuda(), s.cache, s.batch([1]))
    assert torch.equal(dfp4.paged_attention(one(q), s.cache, s.batch([1])), want)
    assert torch.equal(dfp4.paged_attention(one(q), s.cache, s.batch([1]), out=one(into)), want)


# ---- sizes that one launch does not hold -----------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_norm_rope_of_more_tokens_than_a_launch_holds():
    """Without a rotation a workgroup of 256 threads takes four tokens, and a launch has fewer than 2^32 threads."""
    n = (1 << 26) + 5
    x = torch.ones(n, 1, 32, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(3)
    places = [0, 4 * ((1 << 24) - 1) - 3, n - 8]
    for at in places:
        x[at:at + 8] = torch.randn(8, 1, 32, generator=g).bfloat16().cuda()
    w = torch.rand(32, generator=g) + 0.5
    q, _ = dfp4.norm_rope(x, None, None, None, w.cuda())
    for at in places:
        want, _ = _rope(x[at:at + 8].cpu(), w, torch.zeros(8), torch.zeros(0), False, 1e-6)
        assert (np.abs(q[at:at + 8].double().cpu().numpy() - want) <= (HALF + 20 * 2.0 ** -24) * np.abs(want)).all()
    q[places[1]:places[1] + 8], q[-8:], q[:8] = q[1000], q[1000], q[1000]
    assert bool((q == q[1000]).all())


BIG = 1 << 62


@pytest.mark.parametrize("cache,batch,heads,window", [
    (dict(kv_heads=8), dict(batch=1 << 21), 8, 0), ({}, dict(batch=1 << 23), 2, 0), (dict(page_tokens=BIG), {}, 2, 0), ({}, dict(table_width=BIG), 2, 0),
    ({}, dict(tokens=BIG), 2, 0), (dict(kv_heads=BIG), {}, BIG, 0), ({}, dict(batch=BIG), 2, 0), ({}, {}, 2, BIG), ({}, {}, BIG, 0),
    ({}, dict(tokens=1 << 30), 4, 0), (dict(n_pages=BIG), {}, 2, 0), ({}, dict(max_new=-1), 2, 0), (dict(page_tokens=40), {}, 2, 0)])
def test_sizes_that_no_launch_holds_are_refused_before_one(cache, batch, heads, window):
    """The call and the question for its workspace refuse the same sizes."""
    lib, vp = dfp4.load(), ctypes.c_void_p
    batch = dict(dict(table_width=1 << 12), **batch)
    c, b = _cache(**cache), _batch(**batch)
    assert lib.dfp4_paged_attention_workspace_bytes(c, b, heads, window) == 0
    assert lib.dfp4_paged_attention(vp(16), 256, 64, heads, c, b, 1.0, 0.0, window, vp(0), vp(16), 256, 64, vp(0), vp(16), BIG, vp(0)) == -2
    if heads != BIG and window != BIG and batch.get("tokens") != 1 << 30:
        assert lib.dfp4_paged_write(vp(16), 128, 64, vp(16), 128, 64, c, b, vp(0)) == -2
        assert lib.dfp4_paged_read(c, b, vp(16), vp(16), 1, vp(0)) == -2


# ---- norms of numbers whose squares leave fp32 ----------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30, 1e-5])
def test_norms_at_the_ends_of_bf16(dim, eps):
    """Heads of every size beside each other, some of few large numbers among tiny ones."""
    g = torch.Generator().manual_seed(dim)
    sizes = [2.0 ** e for e in (-132, -126, -100, -64, -62, -50, -45, 0, 40, 60, 62, 64, 100, 124)]
    x = torch.randn(3, 2 * len(sizes), dim, generator=g).double()
    for h, size in enumerate(sizes):
        x[:, [h, len(sizes) + h]] *= size
    x[1, :, 1:] *= 2.0 ** -40
    x = x.bfloat16()
    x[..., 0] = torch.where(x[..., 0] == 0, torch.tensor(2.0 ** -133).bfloat16(), x[..., 0])      # (no head of zeros: 0 / 0 where eps is 0)
    assert torch.isfinite(x).all()
    pos, freq = torch.tensor([0, 5, 90000], dtype=torch.int32), (1.0 / 10000.0 ** (torch.arange(0, 32, 2).double() / 32)).float()
    w = 1 + 0.3 * torch.randn(dim, generator=g)
    for wq, wk in ((w, w), (w, None)):
        d = x.cuda()
        q, k = dfp4.norm_rope(d[:, :len(sizes)], d[:, len(sizes):], pos.cuda(), freq.cuda(), wq.cuda(), None if wk is None else wk.cuda(), eps=eps)
        for got, part, weight in ((q, x[:, :len(sizes)], wq), (k, x[:, len(sizes):], wk)):
            want, size = _rope(part, weight, pos, freq, False, float(np.float32(eps)))
            # the same bound as for ordinary numbers, and half a step of the smallest ones
            assert (np.abs(got.double().cpu().numpy() - want) <= HALF * np.abs(want) + 20 * 2.0 ** -24 * size + 2.0 ** -134).all()


# ---- lengths that are taken back ------------------------------------------------------------------------------------------------

def test_slots_hold_one_or_two_chunks():
    lib, vp = dfp4.load(), ctypes.c_void_p
    for chunks, rc in ((0, 0), (1, 0), (2, 0), (3, -2), (-1, -2)):
        c, b = _cache(), _batch(tokens=0)
        c.slot_chunks = chunks
        assert lib.dfp4_paged_write(vp(16), 128, 64, vp(16), 128, 64, c, b, vp(0)) == lib.dfp4_paged_read(c, b, vp(16), vp(16), 1, vp(0)) == rc


@pytest.mark.gpu
@pytest.mark.parametrize("chunks", [1, 2])
@pytest.mark.parametrize("most", [4, 32, 75])
@pytest.mark.parametrize("dim", [64, 128])
def test_drafted_tokens_are_taken_back(dim, most, chunks):
    """Every step writes up to `most` tokens a sequence of which the last ones are wrong, and the next goes on after the last right one."""
    s = Sequences([400, 330], dim, 2, 64, seed=most + chunks)
    s.cache.c.slot_chunks = chunks                       # (with one: the same memory, half of it used)
    lengths, s.lengths, at, largest = s.lengths, [0, 0], [0, 0], [0, 0]
    k, v, s.k, s.v = s.k, s.v, None, None
    draw = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=s.g))  # noqa: E731
    crossed = 0
    for step in range(30 if most > 4 else 90):
        new = [min(draw(0, most), lengths[b] - at[b]) for b in range(2)]
        after = [at[b] + new[b] for b in range(2)]
        largest = [max(largest[b], after[b]) for b in range(2)]
        lowest = [largest[b] - 32 if chunks == 2 else largest[b] // 32 * 32 for b in range(2)]
        right = [draw(max(at[b], lowest[b]), after[b]) if after[b] >= lowest[b] else after[b] for b in range(2)]
        rows = []
        for x in (k, v):
            parts = [x[b][at[b]:after[b]].clone() for b in range(2)]
            for b in range(2):
                parts[b][right[b] - at[b]:] = 100.0
            rows.append(torch.cat(parts).cuda())
        if sum(new):
            dfp4.paged_write(*rows, s.cache, s.batch(new, after))
        crossed += sum(right[b] // 32 < after[b] // 32 and right[b] % 32 != 0 for b in range(2))
        at = s.lengths = right
        s.k, s.v = [x[:n] for x, n in zip(k, at)], [x[:n] for x, n in zip(v, at)]
        _check_read(s, at, at, torch.bfloat16)
        _attend(s, [min(n, 3) for n in at], 4)
    assert (crossed > 0) == (chunks == 2)
    # many rows, over an incomplete chunk that was whole before
    s = Sequences([600, 33, 431, 20, 64], dim, 2, 64, seed=dim, width=40)
    longer = [n + 32 for n in s.lengths]
    true_k, true_v = s.k, s.v
    s.k, s.v = ([torch.cat([x, torch.full((32, 2, dim), 50.0).bfloat16()]) for x in y] for y in (true_k, true_v))
    s.write(longer, longer)
    s.k, s.v = true_k, true_v
    _check_read(s, s.lengths, s.lengths, torch.bfloat16)
    new = [90, 33, 3, 0, 64]
    assert dfp4.paged_attention_rows(s.cache, s.batch(new, max_new=190), sum(new), 8) == 256
    _attend(s, new, 8, max_new=190)


# ---- what a call takes for its sizes ---------------------------------------------------------------------------------------------

def test_rows_of_a_workgroup():
    lib = dfp4.load()

    def rows(batch, tokens, max_new=0, heads=32, kv_heads=8, dim=128, context=8192, window=0):
        return lib.dfp4_paged_attention_rows(_cache(head_dim=dim, kv_heads=kv_heads, page_tokens=64),
                                             _batch(batch=batch, tokens=tokens, table_width=context // 64, max_new=max_new), heads, window)
    # one token of many sequences, whether the caller says so or not
    for batch in (1, 2, 48, 256, 1000):
        assert rows(batch, batch) == rows(batch, batch, max_new=1) == rows(batch, 3 * batch) == 16
    # prompts: the same
    for batch, new in ((1, 2048), (3, 512), (8, 700)):
        assert rows(batch, batch * new) == rows(batch, batch * new, max_new=new) == 256
    assert rows(1, 2048, dim=256) == rows(1, 2048, dim=192, max_new=2048) == 16
    # as many workgroups as a launch holds: of 256 threads, those for many rows have 512
    assert rows(1 << 19, 1 << 26, heads=8) == 256 and rows(1 << 20, 1 << 26, heads=8) == rows((1 << 21) - 1, 1 << 26, heads=8) == 16
    assert rows(1 << 21, 1 << 26, heads=8) == 0
    assert rows(0, 5) == rows(5, 0) == rows(4, 4, heads=12) == rows(4, 4, window=-1) == rows(4, 4, dim=80) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[1] * 7, [70, 1, 1, 1, 1, 1, 1], [1, 0, 0, 0, 0, 0, 90]])
def test_attention_of_batches_that_say_nothing_of_themselves(new):
    """The kernel is chosen for sequences that are alike; one of them may still have most of the tokens."""
    s = Sequences([90, 31, 32, 400, 128, 3000, 99], 64, 2, 64, seed=sum(new)).fill()
    _attend(s, new, 16)


# ---- as many bits as the header says --------------------------------------------------------------------------------------------

def _check_rounding(got, lse, want, probability):
    """A probability is off by `probability` of itself and a score by 2^-19 of sum |q||k| (an instruction adds its products, which are
    exact, with 2^-22 of their sizes, and at most eight follow each other), sums and exponentials in fp32 by 2^-16, and the result is rounded to bf16.  These are bounds of single elements; of all of them together the error is that of the rounding,
    with probabilities of 8 bits another one of its size (sqrt(2), as products of independent signs add up), and a tenth for the rest."""
    out, wlse, size, dot = want
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    score = 2.0 ** -19 * dot
    tol = HALF * np.abs(out) + (1 + HALF) * (probability + 2.0 ** -16 + 2 * score[..., None]) * size
    assert (np.abs(got - out) <= tol).all(), float((np.abs(got - out) / tol).max())
    assert (np.abs(lse - wlse) <= score + 2.0 ** -20 * (1 + np.abs(wlse))).all(), float((np.abs(lse - wlse) / score).max())
    rounding = np.linalg.norm(torch.from_numpy(out).bfloat16().double().numpy() - out)
    assert np.linalg.norm(got - out) <= (1.1 if probability < 2.0 ** -10 else 1.1 * 2 ** 0.5) * rounding, np.linalg.norm(got - out) / rounding


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("options", [dict(), dict(softcap=20.0), dict(window=200)])
def test_probabilities_of_16_bits_with_16_rows(dim, options):
    s = Sequences([300, 45, 700], dim, 2, 64, seed=dim + 1).fill()
    new, heads = [9, 45, 1], 6
    assert dfp4.paged_attention_rows(s.cache, s.batch(new), sum(new), heads, options.get("window", 0)) == 16
    q = torch.randn(sum(new), heads, dim, generator=s.g).bfloat16()
    got, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch(new), return_lse=True, **options)
    _check_rounding(got, lse, _attention(s, q, new, dim ** -0.5, **options), 2.0 ** -16)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("options", [dict(), dict(softcap=20.0), dict(window=300)])
def test_probabilities_of_8_bits_with_256_rows(dim, options):
    s = Sequences([600, 33, 431, 20, 64], dim, 2, 64, seed=dim, width=40).fill()
    new, heads = [200, 33, 300, 0, 64], 8
    b = s.batch(new, max_new=300)
    assert dfp4.paged_attention_rows(s.cache, b, sum(new), heads, options.get("window", 0)) == 256
    q = torch.randn(sum(new), heads, dim, generator=s.g).bfloat16()
    want = _attention(s, q, new, dim ** -0.5, **options)
    got, lse = dfp4.paged_attention(q.cuda(), s.cache, b, return_lse=True, **options)
    _check_rounding(got, lse, want, HALF)
    # the same rows by the other kernel: its bits
    few = s.batch(new, max_new=1)
    assert dfp4.paged_attention_rows(s.cache, few, sum(new), heads, options.get("window", 0)) == 16
    _check_rounding(*dfp4.paged_attention(q.cuda(), s.cache, few, return_lse=True, **options), want, 2.0 ** -16)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,many", [(64, False), (96, False), (128, False), (192, False), (256, False), (64, True), (96, True), (128, True)])
def test_scores_of_numbers_of_many_sizes(dim, many):
    """Queries and keys whose elements differ by a factor of thousands: the small ones meet the other's large ones, and count."""
    s, new, heads, hints = _few_or_many_rows(dim, many)
    s.k = [(k.double() * torch.exp(3 * torch.randn(k.shape, generator=s.g).double())).bfloat16() for k in s.k]
    s.fill()
    q = (torch.randn(sum(new), heads, dim, generator=s.g).double() * torch.exp(3 * torch.randn(sum(new), heads, dim, generator=s.g).double())).bfloat16()
    assert dfp4.paged_attention_rows(s.cache, s.batch(new, **hints), sum(new), heads) == (256 if many else 16)
    scale = 16.0 / float(_attention(s, q, new, 1.0)[3].max())                # (scores up to 16)
    got, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch(new, **hints), scale=scale, return_lse=True)
    _check_rounding(got, lse, _attention(s, q, new, scale), HALF if many else 2.0 ** -16)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", DIMS)
def test_a_score_is_a_sum_in_fp32(dim):
    """One key a sequence: the log-sum-exp is its score."""
    n = 500
    s = Sequences([1] * n, dim, 1, 32, seed=dim, factor=1.0)
    for size in (1.0, 8.0, 1000.0):
        for x in range(n):
            s.k[x][..., :2] *= size
        s.fill()
        q = torch.randn(n, 4, dim, generator=s.g)
        q[..., 1:3] *= size
        q = q.bfloat16()
        _, lse = dfp4.paged_attention(q.cuda(), s.cache, s.batch([1] * n, max_new=1), scale=1.0, return_lse=True)
        k = synth.to_f64(q) * np.concatenate(s.stands_for()[0])
        # (a log-sum-exp passes through base 2: two roundings)
        assert (np.abs(lse.double().cpu().numpy() - k.sum(-1)) <= 2.0 ** -19 * np.abs(k).sum(-1) + 2.0 ** -22 * np.abs(k.sum(-1))).all(), size


# ---- paths that small calls do not take -----------------------------------------------------------------------------------------

def _parts(s, b, tokens, heads, window):
    """In how many parts the keys of a call are split at most (its workspace holds a result and two numbers of each part and row)."""
    need = dfp4.load().dfp4_paged_attention_workspace_bytes(s.cache.c, b.c(tokens), heads, window)
    return max(1, need // (tokens * heads * (s.dim + 2) * 4))


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("lengths,new,window,many,parts", [
    # 256 rows a workgroup; blocks of rows whose windows begin in other chunks and are split in other numbers of parts
    ([3500, 2900], [500, 431], 3000, True, (2, 8)), ([7000], [700], 6000, True, (9, 256)), ([1300, 700, 900, 64, 1200], [700, 650, 300, 64, 333], 333, True, (1, 1)),
    # 16 rows
    ([5000, 700], [9, 3], 2000, False, (2, 8)), ([9000, 33, 5000], [5, 2, 1], 7000, False, (9, 256)), ([3000, 1500], [3, 1], 100, False, (1, 1)),
])
def test_windows_of_both_kernels_whole_and_split(dim, lengths, new, window, many, parts):
    s = Sequences(lengths, dim, 1, 32, seed=dim + window, width=-(-max(lengths) // 32) + 3).fill()
    heads, b = 4, s.batch(new, max_new=max(new))
    assert dfp4.paged_attention_rows(s.cache, b, sum(new), heads, window) == (256 if many else 16)
    assert parts[0] <= _parts(s, b, sum(new), heads, window) <= parts[1]
    q = torch.randn(sum(new), heads, dim, generator=s.g).bfloat16()
    got, lse = dfp4.paged_attention(q.cuda(), s.cache, b, window=window, return_lse=True)
    # (every row where there are few, else some of each block of rows, its first and its last among them)
    want = _attention_rows(s, q, new, dim ** -0.5, window, None if sum(new) < 20 else 29)
    rows = want[0]
    _check_rounding(got[rows], lse[rows], want[1:], HALF if many else 2.0 ** -16)


def _attention_rows(s, q, new, scale, window, every):
    """_attention of every `every`-th new token and of the first and last of each sequence: their numbers, and what _attention gives."""
    picked, row = [], 0
    for n in new:
        picked += [row + i for i in range(n) if every is None or i % every == 0 or i % 64 in (0, 63) or i == n - 1]
        row += n
    ks, vs = s.stands_for()
    q = synth.to_f64(q)
    heads, group = q.shape[1], q.shape[1] // s.kv_heads
    out, size, lse, dot = np.zeros((len(picked),) + q.shape[1:]), np.zeros((len(picked),) + q.shape[1:]), np.zeros((len(picked), heads)), np.zeros((len(picked), heads))
    starts = np.cumsum([0] + list(new))
    for at, row in enumerate(picked):
        b = int(np.searchsorted(starts, row, side="right")) - 1
        p = s.lengths[b] - new[b] + row - starts[b]
        lo = max(0, p - window + 1) if window else 0
        for h in range(heads):
            k, v = ks[b][lo:p + 1, h // group], vs[b][lo:p + 1, h // group]
            z = scale * (k @ q[row, h])
            w = np.exp(z - z.max())
            lse[at, h] = z.max() + math.log(w.sum())
            w /= w.sum()
            out[at, h], size[at, h], dot[at, h] = w @ v, w @ np.abs(v), (np.abs(k) @ np.abs(q[row, h])).max() * abs(scale)
    return picked, out, lse, size, dot


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1500, 2049, 5003])
@pytest.mark.parametrize("dim,rotary,heads,kv_heads,interleaved,norm", [
    (128, 128, 32, 8, False, True), (64, 32, 7, 3, True, True), (96, 16, 5, 1, False, False), (256, 256, 9, 2, False, True), (32, 32, 70, 2, True, True),
    (192, 96, 3, 0, False, True), (128, 0, 11, 5, False, True)])
def test_norm_rope_of_many_tokens(tokens, dim, rotary, heads, kv_heads, interleaved, norm):
    """Several heads and several tokens a workgroup, the last one of fewer: queries and keys as slices of a joint row, and in place."""
    g = torch.Generator().manual_seed(tokens + dim)
    x = (torch.randn(tokens, heads + kv_heads + 1, dim, generator=g) * torch.exp(2 * torch.randn(tokens, 1, 1, generator=g))).bfloat16()
    pos = torch.randint(0, 1 << 20, (tokens,), generator=g).int()
    freq = (1.0 / 500000.0 ** (torch.arange(0, rotary, 2).double() / max(rotary, 1))).float()
    wq, wk = ((1 + 0.3 * torch.randn(dim, generator=g)) if norm else None for _ in range(2))
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    d = x.cuda()
    dq, dk = d[:, 1:1 + heads], d[:, 1 + heads:] if kv_heads else None
    args = (cuda(pos), cuda(freq), cuda(wq), cuda(wk))
    q, k = dfp4.norm_rope(dq, dk, *args, eps=1e-5, interleaved=interleaved)
    into = (dq.contiguous(), None if dk is None else dk.contiguous())
    dfp4.norm_rope(*into, *args, eps=1e-5, interleaved=interleaved, out=into)
    torch.cuda.synchronize()
    for got, same, part, w in ((q, into[0], x[:, 1:1 + heads], wq), (k, into[1], x[:, 1 + heads:], wk)):
        if got is None:
            continue
        want, size = _rope(part, w, pos, freq, interleaved, 1e-5)
        assert (np.abs(got.double().cpu().numpy() - want) <= HALF * np.abs(want) + 20 * 2.0 ** -24 * size).all()
        assert torch.equal(got.view(torch.int16), same.view(torch.int16))


@pytest.mark.gpu
def test_cache_of_a_batch_that_says_nothing_of_itself():
    """300 sequences of which one has most of the tokens: more chunks than there are workgroups for them."""
    lengths = [1 + i % 40 for i in range(299)] + [3000]
    s = Sequences(lengths, 64, 8, 64, seed=41)
    s.write(lengths, lengths)
    _check_read(s, lengths, lengths, torch.bfloat16)
    s = Sequences([40] * 300, 64, 8, 64, seed=42)
    for n in (31, 1, 8):
        at = [sum((31, 1, 8)[:(31, 1, 8).index(n) + 1])] * 300
        s.write([n] * 300, at)
        _check_read(s, [n] * 300, at, torch.bfloat16)
