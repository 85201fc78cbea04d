"""Serving from a 4-bit pool on the GPU against the 64-bit oracle: bytes stored, rows read back, attention.

Bytes are compared for equality: the codes of 16-bit rows are decided by comparisons of exact numbers, and what a norm and a
rotation give is formed in 64 bits, whose rounding moves a value over a border between two codes for about one in 10^13.

Attention is held to what its documentation says of it, with the values that the codes stand for (exact in 16 bits): the
logits are sums of 128 products that are exact in fp32 (2 * 128 * 2^-24 of the sum of their magnitudes bounds the
rounding), the exponentials' arguments and results are off by 2^-22 (1 + logit), sums over the keys by 2 n 2^-24, the
weights and the output by half a step of the type each.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import paged as OP
from oracle import paged4 as O4
from tests import test_gpu_paged as T
from tests.test_gpu_paged import APPEND, D, DECODE, EXTEND, _bits, _f64, _log, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


class Served4(T.Served):
    """A cache of scattered 4-bit pages.  k and v hold the values that it stands for, in the 16-bit type; after a change to
    them or to table or lens, rebuild()."""

    def rebuild(self):
        import torch
        data = []
        for x in (self.k, self.v):
            b = O4.pool(_f64(x), self.name)
            x.copy_(torch.from_numpy(O4.decode(*O4.rows(b, self.page))))
            data.append(torch.from_numpy(b).cuda())
        self.kb, self.vb = data
        self.cache = self.P.PagedCache(*data, torch.from_numpy(self.table).cuda(),
                                       torch.tensor(self.lens, dtype=torch.int32, device="cuda"), self.hq, self.max_len,
                                       dtype=self.dt)

    def compare(self, q, out, scale=D ** -0.5):
        return super().compare(q, out, scale, decode=False)

    def bytes(self):
        return self.kb.cpu().numpy(), self.vb.cpu().numpy()

    def at(self, data, r):
        """Codes and scales of pool row r of every unit."""
        codes, scales = O4.rows(data, self.page)
        return codes[:, :, r // self.page, r % self.page], scales[:, :, r // self.page, r % self.page]


# ---------------------------------------------------------------------------
# Rows out of pages
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,new,page,dtype,layers,hk", [
    ((1,), (1,), 16, "bf16", 1, 1), ((40, 0, 130, 7), (40, 2, 65, 0), 16, "fp16", 3, 2), ((300, 20), (64, 20), 64, "bf16", 2, 4),
    ((3, 700), (5, 700), 256, "fp16", 1, 3)])
def test_read(torch_cuda, four, lens, new, page, dtype, layers, hk):
    """The rows as the pool holds them; zeros where there is none; nothing behind the last one."""
    import torch
    _log(f"paged read {'4 bits ' if four else ''}lens {lens} new {new} page {page} {dtype}")
    f = (Served4 if four else T.Served)(lens, new, page, dtype, layers, hk, hk, seed=41, fill=float("nan"))
    if len(lens) > 2:
        f.table[2, 5] = -1
        f.table[2, 6] = f.n_pages
        f.rebuild()
    n = layers * f.total * hk * D
    buf = torch.full((2, n + 2048), 7.0, dtype=f.dt, device="cuda")
    k, v = (b[1024:-1024].view(layers, f.total, hk, D) for b in buf)
    got = f.P.paged_read(f.cache, f.batch, k_out=k, v_out=v)
    torch.cuda.synchronize()
    assert got[0] is k and got[1] is v and (buf[:, :1024] == 7).all() and (buf[:, -1024:] == 7).all()
    places = OP.new_places(f.table, f.lens, f.cu, page, f.n_pages, f.max_len)
    for x, pool in ((k, f.k), (v, f.v)):
        want = torch.zeros_like(x)
        flat = pool.view(layers, hk, -1, D)
        for i, r in enumerate(places):
            if r is not None:
                want[:, i] = flat[:, :, r]
        assert np.array_equal(_bits(x), _bits(want))
    only = f.P.paged_read(f.cache, f.batch)
    assert torch.equal(only[0], k) and torch.equal(only[1], v)


# ---------------------------------------------------------------------------
# Rows into pages
# ---------------------------------------------------------------------------

def _special(dtype, n, gen):
    """Rows with every border between codes, both signs, at scales of the whole range; zeros, subnormal and greatest values,
    infinities and NaN."""
    import torch
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    info = torch.finfo(dt)
    edge = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0], dtype=torch.float64)
    up = edge * (1 + 2.0 ** (-7 if dtype == "bf16" else -10))
    base = torch.cat([edge, up])
    base = torch.cat([base, -base, edge * 0.9, -up * 1.1, edge.flip(0), up.flip(0)])[:D]
    rows = torch.randn((n, D), generator=gen, dtype=torch.float64)
    lo, hi = (-130, 126) if dtype == "bf16" else (-24, 13)
    for i in range(n):
        rows[i] *= 2.0 ** (lo + (hi - lo) * i / (n - 1))
    for i, e in enumerate(range(lo, hi - 2, 9 if dtype == "bf16" else 2)):
        rows[i] = base[torch.randperm(D, generator=gen)] * 2.0 ** e
    rows[-1], rows[-2] = 0.0, -0.0
    rows[-3] = info.max
    rows[-4] = -info.max / 2
    rows[-5] = info.tiny / 8
    rows[-6, 5], rows[-6, 40], rows[-6, 127] = float("inf"), float("-inf"), float("nan")
    rows[-7, :32] = float("nan")
    return rows.to(dt).cuda()


@pytest.mark.parametrize("lens,beta,page,per_layer,dtype", [
    ((912,), (1, 5), 16, False, "bf16"), ((100, 3, 257, 64), (1, 4), 16, False, "fp16"), ((100, 3, 257, 64), (1, 1), 64, True, "bf16"),
    ((5, 4), (1, 7), 32, False, "bf16"), ((1000, 2000, 31), (2, 3), 256, False, "fp16")])
def test_compact(torch_cuda, lens, beta, page, per_layer, dtype):
    import torch
    _log(f"paged compact, 4 bits, lens {lens} page {page} {dtype}")
    layers, hk = 3, 2
    p = T._problem(lens, layers, hk, beta)
    cb, cu = p.h["cu_budget"], p.h["cu_seqlens"]
    f = Served4([max(int(n), 1) for n in np.diff(cb)], [0] * len(lens), page, dtype, layers, 4, hk, seed=42)
    rng = np.random.default_rng(16)
    lists = layers if per_layer else layers * hk
    kept = np.concatenate([np.sort(np.stack([rng.permutation(n)[:b] for _ in range(lists)]), -1) + a
                           for a, n, b in zip(cu, np.diff(cu), np.diff(cb))], -1).astype(np.int32)
    if kept.size:
        kept[0, -1] = sum(lens)  # out of range: zeros
        kept[-1, 0] = -1
    if len(lens) > 1 and cb[1] > page:
        f.table[0, 1] = -1  # dropped
        f.rebuild()
    f.cache.seq_lens.fill_(-1)
    k, v = (f.randn((layers * hk, sum(lens), D)) for _ in range(2))
    if sum(lens) >= 64:
        gen = torch.Generator()
        gen.manual_seed(7)
        for x in (k, v):
            x[:, :64] = _special(dtype, 64, gen)
    want = [b.copy() for b in f.bytes()]
    f.P.paged_compact(f.cache, p, k, v, torch.from_numpy(kept).cuda().contiguous(), per_layer=per_layer)
    torch.cuda.synchronize()
    for u in range(layers * hk):
        for s in range(len(lens)):
            for j in range(int(cb[s + 1] - cb[s])):
                r = OP.place(f.table, s, j, page, f.n_pages)
                t = int(kept[u // hk if per_layer else u, cb[s] + j])
                if r is None:
                    continue
                for w, src in zip(want, (k, v)):
                    row = _f64(src[u, t]) if 0 <= t < sum(lens) else np.zeros(D)
                    codes, scales = O4.rows(w[u // hk, u % hk], page)
                    codes[r // page, r % page], scales[r // page, r % page] = O4.encode(row, dtype)
    for got, w in zip(f.bytes(), want):
        assert np.array_equal(got, w)
    assert f.cache.seq_lens.tolist() == np.diff(cb).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_code(torch_cuda, dtype):
    """Rows at every border and limit, stored as they are by an append (keys and values) and by a compaction, and read back."""
    import torch
    n = 256
    f = Served4((n,), (n,), 32, dtype, 1, 1, 1, seed=43)
    gen = torch.Generator()
    gen.manual_seed(8)
    rows = _special(dtype, n, gen)
    x = rows.view(1, n, 1, D)
    f.P.paged_append(f.cache, f.batch, None, x, x)
    torch.cuda.synchronize()
    codes, scales = O4.encode(_f64(rows), dtype)
    places = np.array(OP.new_places(f.table, f.lens, f.cu, 32, f.n_pages, f.max_len))
    for data in f.bytes():
        c, s = f.at(data, places)
        assert np.array_equal(c[0, 0], codes) and np.array_equal(s[0, 0], scales)
    stored = f.bytes()
    k, v = f.P.paged_read(f.cache, f.batch)
    want = O4.decode(codes, scales)
    assert np.array_equal(_f64(k)[0, :, 0], want, equal_nan=True) and torch.equal(torch.isnan(k), torch.isnan(v))
    p = T._problem((n,), 1, 1, (1, 1), group=1)
    f.kb.zero_()
    f.vb.zero_()
    f.P.paged_compact(f.cache, p, rows.view(1, n, D), rows.view(1, n, D), torch.arange(n, dtype=torch.int32, device="cuda").view(1, n))
    for got, old in zip(f.bytes(), stored):
        c, s = f.at(got, places)
        assert np.array_equal(c, f.at(old, places)[0]) and np.array_equal(s, f.at(old, places)[1])


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk,axes,interleaved,norms,fused", APPEND)
def test_append(torch_cuda, lens, new, page, dtype, layers, hq, hk, axes, interleaved, norms, fused):
    import torch
    _log(f"paged append, 4 bits, lens {lens} new {new} {dtype} {layers} x {hq}/{hk} axes {axes} norms {norms!r}")
    f = Served4(lens, new, page, dtype, layers, max(hq, hk), hk, seed=44)
    P, n = f.P, f.total
    if fused:
        qkv = f.randn((layers, n, hq + 2 * hk + 1, D), 2.0)
        q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:hq + 2 * hk]
    else:
        q, k, v = (f.randn((layers, n, h, D), 2.0) if h else None for h in (hq, hk, hk))
    sections = {0: None, 1: (64,), 3: (16, 24, 24)}[axes]
    rng = np.random.default_rng(12)
    pos = rng.integers(-5, 200000, (max(axes, 1), n)).astype(np.int32)
    rope = P.Rope(1e6, sections, interleaved) if axes else None
    w = {c: f.randn((layers, D)) + 1 if c in norms else None for c in "qk"}
    want = [b.copy() for b in f.bytes()]
    args = dict(positions=torch.from_numpy(pos).cuda() if axes else None, rope=rope, q_norm=w["q"] if hq else None,
                k_norm=w["k"], eps=1e-5)
    q_out = P.paged_append(f.cache, f.batch, q, k, v, **args)
    torch.cuda.synchronize()
    if hq:
        y = _f64(q) if w["q"] is None else OP.norm(_f64(q), _f64(w["q"])[:, None, None], 1e-5)
        y = OP.rotate(y, pos, 1e6, sections, interleaved) if axes else y
        size = np.abs(_f64(q) if w["q"] is None else OP.norm(_f64(q), _f64(w["q"])[:, None, None], 1e-5)).max(-1, keepdims=True)
        assert (np.abs(_f64(q_out) - y) <= T._half_step(dtype) * np.abs(y) + 2.0 ** -17 * size + 2.0 ** -25).all()
    y = _f64(k)
    if w["k"] is not None:
        # (eps as the call gets it, in fp32)
        y = OP.norm(y, _f64(w["k"])[:, None, None], float(np.float32(1e-5)))
    if axes:
        y = OP.rotate(y, pos, 1e6, sections, interleaved)
    for i, r in enumerate(OP.new_places(f.table, lens, f.cu, page, f.n_pages, f.max_len)):
        if r is None:
            continue
        for data, x in zip(want, (y[:, i], _f64(v[:, i]))):
            codes, scales = O4.rows(data, page)
            codes[:, :, r // page, r % page], scales[:, :, r // page, r % page] = O4.encode(x, dtype)
    for got, data in zip(f.bytes(), want):
        assert np.array_equal(got, data)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", DECODE)
def test_decode(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    """What is no token's row holds NaN, which no output may meet."""
    _log(f"paged decode, 4 bits, lens {lens[:8]} page {page} {dtype} {layers} x {hq}/{hk}")
    f = Served4(lens, new, page, dtype, layers, hq, hk, seed=1, fill=float("nan"))
    q = f.randn((layers, f.total, hq, D), 1.5)
    out = f.attend(q)
    _log(f"worst error / tolerance {f.compare(q, out):.3g}")
    for s, n in enumerate(lens):
        if n == 0 and new[s]:
            assert not out[:, f.cu[s]].any()
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"


@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_decode_at_the_ends_of_tiles(torch_cuda, page):
    """Lengths around the 16- and 32-key runs and the 128 keys that four waves take at once."""
    lens = [n + d for n in (16, 32, 48, 64, 96, 128, 144, 160, 256) for d in (-1, 0, 1)]
    f = Served4(lens, [1] * len(lens), page, "bf16", 1, 3, 1, seed=45, fill=float("nan"))
    q = f.randn((1, f.total, 3, D), 1.5)
    f.compare(q, f.attend(q))


def test_decode_many_short_sequences(torch_cuda):
    """More sequences than threads look them up."""
    rng = np.random.default_rng(2)
    lens = rng.integers(0, 40, 700).tolist()
    f = Served4(lens, [1] * 700, 16, "bf16", 1, 2, 1, fill=float("nan"))
    q = f.randn((1, 700, 2, D))
    f.compare(q, f.attend(q))


# More rows than the kernel of few rows takes, where that of several tokens may go wrong too.
MANY_ROWS = [
    ((3, 0, 2), (5, 3, 9), 16, "bf16", 1, 20, 1),              # shorter than their new tokens
    ((37, 64, 65), (5, 1, 0), 16, "fp16", 2, 40, 2),           # a plain step and an idle sequence beside
    ((9000, 40, 3000, 10), (3, 0, 40, 1), 32, "bf16", 1, 28, 1),  # few items, each in many parts
    ((6000,), (3,), 16, "fp16", 1, 128, 4),                    # few rows over a long cache: joined
]


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", EXTEND + MANY_ROWS)
def test_extend(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    _log(f"paged extend, 4 bits, lens {lens} new {new} page {page} {dtype} {layers} x {hq}/{hk}")
    f = Served4(lens, new, page, dtype, layers, hq, hk, seed=3, fill=float("nan"))
    q = f.randn((layers, f.total, hq, D), 1.5)
    out = f.attend(q)
    _log(f"worst error / tolerance {f.compare(q, out):.3g}")
    for s, n in enumerate(lens):  # tokens that see nothing
        for t in range(max(new[s] - n, 0)):
            assert not out[:, f.cu[s] + t].any()
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"


@pytest.mark.parametrize("group,tokens", [(7, 36), (1, 256), (128, 2)])
def test_extend_at_the_ends_of_blocks(torch_cuda, group, tokens):
    new = [tokens - 1, tokens, tokens + 1, 2 * tokens, 2 * tokens + 1]
    f = Served4([n + c for n, c in zip(new, (0, 63, 1, 0, 130))], new, 16, "bf16", 1, 2 * group, 2, seed=29, fill=float("nan"))
    q = f.randn((1, f.total, 2 * group, D), 1.5)
    f.compare(q, f.attend(q))


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", [
    ((900, 1700, 1030), (900, 200, 0), 16, "bf16", 4, 16, 2),    # 288 items: short ones stay whole, those of the second may be cut
    ((1024, 1025, 5), (513, 600, 5), 64, "fp16", 4, 16, 2),      # keys around the longest that stays whole
    ((900,), (900,), 32, "bf16", 8, 16, 2),                      # one sequence, nothing to join
    ((1023, 1024, 1025, 3000, 1, 0), (1, 1, 1, 1, 1, 0), 16, "bf16", 2, 28, 4),   # one token
    ((1024, 1024, 1000), (1, 1, 1), 256, "fp16", 1, 20, 1),      # one token, nothing to join
    ((1026, 1024, 500, 5000, 3), (4, 3, 4, 4, 3), 64, "bf16", 2, 28, 4),          # a few
    ((463, 461, 462, 40, 2000), (9, 36, 37, 40, 100), 16, "bf16", 1, 7, 1),       # fewer items than CUs
    ((300, 448), (200, 41), 128, "fp16", 1, 14, 2),              # the same, nothing to join
    ((1100, 700, 3), (900, 1050, 9), 16, "fp16", 4, 16, 2),      # shorter than their new tokens
])
def test_items_that_stay_whole(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    """Short items, which are not cut: shares that begin and end where an item does, and within one."""
    f = Served4(lens, new, page, dtype, layers, hq, hk, seed=37, fill=float("nan"))
    q = f.randn((layers, f.total, hq, D), 1.5)
    out = f.attend(q)
    f.compare(q, out)
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"


def test_extend_many_sequences(torch_cuda):
    """More sequences than threads look them up, idle ones among them."""
    rng = np.random.default_rng(4)
    new = rng.integers(0, 4, 1100)
    lens = [int(n + rng.integers(0, 90)) for n in new]
    for heads in (2, 24):
        f = Served4(lens, new.tolist(), 16, "fp16", 1, heads, 1, fill=float("nan"))
        q = f.randn((1, f.total, heads, D))
        f.compare(q, f.attend(q))


@pytest.mark.parametrize("tiles", [1, 2, 7, 8, 9, 10, 11, 17, 25])
def test_extend_of_few_and_many_tiles(torch_cuda, tiles):
    """Caches around the tiles that are fetched ahead, in pages that end inside a tile and behind it."""
    for page, heads in ((16, 7), (128, 7), (16, 40), (128, 40)):
        f = Served4((64 * tiles - 3, 64 * tiles, 64 * tiles + 1), (2, 3, 2), page, "bf16", 1, heads, 1, seed=46, fill=float("nan"))
        q = f.randn((1, f.total, heads, D), 1.5)
        f.compare(q, f.attend(q))


def _room(f, keys):
    """A table for sequences of so many keys, of which the cache's have few: what a program that serves long ones has."""
    wide = np.full((len(f.lens), -(-keys // f.page)), -1, np.int32)
    wide[:, :f.table.shape[1]] = f.table
    f.table, f.max_len = wide, keys
    f.rebuild()
    return f


@pytest.mark.parametrize("group,tokens", [(11, 3), (7, 6), (48, 1), (33, 1), (40, 1), (64, 1), (12, 4), (16, 3), (7, 7), (7, 9), (16, 4), (1, 64), (1, 50), (32, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_few_rows(torch_cuda, group, tokens, dtype):
    """33 to 64 rows to an item, in the kernel that takes them where sequences may be long: masks, ends, idle sequences,
    pages that are none, values that are NaN in a later token's row, and sequences cut into parts."""
    import torch
    lens = (1, tokens, 63 + tokens, 64, 300, 0, 5, 2000, 131)
    new = [min(tokens, max(n, 0)) for n in lens]
    new[6], new[4] = 0, max(tokens - 1, 1)
    f = _room(Served4(lens, new, 32, dtype, 1, 2 * group, 2, seed=51, fill=float("nan")), 1 << 17)
    f.table[7, 3], f.table[7, 40] = -1, f.n_pages
    f.rebuild()
    q = f.randn((1, f.total, 2 * group, D), 1.5)
    out = f.attend(q)
    _log(f"few rows {group} x {tokens} {dtype}: worst error / tolerance {f.compare(q, out):.3g}")
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"
    s, j = 4, lens[4] - max(new[4] // 2, 1)  # a new token's own row, in the middle
    f.v.view(1, 2, -1, D)[0, 1, OP.place(f.table, s, j, 32, f.n_pages), 70] = float("nan")
    f.k.view(1, 2, -1, D)[0, 0, OP.place(f.table, 7, 1990, 32, f.n_pages), 70] = float("nan")
    f.rebuild()
    got = f.attend(q)
    want = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    want[0, int(f.cu[s]) + j - (lens[s] - new[s]):f.cu[s + 1], group:, 64:96] = True
    want[0, int(f.cu[7]) + max(1990 - (2000 - tokens), 0):f.cu[8], :group] = True
    assert torch.equal(torch.isnan(got), want) and torch.equal(got[~want], out[~want])


def test_few_rows_of_long_sequences(torch_cuda):
    """Many parts to an item, ring slots used again, a page table beyond the entries that a wave holds."""
    for page, group, tokens in ((16, 7, 6), (16, 7, 9), (64, 7, 4), (16, 7, 1)):
        f = _room(Served4((20000, 9000, 16384 + tokens), (tokens,) * 3, page, "bf16", 1, group, 1, seed=52), 1 << 19)
        q = f.randn((1, f.total, group, D), 1.5)
        f.compare(q, f.attend(q))


@pytest.mark.parametrize("new", [1, 4, 150])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rising_and_extreme_logits(torch_cuda, new, dtype):
    """Maxima that rise in every step of the cache, fall, and weights that underflow."""
    import torch
    f = Served4((900, 900, 901), (new, new, new), 16, dtype, 1, 4, 1, seed=5)
    q = f.randn((1, f.total, 4, D))
    q[..., 1:] = 0
    q[..., 0] = 8.0
    f.k[..., 1:] = 0
    for s, slope in enumerate((1.0, -1.0, 0.0)):
        for j in range(f.lens[s]):
            r = OP.place(f.table, s, j, 16, f.n_pages)
            f.k.view(1, 1, -1, D)[0, 0, r, 0] = slope * (j - 450) * 0.125
    f.rebuild()
    for scale in (D ** -0.5, 1.0, 4.0, 1e-3):
        out = f.attend(q, scale=scale)
        assert torch.isfinite(out).all()
        f.compare(q, out, scale=scale)


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_masked_values_have_no_influence(torch_cuda, new, dtype):
    """A block of a later token's key or value that is NaN reaches the tokens that see it, and no other."""
    import torch
    lens = (300, 141, 200)
    f = Served4(lens, (new,) * 3, 16, dtype, 1, 6, 2, seed=6, fill=float("nan"))
    q = f.randn((1, f.total, 6, D))
    clean = f.attend(q).clone()
    at = [f.lens[s] - new // 2 - 1 for s in range(3)]  # a new token's own row, in the middle
    rows = [OP.place(f.table, s, at[s], 16, f.n_pages) for s in range(3)]
    v = f.v.view(1, 2, -1, D)
    v[0, 0, rows[0], 5] = float("inf")
    v[0, 1, rows[1], 100] = float("nan")
    f.k.view(1, 2, -1, D)[0, 1, rows[2], 9] = float("nan")
    f.rebuild()
    out = f.attend(q)
    first = [int(f.cu[s]) + max(at[s] - (f.lens[s] - new), 0) for s in range(3)]  # the first token that sees it
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[0, first[0]:f.cu[1], 0:3, 0:32] = True
    hit[0, first[1]:f.cu[2], 3:6, 96:128] = True
    hit[0, first[2]:f.cu[3], 3:6, :] = True
    assert torch.equal(out[~hit], clean[~hit]) and torch.isnan(out[hit]).all()


@pytest.mark.parametrize("new,hq", [(1, 3), (1, 20), (4, 20), (70, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_that_are_seen_and_nan(torch_cuda, new, hq, dtype):
    """They reach every token and head, whatever their weight, and no other block."""
    import torch
    f = Served4((300, 70), (new, new), 16, dtype, 1, hq, 1, seed=18)
    q = f.randn((1, f.total, hq, D), 4.0)
    clean = f.attend(q).clone()
    f.v.view(1, 1, -1, D)[0, 0, OP.place(f.table, 0, 77, 16, f.n_pages), 33] = float("nan")
    f.k.view(1, 1, -1, D)[0, 0, OP.place(f.table, 0, 77, 16, f.n_pages)] = -8 * f.k.view(1, 1, -1, D)[0, 0, 0]
    f.rebuild()
    out = f.attend(q)
    first = slice(0, int(f.cu[1]))
    rest = [d for d in range(D) if d // 32 != 1]
    assert torch.isnan(out[0, first, :, 32:64]).all() and torch.isfinite(out[0, first][..., rest]).all()
    assert torch.equal(out[:, f.cu[1]:], clean[:, f.cu[1]:])


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", [
    ((20000,), (1,), 32, "bf16", 1, 4, 2), ((5000, 300, 7000), (1, 1, 1), 64, "fp16", 1, 40, 1),
    ((6000, 300), (3, 3), 32, "bf16", 1, 28, 4), ((700,) * 9, (150,) * 9, 16, "bf16", 2, 8, 2)])
def test_logits_that_are_nan(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    """A query or keys that are NaN make their own outputs NaN, however many parts a sequence is cut into."""
    import torch
    f = Served4(lens, new, page, dtype, layers, hq, hk, seed=23)
    q = f.randn((layers, f.total, hq, D))
    clean = f.attend(q).clone()
    want = torch.isnan(clean)
    assert not want.any()
    for s in range(0, len(lens), 2):
        q[:, f.cu[s], hq - 1, 5] = float("nan")
        want[:, f.cu[s], hq - 1] = True
    out = f.attend(q)
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], clean[~want])
    rows = [OP.place(f.table, 0, j, page, f.n_pages) for j in range(lens[0] - new[0] + 1)]
    f.k.view(layers, hk, -1, D)[0, hk - 1, rows, 7] = float("nan")
    f.rebuild()
    want[0, :f.cu[1], hq - hq // hk:] = True
    out = f.attend(q)
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], clean[~want])


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_at_the_limits_of_the_type(torch_cuda, new, dtype):
    """Sums of the greatest and the smallest values, and keys of the least scale."""
    import torch
    f = Served4((1500, 300, 200), (new,) * 3, 16, dtype, 1, 7, 1, seed=19)
    info = torch.finfo(f.dt)
    f.v[..., 0:32] = info.max
    f.v[..., 32:64] = -info.max
    f.v[..., 64:96] *= info.max / 16
    f.v[..., 96:] = 2.0 ** -119 if dtype == "bf16" else info.tiny
    f.k[..., 64:] = 2.0 ** -120 if dtype == "bf16" else info.tiny
    f.rebuild()
    q = f.randn((1, f.total, 7, D), 1.5)
    out = f.attend(q)
    assert torch.isfinite(out).all()
    f.compare(q, out)


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_pages_out_of_range_are_left_out(torch_cuda, new, dtype):
    """And rows that are no token's hold bytes that no store writes, in scales too."""
    import torch
    f = Served4((300, 200, 150, 260), (new,) * 4, 16, dtype, 1, 4, 2, seed=7, fill=float("nan"))
    f.table[0, 3] = -1
    f.table[0, 18] = f.n_pages          # the last page: the new tokens' own rows among it
    f.table[1, :] = -5                  # nothing left
    f.table[2, 0] = 2 ** 31 - 1
    f.table[3, 4:9] = np.iinfo(np.int32).min
    f.rebuild()
    used = np.zeros(f.n_pages * 16, bool)
    for s in range(4):
        for j in range(f.lens[s]):
            r = OP.place(f.table, s, j, 16, f.n_pages)
            if r is not None:
                used[r] = True
    for fill in (254, 253, 200, 0):
        for data in (f.kb, f.vb):
            idle = torch.from_numpy(~used).cuda().view(f.n_pages, 16)
            codes, scales = data[..., :1024].unflatten(-1, (16, 64)), data[..., 1024:].unflatten(-1, (16, 4))
            codes[:, :, idle] = 0x77
            scales[:, :, idle] = fill
        q = f.randn((1, f.total, 4, D))
        out = f.attend(q)
        f.compare(q, out)
        assert not out[:, f.cu[1]:f.cu[2]].any() and torch.isfinite(out).all()


def test_lengths_are_cut_to_the_bounds(torch_cuda):
    for new in (1, 4, 30):
        f = Served4((64, 48, 30), (new,) * 3, 16, "bf16", 1, 4, 1, seed=8)
        q = f.randn((1, f.total, 4, D))
        f.lens = [64, 2 ** 31 - 1, -7]
        f.table[1, 3] = f.table[0, 3]  # so that the cut length has its pages
        f.max_len = 60
        f.rebuild()
        out = f.attend(q)
        f.compare(q, out)
        assert not out[:, f.cu[2]:].any()


@pytest.mark.parametrize("new", [1, 40])
def test_pool_of_more_than_4_gib(torch_cuda, new):
    """Rows behind 2^32 bytes of the pool, and of a unit's."""
    import torch
    from paper_2603_00188_amd import paged as P
    page = 256
    n_pages = (1 << 32) // (page * 68) + 3
    f = Served4((700,), (new,), page, "bf16", 1, 4, 2, seed=10)
    used = -(-700 // page)
    k = torch.zeros((1, 2, n_pages, page * 68), dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    k[:, :, -used:], v[:, :, -used:] = f.kb[:, :, f.table[0, :used]], f.vb[:, :, f.table[0, :used]]
    table = torch.arange(n_pages - used, n_pages, dtype=torch.int32, device="cuda").view(1, used)
    big = P.PagedCache(k, v, table, f.cache.seq_lens, 4, f.max_len)
    q = f.randn((1, f.total, 4, D))
    out = f.attend(q)
    f.compare(q, out)
    assert torch.equal(P.paged_attention(big, f.batch, q), out)
    rows = [f.randn((1, f.total, 2, D)) for _ in range(2)]
    P.paged_append(big, f.batch, None, *rows)
    P.paged_append(f.cache, f.batch, None, *rows)
    torch.cuda.synchronize()
    assert torch.equal(big.k[:, :, -used:], f.kb[:, :, f.table[0, :used]])
    assert torch.equal(big.v[:, :, -used:], f.vb[:, :, f.table[0, :used]])
    for a, b in zip(P.paged_read(big, f.batch), P.paged_read(f.cache, f.batch)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_past_the_caches(torch_cuda, dtype):
    """More rows than the caches hold, into pages and back: the first, the last and rows between as the oracle's, the rest as
    a smaller call's."""
    import torch
    from paper_2603_00188_amd import paged as P
    n, layers, hk = 33000, 8, 2
    p = T._problem((n,), layers, hk, (1, 1))
    cache = P.PagedCache.alloc(layers, 4, hk, 1, n, page_size=64, dtype={"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], bits=4)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(53)
    k, v = (torch.randn((layers * hk, n, D), generator=gen, device="cuda").to(cache.dtype) for _ in range(2))
    kept = torch.arange(n, dtype=torch.int32, device="cuda").repeat(layers * hk, 1)
    P.paged_compact(cache, p, k, v, kept)
    out = P.paged_read(cache, P.NewTokens([0, n]))
    for x, src in zip(out, (k, v)):
        for layer in range(layers):  # a layer at a time is a small call
            one = cache.layer(layer)
            assert torch.equal(P.paged_read(one, P.NewTokens([0, n]))[0 if x is out[0] else 1][0], x[layer])
        at = [0, 1, 63, 64, 15999, n - 1]
        want = O4.decode(*O4.encode(_f64(src.view(layers, hk, n, D)[:, :, at]), dtype))
        assert np.array_equal(_f64(x[:, at]), want.transpose(0, 2, 1, 3))
    small = P.PagedCache.alloc(layers, 4, hk, 1, 1000, page_size=64, dtype=cache.dtype, bits=4)
    ps = T._problem((1000,), layers, hk, (1, 1))
    P.paged_compact(small, ps, k[:, 5000:6000].contiguous(), v[:, 5000:6000].contiguous(), kept[:, :1000].contiguous())
    for x, y in zip(P.paged_read(small, P.NewTokens([0, 1000])), out):
        assert torch.equal(x, y[:, 5000:6000])


# ---------------------------------------------------------------------------
# Together, as a program serves
# ---------------------------------------------------------------------------

def test_compress_into_4_bits(torch_cuda):
    """The compression pass straight into 4-bit pages: the codes of the rows that the dense compaction keeps."""
    import torch
    from paper_2603_00188_amd import paged as P
    from paper_2603_00188_amd import stlite as S
    from tests import gpu_harness as H
    from tests.test_gpu_parity import SMALL
    case = H.Case(SMALL["ragged"])
    w, prob, res = case.w, case.prob, case.run()
    cache = P.PagedCache.alloc(case.n_layers, w.n_q_heads, w.n_kv_heads, prob.n_seqs, int(np.diff(case.cu_budget).max()) + 9,
                               page_size=16, bits=4)
    S.compress(prob, case.dq, case.dk, case.dv, case.out, alpha=w.alpha, cache=cache)
    k, v = P.paged_read(cache, P.NewTokens(case.cu_budget))
    torch.cuda.synchronize()
    assert cache.seq_lens.tolist() == np.diff(case.cu_budget).tolist()
    for x, rows in ((k, res["k_out"]), (v, res["v_out"])):
        bits = torch.from_numpy(np.ascontiguousarray(rows).view(np.int16)).view(torch.bfloat16)
        want = O4.decode(*O4.encode(_f64(bits), "bf16")).reshape(case.n_layers, w.n_kv_heads, -1, D)
        assert np.array_equal(_f64(x), want.transpose(0, 2, 1, 3))


def test_layers_one_by_one(torch_cuda):
    """What a model does: layer after layer, each on its own slice of the cache."""
    import torch
    for new in (1, 6, 40):
        f = Served4((500, 120, 77), (new,) * 3, 32, "bf16", 4, 8, 2, seed=17)
        q, k, v = (f.randn((4, f.total, h, D)) for h in (8, 2, 2))
        pos = torch.arange(f.total, dtype=torch.int32, device="cuda").view(1, -1)
        qs = []
        for layer in range(4):
            one, at = f.cache.layer(layer), slice(layer, layer + 1)
            qs.append(f.P.paged_append(one, f.batch, q[at], k[at], v[at], positions=pos, rope=f.P.Rope()))
        outs = torch.cat([f.P.paged_attention(f.cache.layer(i), f.batch, qs[i]) for i in range(4)])
        pools = f.kb.clone(), f.vb.clone()
        whole = f.P.paged_append(f.cache, f.batch, q, k, v, positions=pos, rope=f.P.Rope())
        torch.cuda.synchronize()
        assert torch.equal(torch.cat(qs), whole) and torch.equal(pools[0], f.kb) and torch.equal(pools[1], f.vb)
        for x, b in ((f.k, f.kb), (f.v, f.vb)):
            x.copy_(torch.from_numpy(O4.decode(*O4.rows(b.cpu().numpy(), 32))))
        f.compare(whole, outs)
        f.compare(whole, f.attend(whole))


@pytest.mark.parametrize("new", [1, 4, 40])
def test_streams_and_two_calls_at_once(torch_cuda, new):
    """On busy streams that are not the current one, two workspaces, tensors that are dropped at once."""
    import torch
    f = Served4((3000, 240, 700), (new,) * 3, 32, "bf16", 2, 8, 2, seed=27)
    n = 3 * new
    rows = [f.randn((2, n, h, D)) for h in (8, 2, 2)]
    want_q = f.P.paged_append(f.cache, f.batch, *rows)
    want = f.P.paged_attention(f.cache, f.batch, want_q)
    pools = f.kb.clone(), f.vb.clone()
    busy = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for side in sides:
        with torch.cuda.stream(side):
            for _ in range(10):
                torch.mm(busy, busy)
        q = f.P.paged_append(f.cache, f.P.NewTokens(f.cu), *(x.clone() for x in rows), stream=side)
        got.append((q, f.P.paged_attention(f.cache, f.P.NewTokens(f.cu), q, stream=side)))
        junk = [torch.full_like(x, 9.0) for x in rows for _ in range(4)]
    torch.cuda.synchronize()
    for q, o in got:
        assert torch.equal(q, want_q) and torch.equal(o, want) and len(junk) == 12
    assert torch.equal(f.kb, pools[0]) and torch.equal(f.vb, pools[1])


@pytest.mark.parametrize("layers,seqs,hq,extra", [(2, 65535, 64, 0), (65535, 2, 2, 1), (2, 65535, 128, 1)])
def test_limits_of_a_call(torch_cuda, layers, seqs, hq, extra):
    """As many sequences, or layers, as a call may have.  Every token sees one key, so that its output is that key's value,
    but for the second token of the last sequence, which sees two equal keys with equal values."""
    import torch
    from paper_2603_00188_amd import paged as P
    gen = torch.Generator(device="cuda")
    gen.manual_seed(32)
    new = torch.ones(seqs, dtype=torch.int64)
    new[-1] += extra
    batch = P.NewTokens(torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]))
    n = batch.total
    table = torch.randperm(seqs, generator=gen, device="cuda").to(torch.int32).view(seqs, 1)
    pool = [torch.full((layers, 1, seqs, 16 * 68), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = P.PagedCache(*pool, table, new.to(torch.int32).cuda(), hq)
    k, v = (torch.randn((layers, n, 1, D), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    if extra:
        k[:, -1], v[:, -1] = k[:, -2], v[:, -2]
    P.paged_append(cache, batch, None, k, v)
    rk, rv = P.paged_read(cache, batch)
    for x, y in ((rk, k), (rv, v)):
        for layer in range(0, layers, max(layers // 8, 1)):
            at = torch.randint(0, n, (256,), device="cuda")
            assert np.array_equal(_f64(x[layer, at, 0]), O4.decode(*O4.encode(_f64(y[layer, at, 0]), "bf16")))
    q = torch.randn((1, n, hq, D), generator=gen, device="cuda", dtype=torch.bfloat16).expand(layers, -1, -1, -1).contiguous()
    out = P.paged_attention(cache, batch, q)
    for layer in range(0, layers, max(layers // 64, 1)):
        # (a weight rounded to 1, over a sum of it: exact; of two equal ones too)
        assert torch.equal(out[layer], rv[layer].expand(-1, hq, -1)), layer
