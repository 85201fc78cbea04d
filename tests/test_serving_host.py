"""CPU: the oracles of 4-bit pools, of growing and releasing pages and of drafted tokens, and what the host refuses."""
from __future__ import annotations

import copy
import ctypes
import os
import pickle

import numpy as np
import pytest
import torch

from oracle import paged4 as O4
from oracle import serving as OS
from paper_2603_00188_amd import paged as P
from paper_2603_00188_amd import stlite as S
from tests.test_paged_host import BAD, BAD_BATCH, FAKE, Fake, _err

needs_lib = pytest.mark.skipif(not os.path.exists(S.LIB_PATH), reason="library not built")
BIG = 1 << 44  # apart from FAKE


# ---------------------------------------------------------------------------
# Oracles
# ---------------------------------------------------------------------------

def test_codes_by_hand():
    x = np.zeros(128)
    x[:8] = [6, 5, 3.5, 2.5, 1.75, -0.75, 0.25, -0.2]  # scale 1
    x[32:36] = [7, 1, -0.5, 0.25]                      # 7 fits a scale of 1, and becomes 6
    x[64:67] = [7.1, 1, 0.5]                           # a scale of 2
    codes, scales = O4.encode(x, "bf16")
    assert scales.tolist() == [127, 127, 128, 7]
    assert codes[:4].tolist() == [0x67, 0x46, 0xA4, 0x80]
    assert codes[16:18].tolist() == [0x27, 0x09] and codes[32:34].tolist() == [0x16, 0x00]
    v = O4.decode(codes, scales)
    assert v[:8].tolist() == [6, 4, 4, 2, 2, -1, 0, -0.0] and v[32:36].tolist() == [6, 1, -0.5, 0]
    assert v[64:67].tolist() == [8, 1, 0] and np.signbit(v[7])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_codes_are_the_nearest(dtype):
    """No other code under the block's scale is nearer, the scale is the least that reaches, values store as themselves."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((300, 128)) * np.exp2(rng.integers(-10, 10, (300, 1)))
    codes, scales = O4.encode(x, dtype)
    v = O4.decode(codes, scales)
    s = np.ldexp(1.0, scales.astype(int) - 127).repeat(32, -1).reshape(300, 128)
    grid = np.concatenate([O4.GRID, -O4.GRID])
    assert (np.abs(v - x) <= np.abs(grid[:, None, None] * s - x).min(0) + 1e-300).all()
    top = np.abs(x).reshape(300, 4, 32).max(-1)
    assert (top <= 7 * s[:, ::32]).all() and (top > 3.5 * s[:, ::32]).all()
    again = O4.encode(v, dtype)
    assert np.array_equal(again[0], codes) and np.array_equal(again[1], scales)
    packed = O4.pool(x.reshape(25, 12, 128)[:, :8], dtype)
    assert packed.shape == (25, 8 * 68)
    c, sc = O4.rows(packed, 8)
    assert np.array_equal(c, codes.reshape(25, 12, 64)[:, :8]) and np.array_equal(sc, scales.reshape(25, 12, 4)[:, :8])


def test_codes_at_the_limits():
    for dtype, (lo, hi), top in (("bf16", O4.RANGE["bf16"], 3.3895e38), ("fp16", O4.RANGE["fp16"], 65504.0)):
        x = np.zeros((3, 128))
        x[0, :32], x[0, 32:64], x[0, 64:96] = top, 2.0 ** (lo - 5), 2.0 ** lo
        x[1, 3], x[1, 40], x[1, 90] = np.inf, np.nan, -np.inf
        codes, scales = O4.encode(x, dtype)
        v = O4.decode(codes, scales)
        assert (v[0, :32] == 6 * 2.0 ** hi).all() and (v[0, 32:64] == 0).all() and (v[0, 64:96] == 2.0 ** lo).all()
        assert scales[1, 0] == scales[1, 1] == scales[1, 2] == 255 and scales[1, 3] == lo + 127
        assert np.isnan(v[1, :96]).all() and (v[1, 96:] == 0).all() and (v[2] == 0).all()


def test_pages_by_hand():
    p = OS.Pool([[-1] * 4 for _ in range(3)], [0, 0, 0], [0, 0, 0], [4, 3, 2, 1, 0], 16, 64)
    assert p.grow([17, 16, 1]) == [0 * 16 + j for j in range(16)] + [16] + [32 + j for j in range(16)] + [48]
    assert p.table == [[0, 1, -1, -1], [2, -1, -1, -1], [3, -1, -1, -1]] and p.free == [4]
    # the second asks for two pages, of which one is left: parked, and the third, which needs none, is not held up
    assert p.grow([0, 33, 15]) == [-1] * 33 + [48 + j for j in range(1, 16)]
    assert p.lens == [17, ~16, 16] and p.free == [4]
    assert p.grow([1, 1, 1])[:2] == [17, -1] and p.lens == [18, ~16, 17]  # the third takes the last page
    p.release([0, 16, -1])
    assert p.lens == [0, 16, 17] and p.held == [0, 1, 2] and p.free == [1, 0]
    assert p.grow([17, 0, 0])[:1] == [0] and p.table[0] == [0, 1, -1, -1]
    assert p.grow([48, 0, 0]) == [-1] * 48 and p.lens[0] == ~17  # past max_len
    p.release()
    assert p.lens[0] == ~17 and p.held[0] == 2


def test_drafts_by_hand():
    p = [[0.5, 0.25, 0.25], [0.0, 1.0, 0.0], [0.25, 0.25, 0.5]]
    q = [[0.5, 0.5, 0.0], [1.0, 0.0, 0.0], [0.0, 0.0, 1.0]]
    assert OS.verify(p, q, [0, 0, 9], [0.99, 0.0, 0.0], 0.5) == [0, 1]  # the second is impossible: all of the rest on 1
    assert OS.verify(p, q, [1, 0, 9], [0.5, 0.0, 0.0], 0.5) == [2]      # 0.5 0.5 = 0.25: not below; the rest is on 2
    assert OS.verify(p, q, [1, 1, 9], [0.49, 0.0, 0.0], 0.49) == [1, 1, 1]
    assert OS.verify(p, q, [1, 1, 9], [0.49, 0.0, 0.0], 0.5) == [1, 1, 2]
    assert OS.verify(p, None, [0, 1, 9], [0.5, 0.0, 0.0], 0.49) == [1] and OS.verify(p, None, [0, 1, 9], [0.5, 0.0, 0.0], 0.5) == [2]
    assert OS.verify([[0.0, 0.0]], None, [0], [0], 0.5) == [-1] and OS.verify([[0.0, 2.0]], None, [0], [0], 1.0) == [1]
    assert OS.verify(p, q, [3, 0, 0], [0.0, 0.0, 0.0], 0.0) == [2]      # no token of the vocabulary


def test_drafts_follow_the_target():
    """Whatever the draft proposes, what comes out is distributed as the target: over a fine grid of the numbers the shares
    of the first token are the target's probabilities."""
    p, q = [[0.5, 0.125, 0.375], [1.0, 0.0, 0.0]], [[0.25, 0.5, 0.25], [0.0, 0.0, 0.0]]
    n, m, share = 32, 48, [0.0, 0.0, 0.0]  # (the rest is 2 to 1: m is a multiple of 3)
    for x in range(3):
        for i in range(n):
            for j in range(m):
                got = OS.verify(p, q, [x, 0], [(i + 0.5) / n, 0.0], (j + 0.5) / m)
                share[got[0]] += q[0][x] / n / m
    assert share == pytest.approx(p[0], abs=1e-12)


# ---------------------------------------------------------------------------
# Refusals
# ---------------------------------------------------------------------------

def _pages(**kw):
    f = dict(pages=BIG, n_free=BIG + 4096, held=BIG + 8192, page_table=FAKE)
    f.update(kw)
    return ctypes.byref(S._CFreePages(**f))


@needs_lib
@pytest.mark.parametrize("change, status, text", BAD + BAD_BATCH)
def test_cache_rejections(change, status, text):
    lib, f = S.load(), Fake(**change)
    calls = [lambda: lib.stlite_paged_read(f.ref, BIG, BIG + (1 << 30), None)]
    if change != {"max_len": 1}:  # growing takes more new tokens than that, and parks the sequence
        calls.append(lambda: lib.stlite_paged_grow(f.ref, _pages(), BIG + 16384, None))
    if (change, status, text) in BAD:
        calls.append(lambda: lib.stlite_paged_release(f.ref, _pages(), BIG + 16384, None))
    for call in calls:
        assert call() == status and text in _err()


@needs_lib
def test_dtypes_of_a_4_bit_pool():
    lib, n = S.load(), ctypes.c_size_t(0)
    for dtype, ok in ((16, True), (17, True), (18, False), (15, False), (32, False), (-1, False), (-16, False)):
        st = lib.stlite_paged_workspace_size(Fake(dtype=dtype).ref, ctypes.byref(n))
        assert (st == 0) == ok, dtype


@needs_lib
def test_aliases_of_a_4_bit_pool():
    """A pool in 4 bits has 68 bytes to a row: what lies behind them is another's."""
    lib = S.load()
    f = Fake(dtype=16, v=BIG)
    size = 2 * 4 * 20 * 16 * 68
    q = 2 * 3 * 28 * 128 * 2
    for at, ok in ((FAKE + size - 16, False), (FAKE - q + 16, False)):
        st = lib.stlite_paged_attention(f.ref, BIG + (1 << 40), 1.0, at, BIG + (1 << 41), 1 << 40, None)
        assert st == S.ERR_INVALID_ARG and "alias" in _err()
    for a, b in ((FAKE + size - 16, BIG + (1 << 40)), (BIG + (1 << 40), BIG + size - 16)):
        assert lib.stlite_paged_read(f.ref, a, b, None) == S.ERR_INVALID_ARG and "alias" in _err()
    assert lib.stlite_paged_read(f.ref, BIG + (1 << 40), BIG + (1 << 40) + 64, None) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_read(f.ref, BIG + (1 << 40) + 8, None, None) == S.ERR_INVALID_ARG and "aligned" in _err()
    assert lib.stlite_paged_read(f.ref, None, None, None) == 0  # nothing asked for


@needs_lib
def test_free_pages_rejections():
    lib, table = S.load(), BIG + (1 << 20)
    f = Fake(page_table=table, seq_lens=BIG + (1 << 21), cu_new=BIG + (1 << 22))
    for bad in (dict(pages=None), dict(n_free=None), dict(held=None)):
        assert lib.stlite_paged_grow(f.ref, _pages(page_table=table, **bad), None, None) == S.ERR_INVALID_ARG and "non-NULL" in _err()
        assert lib.stlite_paged_release(f.ref, _pages(page_table=table, **bad), None, None) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_grow(f.ref, None, None, None) == S.ERR_INVALID_ARG
    for other in (None, table + 4):
        assert lib.stlite_paged_grow(f.ref, _pages(page_table=other), None, None) == S.ERR_INVALID_ARG and "page_table" in _err()
        assert lib.stlite_paged_release(f.ref, _pages(page_table=other), None, None) == S.ERR_INVALID_ARG and "page_table" in _err()
    for bad in (dict(n_free=BIG + 76), dict(held=BIG + 4096), dict(pages=table + 36), dict(held=BIG + (1 << 21)),
                dict(n_free=BIG + (1 << 22) + 8)):
        p = _pages(page_table=table, **bad)
        assert lib.stlite_paged_grow(f.ref, p, None, None) == S.ERR_INVALID_ARG and "overlap" in _err()
        assert lib.stlite_paged_release(f.ref, p, None, None) == S.ERR_INVALID_ARG and "overlap" in _err()
    p = _pages(page_table=table)
    assert lib.stlite_paged_grow(f.ref, p, BIG + 8192 + 4, None) == S.ERR_INVALID_ARG and "overlap" in _err()
    assert lib.stlite_paged_release(f.ref, p, BIG + (1 << 21) + 4, None) == S.ERR_INVALID_ARG and "overlap" in _err()
    assert lib.stlite_paged_grow(f.ref, _pages(page_table=table, held=FAKE + 64), None, None) == S.ERR_INVALID_ARG and "pool" in _err()


class Drafts:
    def __init__(self, counts=(0, 2, 2, 5), vocab=100, **kw):
        self.cu = np.asarray(counts, np.int32)
        n = int(self.cu[-1])
        f = dict(n_seqs=len(self.cu) - 1, vocab=vocab, dtype=2, reserved=0, total_new=n, cu_new=BIG, h_cu_new=self.cu.ctypes.data,
                 target=BIG + (1 << 20), draft=BIG + (1 << 24), target_stride=vocab, draft_stride=vocab, tokens=BIG + (1 << 12),
                 accept=BIG + (2 << 12), pick=BIG + (3 << 12), seq_lens=BIG + (4 << 12))
        f.update(kw)
        self.c = S._CVerify(**f)

    def call(self, out=BIG + (5 << 12), n_out=BIG + (6 << 12), ws=BIG + (7 << 12), size=4096):
        return S.load().stlite_verify_drafts(ctypes.byref(self.c), out, n_out, ws, size, None)


@needs_lib
@pytest.mark.parametrize("change, status, text", [
    (dict(dtype=3), S.ERR_INVALID_ARG, "dtype"), (dict(reserved=1), S.ERR_INVALID_ARG, "reserved"),
    (dict(n_seqs=0), S.ERR_INVALID_ARG, "n_seqs"), (dict(n_seqs=65536), S.ERR_UNSUPPORTED, "65535"),
    (dict(vocab=0), S.ERR_INVALID_ARG, "vocab"), (dict(vocab=(1 << 24) + 1), S.ERR_UNSUPPORTED, "2^24"),
    (dict(cu_new=None), S.ERR_INVALID_ARG, "non-NULL"), (dict(h_cu_new=None), S.ERR_INVALID_ARG, "non-NULL"),
    (dict(total_new=4), S.ERR_INVALID_ARG, "total_new"), (dict(counts=(0, 3, 2, 5)), S.ERR_INVALID_ARG, "rows"),
    (dict(counts=(1, 2, 2, 5)), S.ERR_INVALID_ARG, "cu_new[0]")])
def test_drafts_rejections(change, status, text):
    d = Drafts(**change)
    n = ctypes.c_size_t(7)
    assert d.call() == status and text in _err()
    assert S.load().stlite_verify_workspace_size(ctypes.byref(d.c), ctypes.byref(n)) == status and n.value == 0


@needs_lib
def test_drafts_arguments():
    for bad in (dict(target=None), dict(tokens=None), dict(accept=None), dict(pick=None)):
        assert Drafts(**bad).call() == S.ERR_INVALID_ARG and "non-NULL" in _err()
    assert Drafts().call(out=None) == S.ERR_INVALID_ARG and Drafts().call(n_out=None) == S.ERR_INVALID_ARG
    for bad in (dict(target_stride=99), dict(draft_stride=99)):
        assert Drafts(**bad).call() == S.ERR_INVALID_ARG and "stride" in _err()
    for bad in (dict(target=BIG + (1 << 20) + 2), dict(draft=BIG + (1 << 24) + 1, dtype=0)):
        assert Drafts(**bad).call() == S.ERR_INVALID_ARG and "aligned" in _err()
    n = ctypes.c_size_t(0)
    assert S.load().stlite_verify_workspace_size(ctypes.byref(Drafts().c), ctypes.byref(n)) == 0 and n.value > 0
    assert S.load().stlite_verify_workspace_size(ctypes.byref(Drafts().c), None) == S.ERR_INVALID_ARG
    assert Drafts().call(size=n.value - 1) == S.ERR_WORKSPACE and Drafts().call(ws=None) == S.ERR_WORKSPACE
    assert Drafts().call(ws=BIG + (7 << 12) + 128) == S.ERR_WORKSPACE
    at = {"tokens": 1 << 12, "accept": 2 << 12, "pick": 3 << 12, "lens": 4 << 12, "target": (1 << 20) + 400, "draft": 1 << 24, "cu": 8}
    for name, where in at.items():
        assert Drafts().call(out=BIG + where) == S.ERR_INVALID_ARG and "overlap" in _err(), name
        assert Drafts().call(n_out=BIG + where) == S.ERR_INVALID_ARG and "overlap" in _err(), name
        assert Drafts().call(ws=BIG + where & ~255) == S.ERR_INVALID_ARG and "overlap" in _err(), name
    assert Drafts().call(out=BIG + (6 << 12) + 4) == S.ERR_INVALID_ARG
    assert Drafts(seq_lens=BIG + (3 << 12)).call() == S.ERR_INVALID_ARG


# ---------------------------------------------------------------------------
# The binding
# ---------------------------------------------------------------------------

def _four(**kw):
    return P.PagedCache.alloc(2, 8, 2, 3, 60, page_size=16, device="cpu", bits=4, **kw)


@needs_lib
def test_4_bit_cache():
    c = _four()
    assert c.bits == 4 and c.dtype == torch.bfloat16 and c.k.dtype == torch.uint8 and c.k.shape == (2, 2, 12, 16 * 68)
    assert c.page_size == 16 and c._c.dtype == 16 and _four(dtype=torch.float16)._c.dtype == 17
    assert P.PagedCache.alloc(2, 8, 2, 3, 60, page_size=16, device="cpu").bits == 16
    one = c.layer(1)
    assert one.bits == 4 and one.dtype == c.dtype and one.k.data_ptr() == c.k[1].data_ptr()
    for other in (copy.deepcopy(_four(dtype=torch.float16)), pickle.loads(pickle.dumps(_four(dtype=torch.float16)))):
        assert other.bits == 4 and other.dtype == torch.float16 and other._c.k == other.k.data_ptr()
    with pytest.raises(AttributeError):
        c.bits = 16
    free = _four(n_pages=5)
    assert free.n_pages == 5 and (free.page_table == -1).all()


@needs_lib
def test_4_bit_cache_refusals():
    c = _four()
    lens, table = c.seq_lens, c.page_table
    for k in (c.k[..., :-1].contiguous(), c.k.view(2, 2, 12, 16, 68), c.k[..., :0]):
        with pytest.raises(ValueError, match="uint8"):
            P.PagedCache(k, k, table, lens, 8)
    with pytest.raises(ValueError, match="dtype"):
        P.PagedCache(c.k, c.v, table, lens, 8, dtype=torch.float32)
    k = torch.zeros((1, 2, 3, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="dtype"):
        P.PagedCache(k, k, table, lens, 8, dtype=torch.float16)
    with pytest.raises(ValueError, match="bits"):
        P.PagedCache.alloc(1, 1, 1, 1, 16, device="cpu", bits=8)
    with pytest.raises(ValueError, match="v must be"):
        P.PagedCache(c.k, c.v[:1], table, lens, 8)


@needs_lib
def test_binding_refusals():
    c = _four(n_pages=5)
    b = P.NewTokens([0, 1, 1, 4], device="cpu")
    with pytest.raises(ValueError, match="k_out"):
        P.paged_read(c, b, k_out=torch.zeros((2, 4, 2, 128)))
    with pytest.raises(ValueError, match="on a GPU|GPU"):
        P.paged_read(c, b)
    f = P.FreePages.of(c)
    assert f.pages.tolist() == [4, 3, 2, 1, 0] and f.n_free.tolist() == [5] and f.held.tolist() == [0, 0, 0]
    assert copy.deepcopy(f)._c.pages != f._c.pages
    with pytest.raises(AttributeError):
        f.pages = f.pages.clone()
    for bad in ((f.pages.long(), f.n_free, f.held), (f.pages, f.n_free[0], f.held), (f.pages, f.n_free, f.held.float()),
                (f.pages[::2], f.n_free, f.held)):
        with pytest.raises(ValueError):
            P.FreePages(*bad)
    with pytest.raises(ValueError, match="held"):
        P.FreePages(f.pages, f.n_free, f.held[:2].clone())._for(c)
    with pytest.raises(ValueError, match="slots"):
        P.paged_grow(c, f, b, slots=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="lens"):
        P.paged_release(c, f, torch.zeros(3))
    p = torch.zeros((4, 50))
    x, u, r = torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(3)
    for kw, text in ((dict(target=p.double()), "target"), (dict(target=p[:3]), "target"), (dict(target=p.t()), "target"),
                     (dict(target=torch.zeros((50, 4)).t()), "after another"), (dict(target=p[:1].expand(4, 50)), "overlap"),
                     (dict(draft=p.half()), "draft"), (dict(draft=p[:, :49]), "draft"), (dict(tokens=x.long()), "tokens"),
                     (dict(accept=u.double()), "accept"), (dict(pick=u), "pick"), (dict(out=x[:2]), "out"), (dict(n_out=x), "n_out"),
                     (dict(cache=P.PagedCache.alloc(1, 1, 1, 2, 16, device="cpu")), "sequences")):
        args = dict(target=p, tokens=x, accept=u, pick=r)
        args.update(kw)
        with pytest.raises(ValueError, match=text):
            P.verify_drafts(b, **args)
