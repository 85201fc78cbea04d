"""Sequences that are parked for want of pages, and the calls that meet them: growing, compaction into pages, append and
attention, against oracle/serving.py and the 64-bit oracles."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import paged as OP
from oracle import paged4 as O4
from oracle import serving as OS
from tests.test_gpu_paged import D, _bits, _f64, _log, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

PAGE, LAYERS, HK, HQ = 16, 2, 2, 6


def _problem(keep):
    """A problem whose sequences keep the first so many of their tokens, and those tokens (a sequence has 2 more)."""
    from paper_2603_00188_amd import stlite as S
    cu = np.concatenate([[0], np.cumsum(np.array(keep) + 2)])
    p = S.Problem(LAYERS, HQ, HK, 1, cu, np.zeros(len(cu)), np.zeros((0, 3)), np.concatenate([[0], np.cumsum(keep)]))
    return p, [int(a) + j for a, n in zip(cu, keep) for j in range(n)]


class Shared:
    """A pool whose pages are given out, full of rows that sequences before left; the oracle's lengths and pages beside it."""

    def __init__(self, seqs, n_pages, max_len, bits, dtype="bf16", seed=0):
        import torch
        from paper_2603_00188_amd import paged as P
        self.P, self.bits, self.dtype = P, bits, dtype
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.cache = P.PagedCache.alloc(LAYERS, HQ, HK, seqs, max_len, page_size=PAGE, bits=bits, n_pages=n_pages,
                                        dtype={"bf16": torch.bfloat16, "fp16": torch.float16}[dtype])
        old = self.rows(LAYERS, HK, n_pages * PAGE)
        for pool in (self.cache.k, self.cache.v):
            if bits == 4:
                pool.copy_(torch.from_numpy(O4.pool(_f64(old).reshape(LAYERS, HK, n_pages, PAGE, D), dtype)))
            else:
                pool.copy_(old.view(pool.shape))
        self.pages = P.FreePages.of(self.cache)
        self.o = OS.Pool(self.cache.page_table.tolist(), [0] * seqs, [0] * seqs, self.pages.pages.tolist(), PAGE, max_len)

    def rows(self, *shape):
        import torch
        return torch.randn((*shape, D), generator=self.gen, device="cuda").to(self.cache.dtype)

    def batch(self, new):
        return self.P.NewTokens(np.concatenate([[0], np.cumsum(new)]))

    def grow(self, new):
        self.P.paged_grow(self.cache, self.pages, self.batch(new))
        self.o.grow(list(new))
        self.same()

    def release(self, lens=None):
        import torch
        self.P.paged_release(self.cache, self.pages, None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))
        self.o.release(lens)
        self.same()

    def same(self):
        assert self.cache.seq_lens.tolist() == self.o.lens and self.pages.held.tolist() == self.o.held
        n = int(self.pages.n_free)
        assert n == len(self.o.free) and self.pages.pages[:n].tolist() == self.o.free
        assert self.cache.page_table.tolist() == self.o.table

    def bytes(self):
        return [t.cpu().numpy().copy() if self.bits == 4 else _bits(t).copy() for t in (self.cache.k, self.cache.v)]

    def put(self, pool, places, src):
        """Rows `places` of every unit of the oracle's pool (bytes()) become src [units, rows, 128]; None: dropped."""
        at = [i for i, r in enumerate(places) if r is not None]
        r = np.array([places[i] for i in at], np.int64)
        if not at:
            return
        if self.bits == 16:
            pool.reshape(LAYERS * HK, -1, D)[:, r] = _bits(src)[:, at]
            return
        codes, scales = O4.rows(pool.reshape(LAYERS * HK, self.cache.n_pages, -1), PAGE)
        codes[:, r // PAGE, r % PAGE], scales[:, r // PAGE, r % PAGE] = O4.encode(_f64(src)[:, at], self.dtype)

    def compact(self, lens, per_layer=False):
        """So many tokens of each sequence's problem are kept; the pool and the lengths are as the oracle has them afterwards."""
        import torch
        p, tok = _problem(lens)
        k, v = self.rows(LAYERS * HK, p.total_tokens), self.rows(LAYERS * HK, p.total_tokens)
        lists = LAYERS if per_layer else LAYERS * HK
        kept = torch.tensor(tok, dtype=torch.int32, device="cuda").repeat(lists, 1)
        want = self.bytes()
        taken = self.o.compact(list(lens))
        self.P.paged_compact(self.cache, p, k, v, kept, per_layer=per_layer)
        table = np.array(self.o.table)
        places = [OP.place(table, s, j, PAGE, self.cache.n_pages) if taken[s] else None for s, n in enumerate(lens) for j in range(n)]
        for pool, src in zip(want, (k, v)):
            self.put(pool, places, src[:, tok])
        self.same()
        for got, w in zip(self.bytes(), want):
            assert np.array_equal(got, w)
        return taken

    def step(self, new):
        """Growing, append, attention, against the oracle over what the pool holds."""
        self.grow(new)
        b = self.batch(new)
        q, k, v = self.rows(LAYERS, b.total, HQ), self.rows(LAYERS, b.total, HK), self.rows(LAYERS, b.total, HK)
        want = self.bytes()
        places = OP.new_places(np.array(self.o.table), self.o.lens, b.h, PAGE, self.cache.n_pages, self.cache.max_len)
        for pool, src in zip(want, (k, v)):
            self.put(pool, places, src.transpose(1, 2).reshape(LAYERS * HK, b.total, D).contiguous())
        self.P.paged_append(self.cache, b, None, k, v)
        for got, w in zip(self.bytes(), want):
            assert np.array_equal(got, w)
        out = _f64(self.P.paged_attention(self.cache, b, q))
        pools = [_f64(t) if self.bits == 16 else O4.decode(*O4.rows(t.cpu().numpy(), PAGE)) for t in (self.cache.k, self.cache.v)]
        u = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[self.dtype]
        for layer in range(LAYERS):
            ref, weight, keys, dot = OP.attention(_f64(q[layer]), pools[0][layer], pools[1][layer], np.array(self.o.table), self.o.lens,
                                                  b.h, self.cache.max_len, D ** -0.5, HQ // HK)
            rel = u + 2 * 128 * 2.0 ** -24 * dot + 2.0 ** -22 * (1 + dot) + 2 * keys * 2.0 ** -24
            assert (np.abs(out[layer] - ref) <= u * np.abs(ref) + rel[..., None] * weight + 2.0 ** -25).all()
        for s, n in enumerate(self.o.lens):
            if n < 0:
                assert not out[:, b.h[s]:b.h[s + 1]].any()


@pytest.mark.parametrize("bits,dtype", [(16, "bf16"), (4, "bf16"), (4, "fp16")])
@pytest.mark.parametrize("per_layer", [False, True])
def test_compaction_leaves_parked_sequences(torch_cuda, bits, dtype, per_layer):
    """Room for the kept rows, the compression into it, then tokens: with too few pages one sequence is parked, and stays so,
    with nothing stored for it, until a release; the others are served, and then that one is."""
    _log(f"parked, compaction, {bits} bits {dtype}")
    f = Shared(4, 14, 160, bits, dtype, seed=1)
    lens = [70, 100, 33, 40]  # 5 + 7 + 3 + 3 pages of 14
    f.grow(lens)
    assert f.o.lens == [70, 100, ~0, ~0]
    assert f.compact(lens, per_layer) == [True, True, False, False]
    f.step([1, 1, 1, 1])
    f.step([3, 20, 1, 2])
    assert f.o.lens[2:] == [~0, ~0]
    f.release([-1, 0, 0, -1])  # the second ends, the third is parked no more
    f.step([1, 0, 33, 1])
    assert f.o.lens[2] == 33 and f.o.lens[3] == ~0
    f.release([0, 0, 0, 0])
    f.grow([10, 33, 0, 40])
    assert f.compact([10, 33, 0, 40], per_layer) == [True] * 4
    f.step([1, 1, 1, 1])


@pytest.mark.parametrize("bits", [16, 4])
def test_compaction_leaves_a_parked_sequence_its_tokens(torch_cuda, bits):
    """A running sequence that is parked keeps its rows and its length, and goes on once it is released."""
    f = Shared(3, 7, 100, bits, seed=2)
    f.step([50, 20, 0])
    f.grow([45, 0, 5])  # 2 more pages for the first, of 1 that is left: parked, and the third behind it
    assert f.o.lens == [~50, 20, ~0]
    assert f.compact([40, 30, 16]) == [False, True, False]  # (30 of 20: the second's pages reach)
    f.release([50, 20, 0])
    f.step([2, 1, 7])
    assert f.o.lens == [52, 21, 7]


@pytest.mark.parametrize("bits", [16, 4])
def test_compaction_leaves_an_empty_sequence_that_holds_pages(torch_cuda, bits):
    """A slot that is used again with the pages that it has: where these and the free ones are too few, it is parked, and what
    it holds is no beginning for rows whose rest has no place.  Where they reach, they are taken."""
    f = Shared(2, 7, 100, bits, seed=3)
    f.grow([40, 16])
    f.cache.seq_lens[0] = 0
    f.o.lens[0] = 0
    f.grow([97, 0])  # 7 pages, of 3 + 3
    assert f.o.lens == [~0, 16] and f.o.held == [3, 1]
    assert f.compact([90, 16]) == [False, True]
    assert f.compact([49, 16]) == [False, True]
    f.step([5, 1])
    assert f.o.lens == [~0, 17]
    assert f.compact([48, 10]) == [True, True]  # all of it fits in what it holds
    f.step([5, 1])
    assert f.o.lens == [53, 11]
    f.release([0, 0])
    f.grow([60, 40])
    assert f.compact([60, 40]) == [True, True]


@pytest.mark.parametrize("bits", [16, 4])
def test_compaction_of_many_sequences_some_parked(torch_cuda, bits):
    """More sequences than a work-group has threads or a grown chunk holds, lengths of every kind."""
    rng = np.random.default_rng(4)
    seqs = 1100
    f = Shared(seqs, 1200, 64, bits, seed=4)
    lens = rng.integers(0, 50, seqs)
    lens[rng.random(seqs) < 0.3] = 0
    f.grow(lens.tolist())
    assert min(f.o.lens) == ~0
    taken = f.compact(lens.tolist())
    assert 0 < sum(taken) < seqs
    f.release([0 if rng.random() < 0.5 else -1 for _ in range(seqs)])
    f.grow(lens.tolist())
    f.compact(np.minimum(lens, 20).tolist())


@pytest.mark.parametrize("bits", [16, 4])
def test_compaction_in_a_graph_meets_parked_sequences(torch_cuda, bits):
    """Growing, compaction and a look at the rows captured together: each replay goes by the lengths and pages of its own."""
    import torch
    f = Shared(3, 8, 64, bits, seed=5)
    lens = [40, 50, 20]
    p, tok = _problem(lens)
    k, v = f.rows(LAYERS * HK, p.total_tokens), f.rows(LAYERS * HK, p.total_tokens)
    kept = torch.tensor(tok, dtype=torch.int32, device="cuda").repeat(LAYERS * HK, 1)
    b = f.batch(lens)
    outs = [torch.empty((LAYERS, b.total, HK, D), dtype=f.cache.dtype, device="cuda") for _ in range(2)]

    def play():
        f.P.paged_grow(f.cache, f.pages, b)
        f.P.paged_compact(f.cache, p, k, v, kept)
        f.P.paged_read(f.cache, b, *outs)

    state = [t.clone() for t in (*f.cache.tensors, f.pages.pages, f.pages.n_free, f.pages.held)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        play()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        play()
    for t, was in zip((*f.cache.tensors, f.pages.pages, f.pages.n_free, f.pages.held), state):
        t.copy_(was)
    want = [x[:, tok].view(LAYERS, HK, -1, D).transpose(1, 2).contiguous() for x in (k, v)]
    if bits == 4:
        want = [torch.from_numpy(O4.decode(*O4.encode(_f64(x), "bf16"))).to(f.cache.dtype).cuda() for x in want]
    for keep in ([0, 0, 0], [0, -1, 0], [-1, 0, 0], [0, 0, 0]):
        for o in outs:
            o.fill_(7.0)
        g.replay()
        f.o.grow(lens)
        taken = f.o.compact(lens)
        torch.cuda.synchronize()
        f.same()
        for s in range(3):
            rows = slice(int(b.h[s]), int(b.h[s + 1]))
            for o, w in zip(outs, want):
                assert torch.equal(o[:, rows], w[:, rows] if taken[s] else torch.zeros_like(w[:, rows])), (keep, s)
        f.release(keep)


@pytest.mark.parametrize("bits", [16, 4])
def test_a_batch_without_what_cannot_be_served(torch_cuda, bits):
    """More new tokens than max_len park their sequence.  Growing alone takes such a batch; the calls behind it refuse it with
    nothing done, and take the one without those tokens."""
    import torch
    f = Shared(3, 12, 64, bits, seed=6)
    new = [20, 65, 30]
    f.grow(new)
    assert f.o.lens == [20, ~0, 30]
    b, before = f.batch(new), f.bytes()
    q, k = f.rows(LAYERS, b.total, HQ), f.rows(LAYERS, b.total, HK)
    for call in (lambda: f.P.paged_append(f.cache, b, None, k, k), lambda: f.P.paged_attention(f.cache, b, q),
                 lambda: f.P.paged_read(f.cache, b), lambda: f.cache.workspace(b), lambda: f.cache.validate(b)):
        with pytest.raises(RuntimeError, match="grow"):
            call()
    torch.cuda.synchronize()
    f.same()
    assert all(np.array_equal(x, y) for x, y in zip(f.bytes(), before))
    f.step([0, 0, 0])
    rest = f.batch([20, 0, 30])
    k = f.rows(LAYERS, 50, HK)
    f.P.paged_append(f.cache, rest, None, k, k)
    assert torch.equal(f.P.paged_read(f.cache, rest)[0], k) or bits == 4
    f.step([1, 0, 1])


@pytest.mark.parametrize("bits", [16, 4])
def test_compress_into_pages_that_are_too_few(torch_cuda, bits):
    """The whole pass behind growing: who got pages has the kept rows, who did not is parked and nothing else changed."""
    import torch
    from paper_2603_00188_amd import paged as P
    from paper_2603_00188_amd import stlite as S
    from tests import gpu_harness as H
    from tests.test_gpu_parity import SMALL
    case = H.Case(SMALL["ragged"])
    w, prob = case.w, case.prob
    res, keep = case.run(), np.diff(case.cu_budget)
    n_pages = int((-(-keep // PAGE)).sum()) - 1
    cache = P.PagedCache.alloc(case.n_layers, w.n_q_heads, w.n_kv_heads, prob.n_seqs, int(keep.max()) + 40, page_size=PAGE,
                               bits=bits, n_pages=n_pages)
    pages = P.FreePages.of(cache)
    o = OS.Pool(cache.page_table.tolist(), [0] * prob.n_seqs, [0] * prob.n_seqs, pages.pages.tolist(), PAGE, cache.max_len)
    P.paged_grow(cache, pages, P.NewTokens(case.cu_budget))
    o.grow(keep.tolist())
    S.compress(prob, case.dq, case.dk, case.dv, case.out, alpha=w.alpha, cache=cache)
    taken = o.compact(keep.tolist())
    assert 0 < sum(taken) < prob.n_seqs
    assert cache.seq_lens.tolist() == o.lens and cache.page_table.tolist() == o.table and pages.held.tolist() == o.held
    table, used = np.array(o.table), []
    for s in range(prob.n_seqs):
        if not taken[s]:
            continue
        rows = [OP.place(table, s, j, PAGE, n_pages) for j in range(int(keep[s]))]
        used += rows
        a, b = case.cu_budget[s:s + 2]
        for pool, out in ((cache.k, res["k_out"]), (cache.v, res["v_out"])):
            if bits == 16:
                assert np.array_equal(_bits(pool).reshape(prob.units, -1, D)[:, rows].view(np.uint16), out[:, a:b])
                continue
            x = torch.from_numpy(out[:, a:b].astype(np.int32).astype(np.int16)).view(torch.bfloat16)
            codes, scales = O4.rows(pool.cpu().numpy().reshape(prob.units, n_pages, -1), PAGE)
            want = O4.encode(_f64(x), "bf16")
            r = np.array(rows)
            assert np.array_equal(codes[:, r // PAGE, r % PAGE], want[0]) and np.array_equal(scales[:, r // PAGE, r % PAGE], want[1])
    rest = np.setdiff1d(np.arange(n_pages * PAGE), used)
    for pool in (cache.k, cache.v):
        if bits == 16:
            assert not _bits(pool).reshape(prob.units, -1, D)[:, rest].any()
        else:
            codes, scales = O4.rows(pool.cpu().numpy().reshape(prob.units, n_pages, -1), PAGE)
            assert not codes[:, rest // PAGE, rest % PAGE].any() and not scales[:, rest // PAGE, rest % PAGE].any()
