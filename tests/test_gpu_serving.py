"""Growing and releasing pages, drafted tokens, and a serving loop of all calls on the GPU, against oracle/serving.py and
the 64-bit oracles.

Everything that growing, releasing and verifying give is whole numbers, compared for equality.  A drafted token's
acceptance is decided exactly; the next token by 64-bit sums, which may put a number within about 10^-13 of a border on its
other side: the random numbers here are multiples of 2^-24.
"""
from __future__ import annotations

import numpy as np
import pytest

from oracle import paged as OP
from oracle import paged4 as O4
from oracle import serving as OS
from tests import test_gpu_paged as T
from tests.test_gpu_paged import D, _f64, _log, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# Pages
# ---------------------------------------------------------------------------

class Pages:
    """A small cache whose pages are given out, beside the oracle's."""

    def __init__(self, seqs, page, n_pages, max_len, seed=0, shuffled=True):
        import torch
        from paper_2603_00188_amd import paged as P
        self.P, self.page, self.n_pages = P, page, n_pages
        self.cache = P.PagedCache.alloc(1, 1, 1, seqs, max_len, page_size=page, bits=4, n_pages=n_pages)
        self.pages = P.FreePages.of(self.cache)
        order = np.random.default_rng(seed).permutation(n_pages) if shuffled else np.arange(n_pages)[::-1]
        self.pages.pages.copy_(torch.from_numpy(order.astype(np.int32)))
        self.o = OS.Pool(self.cache.page_table.tolist(), [0] * seqs, [0] * seqs, order, page, max_len)

    def grow(self, new, slots=True):
        import torch
        b = self.P.NewTokens(np.concatenate([[0], np.cumsum(new)]))
        buf = torch.full((b.total + 64,), -7, dtype=torch.int32, device="cuda")
        got = buf[32:32 + b.total]
        self.P.paged_grow(self.cache, self.pages, b, slots=got if slots else None)
        want = self.o.grow(list(new))
        assert (buf[:32] == -7).all() and (buf[32 + b.total:] == -7).all()
        if slots:
            assert got.tolist() == want
        self.same()
        return want

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


@pytest.mark.parametrize("seqs,page,n_pages,max_len,most", [
    (1, 16, 3, 40, 25), (3, 16, 40, 300, 100), (64, 16, 500, 400, 90), (64, 256, 30, 2000, 300), (1000, 16, 3000, 160, 60),
    (1023, 32, 400, 90, 20), (1024, 16, 5000, 300, 40), (1025, 16, 700, 100, 3), (2500, 16, 9000, 256, 70),
    (40, 16, 65537, 20000, 2000), (1500, 16, 70000, 3000, 700)])
def test_pages(torch_cuda, seqs, page, n_pages, max_len, most):
    """Rounds of growing, ending, cutting and resuming, with enough pages and with too few."""
    _log(f"pages: {seqs} sequences, {n_pages} pages of {page}")
    f, rng = Pages(seqs, page, n_pages, max_len, seed=seqs), np.random.default_rng(seqs)
    for turn in range(8):
        new = rng.integers(0, most + 1, seqs)
        new[rng.random(seqs) < 0.3] = 0
        f.grow(new.tolist(), slots=turn != 3)
        lens = np.array([x if x >= 0 else ~x for x in f.o.lens])
        keep = np.where(rng.random(seqs) < 0.4, 0, lens - rng.integers(0, 20, seqs).clip(max=lens))
        keep = np.where(rng.random(seqs) < 0.4, -1, keep)  # (some stay as they are, parked ones too)
        if turn % 3 == 2:
            f.release()
        else:
            f.release((keep + (turn == 4) * (keep > 0) * 1000).tolist())
    f.release([0] * seqs)
    assert sorted(f.o.free) == list(range(n_pages)) and not any(f.o.held)


def test_growing_again_takes_the_same_pages(torch_cuda):
    f = Pages(100, 16, 2000, 1000)
    new = np.random.default_rng(3).integers(0, 300, 100).tolist()
    f.grow(new)
    f.grow([5] * 100)
    table, free = f.cache.page_table.clone(), f.pages.pages[:int(f.pages.n_free)].clone()
    f.release(new)
    f.grow([5] * 100)
    assert (f.cache.page_table == table).all() and (f.pages.pages[:len(free)] == free).all()


@pytest.mark.parametrize("total", [4095, 4096, 4097, 70000])
def test_slots_of_many_tokens(torch_cuda, total):
    """Around the number of places that the growing work-group writes itself."""
    f = Pages(7, 16, 5000, 70000)
    cut = np.sort(np.random.default_rng(total).integers(0, total + 1, 6))
    f.grow(np.diff(np.concatenate([[0], cut, [total]])).tolist())


@pytest.mark.parametrize("most", [50, 5000])
def test_more_new_tokens_than_a_sequence_may_have(torch_cuda, most):
    """By itself more than max_len: parked as any other that does not fit, the others are served."""
    f = Pages(5, 16, 40, 48)
    f.grow([3, most, 0, 48, 49])
    assert f.o.lens == [3, ~0, 0, 48, ~0]
    f.release([3, 0, 0, 48, 0])
    f.grow([1, 48, most, 0, most])


def test_slots_are_where_rows_go(torch_cuda):
    """The place that an append writes a token's row to."""
    import torch
    from paper_2603_00188_amd import paged as P
    cache = P.PagedCache.alloc(1, 2, 2, 3, 200, page_size=16, n_pages=20)
    pages, slots = P.FreePages.of(cache), torch.empty(70, dtype=torch.int32, device="cuda")
    for cu in ([0, 40, 40, 70], [0, 1, 38, 70]):
        b = P.NewTokens(cu)
        P.paged_grow(cache, pages, b, slots=slots)
        x = torch.randn((1, 70, 2, D), device="cuda").to(torch.bfloat16)
        P.paged_append(cache, b, None, x, x)
        assert torch.equal(cache.k.view(2, -1, D)[:, slots.long()], x[0].transpose(0, 1))


def test_strange_states(torch_cuda):
    """Numbers that no call leaves behind: cut to what there is, nothing else written."""
    import torch
    f = Pages(4, 16, 10, 64)
    f.grow([20, 3, 0, 64])
    keep = f.cache.k.clone()
    f.pages.n_free.fill_(2 ** 31 - 1)
    f.cache.seq_lens.copy_(torch.tensor([2 ** 31 - 1, -2 ** 31, 5, 64], dtype=torch.int32))
    f.pages.held.copy_(torch.tensor([2 ** 31 - 1, -5, 0, 4], dtype=torch.int32))
    b = f.P.NewTokens([0, 1, 2, 3, 3])
    s = torch.empty(3, dtype=torch.int32, device="cuda")
    f.P.paged_grow(f.cache, f.pages, b, slots=s)
    torch.cuda.synchronize()
    assert f.cache.seq_lens.tolist() == [~64, -2 ** 31, 6, 64] and f.pages.held.tolist()[2:] == [1, 4]
    assert s.tolist()[:2] == [-1, -1] and f.pages.n_free.tolist() == [9]
    f.pages.n_free.fill_(10)  # a full list: what comes back has no room
    f.P.paged_release(f.cache, f.pages, torch.zeros(4, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert f.pages.n_free.tolist() == [10] and f.cache.seq_lens.tolist() == [0, 0, 0, 0]
    assert torch.equal(f.cache.k, keep)


def test_parked_sequences_are_idle(torch_cuda):
    """A parked sequence's rows stay, its new tokens' outputs are 0, and it goes on where it was once it is back."""
    import torch
    from paper_2603_00188_amd import paged as P
    for bits in (16, 4):
        cache = P.PagedCache.alloc(1, 4, 2, 2, 100, page_size=16, bits=bits, n_pages=4)
        pages, gen = P.FreePages.of(cache), torch.Generator(device="cuda")
        rows = lambda n, h: torch.randn((1, n, h, D), generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
        b = P.NewTokens([0, 30, 60])
        P.paged_grow(cache, pages, b)
        P.paged_append(cache, b, None, rows(60, 2), rows(60, 2))
        held = cache.k.clone()
        b = P.NewTokens([0, 3, 5])
        P.paged_grow(cache, pages, b)  # 33 and 32 tokens: no page is left for the first
        assert cache.seq_lens.tolist() == [~30, 32]
        q = rows(5, 4)
        out = P.paged_attention(cache, b, P.paged_append(cache, b, q, rows(5, 2), rows(5, 2)))
        assert not out[:, :3].any() and out[:, 3:].any()
        first = cache.page_table[0, :2].long()
        assert torch.equal(cache.k[:, :, first], held[:, :, first])
        P.paged_release(cache, pages, torch.tensor([30, 0], dtype=torch.int32, device="cuda"))
        P.paged_grow(cache, pages, b)
        assert cache.seq_lens.tolist() == [33, 2]
        out = P.paged_attention(cache, b, P.paged_append(cache, b, q, rows(5, 2), rows(5, 2)))
        assert out[:, :3].any() and torch.equal(cache.k[:, :, first], held[:, :, first]) is False


# ---------------------------------------------------------------------------
# Drafted tokens
# ---------------------------------------------------------------------------

def _drafts(counts, vocab, dtype="fp32", draft="near", seed=0, sharp=3.0):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    n, dt = sum(counts), {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
    logits = torch.randn((n, vocab), generator=gen, device="cuda") * sharp
    p = torch.softmax(logits, -1)
    q = torch.softmax(logits + torch.randn((n, vocab), generator=gen, device="cuda"), -1) if draft != "same" else p.clone()
    x = torch.multinomial(q, 1, generator=gen).view(-1).to(torch.int32)
    u = torch.rand(n, generator=gen, device="cuda")
    r = torch.rand(len(counts), generator=gen, device="cuda")
    return [p.to(dt), None if draft == "token" else q.to(dt), x, u, r]


def _verify(counts, p, q, x, u, r, **kw):
    import torch
    from paper_2603_00188_amd import paged as P
    b = P.NewTokens(np.concatenate([[0], np.cumsum(counts)]))
    out = torch.full((b.total + 64,), -7, dtype=torch.int32, device="cuda")
    n_out = torch.full((len(counts) + 64,), -7, dtype=torch.int32, device="cuda")
    ws = P.verify_workspace(b, p.shape[1])
    big = torch.full((ws.numel() + 512,), 0xAB, dtype=torch.uint8, device="cuda")
    P.verify_drafts(b, p, x, u, r, draft=q, out=out[32:32 + b.total], n_out=n_out[32:32 + len(counts)], workspace=big[:ws.numel()], **kw)
    torch.cuda.synchronize()
    assert (out[:32] == -7).all() and (out[32 + b.total:] == -7).all() and (n_out[:32] == -7).all()
    assert (n_out[32 + len(counts):] == -7).all() and (big[ws.numel():] == 0xAB).all()
    return out[32:32 + b.total].tolist(), n_out[32:32 + len(counts)].tolist()


def _check(counts, p, q, x, u, r, seen=None, **kw):
    """Against the oracle; returns the numbers of tokens."""
    out, n_out = _verify(counts, p, q, x, u, r, **kw)
    rows = lambda t, a, b: None if t is None else t[a:b].double().cpu().numpy()  # noqa: E731
    at = 0
    for s, n in enumerate(counts):
        if n == 0:
            assert n_out[s] == 0
            continue
        want = OS.verify(rows(p, at, at + n), rows(q, at, at + n), x[at:at + n].tolist(), u[at:at + n].tolist(), float(r[s]))
        assert n_out[s] == len(want), (s, n_out[s], want)
        assert out[at:at + n] == want + [-1] * (n - len(want)), s
        at += n
    return n_out


@pytest.mark.parametrize("counts,vocab,dtype,draft", [
    ((1,), 1, "fp32", "near"), ((2, 1), 3, "fp32", "token"), ((5,) * 30, 1000, "fp32", "near"), ((5,) * 30, 1000, "bf16", "near"),
    ((6, 0, 3, 1, 0, 8) * 8, 777, "fp16", "near"), ((4,) * 20, 1023, "fp32", "token"), ((4,) * 20, 1025, "bf16", "token"),
    ((3, 5), 50257, "fp32", "near"), ((2,) * 6, 8191, "fp16", "token"), ((9, 2) * 5, 9000, "fp32", "near"),
    ((300, 5, 520), 64, "fp32", "same"), ((2, 3, 1), 32769, "bf16", "near")])
def test_drafts(torch_cuda, counts, vocab, dtype, draft):
    _log(f"drafts: {len(counts)} sequences, vocabulary {vocab} {dtype} {draft}")
    n = _check(counts, *_drafts(counts, vocab, dtype, draft, seed=vocab))
    _log(f"tokens per sequence {np.mean(n):.2f}")


def test_drafts_of_the_target_itself(torch_cuda):
    """p = q: all accepted (u < 1), but for entries that fp32 holds as 0."""
    counts = (7,) * 20
    assert set(_check(counts, *_drafts(counts, 500, "fp32", "same"))) == {7}


@pytest.mark.parametrize("vocab", [1000, 5000, 20000])
def test_borders(torch_cuda, vocab):
    """Numbers that fall on the borders between tokens: sums of equal powers of two are exact in any order."""
    import torch
    counts = (1,) * 64
    step = 1 << (vocab - 1).bit_length()
    p = torch.zeros((64, vocab), device="cuda")
    p[:, :] = 1.0 / step
    r = torch.arange(64, device="cuda", dtype=torch.float32) / 64
    q, x, u = None, torch.zeros(64, dtype=torch.int32, device="cuda"), torch.zeros(64, device="cuda")
    _check(counts, p, q, x, u, r)
    p[:, ::3] = 0
    _check(counts, p, q, x, u, r)
    p[:, : vocab // 2] = 0
    p[:, vocab - 40:] = 0
    _check(counts, p, q, x, u, r)
    # acceptance exactly at its border is a refusal, the next number below is none
    counts = (2, 2)
    p = torch.zeros((4, vocab), device="cuda")
    q = torch.zeros((4, vocab), device="cuda")
    p[:, 5], p[:, vocab - 1], q[:, 5], q[:, 6] = 0.375, 0.625, 0.75, 0.25
    x = torch.full((4,), 5, dtype=torch.int32, device="cuda")
    u = torch.tensor([0.5, 0, np.nextafter(np.float32(0.5), np.float32(0)), 0], device="cuda", dtype=torch.float32)
    assert _check(counts, p, q, x, u, torch.tensor([0.0, 0.0], device="cuda")) == [1, 2]


def test_strange_probabilities(torch_cuda):
    """Rows without any weight, a rest of nothing, entries that are not finite or negative, tokens that are none, numbers
    outside [0, 1)."""
    import torch
    nan, inf = float("nan"), float("inf")
    for vocab in (9, 3000):
        counts = (2,) * 12
        p, q, x, u, r = _drafts(counts, vocab, seed=vocab)
        u[:] = 1.0
        p[0] = 0
        q[2] = p[2]                      # nothing is left over where u is 1 and p = q: p itself decides
        p[4, 3], p[4, 4], p[4, 5] = nan, inf, -1.0
        q[6, 1], q[6, 2], q[6, 3] = nan, -inf, inf
        x[8], x[10], x[12] = -1, vocab, 2 ** 31 - 1
        u[14], u[16] = nan, -1.0
        r[9], r[10], r[11] = 1.0, 2.0, 0.0
        p[20] = 0
        p[22, :] = nan
        q[18] = 10.0                     # nothing left over
        _check(counts, p, q, x, u, r)
        p[:, :] = 0
        assert _check(counts, p, None, x, u, r) is not None
        out, _ = _verify((1,) * 3, torch.full((3, vocab), nan, device="cuda"), None, x[:3], u[:3], r[:3])
        assert out == [-1] * 3


def test_rows_of_any_stride(torch_cuda):
    """Rows that begin at any entry: slices of wider ones."""
    import torch
    for dtype in ("fp32", "bf16"):
        counts = (3, 4, 1)
        p, q, x, u, r = _drafts(counts, 4099, dtype, seed=5)
        want = _verify(counts, p, q, x, u, r)
        wide = torch.full((8, 9001), float("nan"), dtype=p.dtype, device="cuda")
        wide[:, 1:4100], wide[:, 4801:8900] = p, q
        assert _verify(counts, wide[:, 1:4100], wide[:, 4801:8900], x, u, r) == want
        _check(counts, wide[:, 1:4100], wide[:, 4801:8900], x, u, r)


def test_lengths_go_back(torch_cuda):
    """And parked sequences stay as they are."""
    import torch
    from paper_2603_00188_amd import paged as P
    counts = (4, 3, 0, 5, 2)
    cache = P.PagedCache.alloc(1, 1, 1, 5, 100, page_size=16)
    cache.seq_lens.copy_(torch.tensor([40, ~7, 9, 5, 1], dtype=torch.int32))
    p, q, x, u, r = _drafts(counts, 300, seed=2)
    plain = _verify(counts, p, q, x, u, r)
    out, n = _verify(counts, p, q, x, u, r, cache=cache)
    assert n == [plain[1][0], 0, 0, plain[1][3], plain[1][4]] and out[4:7] == [-1] * 3 and out[:4] == plain[0][:4]
    assert cache.seq_lens.tolist() == [40 - 4 + n[0], ~7, 9, 5 - 5 + n[3], max(1 - 2 + n[4], 0)]


def test_more_than_2_to_32_probabilities(torch_cuda):
    """Rows behind 2^32 entries."""
    import torch
    vocab, n = 1 << 22, 1030
    p = torch.zeros((n, vocab), dtype=torch.bfloat16, device="cuda")
    p[:, 7] = 0.25
    p[-2:, 7] = 0
    p[-2, vocab - 3], p[-1, vocab - 2], p[-1, 5] = 1.0, 0.5, 0.5
    x = torch.full((n,), 7, dtype=torch.int32, device="cuda")
    x[-2] = vocab - 3
    u = torch.full((n,), 0.2, device="cuda")
    out, n_out = _verify((n,), p, None, x, u, torch.tensor([0.5], device="cuda"))
    assert n_out == [n] and out == [7] * (n - 2) + [vocab - 3, vocab - 2]
    u[-2] = 1.0
    p[-2, 11] = 0.5
    out, n_out = _verify((n,), p, None, x, u, torch.tensor([0.5], device="cuda"))
    assert n_out == [n - 1] and out[-2:] == [11, -1]


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

def _round(P, cache, pages, batch, bufs, ws, vws, rope):
    """A program's step: room for the tokens, store them, attend, judge the drafts."""
    P.paged_grow(cache, pages, batch, slots=bufs["slots"])
    P.paged_append(cache, batch, bufs["q"], bufs["k"], bufs["v"], positions=bufs["pos"], rope=rope, q_out=bufs["q_out"])
    P.paged_attention(cache, batch, bufs["q_out"], out=bufs["out"], workspace=ws)
    P.verify_drafts(batch, bufs["p"], bufs["x"], bufs["u"], bufs["r"], draft=bufs["d"], cache=cache, out=bufs["tokens"],
                    n_out=bufs["n_out"], workspace=vws)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("graph", [False, True])
def test_serving_loop(torch_cuda, bits, graph):
    """Prompts, then rounds of drafted tokens, as an eager loop and captured: pages, rows and lengths as the oracles have
    them, the attention of every round against 64 bits."""
    import torch
    from paper_2603_00188_amd import paged as P
    seqs, hk, hq, vocab, page = 5, 2, 6, 400, 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(50)
    cache = P.PagedCache.alloc(2, hq, hk, seqs, 200, page_size=page, bits=bits, n_pages=40)
    pages, rope = P.FreePages.of(cache), P.Rope(1e4)
    o = OS.Pool(cache.page_table.tolist(), [0] * seqs, [0] * seqs, pages.pages.tolist(), page, 200)
    rows = lambda n, h: torch.randn((2, n, h, D), generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    prompt = [40, 17, 100, 1, 64]
    b = P.NewTokens(np.concatenate([[0], np.cumsum(prompt)]))
    P.paged_grow(cache, pages, b)
    P.paged_append(cache, b, None, rows(b.total, hk), rows(b.total, hk))
    o.grow(prompt)
    counts = [4, 1, 3, 4, 2]
    b = P.NewTokens(np.concatenate([[0], np.cumsum(counts)]))
    n = b.total
    bufs = dict(q=rows(n, hq), k=rows(n, hk), v=rows(n, hk), pos=torch.zeros((1, n), dtype=torch.int32, device="cuda"))
    bufs.update(q_out=torch.empty_like(bufs["q"]), out=torch.empty_like(bufs["q"]),
                tokens=torch.empty(n, dtype=torch.int32, device="cuda"), n_out=torch.empty(seqs, dtype=torch.int32, device="cuda"),
                slots=torch.empty(n, dtype=torch.int32, device="cuda"))
    for name, t in zip("pdxur", _drafts(counts, vocab, seed=1)):
        bufs[name] = t
    ws, vws = cache.workspace(b), P.verify_workspace(b, vocab)
    play = lambda: _round(P, cache, pages, b, bufs, ws, vws, rope)  # noqa: E731
    if graph:
        state = [t.clone() for t in (*cache.tensors, pages.pages, pages.n_free, pages.held)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            play()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            play()
        for t, was in zip((*cache.tensors, pages.pages, pages.n_free, pages.held), state):
            t.copy_(was)
        play = g.replay
    for turn in range(6):
        for name, h in (("q", hq), ("k", hk), ("v", hk)):
            bufs[name].copy_(rows(n, h))
        for name, t in zip("pdxur", _drafts(counts, vocab, seed=10 + turn)):
            bufs[name].copy_(t)
        start = list(o.lens)
        slots = o.grow(counts)
        bufs["pos"].copy_(torch.tensor([[start[s] + t for s in range(seqs) for t in range(counts[s])]], dtype=torch.int32))
        play()
        torch.cuda.synchronize()
        assert bufs["slots"].tolist() == slots and cache.page_table.tolist() == o.table
        f64 = _f64
        k, v = (f64(t) if bits == 16 else O4.decode(*O4.rows(t.cpu().numpy(), page)) for t in (cache.k, cache.v))
        u = 2.0 ** -8
        for layer in range(2):
            ref, weight, keys, dot = OP.attention(f64(bufs["q_out"][layer]), k[layer], v[layer], np.array(o.table), o.lens, b.h,
                                                  200, D ** -0.5, hq // hk)
            rel = u + 2 * 128 * 2.0 ** -24 * dot + 2.0 ** -22 * (1 + dot) + 2 * keys * 2.0 ** -24
            err = np.abs(f64(bufs["out"][layer]) - ref)
            assert (err <= u * np.abs(ref) + rel[..., None] * weight + 2.0 ** -25).all(), (turn, layer)
        at = 0
        for s, m in enumerate(counts):
            want = OS.verify(bufs["p"][at:at + m].double().cpu().numpy(), bufs["d"][at:at + m].double().cpu().numpy(),
                             bufs["x"][at:at + m].tolist(), bufs["u"][at:at + m].tolist(), float(bufs["r"][s]))
            assert bufs["tokens"][at:at + m].tolist() == want + [-1] * (m - len(want)) and int(bufs["n_out"][s]) == len(want)
            o.lens[s] -= m - len(want)
            at += m
        assert cache.seq_lens.tolist() == o.lens and pages.held.tolist() == o.held
        if turn == 3:  # one ends, the others give back what they hold too much
            lens = [-1, 0, -1, -1, -1]
            P.paged_release(cache, pages, torch.tensor(lens, dtype=torch.int32, device="cuda"))
            o.release(lens)
            assert pages.pages[:int(pages.n_free)].tolist() == o.free and cache.page_table.tolist() == o.table


def test_streams(torch_cuda):
    """Calls on a busy stream that is not the current one, whose tensors are dropped at once."""
    import torch
    from paper_2603_00188_amd import paged as P
    counts = (5, 4)
    p, q, x, u, r = _drafts(counts, 3000, seed=9)
    want = _verify(counts, p, q, x, u, r)
    f = Pages(2, 16, 20, 100)
    f.grow([30, 20])
    rows = P.paged_read(f.cache, P.NewTokens([0, 30, 50]))
    busy = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            for _ in range(10):
                torch.mm(busy, busy)
        args = [t.clone() for t in (p, x, u, r, q)] if stream is side else [p, x, u, r, q]
        batch = P.NewTokens([0, 5, 9])
        torch.cuda.synchronize() if stream is not side else torch.cuda.current_stream().synchronize()
        out, n_out = P.verify_drafts(batch if stream is not side else P.NewTokens([0, 5, 9]), args[0], args[1], args[2], args[3],
                                     draft=args[4], stream=stream)
        got = P.paged_read(f.cache, P.NewTokens([0, 30, 50]) if stream is side else (batch2 := P.NewTokens([0, 30, 50])), stream=stream)
        del args
        junk = [torch.full((9, 3000), 0.5, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert (out.tolist(), n_out.tolist()) == want and len(junk) == 8
        assert torch.equal(got[0], rows[0]) and torch.equal(got[1], rows[1])


def test_limits_of_the_calls(torch_cuda):
    """65535 sequences."""
    import torch
    from paper_2603_00188_amd import paged as P
    rng = np.random.default_rng(6)
    f = Pages(65535, 16, 100000, 64)
    f.grow(rng.integers(0, 34, 65535).tolist())
    f.grow(rng.integers(0, 3, 65535).tolist())
    f.release(rng.integers(-1, 20, 65535).tolist())
    f.release([0] * 65535)
    counts = rng.integers(0, 4, 65535)
    counts[-3:] = 2
    p, q, x, u, r = _drafts(counts.tolist(), 60, seed=4)
    out, n_out = _verify(counts.tolist(), p, q, x, u, r)
    cu = np.concatenate([[0], np.cumsum(counts)])
    for s in list(range(0, 65535, 997)) + [65532, 65533, 65534]:
        a, n = int(cu[s]), int(counts[s])
        if n == 0:
            assert n_out[s] == 0
            continue
        rows = [t[a:a + n].double().cpu().numpy() for t in (p, q)]
        want = OS.verify(*rows, x[a:a + n].tolist(), u[a:a + n].tolist(), float(r[s]))
        assert out[a:a + n] == want + [-1] * (n - len(want)) and n_out[s] == len(want)
    p = torch.zeros((2, 1 << 24), device="cuda")
    p[0, (1 << 24) - 1], p[1, (1 << 24) - 2] = 1.0, 1.0
    x = torch.tensor([(1 << 24) - 1, 0], dtype=torch.int32, device="cuda")
    z = torch.zeros(2, device="cuda")
    assert _verify((2,), p, None, x, z, z[:1]) == ([(1 << 24) - 1, (1 << 24) - 2], [2])
