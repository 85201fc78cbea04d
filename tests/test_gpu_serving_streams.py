"""The serving calls on a busy stream that is not the current one: what each gives there is what it gives on the current one."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import paged as OP
from oracle import paged4 as O4
from tests.test_gpu_paged import D, _bits, _f64, torch_cuda  # noqa: F401

pytestmark = pytest.mark.gpu

LAYERS, HQ, HK, SEQS, PAGE = 2, 4, 2, 3, 16


class Program:
    """A cache whose pages are given out, and rounds of its calls; every tensor of a round is made anew."""

    def __init__(self, bits):
        import torch
        from paper_2603_00188_amd import paged as P
        self.P, self.bits = P, bits
        self.cache = P.PagedCache.alloc(LAYERS, HQ, HK, SEQS, 200, page_size=PAGE, bits=bits, n_pages=12)
        self.pages = P.FreePages.of(self.cache)
        self.rope = P.Rope(1e4)
        self.kept = []

    def rows(self, gen, n, heads):
        import torch
        return torch.randn((LAYERS, n, heads, D), generator=gen, device="cuda").to(torch.bfloat16)

    def round(self, new, lens, seed, stream=None, drop=True):
        """Growing, append, attention, reading back, release: the outputs, all on `stream`."""
        import torch
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        b = self.P.NewTokens(np.concatenate([[0], np.cumsum(new)]))
        q, k, v = (self.rows(gen, b.total, h) for h in (HQ, HK, HK))
        pos = torch.arange(b.total, dtype=torch.int32, device="cuda").view(1, -1)
        lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        slots = torch.empty(b.total, dtype=torch.int32, device="cuda")
        if not drop:
            self.kept += [b, q, k, v, pos, lens, slots]
        torch.cuda.current_stream().synchronize()  # (the inputs are there; the other stream may be busy)
        self.P.paged_grow(self.cache, self.pages, b, slots=slots, stream=stream)
        qr = self.P.paged_append(self.cache, b, q, k, v, positions=pos, rope=self.rope, stream=stream)
        del q, k, v, pos
        out = self.P.paged_attention(self.cache, b, qr, stream=stream)
        got = self.P.paged_read(self.cache, b, stream=stream)
        self.P.paged_release(self.cache, self.pages, lens, stream=stream)
        return [slots, qr, out, *got]

    def state(self):
        n = int(self.pages.n_free)
        return [t.clone() for t in (*self.cache.tensors, self.pages.held, self.pages.n_free, self.pages.pages[:n])]


# new tokens and what a release keeps: two sequences are parked in the second round for want of pages
ROUNDS = [((60, 30, 17), (-1, 20, -1)), ((20, 90, 100), (70, -1, 0)), ((5, 1, 40), (-1, 0, -1))]


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("how", ["stream", "handle"])
def test_rounds_on_another_stream(torch_cuda, bits, how):
    import torch
    plain, f = Program(bits), Program(bits)
    want = [[t.clone() for t in plain.round(*r, seed=i)] + plain.state() for i, r in enumerate(ROUNDS)]
    torch.cuda.synchronize()
    # the rows are the appended ones, and there are parked sequences among those of the second round
    rows = want[0][3:5]
    assert all(bool((x != 0).any(-1).all()) for x in rows) and want[1][8].min() < 0
    busy = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for i, r in enumerate(ROUNDS):
        with torch.cuda.stream(side):
            for _ in range(10):
                torch.mm(busy, busy)
        got.append(f.round(*r, seed=i, stream=side if how == "stream" else side.cuda_stream, drop=how == "stream"))
        junk = [torch.full((LAYERS, 200, HQ, D), 0.5, device="cuda", dtype=torch.bfloat16) for _ in range(8)]
        assert len(junk) == 8
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for x, y in zip(g, w[:5]):
            assert torch.equal(x, y)
    for x, y in zip(f.state(), want[-1][5:]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [4, 16])
def test_rows_read_back_are_the_stored_ones(torch_cuda, bits):
    """On a busy stream too, by the oracle: each token's row, not another's."""
    import torch
    f = Program(bits)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    new = [60, 30, 17]
    b = f.P.NewTokens(np.concatenate([[0], np.cumsum(new)]))
    f.P.paged_grow(f.cache, f.pages, b)
    k, v = f.rows(gen, b.total, HK), f.rows(gen, b.total, HK)
    busy = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(10):
            torch.mm(busy, busy)
    f.P.paged_append(f.cache, b, None, k, v, stream=side)
    got = f.P.paged_read(f.cache, b, stream=side)
    torch.cuda.synchronize()
    table = f.cache.page_table.cpu().numpy()
    places = OP.new_places(table, new, b.h, PAGE, 12, 200)
    assert len(set(places)) == b.total and None not in places
    for x, src, pool in zip(got, (k, v), (f.cache.k, f.cache.v)):
        want = _f64(src) if bits == 16 else O4.decode(*O4.encode(_f64(src), "bf16"))
        assert np.array_equal(_f64(x), want) and len(np.unique(want.reshape(-1, D), axis=0)) == LAYERS * b.total * HK
        if bits == 16:
            flat = _bits(pool).reshape(LAYERS, HK, -1, D)
            assert np.array_equal(flat[:, :, places].transpose(0, 2, 1, 3), _bits(src))
