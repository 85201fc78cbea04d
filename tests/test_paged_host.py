"""CPU tests of the paged cache: the cuts of an attention call, the refusals of
every entry point and of the binding, validation of tables and lengths, and the
64-bit oracle against closed forms."""
import ctypes
import os
import random
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import paged as OP
from paper_2603_00188_amd import paged as P
from paper_2603_00188_amd import stlite as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_00188_amd", "csrc")
FAKE = 0x100000  # never dereferenced: validation reads only the host mirror

needs_lib = pytest.mark.skipif(not os.path.exists(S.LIB_PATH), reason="libstlite.so not built")

# ---------------------------------------------------------------------------
# Cuts (csrc/paged_cuts.h, the code that the kernels compile)
# ---------------------------------------------------------------------------

# argv: units tokens shares min_share, then n and cached of each sequence.  Walks
# every share as the attention kernels do and every boundary as the joining launch
# does; prints the number of joined items, fails on a tile, an item or a slot out
# of place.
PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include <map>
#include <vector>
#include "paged_cuts.h"
using namespace stlite;
struct Item { int64_t start, keys; int32_t tiles; };
int main(int argc, char** argv) {
  const int64_t units = atoll(argv[1]);
  const int32_t tokens = atoi(argv[2]), shares = atoi(argv[3]), min_share = atoi(argv[4]), cost = atoi(argv[5]);
  std::vector<Item> items;
  int64_t at = 0;
  for (int64_t u = 0; u < units; ++u)
    for (int i = 6; i + 1 < argc; i += 2) {
      const int32_t n = atoi(argv[i]), cached = atoi(argv[i + 1]);
      int64_t base = at;
      for (int32_t k = 0; k < paged_items(n, tokens); ++k) {
        if (at != base + paged_prefix(k, cached, tokens, cost)) { printf("prefix of item %d\n", k); return 1; }
        const int64_t keys = paged_item_keys(k, n, cached, tokens);
        const int64_t seen = cached + (int64_t(k) * tokens + tokens < n ? int64_t(k) * tokens + tokens : n);
        if (keys < seen || keys < 1) { printf("item %d counts %lld keys, sees %lld\n", k, (long long)keys, (long long)seen); return 1; }
        if (paged_item_of(at - base, n, cached, tokens, cost) != k || paged_item_of(at - base + cost + keys - 1, n, cached, tokens, cost) != k) { printf("item_of %d\n", k); return 1; }
        at += cost;
        items.push_back({at, keys, int32_t((keys + kPagedTile - 1) / kPagedTile)});
        at += keys;
      }
      if (at - base != paged_range(n, cached, tokens, cost)) { printf("places of a sequence\n"); return 1; }
    }
  const int64_t total = at, share = paged_share(total, shares, min_share);
  if (share * shares < total) { printf("shares do not cover the range\n"); return 1; }
  std::map<int64_t, size_t> slots;                 // slot -> item
  std::vector<int32_t> next(items.size(), 0);      // tiles covered so far
  std::vector<int> parts(items.size(), 0), whole(items.size(), 0);
  for (int64_t w = 0; w < shares; ++w) {
    int64_t x = w * share;
    const int64_t y = x + share < total ? x + share : total;
    size_t i = 0;
    if (x < y) while (items[i].start + items[i].keys <= x) ++i;
    for (; x < y && items[i].start < y; ++i) {
      const PagedPart p = paged_part(x, y, items[i].start, items[i].keys);
      if (p.t0 != next[i] || p.t1 < p.t0) { printf("share %lld item %zu: tiles %d .. %d, %d covered\n", (long long)w, i, p.t0, p.t1, next[i]); return 1; }
      next[i] = p.t1;
      ++parts[i];
      if (p.whole) ++whole[i];
      else {
        const int64_t slot = paged_slot(w, share, items[i].start);
        if (slot < 0 || slot >= 2 * int64_t(shares) || slots.count(slot)) { printf("slot %lld twice\n", (long long)slot); return 1; }
        slots[slot] = i;
      }
      x = p.end;
    }
  }
  std::vector<int> joined(items.size(), 0);
  for (int64_t w = 0; w + 1 < shares; ++w) {
    const int64_t cut = (w + 1) * share;
    if (cut >= total) continue;
    size_t i = 0;
    while (items[i].start + items[i].keys <= cut) ++i;
    if (items[i].start >= cut || items[i].start / share != w) continue;
    ++joined[i];
    const int64_t w1 = (items[i].start + items[i].keys - 1) / share;
    for (int64_t k = w; k <= w1; ++k) {
      const auto at = slots.find(paged_slot(k, share, items[i].start));
      if (at == slots.end() || at->second != i) { printf("item %zu: share %lld left no part\n", i, (long long)k); return 1; }
    }
    if (w1 - w + 1 != parts[i]) { printf("item %zu: %d parts\n", i, parts[i]); return 1; }
  }
  int n_joined = 0;
  for (size_t i = 0; i < items.size(); ++i) {
    if (next[i] != items[i].tiles) { printf("item %zu: %d of %d tiles\n", i, next[i], items[i].tiles); return 1; }
    if (whole[i] + joined[i] != 1 || (whole[i] && parts[i] != 1)) { printf("item %zu: written %d times\n", i, whole[i] + joined[i]); return 1; }
    n_joined += joined[i];
  }
  printf("%d\n", n_joined);
  return 0;
}
"""


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("paged_cuts")
    src, exe = str(d / "cuts.cpp"), str(d / "cuts")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", f"-I{CSRC}", src, "-o", exe], check=True)

    def run(units, tokens, shares, min_share, seqs, cost=0):
        args = [str(x) for s in seqs for x in s]
        r = subprocess.run([exe, str(units), str(tokens), str(shares), str(min_share), str(cost), *args], capture_output=True, text=True)
        assert r.returncode == 0, (units, tokens, shares, min_share, seqs, r.stdout)
        return int(r.stdout)
    return run


@pytest.mark.parametrize("units,tokens,shares,min_share,seqs", [
    (1, 1, 512, 64, [(1, 0)]), (1, 1, 512, 64, [(1, 677)]), (4, 1, 512, 64, [(1, 677)]), (112, 1, 512, 64, [(1, 30104)]),
    (3, 1, 512, 64, [(1, -1), (0, 50), (1, 0), (1, 63), (1, 64), (0, 0)]), (1, 1, 1, 64, [(1, 5)]),
    (4, 36, 256, 256, [(3136, 30105)]), (2, 32, 256, 256, [(131, 0), (2999, 0), (1, 0), (32, 0), (33, 0)]),
    (5, 18, 512, 256, [(5, -3), (5, 2), (5, 4000), (0, 9)]), (2, 1, 512, 256, [(7, 100)]), (1, 128, 512, 256, [(129, 1)]),
])
@pytest.mark.parametrize("cost", [0, 1, 32, 384])
def test_every_tile_and_output_once(cuts, units, tokens, shares, min_share, seqs, cost):
    cuts(units, tokens, shares, min_share, seqs, cost)


def test_cuts_of_random_batches(cuts):
    r = random.Random(11)
    joined = 0
    for _ in range(150):
        tokens = r.choice([1, 1, 2, 18, 32, 36, 128, 256])
        most = 1 if tokens == 1 else r.choice([3, 40, 700])
        seqs = [(r.randint(0, most), r.choice([-1, 0, 0, 1, 63, r.randint(0, 3000)])) for _ in range(r.randint(1, 9))]
        if not any(n for n, _ in seqs):
            seqs[0] = (1, 10)
        joined += cuts(r.randint(1, 6), tokens, r.choice([1, 2, 3, 17, 256, 512]), r.choice([1, 63, 64, 256]), seqs, r.choice([0, 0, 17, 64, 500]))
    assert joined > 100


# ---------------------------------------------------------------------------
# Refusals
# ---------------------------------------------------------------------------


class Fake:
    """A _CPaged whose host mirror is real and whose device pointers are fake."""

    def __init__(self, counts=(0, 1, 3), **kw):
        self.cu = np.asarray(counts, np.int32)
        f = dict(n_layers=2, n_q_heads=28, n_kv_heads=4, head_dim=128, dtype=0, page_size=16, n_pages=20,
                 n_seqs=len(self.cu) - 1, max_pages=5, max_len=80, total_new=int(self.cu[-1]), k=FAKE, v=FAKE,
                 page_table=FAKE, seq_lens=FAKE, cu_new=FAKE, h_cu_new=self.cu.ctypes.data)
        f.update(kw)
        self.c = S._CPaged(**f)

    @property
    def ref(self):
        return ctypes.byref(self.c)


def _err():
    return S.load().stlite_last_error().decode()


BAD = [
    (dict(head_dim=64), S.ERR_UNSUPPORTED, "head_dim"), (dict(n_q_heads=30), S.ERR_INVALID_ARG, "multiple"),
    (dict(n_q_heads=0), S.ERR_INVALID_ARG, ">= 1"), (dict(n_layers=0), S.ERR_INVALID_ARG, ">= 1"),
    (dict(n_q_heads=129 * 4), S.ERR_UNSUPPORTED, "per kv head"), (dict(dtype=2), S.ERR_INVALID_ARG, "dtype"),
    (dict(page_size=8), S.ERR_UNSUPPORTED, "page_size"), (dict(page_size=48), S.ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=512), S.ERR_UNSUPPORTED, "page_size"), (dict(n_pages=0), S.ERR_INVALID_ARG, "n_pages"),
    (dict(n_pages=2 ** 27), S.ERR_UNSUPPORTED, "2^31"), (dict(n_seqs=0), S.ERR_INVALID_ARG, "n_seqs"),
    (dict(n_seqs=65536), S.ERR_UNSUPPORTED, "65535"), (dict(n_layers=20000), S.ERR_UNSUPPORTED, "65535"),
    (dict(max_pages=0), S.ERR_INVALID_ARG, "max_pages"), (dict(max_len=0), S.ERR_INVALID_ARG, "max_len"),
    (dict(max_len=81), S.ERR_INVALID_ARG, "max_len"),
    (dict(max_pages=2 ** 25, max_len=2 ** 28 + 1), S.ERR_UNSUPPORTED, "2^28"),
    (dict(k=None), S.ERR_INVALID_ARG, "non-NULL"), (dict(v=None), S.ERR_INVALID_ARG, "non-NULL"),
    (dict(page_table=None), S.ERR_INVALID_ARG, "non-NULL"), (dict(k=FAKE + 8), S.ERR_INVALID_ARG, "aligned"),
]
BAD_BATCH = [
    (dict(seq_lens=None), S.ERR_INVALID_ARG, "non-NULL"), (dict(cu_new=None), S.ERR_INVALID_ARG, "non-NULL"),
    (dict(h_cu_new=None), S.ERR_INVALID_ARG, "non-NULL"), (dict(total_new=4), S.ERR_INVALID_ARG, "total_new"),
    (dict(max_len=1), S.ERR_INVALID_ARG, "new tokens"),
]


@needs_lib
@pytest.mark.parametrize("change, status, text", BAD + BAD_BATCH)
def test_cache_rejections(change, status, text):
    """Every call refuses a malformed cache with nothing enqueued."""
    lib, f = S.load(), Fake(**change)
    n = ctypes.c_size_t(7)
    row = ctypes.byref(S._CRows(FAKE, 36 * 128, 3 * 36 * 128))
    calls = [lambda: lib.stlite_paged_validate(f.ref, None, None),
             lambda: lib.stlite_paged_workspace_size(f.ref, ctypes.byref(n)),
             lambda: lib.stlite_paged_append(f.ref, None, None, row, row, row, None, None, 0.0, FAKE + 4096, None),
             lambda: lib.stlite_paged_attention(f.ref, FAKE, 1.0, FAKE + 4096, FAKE, 1 << 40, None)]
    for call in calls:
        assert call() == status
        assert text in _err()
    assert n.value == 0


@needs_lib
@pytest.mark.parametrize("cu", [(1, 2, 3), (0, 2, 1), (0, 81, 82)])
def test_new_token_counts_rejected(cu):
    f = Fake(counts=cu)
    assert S.load().stlite_paged_validate(f.ref, None, None) == S.ERR_INVALID_ARG


@needs_lib
def test_null_arguments_rejected():
    lib, f = S.load(), Fake()
    n = ctypes.c_size_t(0)
    assert lib.stlite_paged_validate(None, None, None) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_workspace_size(f.ref, None) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_workspace_size(None, ctypes.byref(n)) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_attention(None, FAKE, 1.0, FAKE, FAKE, 1, None) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_append(None, None, None, None, None, None, None, None, 0.0, None, None) == S.ERR_INVALID_ARG


@needs_lib
def test_attention_rejections():
    lib, f = S.load(), Fake()
    n = ctypes.c_size_t(0)
    assert lib.stlite_paged_workspace_size(f.ref, ctypes.byref(n)) == S.OK and n.value > 0 and n.value % 256 == 0
    call = lambda q=FAKE, scale=1.0, out=FAKE + 4096, ws=FAKE, nb=n.value: lib.stlite_paged_attention(  # noqa: E731
        f.ref, q, scale, out, ws, nb, None)
    for scale in (0.0, -1.0, float("nan"), float("inf"), 2.5e38):
        assert call(scale=scale) == S.ERR_INVALID_ARG and "scale" in _err()
    assert call(ws=None) == S.ERR_WORKSPACE
    assert call(nb=n.value - 1) == S.ERR_WORKSPACE
    assert call(ws=FAKE + 16) == S.ERR_WORKSPACE
    assert call(q=None) == S.ERR_INVALID_ARG and call(out=None) == S.ERR_INVALID_ARG
    assert call(out=FAKE) == S.ERR_INVALID_ARG and "alias" in _err()
    assert call(q=FAKE + 8) == S.ERR_INVALID_ARG and call(out=FAKE + 4104) == S.ERR_INVALID_ARG
    # no new token: nothing to do, whatever the buffers
    none = Fake(counts=(0, 0, 0))
    assert lib.stlite_paged_attention(none.ref, None, 1.0, None, None, 0, None) == S.OK
    assert lib.stlite_paged_workspace_size(none.ref, ctypes.byref(n)) == S.OK and n.value == 0


@needs_lib
def test_append_rejections():
    lib, f = S.load(), Fake()

    def call(rope=None, positions=None, q=(FAKE, 28 * 128), k=(FAKE, 4 * 128), v=(FAKE, 4 * 128), q_norm=None, k_norm=None,
             eps=1e-6, q_out=FAKE + 8192):
        rows = [None if r is None else ctypes.byref(S._CRows(r[0], r[1], r[2] if len(r) > 2 else 3 * r[1])) for r in (q, k, v)]
        return lib.stlite_paged_append(f.ref, None if rope is None else ctypes.byref(rope), positions, *rows, q_norm, k_norm,
                                       eps, q_out, None)

    def rope(theta=1e6, interleaved=0, n_axes=1, sections=(0, 0, 0), reserved=0):
        return S._CRope(theta, interleaved, n_axes, (ctypes.c_int32 * 3)(*sections), reserved)

    bad = S.ERR_INVALID_ARG
    assert call(rope=rope()) == bad and call(positions=FAKE) == bad
    for theta in (0.5, 0.0, -1.0, float("nan"), float("inf")):
        assert call(rope=rope(theta=theta), positions=FAKE) == bad and "theta" in _err()
    assert call(rope=rope(interleaved=2), positions=FAKE) == bad
    assert call(rope=rope(reserved=1), positions=FAKE) == bad
    assert call(rope=rope(n_axes=2), positions=FAKE) == bad and "n_axes" in _err()
    for sections in ((16, 24, 23), (16, 24, 25), (-1, 33, 32), (2 ** 31 - 1, 1, 0)):
        assert call(rope=rope(n_axes=3, sections=sections), positions=FAKE) == bad and "sections" in _err()
    assert call(k=None) == bad and call(v=None) == bad and call(k=(None, 512)) == bad
    assert call(q=None) == bad and call(q_out=None) == bad and call(q=(None, 28 * 128)) == bad
    assert call(k=(FAKE + 8, 512)) == bad and call(k=(FAKE, 516)) == bad and call(k=(FAKE, 504)) == bad
    assert call(q=(FAKE, 27 * 128)) == bad and call(v=(FAKE, 512, 4)) == bad and call(v=(FAKE, 512, -512)) == bad
    assert call(q_out=FAKE) == bad and "alias" in _err()
    assert call(q_out=FAKE + 8192 + 2) == bad and call(q_norm=FAKE + 2) == bad and call(k_norm=FAKE + 2) == bad
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(q_norm=FAKE, eps=eps) == bad and call(k_norm=FAKE, eps=eps) == bad and "eps" in _err()


@needs_lib
def test_compact_rejections():
    lib = S.load()

    def problem(n_layers=2, n_kv=4, lens=(50, 60)):
        cu = np.concatenate([[0], np.cumsum(lens)])
        return S.Problem(n_layers, 7 * n_kv, n_kv, 1, cu, np.zeros(len(lens) + 1), np.zeros((0, 3)), S.budgets(cu, 4, 5),
                         device="cpu")

    def call(p, f, k=FAKE, v=FAKE, kept=FAKE):
        return lib.stlite_paged_compact(p.ref, f.ref, k, v, kept, 0, None)

    bad = S.ERR_INVALID_ARG
    for change, status, text in BAD:
        assert call(problem(), Fake(**change)) == status and text in _err()
    assert call(problem(n_layers=3), Fake()) == bad and "layers" in _err()
    assert call(problem(n_kv=2), Fake()) == bad
    assert call(problem(lens=(50,)), Fake()) == bad
    assert call(problem(), Fake(max_len=47)) == bad and "keeps 48 rows" in _err()
    for name in ("k", "v", "kept"):
        assert call(problem(), Fake(), **{name: None}) == bad
    assert call(problem(), Fake(), k=FAKE + 2) == bad
    assert call(problem(), Fake(seq_lens=None)) == bad
    p = problem()
    p.c.window = 0
    assert call(p, Fake()) == bad and "window" in _err()


@needs_lib
def test_validate_tables_and_lengths():
    lib = S.load()
    f = Fake(counts=(0, 1, 3), page_size=16, n_pages=6, max_pages=3, max_len=40)

    def check(table, lens):
        t, n = np.asarray(table, np.int32), np.asarray(lens, np.int32)
        return lib.stlite_paged_validate(f.ref, t.ctypes.data, n.ctypes.data)

    good = [[0, 1, 2], [5, 4, -1]]
    assert check(good, [40, 32]) == S.OK
    assert check(good, [40, 33]) == S.ERR_INVALID_ARG and "entry 2 is -1" in _err()
    assert check([[0, 6, 2], [5, 4, 3]], [17, 2]) == S.ERR_INVALID_ARG and "outside [0, 6)" in _err()
    assert check([[0, 6, 2], [5, 4, 3]], [16, 2]) == S.OK  # entries behind the end are not looked at
    assert check(good, [41, 32]) == S.ERR_INVALID_ARG and check(good, [0, 32]) == S.ERR_INVALID_ARG
    assert check(good, [1, 1]) == S.ERR_INVALID_ARG and "2 new tokens" in _err()
    # a shared first page is fine, a shared page that is written to is not
    assert check([[0, 1, 2], [0, 4, 3]], [40, 32]) == S.OK
    assert check([[0, 1, 2], [0, 4, 3]], [16, 32]) == S.ERR_INVALID_ARG and "holds twice" in _err()
    assert check([[0, 1, 1], [3, 4, 3]], [40, 32]) == S.ERR_INVALID_ARG
    assert lib.stlite_paged_validate(f.ref, None, np.asarray([40, 32], np.int32).ctypes.data) == S.OK


@needs_lib
def test_workspace_does_not_depend_on_lengths_and_is_bounded():
    """One new token per sequence, any batch: at most 512 shares x two parts of 16
    heads; more: two parts of an item's rows for each share."""
    lib = S.load()
    n = ctypes.c_size_t(0)
    per = 130 * 4  # a row's maximum, sum and 128 sums
    for cu, rows, shares in (((0, 1, 2), 16, 512), ((0, 0, 1), 16, 512), ((0, 5, 6), 128, 512), ((0, 70, 71), 256, 256)):
        f = Fake(counts=cu, n_layers=28, max_pages=10000, n_pages=10000, max_len=150000)
        assert lib.stlite_paged_workspace_size(f.ref, ctypes.byref(n)) == S.OK
        assert 0 < n.value <= shares * 2 * rows * per + 3 * 256, cu
    tiny = Fake(counts=(0, 1), n_layers=1, n_q_heads=1, n_kv_heads=1, max_pages=1, max_len=16)
    assert lib.stlite_paged_workspace_size(tiny.ref, ctypes.byref(n)) == S.OK and n.value == 0


@needs_lib
def test_workspace_is_what_the_shares_leave():
    """Two parts of an item for each share, a row's maximum, sum and 128 sums in fp32: 512 shares of 16 or 32 heads with
    one token each, 256 of 256 rows with more, however few or many tokens or heads those are."""
    lib, n = S.load(), ctypes.c_size_t(0)
    for cu, heads, shares, rows in (((0, 1, 2), 4, 512, 16), ((0, 0, 1), 64, 512, 16), ((0, 1, 2), 80, 512, 32),
                                    ((0, 1, 2), 512, 512, 32), ((0, 2, 3), 4, 256, 256), ((0, 5, 6), 28, 256, 256),
                                    ((0, 70, 71), 28, 256, 256), ((0, 70, 70), 512, 256, 256)):
        f = Fake(counts=cu, n_layers=28, n_q_heads=heads, max_pages=10000, n_pages=10000, max_len=150000)
        assert lib.stlite_paged_workspace_size(f.ref, ctypes.byref(n)) == S.OK
        assert n.value == shares * 2 * rows * (1 + 1 + 128) * 4, (cu, heads)


# ---------------------------------------------------------------------------
# The binding
# ---------------------------------------------------------------------------


def _cache(**kw):
    return P.PagedCache.alloc(2, 8, 2, 3, 40, page_size=16, device="cpu", **kw)


def test_cache_layout():
    c = _cache(dtype=torch.float16)
    assert c.k.shape == (2, 2, 9, 16, 128) and c.max_pages == 3 and c.max_len == 40
    assert c.page_table.tolist() == [[0, 1, 2], [3, 4, 5], [6, 7, 8]]
    one = c.layer(1)
    assert one.n_layers == 1 and one.k.data_ptr() == c.k[1].data_ptr() and one.seq_lens is c.seq_lens
    with pytest.raises(ValueError):
        c.layer(2)


def test_copied_batches_have_their_own_addresses():
    import copy
    import pickle
    a = P.NewTokens([0, 2, 5], device="cpu")
    for b in (copy.copy(a), copy.deepcopy(a), pickle.loads(pickle.dumps(a))):
        assert b.h is not a.h and b.h.tolist() == [0, 2, 5] and b.d.tolist() == [0, 2, 5] and b.total == 5
        assert (b._h, b._d) == (b.h.ctypes.data, b.d.data_ptr()) and b._h != a._h and b._d != a._d


def test_binding_rejects_tensors():
    c = _cache()
    table, lens = c.page_table, c.seq_lens
    for k, v, t, n in ((c.k.float(), c.v, table, lens), (c.k, c.v.half(), table, lens), (c.k, c.v[:1], table, lens),
                       (c.k[..., :64], c.v[..., :64], table, lens), (c.k.transpose(0, 1), c.v.transpose(0, 1), table, lens),
                       (c.k, c.v, table.long(), lens), (c.k, c.v, table[0], lens), (c.k, c.v, table.t(), lens),
                       (c.k, c.v, table, lens[:2]), (c.k, c.v, table, lens.long())):
        with pytest.raises(ValueError):
            P.PagedCache(k, v, t, n, 8)
    b = P.NewTokens([0, 1, 1, 4], device="cpu")
    q = torch.zeros((2, 4, 8, 128), dtype=torch.bfloat16)
    kn = torch.zeros((2, 4, 2, 128), dtype=torch.bfloat16)
    for bad in (q.half(), q[:1], q[:, :3], q.transpose(1, 2), q.view(2, 4, 128, 8)):
        with pytest.raises(ValueError):
            P.paged_attention(c, b, bad)
    with pytest.raises(ValueError):
        P.paged_attention(c, b, q, out=q.float())
    for bad in (kn.half(), kn[:, :3], kn[..., :64], torch.zeros((2, 4, 128, 2), dtype=torch.bfloat16).transpose(2, 3)):
        with pytest.raises(ValueError):
            P.paged_append(c, b, q, bad, kn)
    pos = torch.zeros((1, 4), dtype=torch.int32)
    for kw in (dict(positions=pos), dict(rope=P.Rope()), dict(positions=pos.long(), rope=P.Rope()),
               dict(positions=pos, rope=P.Rope(sections=(16, 24, 24))), dict(q_norm=torch.zeros((2, 128))),
               dict(k_norm=torch.zeros(128, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            P.paged_append(c, b, q, kn, kn, **kw)
    for sections in ((64, 0), (16, 24, 23), (63,)):
        with pytest.raises(ValueError):
            P.Rope(sections=sections)
    with pytest.raises(ValueError):
        P.NewTokens([0], device="cpu")
    with pytest.raises(ValueError):  # nothing runs on the CPU
        P.paged_attention(c, b, q)


@needs_lib
def test_binding_raises_the_library_errors():
    c = _cache()
    with pytest.raises(ValueError):
        c.workspace_size(P.NewTokens([0, 1, 1], device="cpu"))  # another number of sequences
    with pytest.raises(S.StliteError) as e:
        c.workspace_size(P.NewTokens([0, 1, 0, 4], device="cpu"))
    assert e.value.status == S.ERR_INVALID_ARG
    b = P.NewTokens([0, 1, 1, 4], device="cpu")
    assert c.workspace_size(b) > 0
    c.validate(b, c.page_table.numpy(), [1, 0, 3])
    with pytest.raises(S.StliteError):
        c.validate(b, c.page_table.numpy(), [1, 0, 2])
    with pytest.raises(ValueError):
        c.validate(b, c.page_table.numpy()[:, :2], [1, 0, 3])


# ---------------------------------------------------------------------------
# The oracle
# ---------------------------------------------------------------------------


def test_oracle_rotation_closed_forms():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 128))
    assert np.array_equal(OP.rotate(x, [[0, 0, 0]], 1e4), x)
    for inter in (False, True):
        y = OP.rotate(x, [[5, 70000, -3]], 1e6, interleaved=inter)
        assert np.allclose((y * y).sum(-1), (x * x).sum(-1))
        a, b = (0, 1) if inter else (0, 64)  # pair 0 turns by the position itself
        want = (x[1, 0, a] + 1j * x[1, 0, b]) * np.exp(1j * 70000)
        assert np.allclose([y[1, 0, a], y[1, 0, b]], [want.real, want.imag])
        # relative positions: a dot product depends on the difference alone
        p, q = OP.rotate(x, [[7, 7, 7]], 1e4, interleaved=inter), OP.rotate(x[::-1], [[3, 3, 3]], 1e4, interleaved=inter)
        r, s = OP.rotate(x, [[107] * 3], 1e4, interleaved=inter), OP.rotate(x[::-1], [[103] * 3], 1e4, interleaved=inter)
        assert np.allclose((p * q).sum(-1), (r * s).sum(-1))
    # three axes: equal positions are one axis; each section goes by its own
    one = OP.rotate(x, [[4, 5, 6]], 1e4)
    assert np.allclose(OP.rotate(x, [[4, 5, 6]] * 3, 1e4, (16, 24, 24)), one)
    y = OP.rotate(x, [[4, 5, 6], [0, 0, 0], [0, 0, 0]], 1e4, (16, 24, 24))
    assert np.allclose(y[..., :16], one[..., :16]) and np.array_equal(y[..., 16:64], x[..., 16:64])


def test_oracle_norm_and_attention_closed_forms():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 128))
    y = OP.norm(x, np.ones(128), 0.0)
    assert np.allclose((y * y).mean(-1), 1) and np.allclose(OP.norm(3 * x, 2 * np.ones(128), 0.0), 2 * y)
    # zero queries: the mean of the visible rows, page by page; a bad page holds nothing
    k = rng.standard_normal((1, 4, 16, 128))
    v = rng.standard_normal((1, 4, 16, 128))
    table = np.array([[2, 0], [3, -1]], np.int32)
    q = np.zeros((3, 2, 128))
    out, weight, keys, _ = OP.attention(q, k, v, table, [18, 20], [0, 2, 3], 32, 1.0, 2)
    assert np.allclose(out[1, 0], np.concatenate([v[0, 2], v[0, 0, :2]]).mean(0))
    assert np.allclose(out[0, 1], np.concatenate([v[0, 2], v[0, 0, :1]]).mean(0))
    assert np.allclose(out[2, 0], v[0, 3].mean(0)) and keys[:, 0].tolist() == [17, 18, 16]
    # a sequence shorter than its new tokens: the first see nothing; a length past max_len is cut
    out, _, keys, _ = OP.attention(np.zeros((3, 1, 128)), k, v, table, [1, 99], [0, 2, 3], 16, 1.0, 1)
    assert not out[0].any() and np.allclose(out[1, 0], v[0, 2, 0]) and keys[:, 0].tolist() == [0, 1, 16]
    assert OP.new_places(table, [1, 99], [0, 2, 3], 16, 4, 16) == [None, 32, 63]


# ---------------------------------------------------------------------------
# Compaction: types and shapes, before anything is enqueued
# ---------------------------------------------------------------------------


def _compaction(dtype=torch.bfloat16, layers=2, hk=2, lens=(50, 60), max_len=40):
    cu = np.concatenate([[0], np.cumsum(lens)])
    p = S.Problem(layers, 4 * hk, hk, 1, cu, np.zeros(len(lens) + 1), np.zeros((0, 3)), S.budgets(cu, 1, 2), device="cpu")
    cache = P.PagedCache.alloc(2, 8, 2, 2, max_len, page_size=16, dtype=dtype, device="cpu")
    k = torch.zeros((layers * hk, sum(lens), 128), dtype=torch.bfloat16)
    return p, cache, k


@needs_lib
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_compaction_refuses_another_type(dtype):
    """Rows of one 16-bit type are not stored in a pool of the other; bit patterns carry no type."""
    p, cache, k = _compaction(dtype)
    kept = torch.zeros((4, p.total_budget), dtype=torch.int32)
    other = torch.float16 if dtype == torch.bfloat16 else torch.bfloat16
    for a, b in ((k.to(other), k.to(dtype)), (k.to(dtype), k.to(other)), (k.to(other), k.to(other))):
        with pytest.raises(ValueError, match="must be"):
            P.paged_compact(cache, p, a, b, kept)
    for a in (k.to(dtype), k.to(torch.int16), k.view(torch.uint16)):
        with pytest.raises(ValueError, match="run on a GPU"):  # nothing runs on the CPU
            P.paged_compact(cache, p, a, a, kept)


@needs_lib
def test_compaction_refuses_a_problem_of_another_device():
    """The kernel reads the problem's prefix sums: they lie where the cache does."""
    p, cache, k = _compaction()
    kept = torch.zeros((4, p.total_budget), dtype=torch.int32)
    p.d["cu_budget"] = p.d["cu_budget"].to("meta")
    for call in (lambda: P.paged_compact(cache, p, k, k, kept), lambda: P.check_compression(cache, p, k, k)):
        with pytest.raises(ValueError, match="problem is on meta"):
            call()


@needs_lib
def test_compression_refuses_its_cache_first(monkeypatch):
    """A cache that the pass cannot go into: refused with nothing enqueued."""
    def enqueued(*a, **kw):
        raise AssertionError("a stage was enqueued")
    for stage in ("stlite_score_window", "stlite_tsg_gate", "stlite_css_saliency", "stlite_select_topk"):
        monkeypatch.setattr(S, stage, enqueued)

    class Out:
        kept = torch.zeros((4, 55), dtype=torch.int32)
    for change, text in ((dict(dtype=torch.float16), "bf16"), (dict(layers=3), "layers"), (dict(hk=1), "kv heads"),
                         (dict(lens=(50,)), "sequences"), (dict(max_len=29), "max_len")):
        p, cache, k = _compaction(**change)
        with pytest.raises(ValueError, match=text):
            S.compress(p, k, k, k, Out(), stream=0, cache=cache)


# ---------------------------------------------------------------------------
# What the binding froze at construction
# ---------------------------------------------------------------------------


def test_frozen_fields_are_not_assigned():
    """The C structs hold addresses and sizes from construction: another tensor or size is refused, not ignored."""
    c = _cache()
    for name, other in (("k", c.k.clone()), ("v", c.v.clone()), ("page_table", c.page_table.clone()),
                        ("seq_lens", c.seq_lens + 1), ("max_len", 39), ("n_q_heads", 4), ("n_pages", 8), ("n_seqs", 2),
                        ("dtype", torch.float16)):
        with pytest.raises(AttributeError, match=name):
            setattr(c, name, other)
    with pytest.raises(AttributeError):
        del c.seq_lens
    seq_lens = c.seq_lens
    c.seq_lens += 1  # in place: the same tensor
    c.seq_lens.add_(1)
    assert c.seq_lens is seq_lens and c.seq_lens.tolist() == [2, 2, 2] and c._struct(None).seq_lens == seq_lens.data_ptr()
    b = P.NewTokens([0, 1, 1, 4], device="cpu")
    for name, other in (("h", b.h.copy()), ("d", b.d.clone()), ("total", 3)):
        with pytest.raises(AttributeError, match=name):
            setattr(b, name, other)
    with pytest.raises(ValueError):  # the device's sums would no longer agree
        b.h[1] = 2
    r = P.Rope()
    for name, other in (("n_axes", 3), ("c", P.Rope(sections=(16, 24, 24)).c)):
        with pytest.raises(AttributeError, match=name):
            setattr(r, name, other)


def test_a_programs_own_attributes_are_its_own():
    for x in (_cache(), P.NewTokens([0, 1], device="cpu"), P.Rope()):
        x.step = 1
        x.step = 2
        assert x.step == 2
        del x.step
        assert not hasattr(x, "step")


def test_copied_caches():
    import copy
    import pickle
    c = _cache()
    c.seq_lens[1] = 7
    one = copy.copy(c)  # the same tensors
    assert one.seq_lens is c.seq_lens and one._struct(None).k == c.k.data_ptr()
    for two in (copy.deepcopy(c), pickle.loads(pickle.dumps(c))):  # tensors, and so addresses, of their own
        assert two.seq_lens.tolist() == [0, 7, 0] and two.k.data_ptr() != c.k.data_ptr() and two.max_len == 40
        s = two._struct(None)
        assert (s.k, s.v, s.page_table, s.seq_lens) == tuple(t.data_ptr() for t in (two.k, two.v, two.page_table, two.seq_lens))
    r = P.Rope(1e4, (16, 24, 24), True)
    for q in (copy.copy(r), copy.deepcopy(r)):
        assert (q.n_axes, q.c.theta, q.c.interleaved, list(q.c.sections)) == (3, 1e4, 1, [16, 24, 24])


class FakeStream:
    """A stream as _On sees it."""

    def __init__(self, device, handle=7):
        self.device, self.cuda_stream = torch.device(device), handle


def test_streams_and_devices_of_a_call(monkeypatch):
    """A stream of another device is refused, and what is refused leaves the current device as it was."""
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "set_device", lambda i: current.__setitem__(0, i))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: FakeStream(device, 3))
    device = torch.device("cuda:1")
    for bad in (FakeStream("cuda:0"), FakeStream("cuda:2"), "seven", object()):
        with pytest.raises((ValueError, TypeError)):
            P._On(device, bad)
        assert current == [0]
    for good, handle, own in ((None, 3, True), (3, 3, True), (FakeStream("cuda:1", 3), 3, True), (FakeStream("cuda:1"), 7, False),
                              (9, 9, False), (0, 0, False)):
        with P._On(device, good) as on:
            assert current == [1] and (on.handle, on.own) == (handle, own)
        assert current == [0]
    with pytest.raises(RuntimeError):
        with P._On(device, None):
            raise RuntimeError
    assert current == [0]


# ---------------------------------------------------------------------------
# Buffers that overlap
# ---------------------------------------------------------------------------


@needs_lib
def test_overlaps_rejected():
    """Outputs and workspaces that share a byte with an input, an output or the pool (never dereferenced here: every call
    is refused)."""
    lib, MB = S.load(), 1 << 20
    f = Fake(counts=(0, 1, 3), k=1024 * MB, v=1025 * MB)
    pool = 2 * 4 * 20 * 16 * 256
    nq, nk = 2 * 3 * 28 * 256, 4 * 256
    ws = ctypes.c_size_t(0)
    assert lib.stlite_paged_workspace_size(f.ref, ctypes.byref(ws)) == S.OK and ws.value > nq and pool < MB

    def attend(q=64 * MB, out=65 * MB, work=66 * MB):
        return lib.stlite_paged_attention(f.ref, q, 1.0, out, work, ws.value, None)
    for kw in (dict(q=64 * MB, out=64 * MB + 16), dict(q=64 * MB + nq - 16, out=64 * MB), dict(out=64 * MB + nq - 256),
               dict(out=1024 * MB), dict(out=1024 * MB + pool - 16), dict(out=1025 * MB - nq + 16)):
        assert attend(**kw) == S.ERR_INVALID_ARG and "alias" in _err(), kw
    for kw in (dict(work=64 * MB), dict(work=65 * MB + (nq - 1) // 256 * 256), dict(work=64 * MB - 256), dict(work=1025 * MB),
               dict(work=1024 * MB - (ws.value - 1) // 256 * 256)):
        assert attend(**kw) == S.ERR_WORKSPACE and "alias" in _err(), kw

    def append(q_out, q=64 * MB, k=80 * MB, v=96 * MB, stride=36 * 128, layer=1 << 20):
        rows = [ctypes.byref(S._CRows(x, stride, layer)) for x in (q, k, v)]
        return lib.stlite_paged_append(f.ref, None, None, *rows, None, None, 0.0, q_out, None)
    last = 2 * 36 * 256  # the third token's row
    for at, own in ((64 * MB, 28 * 256), (80 * MB, nk), (96 * MB, nk)):
        for layer in (0, 2 * MB):
            for q_out in (at + layer, at + layer + 16, at + layer - 16, at + layer + last + own - 16, at + layer - nq + 16):
                assert append(q_out) == S.ERR_INVALID_ARG and "alias" in _err(), (at, layer, q_out)
    # (from between the first two tokens' keys on it meets the second one's)
    assert append(80 * MB + nk) == S.ERR_INVALID_ARG and "alias" in _err()
    for q_out in (1024 * MB, 1025 * MB + pool - 256, 1024 * MB - nq + 16):
        assert append(q_out) == S.ERR_INVALID_ARG and "alias" in _err()

    cu = np.array([0, 50, 110])
    p = S.Problem(2, 28, 4, 1, cu, np.zeros(3), np.zeros((0, 3)), S.budgets(cu, 1, 2), device="cpu")
    size = 8 * 110 * 256
    for k, v in ((1024 * MB, 64 * MB), (64 * MB, 1024 * MB), (1025 * MB + pool - 16, 64 * MB), (64 * MB, 1024 * MB - size + 16)):
        assert lib.stlite_paged_compact(p.ref, f.ref, k, v, FAKE, 0, None) == S.ERR_INVALID_ARG and "alias" in _err()


# ---------------------------------------------------------------------------
# Numbers that do not fit the C structs
# ---------------------------------------------------------------------------


def test_numbers_beyond_32_bits_rejected():
    """They are refused, not cut to their low bits (2^32 + 40 to 40)."""
    k = torch.zeros((1, 2, 3, 16, 128), dtype=torch.bfloat16)
    table, lens = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for kw in (dict(n_q_heads=2 ** 32 + 8), dict(n_q_heads=-2 ** 32 + 8), dict(n_q_heads=8, max_len=2 ** 32 + 40),
               dict(n_q_heads=8, max_len=-2 ** 32 + 40)):
        with pytest.raises(ValueError, match="32 bits"):
            P.PagedCache(k, k, table, lens, **kw)
    for cu in ([0, 2 ** 32 + 1], np.array([0, 2 ** 32 + 1]), torch.tensor([0, 2 ** 33]), [0, 1.5], [0.0, float("nan")], [0, 2.0 ** 40]):
        with pytest.raises(ValueError, match="cu_new"):
            P.NewTokens(cu, device="cpu")
    for cu in ([0, 3], (0, 3), np.array([0, 3]), np.array([0.0, 3.0]), torch.tensor([0, 3]), np.array([0, 3], np.uint8)):
        b = P.NewTokens(cu, device="cpu")
        assert b.h.tolist() == b.d.tolist() == [0, 3] and b.h.dtype == np.int32 and b.total == 3
    for sections in ((2 ** 32 + 16, 24, 24 - 2 ** 32), (16.0, 24, 24)):
        with pytest.raises((ValueError, TypeError)):
            P.Rope(sections=sections)


def test_assembly_leaves_m0_to_the_compiler():
    """Inline assembly does not write M0, which indexed accesses and LDS loads go by, behind the compiler's back: what
    reads it has it as an operand."""
    import re
    reads = 0
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\((.*?)\)\s*;", text, re.S):
            assert not re.search(r"\bm0\s*,", m.group(1)), (name, m.group(0))
            if re.search(r"\blds\\?[\"n]", m.group(1)) and "load" in m.group(1):
                reads += 1
                assert '"{m0}"' in m.group(1), (name, m.group(0))
    assert reads >= 1
