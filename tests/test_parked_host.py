"""CPU: parked sequences in the oracle of the pages, and in what the host checks."""
from __future__ import annotations

import os

import numpy as np
import pytest

from oracle import serving as OS
from paper_2603_00188_amd import paged as P
from paper_2603_00188_amd import stlite as S
from tests.test_paged_host import Fake, _err

needs_lib = pytest.mark.skipif(not os.path.exists(S.LIB_PATH), reason="library not built")


def test_compaction_by_hand():
    p = OS.Pool([[-1] * 4 for _ in range(3)], [0, 0, 0], [0, 0, 0], [4, 3, 2, 1, 0], 16, 64)
    p.grow([30, 40, 20])  # 2 + 3 pages, and two more that there are not
    assert p.lens == [30, 40, ~0]
    assert p.compact([30, 40, 20]) == [True, True, False] and p.lens == [30, 40, ~0]
    assert p.compact([7, 0, 0]) == [True, True, False] and p.lens == [7, 0, ~0]
    p.grow([9, 64, 0])  # the second holds 3 pages of 4: parked, empty
    assert p.lens == [16, ~0, ~0] and p.table[1] == [2, 3, 4, OS.ENDS]
    assert p.compact([10, 49, 1]) == [True, False, False] and p.lens == [10, ~0, ~0]
    assert p.compact([10, 48, 1]) == [True, True, False] and p.lens == [10, 48, ~0]
    p.grow([60, 0, 0])  # past max_len: parked with its tokens
    assert p.lens == [~10, 48, ~0]
    assert p.compact([10, 20, 0]) == [False, True, False] and p.lens == [~10, 20, ~0]
    # a table that no call has grown: a length of -1 is as good as 0
    q = OS.Pool([[0, 1, -1, 3]], [-1], [0], [], 16, 64)
    assert q.compact([50]) == [True] and q.lens == [50]


@needs_lib
def test_validate_takes_parked_sequences():
    """They are idle slots, whatever the batch has for them; their tokens' pages are still their own."""
    lib = S.load()
    f = Fake(counts=(0, 1, 3), page_size=16, n_pages=6, max_pages=3, max_len=40)

    def check(table, lens):
        t, n = np.asarray(table, np.int32), np.asarray(lens, np.int32)
        return lib.stlite_paged_validate(f.ref, t.ctypes.data, n.ctypes.data)

    table = [[0, 1, 2], [5, 4, -1]]
    for lens in ([40, ~0], [40, ~32], [~0, 32], [~40, 32], [~5, ~5], [17, ~40], [17, ~(2 ** 31 - 1)]):
        assert check(table, lens) == S.OK, lens
    assert lib.stlite_paged_validate(f.ref, None, np.asarray([~3, 32], np.int32).ctypes.data) == S.OK
    # a page of a parked sequence's tokens is none for another's new ones; behind its tokens it may be
    shared = [[0, 1, 2], [1, 4, -1]]
    assert check(shared, [17, ~16]) == S.ERR_INVALID_ARG and "holds twice" in _err()
    assert check(shared, [17, ~0]) == S.OK and check([[0, 1, 2], [5, 1, -1]], [17, ~16]) == S.OK
    assert check(shared, [16, ~16]) == S.OK  # read alone
    # the others are checked as ever
    assert check(table, [0, ~0]) == S.ERR_INVALID_ARG and check(table, [41, ~0]) == S.ERR_INVALID_ARG
    assert check([[0, 6, 2], [5, 4, 3]], [17, ~2]) == S.ERR_INVALID_ARG and "outside [0, 6)" in _err()
    assert check([[0, 1, 2], [6, 4, 3]], [17, ~2]) == S.OK


@needs_lib
def test_binding_validates_parked_sequences():
    c = P.PagedCache.alloc(1, 2, 2, 2, 40, page_size=16, device="cpu", n_pages=6)
    b = P.NewTokens([0, 1, 3], device="cpu")
    c.validate(b, [[0, 1, -1], [2, -1, -1]], [20, ~7])
    with pytest.raises(RuntimeError, match="new tokens"):
        c.validate(b, [[0, 1, -1], [2, -1, -1]], [20, 1])


@needs_lib
def test_refusals_name_the_call_that_takes_more_than_max_len():
    lib = S.load()
    assert lib.stlite_paged_read(Fake(counts=(0, 1, 82)).ref, None, None, None) == S.ERR_INVALID_ARG
    assert "81 new tokens" in _err() and "stlite_paged_grow" in _err()
    assert lib.stlite_paged_read(Fake(counts=(0, 2, 1)).ref, None, None, None) == S.ERR_INVALID_ARG
    assert "-1 new tokens" in _err() and "grow" not in _err()
