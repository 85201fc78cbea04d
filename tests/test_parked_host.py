"""CPU: parked sequences in the oracle of the pages, and in what the host checks."""
from __future__ import annotations

from oracle import serving as OS


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
