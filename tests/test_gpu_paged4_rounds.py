"""The kernel of few rows over a 4-bit pool at the ends of its own steps: 16-key runs, 64-key tiles, the 256 keys that four
waves take at once, and two and three such rounds, whole and cut, for one token and a few."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_paged import D, _bits, torch_cuda  # noqa: F401
from tests.test_gpu_paged4 import Served4, _room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,new,far", [(4, 1, False), (20, 1, False), (5, 3, False), (7, 4, True), (7, 5, True), (16, 4, True)])
@pytest.mark.parametrize("page,dtype", [(16, "bf16"), (64, "fp16"), (256, "bf16")])
def test_ends_of_rounds(torch_cuda, heads, new, far, page, dtype):
    lens = [n + d for n in (256, 320, 512, 528, 768, 1024) for d in (-1, 0, 1)]
    f = Served4(lens, [new] * len(lens), page, dtype, 1, heads, 1, seed=70, fill=float("nan"))
    if far:
        _room(f, 1 << 17)
    q = f.randn((1, f.total, heads, D), 1.5)
    out = f.attend(q)
    f.compare(q, out)
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"


@pytest.mark.parametrize("new", [1, 4])
@pytest.mark.parametrize("n", [255, 256, 257, 511, 512, 513, 1023, 1024, 1025])
def test_one_sequence(torch_cuda, new, n):
    """Nothing to look up, and the places of a share are the sequence's own; room for long ones, so that a joining launch goes."""
    f = _room(Served4((n,), (new,), 32, "bf16", 2, 4, 2, seed=71, fill=float("nan")), 1 << 16)
    q = f.randn((2, f.total, 4, D), 1.5)
    f.compare(q, f.attend(q))
