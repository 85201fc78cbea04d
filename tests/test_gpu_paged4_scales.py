"""Scale bytes that no store writes, in rows that are seen: code times 2^(byte - 127) as everywhere, rounded to the type of the
call (an infinity beyond it), whichever kernel meets them and in whatever tile.

Attention of the finite ones is held to the tolerances of the 4-bit pool's other tests: the values are exact in 16 bits."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import paged as OP
from oracle import paged4 as O4
from tests.test_gpu_paged import D, _f64, _log, torch_cuda  # noqa: F401
from tests.test_gpu_paged4 import Served4, _room

pytestmark = pytest.mark.gpu

MOST = {"bf16": 252, "fp16": 140}  # the greatest byte that a store writes
FINITE = {1: 5, 2: 3, 3: 1}        # so much above it, the greatest code that is finite (3 2^126, 3/2 2^127; 3 2^14, .. 1/2 2^16)

# What runs: heads of one kv head, new tokens, and whether the sequences may be long.
FORMS = [(3, 1, False), (20, 1, False), (3, 4, False), (7, 4, False), (7, 5, True), (7, 9, True), (2, 140, False), (7, 70, False)]


def _set(f, s, j, block, byte, codes):
    """Block `block` of the value of token j of sequence s, in kv head 0: codes [32] of 4 bits under a scale byte."""
    import torch
    r = OP.place(f.table, s, j, f.page, f.n_pages)
    data = f.vb.cpu().numpy()
    c, scales = O4.rows(data, f.page)
    c[0, 0, r // f.page, r % f.page, 16 * block:16 * block + 16] = codes[0::2] | codes[1::2] << 4
    scales[0, 0, r // f.page, r % f.page, block] = byte
    f.vb.copy_(torch.from_numpy(data))
    f.v.copy_(torch.from_numpy(O4.decode(*O4.rows(data, f.page))))


def _served(heads, new, far, dtype, seed):
    f = Served4((200 + new, 64 + new, new), (new,) * 3, 32, dtype, 1, heads, 1, seed=seed, fill=float("nan"))
    return _room(f, 1 << 17) if far else f


def _tokens(f, s):
    """One that every new token sees, the new ones' first, middle and last."""
    n, size = f.new[s], f.lens[s]
    return sorted({max(size - n - 3, 0), size - n, size - n // 2 - 1, size - 1})


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_of_every_scale(torch_cuda, dtype):
    """Read back: each of 16 codes under each of 256 bytes."""
    import torch
    f = Served4((64,), (64,), 16, dtype, 1, 1, 1, seed=60)
    codes = np.tile((np.arange(16) * 2 % 16 | (np.arange(16) * 2 + 1) % 16 << 4).astype(np.uint8), (64, 4))
    scales = np.arange(256, dtype=np.uint8).reshape(64, 4)
    places = np.array(OP.new_places(f.table, f.lens, f.cu, 16, f.n_pages, f.max_len))
    for data in (f.kb, f.vb):
        b = data.cpu().numpy()
        c, sc = O4.rows(b, 16)
        c[0, 0, places // 16, places % 16], sc[0, 0, places // 16, places % 16] = codes, scales
        data.copy_(torch.from_numpy(b))
    want = torch.from_numpy(O4.decode(codes, scales)).to(f.dt)
    for got in f.P.paged_read(f.cache, f.batch):
        got = got[0, :, 0].cpu()
        assert ((got == want) | (torch.isnan(got) & torch.isnan(want))).all()


@pytest.mark.parametrize("heads,new,far", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_finite_values_above_the_stored_scales(torch_cuda, dtype, heads, new, far):
    """They count with their weights for whom they are seen, and for nobody else."""
    import torch
    f = _served(heads, new, far, dtype, 61)
    rng = np.random.default_rng(62)
    for s in range(3):
        for i, j in enumerate(_tokens(f, s)):
            above = 1 + (i + s) % (3 if dtype == "fp16" else 2)
            codes = (rng.integers(0, FINITE[above] + 1, 32) | rng.integers(0, 2, 32) << 3).astype(np.uint8)
            _set(f, s, j, i % 4, MOST[dtype] + above, codes)
    _set(f, 0, f.lens[0] - 1, 3, 254, np.zeros(32, np.uint8))  # nothing but zeros
    q = f.randn((1, f.total, heads, D))
    out = f.attend(q)
    assert torch.isfinite(out).all()
    _log(f"scales above, {heads} x {new} {dtype}: worst error / tolerance {f.compare(q, out):.3g}")


@pytest.mark.parametrize("heads,new,far", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_infinities_above_the_stored_scales(torch_cuda, dtype, heads, new, far):
    """A code beyond the type is an infinity of its sign, the block's other values are what they are; both signs in one place
    are NaN."""
    import torch
    f = _served(heads, new, far, dtype, 63)
    q = f.randn((1, f.total, heads, D), 0.25)  # (no weight is rounded to 0)
    small = np.array([1, 9] * 16, np.uint8)    # +- 1/2: finite under the least scale above
    want = np.zeros((f.total, D))              # the sum of the infinities that a token sees
    for s in range(3):
        for i, j in enumerate(_tokens(f, s)):
            codes = small.copy()
            codes[3], codes[20], codes[7 + i] = 7, 15, 7
            _set(f, s, j, (s + i) % 4, MOST[dtype] + 1, codes)
            base = 32 * ((s + i) % 4)
            first = int(f.cu[s]) + max(j - (f.lens[s] - f.new[s]), 0)
            for d, x in ((3, np.inf), (20, -np.inf), (7 + i, np.inf)):
                with np.errstate(invalid="ignore"):
                    want[first:f.cu[s + 1], base + d] += x
    # the last new token's row once more: the other sign where the middle one's has an infinity
    s, j = 0, f.lens[0] - 1
    if new > 2:
        codes = np.zeros(32, np.uint8)
        at = _tokens(f, 0).index(f.lens[0] - new // 2 - 1)
        codes[3] = 15
        _set(f, s, j, at % 4, MOST[dtype] + 1, codes)
        with np.errstate(invalid="ignore"):
            want[int(f.cu[1]) - 1, 32 * (at % 4) + 3] -= np.inf
    got = _f64(f.attend(q))[0]
    want = np.broadcast_to(want[:, None], got.shape)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True) and np.isfinite(got[~odd]).all()
    # the finite ones beside them: as without the infinities
    f.v.copy_(torch.where(torch.isfinite(f.v) | torch.isnan(f.v), f.v, torch.zeros_like(f.v)))
    ref, weight, keys, dot = OP.attention(_f64(q[0]), _f64(f.k[0]), _f64(f.v[0]), f.table, f.lens, f.cu, f.max_len, D ** -0.5, heads)
    u = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    rel = u + 2 * 128 * 2.0 ** -24 * dot + 2.0 ** -22 * (1 + dot) + 2 * keys * 2.0 ** -24
    err = np.where(odd, 0.0, np.abs(np.where(odd, 0.0, got) - ref))
    assert (err <= u * np.abs(ref) + rel[..., None] * weight + 2.0 ** -25).all()
