"""Keys into a 4-bit pool at positions of the whole range of 32 bits: the codes are those of the exact rotation.

The rows here are looked for on the CPU: each has values that lie 10^-11 to 2 10^-7 of a step beside a border between two
codes, where an angle that is off by a few 2^-53 of the position (10^-7 rad at 2^31) takes the wrong side of many.  The
exact angles come from 60 decimal digits; what 64 bits round after that is 10^-15, so bytes are compared for equality."""
from __future__ import annotations

from decimal import Decimal, localcontext

import numpy as np
import pytest

from oracle import paged as OP
from oracle import paged4 as O4
from tests.test_gpu_paged import D, _f64, _log, torch_cuda  # noqa: F401
from tests.test_gpu_paged4 import Served4

pytestmark = pytest.mark.gpu

TWO_PI = Decimal("6.28318530717958647692528676655900576839433879875021164194989")
POSITIONS = [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 12345, 2000000011, 1999999973, 1500450271, 1234567891, 1073741827, -(2 ** 31),
             -1999999943, -(2 ** 30) - 1, 987654321, 700000001, 536870909, -400000009, 268435459]
PAIRS = range(12)  # whose frequencies are the greatest


def _angles(positions, theta):
    """(cos, sin) [positions][pair], each to 2^-52."""
    with localcontext() as c:
        c.prec = 60
        turns = [Decimal(theta) ** (Decimal(-i) / 64) / TWO_PI for i in range(64)]
        frac = [[float(p * t - (p * t).to_integral_value()) for t in turns] for p in positions]
    a = 2 * np.pi * np.array(frac)
    return np.cos(a), np.sin(a)


def _bf16(x):
    """The nearest bf16 of a float64 array."""
    import torch
    return torch.from_numpy(np.asarray(x)).to(torch.bfloat16).double().numpy()


def _beside_a_border(c, s):
    """(a, b) in bf16 with a c - b s nearest to a border between two codes under a scale of 1, and how near."""
    b = np.concatenate([np.arange(128, 256) * 2.0 ** e for e in range(-9, -5)])
    b = np.concatenate([b, -b])[:, None]
    border = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5])
    border = np.concatenate([border, -border])[None]
    a = _bf16((border + b * s) / c)
    off = np.abs(a * c - b * s - border)
    off[(off < 1e-11) | (np.abs(a) > 4)] = 1
    off[np.abs(b * c + a * s) > 4] = 1  # (its partner keeps the block's scale)
    i = np.unravel_index(np.argmin(off), off.shape)
    return a[i], b[i[0], 0], off[i]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("theta", [10000.0, 1e6, 1.0, 1.7e308])
def test_codes_at_far_positions(torch_cuda, theta, interleaved):
    import torch
    n = len(POSITIONS)
    cos, sin = _angles(POSITIONS, theta)
    a, b, near = np.zeros((n, 64)), np.zeros((n, 64)), []
    for t in range(n):
        for i in (PAIRS if theta < 1e300 else range(4)):
            if abs(cos[t, i]) > 0.05:
                a[t, i], b[t, i], off = _beside_a_border(cos[t, i], sin[t, i])
                near.append(off)
        for i in (15, 31, 47, 63):  # makes the scales 1 in either order
            a[t, i], b[t, i] = _bf16(4.5 * (cos[t, i] + sin[t, i])), _bf16(4.5 * (cos[t, i] - sin[t, i]))
    assert np.mean(np.array(near) < 2e-7) > 0.2, "too few values beside a border"
    ya, yb = a * cos - b * sin, b * cos + a * sin
    x, y = np.zeros((n, D)), np.zeros((n, D))
    lo, hi = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, 64), slice(64, D))
    x[:, lo], x[:, hi], y[:, lo], y[:, hi] = a, b, ya, yb
    codes, scales = O4.encode(y, "bf16")
    assert (scales == 127).all()
    f = Served4((n,), (n,), 16, "bf16", 1, 1, 1, seed=64)
    k = torch.from_numpy(x).to(torch.bfloat16).cuda().view(1, n, 1, D)
    assert np.array_equal(_f64(k)[0, :, 0], x)
    pos = torch.tensor([POSITIONS], dtype=torch.int32, device="cuda")
    f.P.paged_append(f.cache, f.batch, None, k, k, positions=pos, rope=f.P.Rope(theta, interleaved=interleaved))
    torch.cuda.synchronize()
    got, got_scales = f.at(f.bytes()[0], np.array(OP.new_places(f.table, f.lens, f.cu, 16, f.n_pages, f.max_len)))
    wrong = int((got[0, 0] != codes).sum())
    _log(f"far positions, theta {theta:g}{' interleaved' if interleaved else ''}: {wrong} of {codes.size} bytes differ")
    assert wrong == 0 and np.array_equal(got_scales[0, 0], scales)
