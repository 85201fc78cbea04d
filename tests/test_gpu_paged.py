"""GPU tests of serving from a paged cache, against the 64-bit oracle.

Tolerances, from the roundings of the definition (u: half a step of the output
type relative to the value, 2^-8 bf16, 2^-11 fp16):

* append: the fp32 result is rounded once, u |y|.  In fp32 a pair's rotation
  rounds 2 products, a sum and the two factors (the reduced angle to 2^-25 of a
  turn, the sine to two units of 2^-24): within 8 * 2^-24 (|n_a| + |n_b|); a norm
  (16 squares in a row, three additions, the mean, root, quotient, two products)
  within 24 * 2^-24 relative.  Together under 2^-18 (|n_a| + |n_b|), and half the
  smallest step of fp16, 2^-25.
* attention: the output is rounded once, u |o|; with several new tokens the
  weights are too, u sum_j p_j |v_j| (with one they are fp32, or fp16 terms whose sum
  is off by 2^-22 relative or 2^-40 of the greatest: inside what follows).  A logit is a sum of 128 exact products in
  fp32, off by at most 128 * 2^-24 of scale sum_c |q_c k_c|, and its weight by
  twice that (numerator and denominator); the exponential and its argument,
  |x| <= the same sum, by 2^-22 (1 + that); sums of n weights by n 2^-24 each in
  the denominator and the numerator.
"""
import numpy as np
import pytest

from oracle import paged as OP

pytestmark = pytest.mark.gpu

D = 128


@pytest.fixture(scope="module")
def torch_cuda():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _log(msg):
    from tests import gpu_harness as H
    H.log(msg)


def _type(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _half_step(name):
    return {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[name]


def _f64(t):
    return t.double().cpu().numpy()


def _bits(t):
    import torch
    return t.view(torch.int16).cpu().numpy()


class Served:
    """A cache with scattered pages, random rows in it, and a batch of new tokens."""

    def __init__(self, lens, new, page, dtype="bf16", layers=1, hq=7, hk=1, seed=0, spare=2, fill=None, v_scale=1.0):
        import torch
        from paper_2603_00188_amd import paged as P
        self.P, self.name, self.layers, self.hq, self.hk, self.page = P, dtype, layers, hq, hk, page
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.dt, self.lens, self.new = _type(dtype), list(lens), list(new)
        need = [-(-n // page) for n in lens]
        max_pages = max(max(need), 1)
        self.n_pages = sum(need) + spare
        rng = np.random.default_rng(seed)
        order = rng.permutation(self.n_pages).astype(np.int32)
        table = np.full((len(lens), max_pages), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        self.table = table
        shape = (layers, hk, self.n_pages, page, D)
        self.k, self.v = self.randn(shape), self.randn(shape) * v_scale
        if fill is not None:  # whatever is no token's row
            used = np.zeros(self.n_pages * page, bool)
            for s, n in enumerate(lens):
                for j in range(n):
                    used[OP.place(table, s, j, page, self.n_pages)] = True
            idle = torch.from_numpy(~used).cuda()
            for pool in (self.k, self.v):
                pool.view(layers, hk, -1, D)[:, :, idle] = fill
        self.max_len = max_pages * page
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.total = int(self.cu[-1])
        self.batch = P.NewTokens(self.cu)
        self.rebuild()

    def rebuild(self):
        import torch
        self.cache = self.P.PagedCache(self.k, self.v, torch.from_numpy(self.table).cuda(),
                                       torch.tensor(self.lens, dtype=torch.int32, device="cuda"), self.hq, self.max_len)

    def randn(self, shape, scale=1.0):
        import torch
        return (torch.randn(shape, generator=self.gen, device="cuda") * scale).to(self.dt)

    def attend(self, q, scale=D ** -0.5, **kw):
        """Output, inside a larger buffer whose other rows must stay as they were."""
        import torch
        n = q.numel()
        buf = torch.full((n + 4096,), 7.0, dtype=self.dt, device="cuda")
        out = buf[2048:2048 + n].view(q.shape)
        size = self.cache.workspace_size(self.batch)
        ws = torch.full((max(size, 256) + 1024,), 0xAB, dtype=torch.uint8, device="cuda")
        self.P.paged_attention(self.cache, self.batch, q, out=out, workspace=ws[:max(size, 256)], scale=scale, **kw)
        torch.cuda.synchronize()
        assert (buf[:2048] == 7).all() and (buf[2048 + n:] == 7).all(), "written outside the output"
        assert (ws[max(size, 256):] == 0xAB).all(), "written behind the workspace"
        return out

    def compare(self, q, out, scale=D ** -0.5, decode=None):
        """Worst error in units of the tolerance, over every layer."""
        decode = max(self.new) <= 1 if decode is None else decode
        u, worst = _half_step(self.name), 0.0
        got = _f64(out)
        for layer in range(self.layers):
            ref, weight, keys, dot = OP.attention(_f64(q[layer]), _f64(self.k[layer]), _f64(self.v[layer]), self.table,
                                                  self.lens, self.cu, self.max_len, scale, self.hq // self.hk)
            rel = (0 if decode else u) + 2 * 128 * 2.0 ** -24 * dot + 2.0 ** -22 * (1 + dot) + 2 * keys * 2.0 ** -24
            lim = u * np.abs(ref) + rel[..., None] * weight + 2.0 ** -25
            err = np.abs(got[layer] - ref)
            if not (err <= lim).all():
                i = np.unravel_index(np.argmax(np.where(np.isnan(err), np.inf, err / lim)), err.shape)
                raise AssertionError(f"layer {layer} token {i[0]} head {i[1]} dim {i[2]}: got {got[layer][i]!r} ref {ref[i]!r} "
                                     f"tol {lim[i]:.3g}, {keys[i[:2]]} keys")
            worst = max(worst, float((err / lim).max()) if err.size else 0.0)
        return worst


# ---------------------------------------------------------------------------
# Attention of one new token
# ---------------------------------------------------------------------------

DECODE = [
    # lens, new, page, dtype, layers, hq, hk
    ((1,), (1,), 16, "bf16", 1, 1, 1),
    ((1, 2, 15, 16, 17, 31, 32, 33), (1,) * 8, 16, "bf16", 1, 7, 1),
    ((63, 64, 65, 127, 128, 129, 130), (1,) * 7, 32, "fp16", 2, 16, 2),
    ((0, 5, 0, 200, 77), (1, 0, 1, 1, 0), 64, "bf16", 1, 8, 8),
    ((678,), (1,), 16, "bf16", 3, 28, 4),
    ((5000, 1, 0, 333), (1, 1, 1, 1), 128, "fp16", 2, 12, 2),
    ((1000, 300), (1, 1), 256, "bf16", 1, 17, 1),      # two head groups, one head in the second
    ((700, 64, 1), (1, 1, 1), 16, "fp16", 1, 128, 1),  # eight head groups
    ((20000,), (1,), 32, "bf16", 1, 4, 2),
    ((3000,), (1,), 16, "bf16", 1, 40, 1),             # one sequence, three head groups, each cut
    ((9000,), (1,), 16, "fp16", 2, 2, 2),              # one row to an item, more parts than are joined at once
    (tuple(range(1, 300, 3)), (1,) * 100, 16, "bf16", 1, 4, 1),
    ((9000, 40, 0, 6000), (1, 0, 1, 1), 16, "bf16", 1, 7, 1),  # few items, each in many parts, idle sequences between
    ((5000, 300, 7000), (1, 1, 1), 64, "fp16", 1, 40, 1),      # the same with two head groups
]


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", DECODE)
def test_decode(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    """What is no token's row holds NaN, which no output may meet."""
    _log(f"paged decode lens {lens[:8]} page {page} {dtype} {layers} x {hq}/{hk}")
    f = Served(lens, new, page, dtype, layers, hq, hk, seed=1, fill=float("nan"))
    q = f.randn((layers, f.total, hq, D), 1.5)
    out = f.attend(q)
    _log(f"worst error / tolerance {f.compare(q, out):.3g}")
    for s, n in enumerate(lens):
        if n == 0 and new[s]:
            assert not out[:, f.cu[s]].any()
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"


def test_decode_many_short_sequences(torch_cuda):
    """More sequences than threads look them up."""
    rng = np.random.default_rng(2)
    lens = rng.integers(0, 40, 700).tolist()
    f = Served(lens, [1] * 700, 16, "bf16", 1, 2, 1, fill=float("nan"))
    q = f.randn((1, 700, 2, D))
    f.compare(q, f.attend(q))


def test_half_weights_are_rounded_to_nearest(torch_cuda):
    """One token in fp16: a weight is two half terms, off by at most 2^-22 of itself and to
    either side alike.  A key of weight p meets 2^14, keys of weight 1 meet what cancels all
    but the last bits of it: the sums are exact, so that the output shows the terms' error.
    In units of an fp32 step of the weight, terms that are cut off at 13 bits of which the
    second holds the first 11 from its leading one lose 0.875 on average (half of all: 1.5 of
    two bits, a quarter: 0.5 of one), terms that are rounded nothing; half of that is told
    apart here.  The exponential's error is within one such step for each weight."""
    import torch
    n, big = 4096, 2.0 ** 14
    f = Served((3,) * n, (1,) * n, 16, "fp16", 1, 1, 1, seed=24)
    scale = np.float32(np.log(2.0))
    x = (-np.linspace(0.01, 0.99, n)).astype(np.float16)
    p = np.exp2((x.astype(np.float32) * np.float32(scale * np.float32(1.4426950408889634))).astype(np.float64))
    c1 = (p * big).astype(np.float16)
    c2 = (p * big - c1.astype(np.float64)).astype(np.float16)
    at = np.array([[OP.place(f.table, s, j, 16, f.n_pages) for j in range(3)] for s in range(n)])
    k, v = np.zeros((f.n_pages * 16, D), np.float16), np.zeros((f.n_pages * 16, D), np.float16)
    k[at[:, 2], 0] = x
    v[at[:, 0]], v[at[:, 1]], v[at[:, 2]] = -c1[:, None], -c2[:, None], big
    f.k.copy_(torch.from_numpy(k).view(f.k.shape))
    f.v.copy_(torch.from_numpy(v).view(f.v.shape))
    q = torch.zeros((1, n, 1, D), dtype=f.dt, device="cuda")
    q[..., 0] = 1
    got = _f64(f.attend(q, scale=float(scale)))[0, :, 0, 0] * (2 + p)
    err = (got - (p * big - c1.astype(np.float64) - c2.astype(np.float64))) / (big * 2.0 ** -24)
    _log(f"half terms: mean error {err.mean():.3f} fp32 steps, worst {np.abs(err).max():.2f}")
    assert abs(err.mean()) < 0.875 / 2 and np.abs(err).max() <= 2 + 1 + 0.5


# ---------------------------------------------------------------------------
# Attention of several new tokens
# ---------------------------------------------------------------------------

EXTEND = [
    ((2,), (2,), 16, "bf16", 1, 1, 1),
    ((5,), (5,), 16, "fp16", 1, 7, 1),
    ((37, 64, 65), (5, 1, 0), 16, "bf16", 2, 14, 2),      # drafted tokens beside a plain step and an idle sequence
    ((300, 33, 128), (33, 33, 20), 32, "bf16", 1, 7, 1),  # more than one block of 128 rows
    ((130,), (130,), 64, "fp16", 1, 3, 1),                # a prompt, 256-row blocks
    ((1000, 200, 64), (500, 200, 1), 16, "bf16", 1, 8, 2),
    ((777, 90), (300, 90), 128, "fp16", 2, 4, 4),
    ((400,), (100,), 256, "bf16", 1, 17, 1),              # 15 tokens to a block, its last row idle
    ((200,), (150,), 16, "bf16", 1, 128, 1),              # two tokens to a block
    ((6000,), (3,), 32, "bf16", 1, 28, 4),                # few rows over a long cache: joined
    ((2500,), (700,), 64, "bf16", 1, 7, 1),
    ((3000,), (60,), 16, "fp16", 1, 128, 1),              # items of one sequence, each in many parts
    ((900,) * 6, (200,) * 6, 32, "bf16", 3, 8, 2),        # items cut in two
    ((3, 0, 2), (5, 3, 9), 16, "bf16", 1, 2, 1),          # shorter than their new tokens
    ((9000, 40, 3000, 10), (3, 0, 40, 1), 32, "fp16", 1, 7, 1),  # few items, each in many parts
]


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", EXTEND)
def test_extend(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    _log(f"paged extend lens {lens} new {new} page {page} {dtype} {layers} x {hq}/{hk}")
    f = Served(lens, new, page, dtype, layers, hq, hk, seed=3, fill=float("nan"))
    q = f.randn((layers, f.total, hq, D), 1.5)
    out = f.attend(q)
    _log(f"worst error / tolerance {f.compare(q, out):.3g}")
    for s, n in enumerate(lens):  # tokens that see nothing
        for t in range(max(new[s] - n, 0)):
            assert not out[:, f.cu[s] + t].any()
    assert np.array_equal(_bits(f.attend(q)), _bits(out)), "two calls differ"


@pytest.mark.parametrize("group,tokens", [(7, 36), (1, 256), (3, 85), (20, 12), (128, 2)])
def test_extend_at_the_ends_of_blocks(torch_cuda, group, tokens):
    """A block has 256 rows, whole tokens of `group` heads: one token less, as many, one more, two blocks and one more,
    each beside the others and behind a few keys or none."""
    _log(f"paged extend, {tokens} tokens of {group} heads to a block")
    new = [tokens - 1, tokens, tokens + 1, 2 * tokens, 2 * tokens + 1]
    f = Served([n + c for n, c in zip(new, (0, 63, 1, 0, 130))], new, 16, "bf16", 1, 2 * group, 2, seed=29, fill=float("nan"))
    q = f.randn((1, f.total, 2 * group, D), 1.5)
    f.compare(q, f.attend(q))


def test_extend_many_sequences(torch_cuda):
    """More sequences than threads look them up, idle ones among them."""
    rng = np.random.default_rng(4)
    new = rng.integers(0, 4, 1100)
    lens = [int(n + rng.integers(0, 90)) for n in new]
    f = Served(lens, new.tolist(), 16, "fp16", 1, 2, 1, fill=float("nan"))
    q = f.randn((1, f.total, 2, D))
    f.compare(q, f.attend(q))


@pytest.mark.parametrize("new", [1, 4, 150])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rising_and_extreme_logits(torch_cuda, new, dtype):
    """Maxima that rise in every step of the cache, fall, and weights that underflow."""
    import torch
    f = Served((900, 900, 901), (new, new, new), 16, dtype, 1, 4, 1, seed=5)
    q = f.randn((1, f.total, 4, D))
    q[..., 1:] = 0
    q[..., 0] = 8.0
    f.k[..., 1:] = 0
    for s, slope in enumerate((1.0, -1.0, 0.0)):
        for j in range(f.lens[s]):
            r = OP.place(f.table, s, j, 16, f.n_pages)
            f.k.view(1, 1, -1, D)[0, 0, r, 0] = slope * (j - 450) * 0.125
    for scale in (D ** -0.5, 1.0, 4.0, 1e-3):
        out = f.attend(q, scale=scale)
        assert torch.isfinite(out).all()
        f.compare(q, out, scale=scale)


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_logits_of_any_size(torch_cuda, new, dtype):
    """Logits up to 2^107.  Equal ones give the mean of the values that are seen; others
    differ by more than 2^14, so that one key has all the weight.  Either way no logit's
    rounding matters, and the tolerance has no part for it."""
    import torch
    f = Served((300, 200, 171), (new,) * 3, 16, dtype, 1, 4, 1, seed=22)
    u, where = _half_step(dtype), [(s, j, OP.place(f.table, s, j, 16, f.n_pages)) for s in range(3) for j in range(f.lens[s])]
    rows = f.k.view(1, 1, -1, D)

    def check(q, scale, what):
        out = f.attend(q, scale=scale)
        ref, weight, keys, _ = OP.attention(_f64(q[0]), _f64(f.k[0]), _f64(f.v[0]), f.table, f.lens, f.cu, f.max_len, scale, 4)
        lim = u * np.abs(ref) + ((0 if new == 1 else u) + 2.0 ** -22 + 2 * keys * 2.0 ** -24)[..., None] * weight + 2.0 ** -25
        err = np.abs(_f64(out[0]) - ref)
        assert (err <= lim).all(), (what, scale, np.argwhere(~(err <= lim))[:3].tolist(), _f64(out[0])[~(err <= lim)][:3])

    q = torch.empty((1, f.total, 4, D), dtype=f.dt, device="cuda")
    sizes = [(7000.0, 7000.0, D ** -0.5), (60000.0, 60000.0, D ** -0.5), (60000.0, -60000.0, D ** -0.5), (1.0, 1.0, 2.0 ** 15),
             (1.0, -1.0, 2.0 ** 17), (3.0, 5.0, 2.0 ** 20), (1.0, 1.0, 2.0 ** 24), (1.0, -1.0, 2.0 ** 30), (1.0, 1.0, 2.0 ** 100)]
    for a, b, scale in sizes + ([(1e10, 1e10, D ** -0.5)] if dtype == "bf16" else []):
        q.fill_(a)
        rows.fill_(b)
        check(q, scale, ("equal", a, b))
        rows.fill_(b / 2 if b > 0 else b)
        for s in range(3):  # one that stands out, in the first tile, behind it, and among the new tokens
            rows[0, 0, OP.place(f.table, s, (3, 100, f.lens[s] - 1)[s], 16, f.n_pages)] = b if b > 0 else b / 2
        check(q, scale, ("one", a, b))
    q.zero_()
    q[..., :2] = 1
    rows.zero_()
    for slope in (1, -1):  # every key above the one before it, or below
        for s, j, r in where:
            rows[0, 0, r, 0], rows[0, 0, r, 1] = slope * (j % 128), slope * (j - j % 128)
        for scale in (2.0 ** 14, 2.0 ** 15, 2.0 ** 18, 2.0 ** 24, 2.0 ** 60, 2.0 ** 99):
            check(q, scale, ("slope", slope))


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("long", [False, True])
def test_infinite_logits(torch_cuda, new, dtype, long):
    """Keys whose logit is -infinity weigh nothing, and a token all of whose logits are gets 0; a logit of infinity makes
    the tokens that see it NaN.  In one part and in many."""
    import torch
    f = Served((9000, 5000, 6000) if long else (300, 200, 171), (new,) * 3, 16, dtype, 1, 4, 1, seed=30)
    rows = f.k.view(1, 1, -1, D)
    rows.zero_()
    at = lambda s, j: OP.place(f.table, s, j, 16, f.n_pages)  # noqa: E731
    for j in (0, 5, 63, 64, 70, f.lens[0] - new):
        rows[0, 0, at(0, j), 0] = float("-inf")
    for j in range(f.lens[1]):
        rows[0, 0, at(1, j), 0] = float("-inf")
    last = f.lens[2] - new // 2 - 1
    rows[0, 0, at(2, last), 0] = float("inf")
    q = torch.zeros((1, f.total, 4, D), dtype=f.dt, device="cuda")
    q[..., 0] = 1
    out = f.attend(q)
    sees = int(f.cu[2]) + max(last - (f.lens[2] - new), 0)
    assert not out[0, f.cu[1]:f.cu[2]].any() and torch.isnan(out[0, sees:]).all()
    ref, weight, keys, _ = OP.attention(_f64(q[0]), _f64(f.k[0]), _f64(f.v[0]), f.table, f.lens, f.cu, f.max_len, D ** -0.5, 4)
    u = _half_step(dtype)
    lim = u * np.abs(ref) + ((0 if new == 1 else u) + 2.0 ** -22 + 2 * keys * 2.0 ** -24)[..., None] * weight + 2.0 ** -25
    for part in (slice(0, f.cu[1]), slice(f.cu[2], sees)):
        assert (np.abs(_f64(out[0]) - ref) <= lim)[part].all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("scale", [D ** -0.5, 0.7, 100.0, 1e6])
def test_the_greatest_weight_is_not_rounded(torch_cuda, dtype, scale):
    """A token that sees one key, or many that another outweighs by 2^100, gets that one's value bit by bit: its weight is
    a power of two to 2^-15, well inside half a step of either type."""
    import torch
    f = Served((150, 90, 40), (150, 20, 1), 16, dtype, 1, 4, 1, seed=31)
    q = f.randn((1, f.total, 4, D), 1.5)
    out = f.attend(q, scale=scale)
    value = lambda s, j: f.v.view(-1, D)[OP.place(f.table, s, j, 16, f.n_pages)]  # noqa: E731
    assert torch.equal(out[0, 0], value(0, 0).expand(4, D))
    q.zero_()
    q[..., 0] = 3.0
    rows, rng = f.k.view(-1, D), np.random.default_rng(31)
    for s, at in enumerate((7, 70, 5)):
        for j in range(f.lens[s]):  # below the one that stands out by 2^100 in base 2
            rows[OP.place(f.table, s, j, 16, f.n_pages), 0] = float((rng.random() - (0 if j == at else 101)) * 0.7 / 3 / scale)
        seen = slice(int(f.cu[s]) + max(at - (f.lens[s] - f.new[s]), 0), int(f.cu[s + 1]))
        want = value(s, at)
        assert torch.equal(f.attend(q, scale=scale)[0, seen], want.expand(seen.stop - seen.start, 4, D)), s


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_masked_values_have_no_influence(torch_cuda, new, dtype):
    """Keys and values of later tokens that are infinite or NaN reach the tokens that
    see them, and no other."""
    import torch
    lens = (300, 141, 200)
    f = Served(lens, (new,) * 3, 16, dtype, 1, 6, 2, seed=6, fill=float("nan"))
    q = f.randn((1, f.total, 6, D))
    clean = f.attend(q).clone()
    at = [f.lens[s] - new // 2 - 1 for s in range(3)]  # a new token's own row, in the middle
    rows = [OP.place(f.table, s, at[s], 16, f.n_pages) for s in range(3)]
    v = f.v.view(1, 2, -1, D)
    v[0, 0, rows[0], 5] = float("inf")
    v[0, 0, rows[0], 6] = float("-inf")
    v[0, 1, rows[1], 7] = float("nan")
    f.k.view(1, 2, -1, D)[0, 1, rows[2], 9] = float("nan")
    out = f.attend(q)
    first = [int(f.cu[s]) + max(at[s] - (f.lens[s] - new), 0) for s in range(3)]  # the first token that sees it
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[0, first[0]:f.cu[1], 0:3, 5:7] = True
    hit[0, first[1]:f.cu[2], 3:6, 7] = True
    hit[0, first[2]:f.cu[3], 3:6, :] = True
    assert torch.equal(out[~hit], clean[~hit])
    assert (out[0, first[0]:f.cu[1], 0:3, 5] == float("inf")).all() and (out[0, first[0]:f.cu[1], 0:3, 6] == float("-inf")).all()
    assert torch.isnan(out[0, first[1]:f.cu[2], 3:6, 7]).all() and torch.isnan(out[0, first[2]:f.cu[3], 3:6, :]).all()


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk", [
    ((20000,), (1,), 32, "bf16", 1, 4, 2), ((9000, 40, 0, 6000), (1, 0, 1, 1), 16, "bf16", 1, 7, 1),
    ((5000, 300, 7000), (1, 1, 1), 64, "fp16", 1, 40, 1), ((900,) * 40, (1,) * 40, 16, "fp16", 2, 16, 2),
    ((6000, 300), (3, 3), 32, "bf16", 1, 28, 4), ((3000,), (60,), 16, "fp16", 1, 128, 1), ((700,) * 9, (150,) * 9, 16, "bf16", 2, 8, 2)])
def test_logits_that_are_nan(torch_cuda, lens, new, page, dtype, layers, hq, hk):
    """A query or keys that are NaN make their own outputs NaN, however many parts a sequence is cut into, even where no
    part has another logit; a token that sees nothing still gets 0."""
    import torch
    f = Served(lens, new, page, dtype, layers, hq, hk, seed=23)
    q = f.randn((layers, f.total, hq, D))
    clean = f.attend(q).clone()
    want = torch.isnan(clean)
    assert not want.any()
    for s in range(0, len(lens), 2):
        if new[s]:
            q[:, f.cu[s], hq - 1, 5] = float("nan")
            want[:, f.cu[s], hq - 1] = lens[s] > 0
    out = f.attend(q)
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], clean[~want])
    for j in range(lens[0] - new[0] + 1):  # every key that the first sequence's first token sees, of one kv head
        f.k.view(layers, hk, -1, D)[0, hk - 1, OP.place(f.table, 0, j, page, f.n_pages), 7] = float("nan")
    want[0, :f.cu[1], hq - hq // hk:] = True
    out = f.attend(q)
    assert torch.equal(torch.isnan(out), want) and torch.equal(out[~want], clean[~want])


@pytest.mark.parametrize("new,hq", [(1, 3), (1, 20), (1, 40), (4, 20), (70, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_that_are_seen_and_not_finite(torch_cuda, new, hq, dtype):
    """They reach every token and head, with the greatest weight or none to speak of, and
    no other dimension.  With several tokens the weights are rounded to the type of the
    call first, and one below half its smallest step becomes 0: 0 * infinity is NaN."""
    import torch
    f = Served((300, 70), (new, new), 16, dtype, 1, hq, 1, seed=18)
    q = f.randn((1, f.total, hq, D), 4.0)
    clean = f.attend(q).clone()
    v = f.v.view(1, 1, -1, D)
    row = lambda s, j: OP.place(f.table, s, j, 16, f.n_pages)  # noqa: E731
    v[0, 0, row(0, 0), 3] = v[0, 0, row(0, 77), 3] = float("inf")
    v[0, 0, row(0, 78), 4] = float("-inf")
    v[0, 0, row(0, 16), 127], v[0, 0, row(0, 17), 127] = float("inf"), float("-inf")
    f.k.view(1, 1, -1, D)[0, 0, row(0, 78)] *= -8
    k = f.k.clone()
    dims = torch.tensor([d for d in range(D) if d not in (3, 4, 127)], device="cuda")
    out = f.attend(q)
    first = slice(0, int(f.cu[1]))
    zero = torch.isnan(out[0, first]) & (new > 1)
    assert ((out[0, first, :, 3] == float("inf")) | zero[..., 3]).all()
    assert ((out[0, first, :, 4] == float("-inf")) | zero[..., 4]).all()
    assert torch.isnan(out[0, first, :, 127]).all()
    assert torch.equal(out[:, f.cu[1]:], clean[:, f.cu[1]:])
    v[0, 0, row(0, 0), 3] = v[0, 0, row(0, 77), 3] = v[0, 0, row(0, 78), 4] = 0
    v[0, 0, row(0, 16), 127] = v[0, 0, row(0, 17), 127] = 0
    assert torch.equal(f.k, k)
    assert torch.equal(out[..., dims], f.attend(q)[..., dims])


@pytest.mark.parametrize("new", [1, 3, 140])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_at_the_limits_of_the_type(torch_cuda, new, dtype):
    """Sums of the greatest and the smallest normal values."""
    import torch
    f = Served((1500, 300, 200), (new,) * 3, 16, dtype, 1, 7, 1, seed=19)
    info = torch.finfo(f.dt)
    f.v[..., 0::4] = info.max
    f.v[..., 1::4] = -info.max
    f.v[..., 2::4] *= info.max / 16
    f.v[..., 3] = 2.0 ** -40 if dtype == "bf16" else info.tiny
    q = f.randn((1, f.total, 7, D), 1.5)
    out = f.attend(q)
    assert torch.isfinite(out).all()
    f.compare(q, out)


@pytest.mark.parametrize("new", [1, 3, 140])
def test_pages_out_of_range_are_left_out(torch_cuda, new):
    import torch
    f = Served((300, 200, 150, 260), (new,) * 4, 16, "bf16", 1, 4, 2, seed=7, fill=float("nan"))
    f.table[0, 3] = -1
    f.table[0, 18] = f.n_pages          # the last page: the new tokens' own rows among it
    f.table[1, :] = -5                  # nothing left
    f.table[2, 0] = 2 ** 31 - 1
    f.table[3, 4:9] = np.iinfo(np.int32).min
    # what page 0 holds must not matter either: it is read where an index is out of range
    keep = [f.table[s, e] for s in range(4) for e in range(-(-f.lens[s] // 16))]
    if 0 not in keep:
        f.k[:, :, 0], f.v[:, :, 0] = float("nan"), float("inf")
    f.rebuild()
    q = f.randn((1, f.total, 4, D))
    out = f.attend(q)
    f.compare(q, out)
    assert not out[:, f.cu[1]:f.cu[2]].any()
    assert torch.isfinite(out).all()


def test_lengths_are_cut_to_the_bounds(torch_cuda):
    for new in (1, 4):
        f = Served((64, 48, 30), (new,) * 3, 16, "bf16", 1, 4, 1, seed=8)
        q = f.randn((1, f.total, 4, D))
        f.lens = [64, 2 ** 31 - 1, -7]
        f.table[1, 3] = f.table[0, 3]  # so that the cut length has its pages
        f.max_len = 60
        f.rebuild()
        out = f.attend(q)
        f.compare(q, out)
        assert not out[:, f.cu[2]:].any()


def test_shared_pages(torch_cuda):
    """A prefix that two sequences share."""
    for new in (1, 4):
        f = Served((200, 180), (new, new), 32, "bf16", 2, 8, 2, seed=9)
        f.table[1, :3] = f.table[0, :3]
        f.rebuild()
        q = f.randn((2, f.total, 8, D))
        f.compare(q, f.attend(q))


@pytest.mark.parametrize("new", [1, 40])
def test_pool_of_more_than_4_gib(torch_cuda, new):
    """Rows behind 2^32 bytes of a unit's pool, and of the units before it."""
    import torch
    page, n_pages = 256, (1 << 24) // 256 + 3
    from paper_2603_00188_amd import paged as P
    k = torch.zeros((1, 2, n_pages, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    f = Served((700,), (new,), page, "bf16", 1, 4, 2, seed=10)
    used = -(-700 // page)
    k[:, :, -used:], v[:, :, -used:] = f.k[:, :, f.table[0, :used]], f.v[:, :, f.table[0, :used]]
    table = torch.arange(n_pages - used, n_pages, dtype=torch.int32, device="cuda").view(1, used)
    big = P.PagedCache(k, v, table, f.cache.seq_lens, 4, f.max_len)
    q = f.randn((1, f.total, 4, D))
    out = f.attend(q)
    f.compare(q, out)
    assert torch.equal(P.paged_attention(big, f.batch, q), out)
    # and stores there
    rows = [f.randn((1, f.total, 2, D)) for _ in range(2)]
    P.paged_append(big, f.batch, None, *rows)
    P.paged_append(f.cache, f.batch, None, *rows)
    torch.cuda.synchronize()
    assert torch.equal(big.k[:, :, -used:], f.k[:, :, f.table[0, :used]])
    assert torch.equal(big.v[:, :, -used:], f.v[:, :, f.table[0, :used]])


# ---------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------

APPEND = [
    # lens, new, page, dtype, layers, hq, hk, axes, interleaved, norms, fused
    ((1,), (1,), 16, "bf16", 1, 7, 1, 1, False, "", False),
    ((33, 0, 17, 64), (1, 1, 0, 1), 16, "fp16", 3, 8, 2, 3, False, "qk", False),
    ((40, 7, 100), (40, 7, 3), 32, "bf16", 2, 28, 4, 3, False, "", True),
    ((40, 7, 100), (40, 7, 3), 32, "bf16", 2, 28, 4, 1, True, "qk", True),
    ((300,), (290,), 64, "fp16", 8, 5, 5, 1, False, "k", False),      # the path of many tokens
    ((1500, 900), (1100, 900), 128, "bf16", 2, 28, 4, 3, True, "q", True),
    ((5, 2), (9, 4), 16, "bf16", 2, 3, 1, 1, False, "", False),       # shorter than their new tokens
    ((90,), (50,), 256, "bf16", 1, 12, 3, 0, False, "qk", True),      # no rotation
    ((90,), (50,), 16, "fp16", 1, 0, 3, 0, False, "", False),         # rows as they are, no queries
]


@pytest.mark.parametrize("lens,new,page,dtype,layers,hq,hk,axes,interleaved,norms,fused", APPEND)
def test_append(torch_cuda, lens, new, page, dtype, layers, hq, hk, axes, interleaved, norms, fused):
    import torch
    _log(f"paged append lens {lens} new {new} {dtype} {layers} x {hq}/{hk} axes {axes} norms {norms!r}")
    f = Served(lens, new, page, dtype, layers, max(hq, hk), hk, seed=11)
    P, n = f.P, f.total
    if fused:
        qkv = f.randn((layers, n, hq + 2 * hk + 1, D), 2.0)
        q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:hq + 2 * hk]
    else:
        q, k, v = (f.randn((layers, n, h, D), 2.0) if h else None for h in (hq, hk, hk))
    sections = {0: None, 1: (64,), 3: (16, 24, 24)}[axes]
    rng = np.random.default_rng(12)
    pos = rng.integers(-5, 200000, (max(axes, 1), n)).astype(np.int32)
    pos[0, 0] = 2 ** 31 - 1
    pos[-1, -1] = -2 ** 31
    rope = P.Rope(1e6, sections, interleaved) if axes else None
    w = {c: f.randn((layers, D)) + 1 if c in norms else None for c in "qk"}
    before = _bits(f.k), _bits(f.v)
    buf = torch.full((layers * n * max(hq, 1) * D + 2048,), 7.0, dtype=f.dt, device="cuda")
    q_out = buf[1024:-1024].view(layers, n, hq, D) if hq else None
    args = dict(positions=torch.from_numpy(pos).cuda() if axes else None, rope=rope, q_norm=w["q"] if hq else None,
                k_norm=w["k"], eps=1e-5)
    got = P.paged_append(f.cache, f.batch, q, k, v, q_out=q_out, **args)
    torch.cuda.synchronize()
    assert got is q_out and (buf[:1024] == 7).all() and (buf[-1024:] == 7).all()

    def want(x, weight):
        y = _f64(x)
        if weight is not None:
            y = OP.norm(y, _f64(weight)[:, None, None], 1e-5)
        size = np.abs(y)
        if axes:
            y = OP.rotate(y, pos, 1e6, sections, interleaved)
            a, b = (size[..., 0::2], size[..., 1::2]) if interleaved else (size[..., :64], size[..., 64:])
            size = np.repeat(a + b, 2, -1) if interleaved else np.concatenate([a + b] * 2, -1)
        return y, _half_step(dtype) * np.abs(y) + 2.0 ** -18 * size + 2.0 ** -25

    if hq:
        ref, lim = want(q, w["q"])
        assert (np.abs(_f64(q_out) - ref) <= lim).all()
    ref, lim = want(k, w["k"])
    places = OP.new_places(f.table, lens, f.cu, page, f.n_pages, f.max_len)
    assert (None in places) == any(a < b for a, b in zip(lens, new))
    kept = [(i, r) for i, r in enumerate(places) if r is not None]
    i, r = (np.array(x, np.int64) for x in zip(*kept))
    after = _f64(f.k).reshape(layers, hk, -1, D)
    assert (np.abs(after[:, :, r] - ref[:, i].transpose(0, 2, 1, 3)) <= lim[:, i].transpose(0, 2, 1, 3)).all()
    assert np.array_equal(_bits(f.v).reshape(layers, hk, -1, D)[:, :, r], _bits(v.contiguous())[:, i].transpose(0, 2, 1, 3))
    rest = np.setdiff1d(np.arange(f.n_pages * page), r)
    for now, old in zip((_bits(f.k), _bits(f.v)), before):
        assert np.array_equal(now.reshape(layers, hk, -1, D)[:, :, rest], old.reshape(layers, hk, -1, D)[:, :, rest])


@pytest.mark.parametrize("n_seqs", [63, 64, 65, 700, 4097])
def test_append_finds_its_sequence(torch_cuda, n_seqs):
    """Sequences without new tokens between the others, and at both ends."""
    rng = np.random.default_rng(n_seqs)
    new = rng.integers(0, 3, n_seqs)
    new[0] = new[-1] = 0
    lens = [int(n + rng.integers(0, 20)) for n in new]
    f = Served(lens, new.tolist(), 16, "bf16", 1, 1, 1, seed=17)
    k, v = (f.randn((1, f.total, 1, D)) for _ in range(2))
    want = [_bits(x).reshape(-1, D).copy() for x in (f.k, f.v)]
    f.P.paged_append(f.cache, f.batch, None, k, v)
    places = OP.new_places(f.table, f.lens, f.cu, 16, f.n_pages, f.max_len)
    for pool, x in zip(want, (k, v)):
        pool[np.array(places)] = _bits(x).reshape(-1, D)
    for pool, got in zip(want, (f.k, f.v)):
        assert np.array_equal(_bits(got).reshape(-1, D), pool)


@pytest.mark.parametrize("more", [-1, 0, 5])
def test_append_of_2_to_26_tokens(torch_cuda, more):
    """More threads than a grid has along one axis.  The last tokens have pages, the others none."""
    import torch
    from paper_2603_00188_amd import paged as P
    page, n, kept = 256, (1 << 26) + more, 1000
    table = torch.full((1, -(-n // page)), -1, dtype=torch.int32, device="cuda")
    first = (n - kept) // page
    pages = table.shape[1] - first
    table[0, first:] = torch.randperm(pages, device="cuda").to(torch.int32)
    pool = [torch.zeros((1, 1, pages, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = P.PagedCache(*pool, table, torch.tensor([n], dtype=torch.int32, device="cuda"), 1)
    batch = P.NewTokens([0, n])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(26)
    k = torch.zeros((1, n, 1, D), dtype=torch.bfloat16, device="cuda")  # (values too)
    last = torch.randn((n - first * page, D), generator=gen, device="cuda").to(torch.bfloat16)
    k[0, first * page:, 0] = last
    P.paged_append(cache, batch, None, k, k)
    for x in pool:
        got = x[0, 0][table[0, first:].long()].view(-1, D)
        assert torch.equal(got[:len(last)], last) and not got[len(last):].any()


def test_append_drops_rows_without_a_page(torch_cuda):
    import torch
    f = Served((40, 70), (40, 5), 16, "bf16", 1, 4, 2, seed=13)
    f.table[0, 1] = -1
    f.table[1, 4] = f.n_pages
    f.rebuild()
    before = _bits(f.k)
    q, k, v = (f.randn((1, 45, h, D)) for h in (4, 2, 2))
    out = f.P.paged_append(f.cache, f.batch, q, k, v)
    torch.cuda.synchronize()
    assert torch.equal(out, q)  # neither norm nor rotation: the rows as they are
    places = OP.new_places(f.table, f.lens, f.cu, 16, f.n_pages, f.max_len)
    assert sum(p is None for p in places) == 16 + 5
    after = _bits(f.k).reshape(1, 2, -1, D)
    want = before.reshape(1, 2, -1, D).copy()
    for i, r in enumerate(places):
        if r is not None:
            want[:, :, r] = _bits(k)[:, i]
    assert np.array_equal(after, want)


def test_append_special_values(torch_cuda):
    """Norms of zero and huge rows, infinities and NaN that stay in their own head."""
    import torch
    f = Served((16,), (16,), 16, "bf16", 1, 2, 1, seed=14)
    q, k, v = (f.randn((1, 16, h, D)) for h in (2, 1, 1))
    q[0, 0] = 0
    q[0, 1, 0, 3] = float("inf")
    q[0, 2, 1, 3] = float("nan")
    v[0, 5, 0, 7] = float("nan")
    one = torch.ones((1, D), dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(16, dtype=torch.int32, device="cuda").view(1, 16)
    out = f.P.paged_append(f.cache, f.batch, q, k, v, positions=pos, rope=f.P.Rope(), q_norm=one, k_norm=one)
    torch.cuda.synchronize()
    assert not out[0, 0].any()
    assert torch.isfinite(out[0, 1, 1]).all() and torch.isfinite(out[0, 2, 0]).all() and torch.isfinite(out[0, 3:]).all()
    assert torch.isnan(out[0, 2, 1]).all()
    row = OP.place(f.table, 0, 5, 16, f.n_pages)
    assert np.array_equal(_bits(f.v).reshape(-1, D)[row], _bits(v)[0, 5, 0])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
@pytest.mark.parametrize("many", [False, True])
def test_norms_of_rows_of_any_size(torch_cuda, dtype, eps, many):
    """Rows whose squares pass fp32's range, or fall out of it: at the limits of the type, alone and beside others."""
    import torch
    n = 2000 if many else 40  # both forms of the kernel
    f = Served((n,), (n,), 16, dtype, 1, 3, 1, seed=25)
    q, k, v = (f.randn((1, n, h, D)) for h in (3, 1, 1))
    info = torch.finfo(f.dt)
    sizes = [1e10, 2e18, 1e19, 3e25, 1e37, info.max / 8, 1e-15, 1e-20, 1e-25, 1e-35] if dtype == "bf16" else [info.max / 8, info.tiny, 1.0]
    for i, size in enumerate(sizes * 3):
        q[0, i, i % 3] = (q[0, i, i % 3].float() * size).clamp(-info.max, info.max).to(f.dt)
        k[0, i, 0] = (k[0, i, 0].float() * size).clamp(-info.max, info.max).to(f.dt)
    q[0, 35], k[0, 35] = info.max, -info.max
    q[0, 36] = 0
    q[0, 36, :, 9] = info.max  # one element of a row
    k[0, 36] = info.smallest_normal
    w = f.randn((1, D)) + 1
    out = f.P.paged_append(f.cache, f.batch, q, k, v, q_norm=w, k_norm=w, eps=eps)
    u = _half_step(dtype)
    places = OP.new_places(f.table, f.lens, f.cu, 16, f.n_pages, f.max_len)
    for x, y in ((_f64(q)[0], _f64(out)[0]), (_f64(k)[0], _f64(f.k).reshape(1, -1, D)[0][np.array(places)][:, None])):
        ref = OP.norm(x, _f64(w)[0], float(np.float32(eps)))
        assert (np.abs(y - ref) <= (u + 2.0 ** -18) * np.abs(ref) + 2.0 ** -25).all()


# ---------------------------------------------------------------------------
# Compaction into pages
# ---------------------------------------------------------------------------


def _problem(lens, layers, hk, beta, group=2):
    from paper_2603_00188_amd import stlite as S
    cu = np.concatenate([[0], np.cumsum(lens)])
    return S.Problem(layers, group * hk, hk, 1, cu, np.zeros(len(lens) + 1), np.zeros((0, 3)), S.budgets(cu, *beta))


@pytest.mark.parametrize("lens,beta,page,per_layer", [
    ((912,), (1, 5), 16, False), ((100, 3, 257, 64), (1, 4), 16, False), ((100, 3, 257, 64), (1, 1), 64, True),
    ((5, 4), (1, 7), 32, False), ((1000, 2000, 31), (2, 3), 256, False)])
def test_compact_into_pages(torch_cuda, lens, beta, page, per_layer):
    import torch
    layers, hk = 3, 2
    p = _problem(lens, layers, hk, beta)
    cb, cu = p.h["cu_budget"], p.h["cu_seqlens"]
    f = Served([max(int(n), 1) for n in np.diff(cb)], [0] * len(lens), page, "fp16", layers, 4, hk, seed=15)
    f.cache.seq_lens.fill_(-1)
    rng = np.random.default_rng(16)
    lists = layers if per_layer else layers * hk
    kept = np.concatenate([np.sort(np.stack([rng.permutation(n)[:b] for _ in range(lists)]), -1) + a
                           for a, n, b in zip(cu, np.diff(cu), np.diff(cb))], -1).astype(np.int32)
    if kept.size:
        kept[0, -1] = sum(lens)  # out of range: zeros
        kept[-1, 0] = -1
    k, v = (f.randn((layers * hk, sum(lens), D)) for _ in range(2))
    want = [_bits(f.k).reshape(layers * hk, -1, D).copy(), _bits(f.v).reshape(layers * hk, -1, D).copy()]
    if len(lens) > 1 and cb[1] > page:
        f.table[0, 1] = -1  # dropped
        f.rebuild()
    f.P.paged_compact(f.cache, p, k, v, torch.from_numpy(kept).cuda().contiguous(), per_layer=per_layer)
    torch.cuda.synchronize()
    for u in range(layers * hk):
        for s in range(len(lens)):
            for j in range(int(cb[s + 1] - cb[s])):
                r = OP.place(f.table, s, j, page, f.n_pages)
                t = int(kept[u // hk if per_layer else u, cb[s] + j])
                for w, src in zip(want, (k, v)):
                    if r is not None:
                        w[u, r] = _bits(src[u, t]) if 0 <= t < sum(lens) else 0
    assert np.array_equal(_bits(f.k).reshape(layers * hk, -1, D), want[0])
    assert np.array_equal(_bits(f.v).reshape(layers * hk, -1, D), want[1])
    assert f.cache.seq_lens.tolist() == np.diff(cb).tolist()


# ---------------------------------------------------------------------------
# Together, as a program serves
# ---------------------------------------------------------------------------


def _step(f, q, k, v, pos, rope, norms):
    """One serving step on f's cache: lengths, append, attention."""
    counts = np.diff(f.cu)
    import torch
    f.cache.seq_lens += torch.from_numpy(counts).cuda()
    qr = f.P.paged_append(f.cache, f.batch, q, k, v, positions=pos, rope=rope, q_norm=norms[0], k_norm=norms[1])
    return qr, f.P.paged_attention(f.cache, f.batch, qr)


def test_compress_then_serve(torch_cuda):
    """The compression pass straight into pages, then a prompt of several tokens,
    single tokens and drafted ones, each attending to all that is there: the
    compressed rows, and every token appended since."""
    import torch
    from paper_2603_00188_amd import paged as P
    from paper_2603_00188_amd import stlite as S
    from tests import gpu_harness as H
    from tests.test_gpu_parity import SMALL
    case = H.Case(SMALL["ragged"])
    w, prob = case.w, case.prob
    res = case.run()
    cache = P.PagedCache.alloc(case.n_layers, w.n_q_heads, w.n_kv_heads, prob.n_seqs, int(np.diff(case.cu_budget).max()) + 90,
                               page_size=16)
    case.out.kept.fill_(-1)
    S.compress(prob, case.dq, case.dk, case.dv, case.out, alpha=w.alpha, cache=cache)
    torch.cuda.synchronize()
    assert np.array_equal(case.out.kept[:, :prob.total_budget].cpu().numpy(), res["kept"])
    assert cache.seq_lens.tolist() == np.diff(case.cu_budget).tolist()
    table = cache.page_table.cpu().numpy()
    for s in range(prob.n_seqs):
        rows = [OP.place(table, s, j, 16, cache.n_pages) for j in range(int(np.diff(case.cu_budget)[s]))]
        a, b = case.cu_budget[s:s + 2]
        assert np.array_equal(_bits(cache.k).reshape(prob.units, -1, D)[:, rows].view(np.uint16), res["k_out"][:, a:b])
        assert np.array_equal(_bits(cache.v).reshape(prob.units, -1, D)[:, rows].view(np.uint16), res["v_out"][:, a:b])

    f = Served([16], [1], 16, "bf16", 1, w.n_q_heads, w.n_kv_heads)  # (its generator and comparison)
    f.layers, f.k, f.v, f.cache, f.table, f.max_len = case.n_layers, cache.k, cache.v, cache, table, cache.max_len
    f.n_pages, norms = cache.n_pages, (None, None)
    rope, seen = P.Rope(1e6, (16, 24, 24)), np.diff(case.cu_seqlens if hasattr(case, "cu_seqlens") else case.lay.cu_seqlens).copy()
    for new in ([30] + [7] * (prob.n_seqs - 1), [1] * prob.n_seqs, [0] + [1] * (prob.n_seqs - 1), [4] * prob.n_seqs, [1] * prob.n_seqs):
        f.new, f.cu = new, np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        f.total, f.batch = int(f.cu[-1]), P.NewTokens(f.cu)
        q, k, v = (f.randn((f.layers, f.total, h, D)) for h in (w.n_q_heads, w.n_kv_heads, w.n_kv_heads))
        pos = np.concatenate([seen[s] + np.arange(n) for s, n in enumerate(new)]).astype(np.int32)
        pos = torch.from_numpy(np.stack([pos, pos // 80, pos % 80])).cuda().contiguous()
        qr, out = _step(f, q, k, v, pos, rope, norms)
        torch.cuda.synchronize()
        f.lens = cache.seq_lens.tolist()
        cache.validate(f.batch, table, f.lens)
        f.compare(qr, out)
        seen += np.array(new)
    assert f.lens == [int(b) + n for b, n in zip(np.diff(case.cu_budget), (np.array([36] + [14] * (prob.n_seqs - 1))))]


def test_layers_one_by_one(torch_cuda):
    """What a model does: layer after layer, each on its own slice of the cache."""
    import torch
    for new in (1, 6):
        f = Served((500, 20, 77), (new,) * 3, 32, "bf16", 4, 8, 2, seed=17)
        q, k, v = (f.randn((4, f.total, h, D)) for h in (8, 2, 2))
        pos = torch.arange(f.total, dtype=torch.int32, device="cuda").view(1, -1)
        qs = []
        for layer in range(4):
            one, at = f.cache.layer(layer), slice(layer, layer + 1)
            qs.append(f.P.paged_append(one, f.batch, q[at], k[at], v[at], positions=pos, rope=f.P.Rope()))
        outs = torch.cat([f.P.paged_attention(f.cache.layer(i), f.batch, qs[i]) for i in range(4)])
        pools = f.k.clone(), f.v.clone()
        whole = f.P.paged_append(f.cache, f.batch, q, k, v, positions=pos, rope=f.P.Rope())
        torch.cuda.synchronize()
        assert torch.equal(torch.cat(qs), whole) and torch.equal(pools[0], f.k) and torch.equal(pools[1], f.v)
        f.compare(whole, outs)
        f.compare(whole, f.attend(whole))


@pytest.mark.parametrize("new", [1, 5])
def test_graph_of_a_step(torch_cuda, new):
    """A captured step (lengths, append, attention) follows the lengths and inputs of
    each replay; eager work in between, and a second graph on the same workspace."""
    import torch
    f = Served((300, 40, 0), (new,) * 3, 16, "bf16", 2, 8, 2, seed=18, spare=0)
    f.table = np.arange(3 * 40, dtype=np.int32).reshape(3, 40)[:, ::-1].copy()
    f.n_pages, f.max_len = 120, 640
    f.k, f.v = f.randn((2, 2, 120, 16, D)), f.randn((2, 2, 120, 16, D))
    f.rebuild()
    counts = torch.full((3,), new, dtype=torch.int32, device="cuda")
    q, k, v = (f.randn((2, f.total, h, D)) for h in (8, 2, 2))
    pos = torch.zeros((1, f.total), dtype=torch.int32, device="cuda")
    rope, ws = f.P.Rope(), f.cache.workspace(f.batch)
    q_out, out, out2 = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)

    def step(out):
        f.cache.seq_lens.add_(counts)
        pos.add_(1)
        f.P.paged_append(f.cache, f.batch, q, k, v, positions=pos, rope=rope, q_out=q_out)
        f.P.paged_attention(f.cache, f.batch, q_out, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for o in (out, out2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(o)
        graphs.append(g)
    f.cache.seq_lens.copy_(torch.tensor([300, 40, 0], dtype=torch.int32))
    pos.zero_()
    start_k, start_v = f.k.clone(), f.v.clone()
    inputs = [[f.randn(t.shape) for t in (q, k, v)] for _ in range(4)]
    got = []
    for i, xs in enumerate(inputs):
        for t, x in zip((q, k, v), xs):
            t.copy_(x)
        (out, out2)[i % 2].fill_(3.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got.append((out, out2)[i % 2].clone())
    assert f.cache.seq_lens.tolist() == [300 + 4 * new, 40 + 4 * new, 4 * new]
    end_k = f.k.clone()
    f.k.copy_(start_k)
    f.v.copy_(start_v)
    f.cache.seq_lens.copy_(torch.tensor([300, 40, 0], dtype=torch.int32))
    pos.zero_()
    for xs, g in zip(inputs, got):
        for t, x in zip((q, k, v), xs):
            t.copy_(x)
        out.fill_(5.0)
        step(out)
        torch.cuda.synchronize()
        assert torch.equal(out, g)
        f.lens = f.cache.seq_lens.tolist()
        f.compare(q_out, out)
    assert torch.equal(f.k, end_k)


def test_streams(torch_cuda):
    """A call on a stream that is not the current one, its tensors made for it."""
    import torch
    f = Served((3000, 40), (3, 3), 32, "bf16", 2, 8, 2, seed=19)
    q, k, v = (f.randn((2, 6, h, D)) for h in (8, 2, 2))
    want_q = f.P.paged_append(f.cache, f.batch, q, k, v)
    want = f.P.paged_attention(f.cache, f.batch, want_q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        side.wait_stream(torch.cuda.current_stream())
        got_q = f.P.paged_append(f.cache, f.batch, q, k, v, stream=stream)
        got = f.P.paged_attention(f.cache, f.batch, got_q, stream=stream)
        junk = [torch.full_like(want, 9.0) for _ in range(8)]  # whatever the current stream allocates meanwhile
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(got_q, want_q) and len(junk) == 8


@pytest.mark.parametrize("new", [1, 3])
def test_dropped_tensors_on_another_stream(torch_cuda, new):
    """A call on a busy stream whose batch and inputs are dropped at once: their memory is not given to others before the
    kernels have run.  (What would take their place is another batch of as many tokens: in bounds either way.)"""
    import torch
    f = Served((3000, 40, 700), (new,) * 3, 32, "bf16", 2, 8, 2, seed=27)
    n = 3 * new
    other = [0, n - 1, n - 1, n] if new == 3 else [0, 0, 2, 3]
    rows = [f.randn((2, n, h, D)) for h in (8, 2, 2)]
    want_q = f.P.paged_append(f.cache, f.batch, *rows)
    want = f.P.paged_attention(f.cache, f.batch, want_q)
    pools = f.k.clone(), f.v.clone()
    f.k.zero_()
    f.k.copy_(pools[0])
    busy = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.mm(busy, busy)
    got_q = f.P.paged_append(f.cache, f.P.NewTokens(f.cu), *(x.clone() for x in rows), stream=side)
    got = f.P.paged_attention(f.cache, f.P.NewTokens(f.cu), got_q, stream=side)
    others = [f.P.NewTokens(other) for _ in range(8)] + [torch.full_like(x, 9.0) for x in rows for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got_q, want_q) and torch.equal(got, want) and len(others) == 20
    assert torch.equal(f.k, pools[0]) and torch.equal(f.v, pools[1])


@pytest.mark.parametrize("new", [1, 5])
def test_buffers_that_only_touch(torch_cuda, new):
    """One allocation holds queries, output, workspace and pool without a byte between them, and an append's output lies
    between its inputs' layers."""
    import torch
    f = Served((300, 40), (new, new), 16, "bf16", 2, 8, 2, seed=28)
    n, size = 2 * 2 * new * 8 * D, max(f.cache.workspace_size(f.batch), 256) // 2
    pool = f.k.numel()
    buf = torch.empty(2 * pool + 2 * n + size, dtype=f.dt, device="cuda")
    at = np.cumsum([0, n, n, size, pool, pool])
    q, out, ws, k, v = (buf[a:b] for a, b in zip(at, at[1:]))
    q, out, k, v = q.view(2, -1, 8, D), out.view(2, -1, 8, D), k.view(f.k.shape), v.view(f.v.shape)
    k.copy_(f.k)
    v.copy_(f.v)
    q.copy_(f.randn(q.shape))
    cache = f.P.PagedCache(k, v, f.cache.page_table, f.cache.seq_lens, 8, f.max_len)
    f.P.paged_attention(cache, f.batch, q, out=out, workspace=ws)
    f.compare(q, out)
    m = f.total * (8 + 2 * 2) * D  # a layer of a fused projection
    buf = f.randn((2 * m + n,))
    qkv = torch.as_strided(buf, (2, f.total, 12, D), (m + n, 12 * D, D, 1))
    parts = qkv.split([8, 2, 2], 2)
    f.P.paged_append(cache, f.batch, *parts, q_out=buf[m:m + n].view(2, f.total, 8, D))
    assert torch.equal(buf[m:m + n].view(2, f.total, 8, D), parts[0])
    places = np.array(OP.new_places(f.table, f.lens, f.cu, 16, f.n_pages, f.max_len))
    assert np.array_equal(_bits(k).reshape(2, 2, -1, D)[:, :, places], _bits(parts[1].contiguous()).transpose(0, 2, 1, 3))


@pytest.mark.parametrize("layers,seqs,hq,extend", [(4, 65535, 128, False), (4, 65535, 128, True), (65535, 2, 2, False),
                                                   (65535, 2, 2, True)])
def test_limits_of_a_call(torch_cuda, layers, seqs, hq, extend):
    """As many sequences, or layers, as a call may have, and queries of more than 2^32 elements.  Every token sees one key,
    so that its output is that key's value, but for the second token of the last sequence, which sees two equal keys."""
    import torch
    from paper_2603_00188_amd import paged as P
    gen = torch.Generator(device="cuda")
    gen.manual_seed(32)
    new = torch.ones(seqs, dtype=torch.int64)
    new[-1] += extend
    batch = P.NewTokens(torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]))
    n = batch.total
    table = torch.randperm(seqs, generator=gen, device="cuda").to(torch.int32).view(seqs, 1)
    pool = [torch.full((layers, 1, seqs, 16, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache = P.PagedCache(*pool, table, new.to(torch.int32).cuda(), hq)
    k, v = (torch.randn((layers, n, 1, D), generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    if extend:
        k[:, -1] = k[:, -2]
    q = torch.randn((1, n, hq, D), generator=gen, device="cuda", dtype=torch.bfloat16).expand(layers, -1, -1, -1)
    rotated = P.paged_append(cache, batch, q, k, v)
    assert torch.equal(rotated, q)
    first = slice(0, n - extend)
    at = table[:, 0].long()
    for x, rows in zip(pool, (k, v)):
        assert torch.equal(x[:, 0, at, 0], rows[:, first, 0]) and torch.isnan(x[:, 0, at[:-1], 1:]).all()
        if extend:
            assert torch.equal(x[:, 0, at[-1], 1], rows[:, -1, 0])
    out = P.paged_attention(cache, batch, rotated)
    for layer in range(0, layers, max(layers // 64, 1)):
        assert torch.equal(out[layer, first], v[layer, first].expand(-1, hq, -1)), layer
    assert torch.equal(out[-1, first], v[-1, first].expand(-1, hq, -1))
    if extend:
        mean = (v[:, -1].float() + v[:, -2].float()) / 2
        bound = 2.0 ** -8 * mean.abs() + (2.0 ** -8 + 2.0 ** -20) * (v[:, -1].float().abs() + v[:, -2].float().abs()) / 2
        assert ((out[:, -1].float() - mean).abs() <= bound + 2.0 ** -100).all()


def test_dense_decode_agrees(torch_cuda):
    """The dense decode call and the paged one over identity pages, on the same cache."""
    import torch
    from paper_2603_00188_amd import paged as P
    from paper_2603_00188_amd import stlite as S
    lens, hk, G = (512,), 2, 7
    p = _problem(lens, 2, hk, (1, 5), group=G)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(20)
    k, v = (torch.randn((2, hk, 512, D), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((2, 1, G * hk, D), generator=gen, device="cuda").to(torch.bfloat16)
    dense = S.decode(p, q, k, v, S.CACHE_FULL)
    cache = P.PagedCache(k.view(2, hk, 32, 16, D), v.view(2, hk, 32, 16, D),
                         torch.arange(32, dtype=torch.int32, device="cuda").view(1, 32),
                         torch.tensor([512], dtype=torch.int32, device="cuda"), G * hk)
    out = P.paged_attention(cache, P.NewTokens([0, 1]), q)
    torch.cuda.synchronize()
    assert (out.float() - dense).abs().le(2.0 ** -8 * dense.abs() + 2.0 ** -16 * v.float().abs().max()).all()


@pytest.mark.parametrize("hq,hk,shares", [(4, 1, 4), (28, 4, 8)])
def test_two_calls_at_once(torch_cuda, hq, hk, shares):
    """Two streams, two workspaces, one cache."""
    import torch
    f = Served((4000, 1000), (1, 1), 32, "bf16", 2, hq, hk, seed=21)
    qs = [f.randn((2, 2, hq, D)) for _ in range(shares)]
    want = [f.attend(q) for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [f.cache.workspace(f.batch) for _ in range(2)]
    outs = [torch.empty_like(q) for q in qs]
    torch.cuda.synchronize()
    for i, q in enumerate(qs):
        f.P.paged_attention(f.cache, f.batch, q, out=outs[i], workspace=ws[i % 2], stream=streams[i % 2])
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert torch.equal(a, b)
