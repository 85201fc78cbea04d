"""Timed cases of serving from pages that hold keys and values in 4 bits, and of the steps around attention in a loop that
drafts tokens.

* ``append``  -- new tokens' keys normalised, rotated and stored in 4 bits, values too; queries in 16 bits; the new rows read back;
* ``compact`` -- the kept rows of the compression into 4-bit pages, and read back;
* ``decode``  -- attention of one new token per sequence over 4-bit pages;
* ``extend``  -- causal attention of several new tokens per sequence over them;
* ``grow``    -- pages for the tokens that sequences get next, out of a list of free ones, and every new token's place;
  what a sequence gave back before (the last step's pages) goes into the list first;
* ``verify``  -- drafted tokens against the target's probabilities with given random numbers, and the next token.

A page of a 4-bit pool is ``page`` rows of 64 bytes of codes and then ``page`` rows of 4 scale bytes.  A row is four blocks of
32 values; a value is its code's (element 2 i in the low half of byte i: a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6) times
2^(byte - 127) of its block.  The scale is the least power of two of which 7 times reaches the block's greatest value.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
ROW = 68  # bytes of a row in a 4-bit pool
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

# The benchmark's models: 28 query heads over 4 kv heads, three position axes.
BASE = dict(kind="decode", dtype="bf16", layers=28, q_heads=28, kv_heads=4, page=64, seqs=1, len_min=678, len_max=678,
            new_min=1, new_max=1, layout=0, axes=3, interleaved=False, norm=False, fused=False, beta_num=1, beta_den=5,
            room=1.0, vocab=0, draft="full")


def listed():
    return [
        # a serving batch's next tokens, a model with normalised heads and one position axis
        dict(BASE, name="append_batch", kind="append", dtype="fp16", q_heads=32, kv_heads=8, seqs=64, len_min=50,
             len_max=900, axes=1, interleaved=True, norm=True, page=16),
        # the next screenshot and its text, all layers, out of one fused projection
        dict(BASE, name="append_screen", kind="append", len_min=30105, len_max=30105, new_min=3136, new_max=3136,
             fused=True),
        # the first step's cache into pages (one screenshot and the instruction)
        dict(BASE, name="compact_step", kind="compact", len_min=3392, len_max=3392),
        # the fifty-step trajectory's cache into pages
        dict(BASE, name="compact_trajectory", kind="compact", len_min=150528, len_max=150528),
        # one layer's attention for the token behind the compressed first step: latency
        dict(BASE, name="decode_token", layers=1, page=16),
        # a decode step of all layers over the compressed trajectory
        dict(BASE, name="decode_step", len_min=30105, len_max=30105),
        # a batch in which every sequence checks a few drafted tokens, small pages
        dict(BASE, name="extend_few", kind="extend", dtype="fp16", layers=2, q_heads=32, kv_heads=8, seqs=16, len_min=1,
             len_max=8000, new_min=1, new_max=5, page=16, layout=5),
        # the next screenshot and its text over the compressed trajectory, one layer
        dict(BASE, name="extend_screen", kind="extend", layers=1, len_min=30105, len_max=30105, new_min=3136,
             new_max=3136),
        # a serving batch's next tokens: few of the sequences need a page
        dict(BASE, name="grow_step", kind="grow", seqs=64, len_min=1, len_max=8000, page=16, layout=1),
        # prompts and drafted tokens of a large batch, more than the free pages hold
        dict(BASE, name="grow_prompts", kind="grow", seqs=1000, len_min=0, len_max=2000, new_min=0, new_max=2999, page=16,
             layout=2, room=0.9),
        # one sequence's few drafted tokens, a small vocabulary: latency
        dict(BASE, name="verify_few", kind="verify", dtype="fp32", vocab=32000, new_min=5, new_max=5),
        # a batch's drafts, a large vocabulary
        dict(BASE, name="verify_batch", kind="verify", dtype="fp32", vocab=131072, seqs=64, new_min=1, new_max=6, layout=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def _cost(case):
    w = work(case)
    # the plain form of attention holds every sequence padded to the longest
    pad = case["layers"] * case["seqs"] * (case["len_max"] + case["new_max"])
    pairs = pad * case["q_heads"] * case["new_max"] if case["kind"] in ("decode", "extend") else 0
    return {"bytes": w["bytes"], "flops": w["flops"], "pairs": pairs, "rows": pad * case["kv_heads"],
            "tokens": case["seqs"] * case["new_max"], "probs": case["seqs"] * case["new_max"] * case["vocab"]}


def draw(rng):
    """Another case of the ranges above, no dearer than the largest of its kind."""
    top = {}
    for c in listed():
        for key, v in _cost(c).items():
            top[c["kind"], key] = max(v, top.get((c["kind"], key), 0))
    while True:
        kind = rng.choice(["append", "compact", "decode", "decode", "extend", "extend", "grow", "verify", "verify"])
        q_heads, kv_heads = rng.choice([(28, 4), (28, 4), (16, 2), (32, 8), (24, 4), (8, 8), (12, 1), (20, 1)])
        c = dict(BASE, kind=kind, dtype=rng.choice(["bf16", "bf16", "fp16"]), layers=_log_int(rng, 1, 28), q_heads=q_heads,
                 kv_heads=kv_heads, page=rng.choice([16, 32, 64, 128, 256]), layout=rng.randrange(1 << 16),
                 axes=rng.choice([1, 3]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.5,
                 fused=rng.random() < 0.5, beta_num=rng.choice([1, 1, 2, 3]), beta_den=rng.choice([5, 7, 10]))
        c["seqs"] = _log_int(rng, 1, 8 if kind == "compact" else 64)
        c["len_max"] = _log_int(rng, 100, 150000)
        c["len_min"] = rng.choice([c["len_max"], _log_int(rng, 1, c["len_max"])])
        if kind == "compact":
            c["len_min"] = max(c["len_min"], 40)
        elif kind == "extend":
            c["new_max"] = _log_int(rng, 2, 3500)
            c["new_min"] = rng.choice([c["new_max"], rng.randint(1, c["new_max"])])
            if rng.random() < 0.3:
                c["len_min"] = c["len_max"] = 0
        elif kind == "append":
            c["new_max"] = rng.choice([1, _log_int(rng, 1, 3500)])
            c["new_min"] = rng.choice([c["new_max"], rng.randint(1, c["new_max"])])
        elif kind == "grow":
            c.update(seqs=_log_int(rng, 1, 1000), len_max=_log_int(rng, 1, 8000), layers=1, room=rng.choice([1.0, 1.0, 0.8]))
            c["len_min"] = rng.randint(0, c["len_max"])
            c["new_max"] = rng.choice([1, _log_int(rng, 1, 3000)])
            c["new_min"] = rng.randint(0, c["new_max"])
        elif kind == "verify":
            c.update(seqs=_log_int(rng, 1, 64), new_max=rng.randint(1, 8), vocab=_log_int(rng, 300, 131072), len_min=678,
                     len_max=678, layers=1, dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                     draft=rng.choice(["full", "full", "token"]))
            c["new_min"] = rng.randint(1, c["new_max"])
        if all(v <= top[kind, key] for key, v in _cost(c).items()):
            return c


def _lengths(case):
    """Cached and new tokens of every sequence; with several sequences the longest is among them."""
    r = random.Random(case["layout"])
    old = [r.randint(case["len_min"], case["len_max"]) for _ in range(case["seqs"])]
    new = [r.randint(case["new_min"], case["new_max"]) for _ in range(case["seqs"])]
    old[0], new[0] = case["len_max"], case["new_max"]
    return old, new


def _budgets(case):
    return [n * case["beta_num"] // case["beta_den"] for n in _lengths(case)[0]]


# ---------------------------------------------------------------------------
# The 4-bit rows
# ---------------------------------------------------------------------------

RANGE = {"bf16": (-120, 125), "fp16": (-14, 13)}  # of a scale's exponent


def _quantised(x, dtype):
    """Rows [..., 128] in 32 or 64 bits as codes [..., 64] and scale bytes [..., 4], and the values that they stand for."""
    x = x.unflatten(-1, (4, 32))
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e, m in [1/2, 1); 7 2^(e - 3) = 0.875 2^e
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(*RANGE[dtype])
    e = torch.where(top == 0, RANGE[dtype][0], e)
    y = torch.ldexp(x, -e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.clamp(torch.round(a / step) * step, max=6.0)  # (half to even, as the codes' last bit goes)
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(y)
    value = torch.ldexp(torch.copysign(a, y), e).flatten(-2)
    code = code.flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e.squeeze(-1) + 127).to(torch.uint8), value


def _split(pool, page):
    """Codes [.., pages, page, 64] and scales [.., pages, page, 4] of a pool [.., pages, page * 68], as views."""
    return pool[..., :page * 64].unflatten(-1, (page, 64)), pool[..., page * 64:].unflatten(-1, (page, 4))


def _values(codes, scales):
    """The values of rows, in 32 bits."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).to(torch.int32)
    a = c & 7
    a = torch.where(a < 4, a * 0.5, torch.where(a < 6, a - 2.0, a * 2.0 - 8.0))
    a = torch.where(c >= 8, -a, a)
    return torch.ldexp(a.unflatten(-1, (4, 32)), scales.to(torch.int32).unsqueeze(-1) - 127).flatten(-2)


# ---------------------------------------------------------------------------
# States
# ---------------------------------------------------------------------------

def _prepare_verify(case, gen):
    _, new = _lengths(case)
    total, vocab, dt = sum(new), case["vocab"], TYPES[case["dtype"]]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    # the draft's distribution is near the target's; its tokens are drawn from it
    logits = torch.randn((total, vocab), generator=gen, device=DEV) * 3.0
    target = torch.softmax(logits, -1)
    draft = torch.softmax(logits + 0.5 * torch.randn((total, vocab), generator=gen, device=DEV), -1)
    st = dict(case=case, cu_new=cu, cu_new_dev=torch.from_numpy(cu).to(DEV), target=target.to(dt),
              tokens=torch.multinomial(draft, 1, generator=gen).view(-1).to(torch.int32),
              accept=torch.rand(total, generator=gen, device=DEV), pick=torch.rand(case["seqs"], generator=gen, device=DEV),
              draft=draft.to(dt) if case["draft"] == "full" else None)
    st["out"] = torch.empty(total, dtype=torch.int32, device=DEV)
    st["n_out"] = torch.empty(case["seqs"], dtype=torch.int32, device=DEV)
    return st


def _prepare_grow(case, gen):
    old, new = _lengths(case)
    page = case["page"]
    max_len = max(case["len_max"] + case["new_max"] // 2, 1) if case["room"] < 1 else max(case["len_max"] + case["new_max"], 1)
    held = [-(-n // page) for n in old]
    need = [max(-(-(a + b) // page) - h, 0) if a + b <= max_len else 0 for a, b, h in zip(old, new, held)]
    spare = int(sum(need) * case["room"]) if case["room"] < 1 else sum(need) + 3
    n_pages, max_pages = sum(held) + spare + 1, -(-max_len // page)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((case["seqs"], max_pages), -1, dtype=torch.int32)
    at = 0
    host = order.cpu()
    for s, n in enumerate(held):
        table[s, :n] = host[at:at + n]
        at += n
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    free[:n_pages - at] = order[at:]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return dict(case=case, page_table=table.to(DEV), seq_lens=dev(old), base=dev(old), held=dev(held), free=free,
                n_free=dev([n_pages - at]), cu_new=cu, cu_new_dev=torch.from_numpy(cu).to(DEV), max_len=max_len,
                slots=torch.empty(int(cu[-1]), dtype=torch.int32, device=DEV),
                k_pool=torch.zeros((1, 1, n_pages, page * ROW), dtype=torch.uint8, device=DEV),
                v_pool=torch.zeros((1, 1, n_pages, page * ROW), dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if case["kind"] == "verify":
        return _prepare_verify(case, gen)
    if case["kind"] == "grow":
        return _prepare_grow(case, gen)
    dt, layers, hq, hk, page = TYPES[case["dtype"]], case["layers"], case["q_heads"], case["kv_heads"], case["page"]
    old, new = _lengths(case)
    if case["kind"] == "compact":
        old, new = _budgets(case), [0] * case["seqs"]
    lens = [a + b for a, b in zip(old, new)]
    max_len = max(max(lens), 1)
    max_pages = -(-max_len // page)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3

    def randn(shape, scale=1.0):
        x = torch.empty(shape, dtype=dt, device=DEV)
        for layer in range(shape[0]):
            x[layer] = torch.randn(shape[1:], generator=gen, device=DEV) * scale
        return x

    def pool(scale):
        """Every page is in use somewhere: what lies behind a sequence's end is another's old rows."""
        p = torch.empty((layers, hk, n_pages, page * ROW), dtype=torch.uint8, device=DEV)
        codes, scales = _split(p, page)
        for layer in range(layers):
            x = torch.randn((hk, n_pages, page, D), generator=gen, device=DEV) * scale
            codes[layer], scales[layer], _ = _quantised(x.to(dt).float(), case["dtype"])
        return p

    st = dict(case=case, k_pool=pool(D ** -0.5), v_pool=pool(1.0), max_len=max_len)
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros((case["seqs"], max_pages), dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    st["page_table"] = table
    st["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if case["kind"] == "compact":
        lengths = _lengths(case)[0]
        total, budget = sum(lengths), sum(old)
        st["cu_seqlens"] = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        st["cu_budget"] = np.concatenate([[0], np.cumsum(old)]).astype(np.int32)
        st["cu_budget_dev"] = torch.from_numpy(st["cu_budget"]).to(DEV)
        st["k"], st["v"] = randn((layers * hk, total, D), D ** -0.5), randn((layers * hk, total, D))
        kept = torch.empty((layers * hk, budget), dtype=torch.int32, device=DEV)
        for s in range(case["seqs"]):
            a, b = (int(x) for x in st["cu_seqlens"][s:s + 2])
            c, d = (int(x) for x in st["cu_budget"][s:s + 2])
            for u in range(layers * hk):
                kept[u, c:d] = (torch.randperm(b - a, generator=gen, device=DEV)[:d - c].sort().values + a).to(torch.int32)
        st["kept"] = kept
        st["k_out"], st["v_out"] = (torch.empty((layers, budget, hk, D), dtype=dt, device=DEV) for _ in range(2))
        return st
    st["cu_new"] = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    st["cu_new_dev"] = torch.from_numpy(st["cu_new"]).to(DEV)
    total = int(st["cu_new"][-1])
    if case["kind"] == "append":
        scale = 3.0 if case["norm"] else D ** -0.5
        if case["fused"]:
            qkv = randn((layers, total, hq + 2 * hk, D), scale)
            st["q"], st["k"], st["v"] = qkv.split([hq, hk, hk], dim=2)
        else:
            st["q"], st["k"], st["v"] = (randn((layers, total, h, D), scale) for h in (hq, hk, hk))
        # positions go on from the uncompressed context; a screenshot's rows and columns on axes of their own
        base = torch.repeat_interleave(torch.tensor([5 * n for n in old], device=DEV), torch.tensor(new, device=DEV))
        step = torch.arange(total, device=DEV)
        axes = [base + step, base + step // 80, base + step % 80][:case["axes"]]
        st["positions"] = torch.stack(axes).to(torch.int32).contiguous()
        st["theta"], st["sections"] = 1e6, (16, 24, 24) if case["axes"] == 3 else (64,)
        st["q_norm"] = st["k_norm"] = None
        if case["norm"]:
            st["q_norm"], st["k_norm"] = (1.0 + randn((layers, D), 0.2) for _ in range(2))
        st["q_out"] = torch.empty((layers, total, hq, D), dtype=dt, device=DEV)
        st["k_out"], st["v_out"] = (torch.empty((layers, total, hk, D), dtype=dt, device=DEV) for _ in range(2))
        return st
    # queries near the sum of a few of their sequence's keys, so that the softmax has peaks; the noise keeps its tail
    codes, scales = _split(st["k_pool"], page)
    at = table[:, 0].long()
    first = _values(codes[:, :, at, :4], scales[:, :, at, :4]).sum(3)  # [layers, kv, seqs, D]
    rows = torch.repeat_interleave(torch.arange(case["seqs"], device=DEV), torch.tensor(new, device=DEV))
    st["q"] = torch.empty((layers, total, hq, D), dtype=dt, device=DEV)
    for layer in range(layers):
        aim = first[layer][:, rows].permute(1, 0, 2).unsqueeze(2)  # [total, kv, 1, D]
        noise = torch.randn((total, hk, hq // hk, D), generator=gen, device=DEV)
        st["q"][layer] = (64.0 * aim + 24.0 * noise).reshape(total, hq, D)
    st["out"] = torch.empty((layers, total, hq, D), dtype=dt, device=DEV)
    return st


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _new_slots(st):
    """Sequence of every new token, its index in the sequence and its row in the pool."""
    cu = st["cu_new_dev"].long()
    i = torch.arange(int(st["cu_new"][-1]), device=DEV)
    seq = torch.searchsorted(cu, i, right=True) - 1
    at = st["seq_lens"].long()[seq] - cu[seq + 1] + i
    page = st["case"]["page"]
    return seq, at, st["page_table"].long()[seq, at // page] * page + at % page


def _plain_rotated(x, w, st, wide=False):
    """Norm (where given) and rotation of [layers, tokens, heads, D] in 32 bits, the angles in 64; wide: all in 64."""
    x = x.double() if wide else x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.to(x.dtype)[:, None, None]
    half = D // 2
    freq = st["theta"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    axis = torch.repeat_interleave(torch.arange(len(st["sections"]), device=DEV), torch.tensor(st["sections"], device=DEV))
    angle = st["positions"].double()[axis].T * freq
    cos, sin = angle.cos().to(x.dtype)[None, :, None], angle.sin().to(x.dtype)[None, :, None]
    if st["case"]["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _plain_store(st, pool, unit_rows, slot):
    """Rows [layers, kv, tokens, 128] in 32 or 64 bits into the pool's rows `slot`; the values stored."""
    case = st["case"]
    codes, scales, value = _quantised(unit_rows, case["dtype"])
    c, s = _split(pool, case["page"])
    at, row = slot // case["page"], slot % case["page"]
    c[:, :, at, row] = codes
    s[:, :, at, row] = scales
    return value


def _plain_append(st):
    dt = TYPES[st["case"]["dtype"]]
    st["q_out"].copy_(_plain_rotated(st["q"], st["q_norm"], st).to(dt))
    _, _, slot = _new_slots(st)
    # (which code a key gets turns on the side of a border that it lies on: in 64 bits)
    k = _plain_store(st, st["k_pool"], _plain_rotated(st["k"], st["k_norm"], st, wide=True).transpose(1, 2), slot)
    v = _plain_store(st, st["v_pool"], st["v"].float().transpose(1, 2), slot)
    st["k_out"].copy_(k.transpose(1, 2).to(dt))
    st["v_out"].copy_(v.transpose(1, 2).to(dt))
    return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}


def _plain_compact(st):
    case, page, dt = st["case"], st["case"]["page"], TYPES[st["case"]["dtype"]]
    layers, hk = case["layers"], case["kv_heads"]
    cu = st["cu_budget_dev"].long()
    j = torch.arange(int(st["cu_budget"][-1]), device=DEV)
    seq = torch.searchsorted(cu, j, right=True) - 1
    at = j - cu[seq]
    slot = st["page_table"].long()[seq, at // page] * page + at % page
    unit = torch.arange(layers * hk, device=DEV)[:, None]
    kept = st["kept"].long()
    k = _plain_store(st, st["k_pool"], st["k"][unit, kept].float().unflatten(0, (layers, hk)), slot)
    st["k_out"].copy_(k.transpose(1, 2).to(dt))
    del k
    v = _plain_store(st, st["v_pool"], st["v"][unit, kept].float().unflatten(0, (layers, hk)), slot)
    st["v_out"].copy_(v.transpose(1, 2).to(dt))
    st["seq_lens"].copy_(cu[1:] - cu[:-1])
    return {"k": st["k_out"], "v": st["v_out"], "seq_lens": st["seq_lens"]}


def _plain_attention(st):
    case = st["case"]
    layers, hq, hk, seqs, page = case["layers"], case["q_heads"], case["kv_heads"], case["seqs"], case["page"]
    G, n = hq // hk, case["new_max"]
    cu, lens = st["cu_new_dev"].long(), st["seq_lens"].long()
    count = cu[1:] - cu[:-1]
    total = int(st["cu_new"][-1])
    t = torch.arange(n, device=DEV)
    rows = (cu[:-1, None] + t).clamp(max=total - 1)  # [seqs, n], padded
    q = st["q"].float()[:, rows].view(layers, seqs, n, hk, G, D).permute(0, 3, 1, 4, 2, 5).reshape(layers, hk, seqs, G * n, D)
    table = st["page_table"].long()
    codes, scales = _split(st["k_pool"][:, :, table], page)
    k = _values(codes, scales).view(layers, hk, seqs, -1, D)
    x = torch.matmul(q, k.transpose(-1, -2))
    del k
    x *= D ** -0.5
    last = (lens - count)[:, None] + t  # the last key that a new token sees
    seen = torch.arange(x.shape[-1], device=DEV) <= last[..., None]  # [seqs, n, keys]
    x = x.view(layers, hk, seqs, G, n, -1).masked_fill_(~seen[:, None], -math.inf).view(layers, hk, seqs, G * n, -1)
    x -= x.amax(-1, keepdim=True)
    p = x.exp_()
    total_p = p.sum(-1, keepdim=True)
    codes, scales = _split(st["v_pool"][:, :, table], page)
    v = _values(codes, scales).view(layers, hk, seqs, -1, D)
    o = torch.matmul(p, v) / total_p
    o = o.view(layers, hk, seqs, G, n, D).permute(0, 2, 4, 1, 3, 5).reshape(layers, seqs, n, hq, D)
    seq, at, _ = _new_slots(st)
    st["out"].copy_(o[:, seq, at - (lens - count)[seq]].to(st["out"].dtype))
    return st["out"]


def _plain_grow(st):
    """Gives back what lies behind the lengths `base`, then serves the sequences in turn from the top of the list."""
    page, table, free = st["case"]["page"], st["page_table"], st["free"]
    n_free, held = st["n_free"].long(), st["held"].long()
    seqs, max_pages = table.shape
    entry = torch.arange(max_pages, device=DEV)
    spill = torch.cat((free, free.new_zeros(1)))  # (a place behind the list for what does not go there)

    keep = (st["base"].long() + page - 1) // page
    back = (entry >= keep[:, None]) & (entry < held[:, None])
    order = back.view(-1).long().cumsum(0).view_as(back) - 1
    count = order.view(-1)[-1:] + 1
    spill[torch.where(back, n_free + count - 1 - order, len(free))] = table
    table.masked_fill_(back, -1)
    held = torch.minimum(held, keep)
    n_free = n_free + count

    cu, old = st["cu_new_dev"].long(), st["base"].long()
    new = cu[1:] - cu[:-1]
    fits = old + new <= st["max_len"]
    need = torch.where(fits, (old + new + page - 1) // page - held, 0).clamp(min=0)
    before = need.cumsum(0) - need
    granted = fits & ((need == 0) | (before + need <= n_free))
    take = granted[:, None] & (entry >= held[:, None]) & (entry < (held + need)[:, None])
    at = n_free - 1 - (before[:, None] + entry - held[:, None])
    table.copy_(torch.where(take, spill[at.clamp(0, len(free) - 1)], table))
    held = held + torch.where(granted, need, 0)
    st["n_free"].copy_(n_free - torch.where(granted, need, 0).sum())
    st["held"].copy_(held)
    free.copy_(spill[:-1])
    st["seq_lens"].copy_(torch.where(granted, old + new, -1 - old))

    i = torch.arange(len(st["slots"]), device=DEV)
    seq = torch.searchsorted(cu, i, right=True) - 1
    at = old[seq] + i - cu[seq]
    slot = table.long()[seq, (at // page).clamp(max=max_pages - 1)] * page + at % page
    st["slots"].copy_(torch.where(granted[seq], slot, -1))
    return _grown(st)


def _grown(st):
    return {n: st[n] for n in ("page_table", "seq_lens", "held", "free", "n_free", "slots")}


def _plain_verify(st):
    case, vocab = st["case"], st["case"]["vocab"]
    cu = st["cu_new_dev"].long()
    count = cu[1:] - cu[:-1]
    total = len(st["tokens"])
    t = torch.arange(case["new_max"], device=DEV)
    row = (cu[:-1, None] + t).clamp(max=total - 1)  # [seqs, n], padded
    token = st["tokens"].long()[row]
    p = st["target"][row, token].double()
    q = st["draft"][row, token].double() if st["draft"] is not None else torch.ones_like(p)
    good = (st["accept"][row].double() * q < p) & (t < count[:, None] - 1)
    accepted = good.long().cumprod(1).sum(1)
    stop = cu[:-1] + accepted
    w = st["target"][stop].double()
    if st["draft"] is not None:
        less = st["draft"][stop].double()
    else:
        less = torch.zeros_like(w).scatter_(1, st["tokens"].long()[stop][:, None], math.inf)
    rest = (w - less).clamp(min=0)
    some = (accepted < count - 1) & (rest.sum(1) > 0)
    c = torch.where(some[:, None], rest, w).cumsum(1)
    last = vocab - 1 - (c.diff(dim=1, prepend=torch.zeros_like(c[:, :1])) > 0).flip(1).long().argmax(1)
    chosen = torch.minimum((c <= st["pick"].double()[:, None] * c[:, -1:]).sum(1), last)
    i = torch.arange(total, device=DEV)
    seq = torch.searchsorted(cu, i, right=True) - 1
    at = i - cu[seq]
    out = torch.where(at < accepted[seq], st["tokens"].long(), torch.where(at == accepted[seq], chosen[seq], -1))
    st["out"].copy_(out)
    st["n_out"].copy_(accepted + 1)
    return {"tokens": st["out"], "n_out": st["n_out"]}


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------

def _handle(st):
    """What a program that serves from the cache keeps: the cache, the batch of new tokens, free pages, a workspace."""
    from paper_2603_00188_amd import paged as P
    from paper_2603_00188_amd import stlite as S
    case = st["case"]
    h = dict(P=P)
    if case["kind"] == "verify":
        h["batch"] = P.NewTokens(st["cu_new"], device=DEV)
        h["ws"] = P.verify_workspace(h["batch"], case["vocab"])
        return h
    h["cache"] = P.PagedCache(st["k_pool"], st["v_pool"], st["page_table"], st["seq_lens"], case["q_heads"],
                              max_len=st["max_len"], dtype=TYPES[case["dtype"]])
    if case["kind"] == "compact":
        none = np.zeros(case["seqs"] + 1, np.int32)
        h["p"] = S.Problem(case["layers"], case["q_heads"], case["kv_heads"], 1, st["cu_seqlens"], none,
                           np.zeros((0, 3), np.int32), st["cu_budget"], device=DEV)
        h["batch"] = P.NewTokens(st["cu_budget"], device=DEV)
        return h
    h["batch"] = P.NewTokens(st["cu_new"], device=DEV)
    if case["kind"] == "append":
        h["rope"] = P.Rope(theta=st["theta"], sections=st["sections"], interleaved=case["interleaved"])
    elif case["kind"] == "grow":
        h["pages"] = P.FreePages(st["free"], st["n_free"], st["held"])
    else:
        h["ws"] = h["cache"].workspace(h["batch"])
    return h


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"append": _plain_append, "compact": _plain_compact, "grow": _plain_grow,
                "verify": _plain_verify}.get(kind, _plain_attention)(st)
    h = st.get("handle")
    if h is None:
        h = st["handle"] = _handle(st)
    P = h["P"]
    if kind == "append":
        P.paged_append(h["cache"], h["batch"], st["q"], st["k"], st["v"], positions=st["positions"], rope=h["rope"],
                       q_norm=st["q_norm"], k_norm=st["k_norm"], eps=1e-6, q_out=st["q_out"])
        P.paged_read(h["cache"], h["batch"], k_out=st["k_out"], v_out=st["v_out"])
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    if kind == "compact":
        P.paged_compact(h["cache"], h["p"], st["k"], st["v"], st["kept"])
        P.paged_read(h["cache"], h["batch"], k_out=st["k_out"], v_out=st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"], "seq_lens": st["seq_lens"]}
    if kind == "grow":
        P.paged_release(h["cache"], h["pages"], st["base"])
        P.paged_grow(h["cache"], h["pages"], h["batch"], slots=st["slots"])
        return _grown(st)
    if kind == "verify":
        P.verify_drafts(h["batch"], st["target"], st["tokens"], st["accept"], st["pick"], draft=st["draft"], out=st["out"],
                        n_out=st["n_out"], workspace=h["ws"])
        return {"tokens": st["out"], "n_out": st["n_out"]}
    return P.paged_attention(h["cache"], h["batch"], st["q"], out=st["out"], workspace=h["ws"])


def work(case):
    old, new = _lengths(case)
    layers, hq, hk, row = case["layers"], case["q_heads"], case["kv_heads"], 2 * D
    total = sum(new)
    if case["kind"] == "verify":
        # a row of each side's probabilities for every sequence, where its run of accepted tokens ends; a few words a token
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": case["seqs"] * case["vocab"] * size * (2 if case["draft"] == "full" else 1) + total * 20,
                "flops": 2 * case["seqs"] * case["vocab"]}
    if case["kind"] == "grow":
        # lengths, pages held, prefix sums; the pages taken and given back: list and table, read and written; a place a token
        pages = sum(-(-(a + b) // case["page"]) - -(-a // case["page"]) for a, b in zip(old, new))
        return {"bytes": case["seqs"] * 24 + pages * 16 + total * 4, "flops": 0}
    if case["kind"] == "compact":
        kept = sum(_budgets(case))  # K and V rows: read, stored in 4 bits; read there, written; their list
        return {"bytes": layers * hk * kept * (2 * (2 * row + 2 * ROW) + 4), "flops": 0}
    if case["kind"] == "append":
        # queries in and out; K and V rows as in a compaction; a product and a sum for each rotated element and each
        # element's norm
        return {"bytes": layers * total * (hq * row * 2 + 2 * hk * (2 * row + 2 * ROW)) + total * case["axes"] * 4,
                "flops": layers * total * (hq + hk) * D * (7 if case["norm"] else 3)}
    pairs = sum(n * o + n * (n + 1) // 2 for o, n in zip(old, new))
    return {"bytes": layers * (hk * sum(a + b for a, b in zip(old, new)) * 2 * ROW + 2 * total * hq * row),
            "flops": layers * hq * pairs * 4 * D}


# ---------------------------------------------------------------------------
# In 64 bits, from the definitions
# ---------------------------------------------------------------------------

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_rows(pool, page, unit, pages, n):
    """The first n rows of a unit's pages, from the bytes."""
    rows = pool[unit][pages]
    codes = rows[:, :64 * page].reshape(-1, 64).long()
    scales = rows[:, 64 * page:].reshape(-1, 4).double()
    grid = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float64, device=DEV)
    x = torch.empty((codes.shape[0], D), dtype=torch.float64, device=DEV)
    x[:, 0::2], x[:, 1::2] = grid[codes % 16], grid[codes // 16]
    return (x * torch.exp2(scales - 127).repeat_interleave(32, 1))[:n]


def _exact_stored(x, dtype):
    """The values that rows [.., 128] in 64 bits are held as: the nearest of the grid, between neighbours by comparison."""
    lo, hi = RANGE[dtype]
    b = x.reshape(-1, 32)
    top = b.abs().amax(1)
    e = torch.full_like(top, lo)
    for k in range(lo, hi):  # one step up while 7 scales do not reach
        more = top > 7.0 * 2.0 ** k
        if not bool(more.any()):
            break
        e += more
    y = b.abs() / torch.exp2(e)[:, None]
    v = torch.zeros_like(y)
    for i in range(7):
        mid = (GRID[i] + GRID[i + 1]) / 2
        v[(y >= mid) if i % 2 else (y > mid)] = GRID[i + 1]
    return (v * torch.sign(b) * torch.exp2(e)[:, None]).view_as(x)


def _exact_rotated(st, x, w, at):
    """One token's heads [layers, heads, D] in 64 bits, from the definition: pairs as complex numbers."""
    x = x.double()
    if w is not None:
        x = w.double()[:, None] * x / (x.square().sum(-1, keepdim=True) / D + 1e-6).sqrt()
    pos = st["positions"][:, at].tolist()
    axis = [a for a, n in enumerate(st["sections"]) for _ in range(n)]
    angle = [pos[axis[i]] * st["theta"] ** (-2.0 * i / D) for i in range(D // 2)]
    turn = torch.tensor([complex(math.cos(a), math.sin(a)) for a in angle], dtype=torch.complex128, device=DEV)
    if st["case"]["interleaved"]:
        z = torch.complex(x[..., 0::2], x[..., 1::2]) * turn
        return torch.view_as_real(z).reshape(x.shape)
    z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * turn
    return torch.cat((z.real, z.imag), -1)


def exact(case, seed):
    if case["kind"] in ("grow", "verify"):
        return None  # (whole numbers)
    st = prepare(case, seed)
    page, layers, hq, hk = case["page"], case["layers"], case["q_heads"], case["kv_heads"]
    if case["kind"] == "compact":
        out = {}
        for name in ("k", "v"):
            x = torch.empty(st[name + "_out"].shape, dtype=torch.float64, device=DEV)
            for u in range(layers * hk):
                x[u // hk, :, u % hk] = _exact_stored(st[name][u].double()[st["kept"][u].long()], case["dtype"])
            out[name] = x
        return dict(out, seq_lens=None)
    cu = st["cu_new"].tolist()
    if case["kind"] == "append":
        if cu[-1] > 15000:
            return None
        q = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
        k = torch.empty(st["k_out"].shape, dtype=torch.float64, device=DEV)
        for i in range(cu[-1]):
            q[:, i] = _exact_rotated(st, st["q"][:, i], st["q_norm"], i)
            k[:, i] = _exact_rotated(st, st["k"][:, i], st["k_norm"], i)
        return {"q": q, "k": _exact_stored(k, case["dtype"]), "v": _exact_stored(st["v"].double().contiguous(), case["dtype"])}
    table = st["page_table"].tolist()
    lens = st["seq_lens"].tolist()
    out = torch.empty(st["out"].shape, dtype=torch.float64, device=DEV)
    G = hq // hk
    for s in range(case["seqs"]):
        n, pages = cu[s + 1] - cu[s], table[s][:-(-lens[s] // page)]
        at = torch.arange(lens[s], device=DEV)
        for layer in range(layers):
            for h in range(hk):
                k = _exact_rows(st["k_pool"][layer], page, h, pages, lens[s])
                v = _exact_rows(st["v_pool"][layer], page, h, pages, lens[s])
                for a in range(cu[s], cu[s + 1], 512):
                    b = min(a + 512, cu[s + 1])
                    x = st["q"][layer, a:b, h * G:(h + 1) * G].double() @ k.T / math.sqrt(D)
                    far = at > (lens[s] - n + torch.arange(a - cu[s], b - cu[s], device=DEV))[:, None]
                    x[far[:, None].expand_as(x)] = -math.inf
                    out[layer, a:b, h * G:(h + 1) * G] = torch.softmax(x, -1) @ v
    return out
