"""Timed cases of serving from a paged cache: what a program does with a
compressed cache after the compression pass.

* ``append``  -- new tokens' queries and keys are normalised per head and rotated, the keys and values stored in pages;
* ``compact`` -- the kept rows of the compression go straight into pages;
* ``decode``  -- attention of one new token per sequence over its pages;
* ``extend``  -- causal attention of several new tokens per sequence over its pages.

A page holds ``page`` tokens of one (layer, kv head); the page table is shared by all layers and kv heads, and the pages
of a sequence are scattered over the pool.  ``seq_lens`` counts a sequence's tokens with the new ones.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

# The benchmark's models: 28 query heads over 4 kv heads, three position axes.
BASE = dict(kind="decode", dtype="bf16", layers=28, q_heads=28, kv_heads=4, page=64, seqs=1, len_min=678, len_max=678,
            new_min=1, new_max=1, layout=0, axes=3, interleaved=False, norm=False, fused=False, beta_num=1, beta_den=5)


def listed():
    return [
        # one layer's new token behind the compressed first step: nothing but a launch
        dict(BASE, name="append_token", kind="append", layers=1, page=16),
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
        # a serving batch of short and long sequences, small pages
        dict(BASE, name="decode_ragged", dtype="fp16", layers=4, q_heads=32, kv_heads=8, seqs=64, len_min=1,
             len_max=8000, page=16, layout=3),
        # one layer over the uncompressed trajectory: few heads, a long cache
        dict(BASE, name="decode_long", layers=1, len_min=150528, len_max=150528, page=128),
        # a batch in which every sequence checks a few drafted tokens
        dict(BASE, name="extend_few", kind="extend", layers=2, seqs=16, len_min=500, len_max=6000, new_min=5, new_max=5,
             page=16, layout=5),
        # the next screenshot and its text over the compressed trajectory, one layer
        dict(BASE, name="extend_screen", kind="extend", layers=1, len_min=30105, len_max=30105, new_min=3136,
             new_max=3136),
        # prompts of several lengths into an empty cache
        dict(BASE, name="extend_prompts", kind="extend", dtype="fp16", layers=2, q_heads=16, kv_heads=2, seqs=5,
             len_min=0, len_max=0, new_min=131, new_max=2999, page=32, layout=7),
    ]


def _log_int(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def _cost(case):
    w = work(case)
    # the plain form of attention holds every sequence padded to the longest
    pad = case["layers"] * case["seqs"] * (case["len_max"] + case["new_max"])
    pairs = pad * case["q_heads"] * case["new_max"] if case["kind"] in ("decode", "extend") else 0
    return {"bytes": w["bytes"], "flops": w["flops"], "pairs": pairs, "rows": pad * case["kv_heads"]}


def draw(rng):
    """Another case of the ranges above, no dearer than the largest of its kind."""
    top = {}
    for c in listed():
        for key, v in _cost(c).items():
            top[c["kind"], key] = max(v, top.get((c["kind"], key), 0))
    while True:
        kind = rng.choice(["append", "compact", "decode", "decode", "decode", "extend", "extend", "extend"])
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


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, layers, hq, hk, page = TYPES[case["dtype"]], case["layers"], case["q_heads"], case["kv_heads"], case["page"]
    old, new = _lengths(case)
    if case["kind"] == "compact":
        old, new = _budgets(case), [0] * case["seqs"]
    lens = [a + b for a, b in zip(old, new)]
    max_len = max(lens)
    max_pages = max(-(-max_len // page), 1)
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3

    def randn(shape, scale=1.0):
        x = torch.empty(shape, dtype=dt, device=DEV)
        for layer in range(shape[0]):
            x[layer] = torch.randn(shape[1:], generator=gen, device=DEV) * scale
        return x

    # every page is in use somewhere: what lies behind a sequence's end is another's old rows
    st = dict(case=case, k_pool=randn((layers, hk, n_pages, page, D), D ** -0.5),
              v_pool=randn((layers, hk, n_pages, page, D)), max_len=max_len)
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
        return st
    # queries near the sum of a few of their sequence's keys, so that the softmax has peaks; the noise keeps its tail
    first = st["k_pool"][:, :, table[:, 0].long(), :4].float().sum(3)  # [layers, kv, seqs, D]
    rows = torch.repeat_interleave(torch.arange(case["seqs"], device=DEV), torch.tensor(new, device=DEV))
    st["q"] = torch.empty((layers, total, hq, D), dtype=dt, device=DEV)
    for layer in range(layers):
        aim = first[layer][:, rows].permute(1, 0, 2).unsqueeze(2)  # [total, kv, 1, D]
        noise = torch.randn((total, hk, hq // hk, D), generator=gen, device=DEV)
        st["q"][layer] = (64.0 * aim + 24.0 * noise).reshape(total, hq, D)
    st["out"] = torch.empty((layers, total, hq, D), dtype=dt, device=DEV)
    return st


def _new_slots(st):
    """Sequence of every new token, its index in the sequence and its row in the pool."""
    cu = st["cu_new_dev"].long()
    i = torch.arange(int(st["cu_new"][-1]), device=DEV)
    seq = torch.searchsorted(cu, i, right=True) - 1
    at = st["seq_lens"].long()[seq] - cu[seq + 1] + i
    page = st["case"]["page"]
    return seq, at, st["page_table"].long()[seq, at // page] * page + at % page


def _plain_rotated(x, w, st):
    """Norm (where given) and rotation of [layers, tokens, heads, D] in 32 bits; the angles in 64."""
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()[:, None, None]
    half = D // 2
    freq = st["theta"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    axis = torch.repeat_interleave(torch.arange(len(st["sections"]), device=DEV), torch.tensor(st["sections"], device=DEV))
    angle = st["positions"].double()[axis].T * freq
    cos, sin = angle.cos().float()[None, :, None], angle.sin().float()[None, :, None]
    if st["case"]["interleaved"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _plain_append(st):
    dt, layers, hk = TYPES[st["case"]["dtype"]], st["case"]["layers"], st["case"]["kv_heads"]
    st["q_out"].copy_(_plain_rotated(st["q"], st["q_norm"], st).to(dt))
    _, _, slot = _new_slots(st)
    st["k_pool"].view(layers, hk, -1, D)[:, :, slot] = _plain_rotated(st["k"], st["k_norm"], st).to(dt).transpose(1, 2)
    st["v_pool"].view(layers, hk, -1, D)[:, :, slot] = st["v"].transpose(1, 2)
    return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"]}


def _plain_compact(st):
    case, page = st["case"], st["case"]["page"]
    layers, hk = case["layers"], case["kv_heads"]
    cu = st["cu_budget_dev"].long()
    j = torch.arange(int(st["cu_budget"][-1]), device=DEV)
    seq = torch.searchsorted(cu, j, right=True) - 1
    at = j - cu[seq]
    slot = st["page_table"].long()[seq, at // page] * page + at % page
    unit = torch.arange(layers * hk, device=DEV)[:, None]
    kept = st["kept"].long()
    st["k_pool"].view(layers * hk, -1, D)[:, slot] = st["k"][unit, kept]
    st["v_pool"].view(layers * hk, -1, D)[:, slot] = st["v"][unit, kept]
    return {"k_pool": st["k_pool"], "v_pool": st["v_pool"]}


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
    k = st["k_pool"][:, :, table].float().view(layers, hk, seqs, -1, D)
    x = torch.matmul(q, k.transpose(-1, -2))
    del k
    x *= D ** -0.5
    last = (lens - count)[:, None] + t  # the last key that a new token sees
    seen = torch.arange(x.shape[-1], device=DEV) <= last[..., None]  # [seqs, n, keys]
    x = x.view(layers, hk, seqs, G, n, -1).masked_fill_(~seen[:, None], -math.inf).view(layers, hk, seqs, G * n, -1)
    x -= x.amax(-1, keepdim=True)
    p = x.exp_()
    total_p = p.sum(-1, keepdim=True)
    v = st["v_pool"][:, :, table].float().view(layers, hk, seqs, -1, D)
    o = torch.matmul(p, v) / total_p
    o = o.view(layers, hk, seqs, G, n, D).permute(0, 2, 4, 1, 3, 5).reshape(layers, seqs, n, hq, D)
    seq, at, _ = _new_slots(st)
    st["out"].copy_(o[:, seq, at - (lens - count)[seq]].to(st["out"].dtype))
    return st["out"]


def _handle(st):
    """What a program that serves from the cache keeps: the cache, the batch of new tokens and a workspace."""
    from paper_2603_00188_amd import paged as P
    from paper_2603_00188_amd import stlite as S
    case = st["case"]
    h = dict(P=P, cache=P.PagedCache(st["k_pool"], st["v_pool"], st["page_table"], st["seq_lens"], case["q_heads"],
                                     max_len=st["max_len"]))
    if case["kind"] == "compact":
        none = np.zeros(case["seqs"] + 1, np.int32)
        h["p"] = S.Problem(case["layers"], case["q_heads"], case["kv_heads"], 1, st["cu_seqlens"], none,
                           np.zeros((0, 3), np.int32), st["cu_budget"], device=DEV)
        return h
    h["batch"] = P.NewTokens(st["cu_new"], device=DEV)
    if case["kind"] == "append":
        h["rope"] = P.Rope(theta=st["theta"], sections=st["sections"], interleaved=case["interleaved"])
    else:
        h["ws"] = h["cache"].workspace(h["batch"])
    return h


def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"append": _plain_append, "compact": _plain_compact}.get(kind, _plain_attention)(st)
    h = st.get("handle")
    if h is None:
        h = st["handle"] = _handle(st)
    P = h["P"]
    if kind == "append":
        P.paged_append(h["cache"], h["batch"], st["q"], st["k"], st["v"], positions=st["positions"], rope=h["rope"],
                       q_norm=st["q_norm"], k_norm=st["k_norm"], eps=1e-6, q_out=st["q_out"])
        return {"q": st["q_out"], "k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    if kind == "compact":
        P.paged_compact(h["cache"], h["p"], st["k"], st["v"], st["kept"])
        return {"k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    return P.paged_attention(h["cache"], h["batch"], st["q"], out=st["out"], workspace=h["ws"])


def work(case):
    old, new = _lengths(case)
    layers, hq, hk, row = case["layers"], case["q_heads"], case["kv_heads"], 2 * D
    total = sum(new)
    if case["kind"] == "compact":
        kept = sum(_budgets(case))  # K and V rows read and written, their list
        return {"bytes": layers * hk * kept * (4 * row + 4), "flops": 0}
    if case["kind"] == "append":
        # the rows in and out; a product and a sum for each rotated element and each element's norm
        return {"bytes": layers * total * (hq + 2 * hk) * row * 2 + total * case["axes"] * 4,
                "flops": layers * total * (hq + hk) * D * (7 if case["norm"] else 3)}
    pairs = sum(n * o + n * (n + 1) // 2 for o, n in zip(old, new))
    return {"bytes": layers * (hk * sum(a + b for a, b in zip(old, new)) * 2 * row + 2 * total * hq * row),
            "flops": layers * hq * pairs * 4 * D}


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
    st = prepare(case, seed)
    page, layers, hq, hk = case["page"], case["layers"], case["q_heads"], case["kv_heads"]
    table = st["page_table"].tolist()
    lens = st["seq_lens"].tolist()
    if case["kind"] == "compact":
        k, v = st["k_pool"].flatten(0, 1), st["v_pool"].flatten(0, 1)
        for s in range(case["seqs"]):
            a, b = (int(x) for x in st["cu_budget"][s:s + 2])
            for j in range(0, b - a, page):
                m = min(page, b - a - j)
                rows = st["kept"][:, a + j:a + j + m].long()
                for pool, src in ((k, st["k"]), (v, st["v"])):
                    pool[:, table[s][j // page], :m] = torch.gather(src, 1, rows[..., None].expand(-1, -1, D))
        return {"k_pool": st["k_pool"].double(), "v_pool": st["v_pool"].double()}
    cu = st["cu_new"].tolist()
    if case["kind"] == "append":
        if cu[-1] > 15000:
            return None
        q = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
        k, v = st["k_pool"].double(), st["v_pool"].double()
        for s in range(case["seqs"]):
            for i in range(cu[s], cu[s + 1]):
                j = lens[s] - cu[s + 1] + i
                q[:, i] = _exact_rotated(st, st["q"][:, i], st["q_norm"], i)
                k[:, :, table[s][j // page], j % page] = _exact_rotated(st, st["k"][:, i], st["k_norm"], i)
                v[:, :, table[s][j // page], j % page] = st["v"][:, i].double()
        return {"q": q, "k_pool": k, "v_pool": v}
    out = torch.empty(st["out"].shape, dtype=torch.float64, device=DEV)
    G = hq // hk
    for s in range(case["seqs"]):
        n, pages = cu[s + 1] - cu[s], table[s][:-(-lens[s] // page)]
        at = torch.arange(lens[s], device=DEV)
        for layer in range(layers):
            for h in range(hk):
                k = st["k_pool"][layer, h, pages].reshape(-1, D)[:lens[s]].double()
                v = st["v_pool"][layer, h, pages].reshape(-1, D)[:lens[s]].double()
                for a in range(cu[s], cu[s + 1], 512):
                    b = min(a + 512, cu[s + 1])
                    x = st["q"][layer, a:b, h * G:(h + 1) * G].double() @ k.T / math.sqrt(D)
                    far = at > (lens[s] - n + torch.arange(a - cu[s], b - cu[s], device=DEV))[:, None]
                    x[far[:, None].expand_as(x)] = -math.inf
                    out[layer, a:b, h * G:(h + 1) * G] = torch.softmax(x, -1) @ v
    return out
