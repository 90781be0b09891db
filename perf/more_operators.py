"""Cases of the operators of a KV cache held in 4 bits, and their plain forms.

    append   new keys and values go into the cache, rotated to their positions and quantised on the way; the rows just
             written are read back (a prompt's own attention runs over the same values that later steps will see)
    read     the cached rows of a batch come back as bf16
    attend   one query token per sequence attends over its cached rows
    evict    after a compression round the kept rows move to the front of their unit, or into another cache

A cached row is 80 bytes: 128 codes of 4 bits, and a scale s and a centre c (bf16) for each of its four groups of 32
components.  A component stands for (code - 8) s + c.  For a group with smallest and largest value lo and hi
    c = bf16((8 hi + 7 lo) / 15),  s = the smallest bf16 that is not below (hi - c) / 7 and (c - lo) / 8,
    code = 8 + (x - c) / s rounded to nearest even, within 0..15 (8 where s = 0).
Component 32 g + 8 t + 2 i + h has bits 4 (i + 4 h) .. + 3 of the 32-bit word 4 t + g; the scales follow at byte 64, the
centres at byte 72.  Head dimension 128 throughout.

``run`` computes the plain form in torch, or makes the framework's calls where ``own`` is true.  Lengths follow from the
case alone; the seed makes the contents, the page order, the positions and the kept rows.
"""
import functools
import math

import torch

own = False

D = 128
ROW = 80
GOLDEN = 0.6180339887498949


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------
def _append(name, seqs, tokens, kv_heads, group, **kw):
    return dict({"name": name, "op": "append", "seqs": seqs, "tokens": tokens, "kv_heads": kv_heads, "group": group,
                 "page": 0, "len_lo": 0, "len_hi": 0, "ragged_new": False, "half_split": False, "theta": 1e6,
                 "pos_hi": 32768}, **kw)


def _read(name, seqs, kv_heads, len_lo, len_hi, **kw):
    return dict({"name": name, "op": "read", "seqs": seqs, "kv_heads": kv_heads, "group": 1, "page": 0,
                 "len_lo": len_lo, "len_hi": len_hi}, **kw)


def _attend(name, seqs, kv_heads, group, len_lo, len_hi, **kw):
    return dict({"name": name, "op": "attend", "seqs": seqs, "kv_heads": kv_heads, "group": group, "page": 0,
                 "len_lo": len_lo, "len_hi": len_hi, "per_head": False}, **kw)


def _evict(name, seqs, kv_heads, len_lo, len_hi, budget, **kw):
    return dict({"name": name, "op": "evict", "seqs": seqs, "kv_heads": kv_heads, "group": 1, "page": 0,
                 "len_lo": len_lo, "len_hi": len_hi, "budget": budget, "in_place": False}, **kw)


def listed():
    return [
        # one sequence decodes one token far into its text: latency is all there is
        _append("append_1x1", 1, 1, 8, 4, len_lo=2100, len_hi=2100, pos_hi=131072),
        # a batch of 64 decodes a token each into a paged cache
        _append("append_b64_paged", 64, 1, 8, 8, page=16, len_lo=1, len_hi=2175),
        # a mixed step of a paged server: prompt pieces of any length from nothing to 517 tokens
        _append("append_ragged_pieces", 16, 517, 8, 8, page=16, len_lo=0, len_hi=4000, ragged_new=True, half_split=True),
        # a whole prompt of 16,384 tokens fills an empty contiguous cache
        _append("append_prompt_16k", 1, 16384, 8, 4),
        # one short sequence read back
        _read("read_1x600", 1, 8, 600, 600),
        # 16 sequences of up to 8K tokens read back from 16-token pages, as a scoring round or a prompt's attention wants them
        _read("read_b16_paged", 16, 8, 1024, 8192, page=16),
        # one sequence, a short cache
        _attend("attend_1x600", 1, 8, 4, 600, 600),
        # 64 sequences between two compression rounds: 2,048 kept rows and up to 128 new ones, heads of different lengths
        _attend("attend_b64_heads", 64, 8, 4, 1024, 4096, page=32, per_head=True),
        # one sequence of 131,072 tokens that was never compressed
        _attend("attend_long_128k", 1, 8, 4, 131072, 131072),
        # 16 sequences of 8K to 64K tokens in 16-token pages, eight query heads per KV head
        _attend("attend_ragged_paged", 16, 8, 8, 8192, 65536, page=16),
        # a prompt of 32K tokens is cut to 2,048 rows on its way into a small cache
        _evict("evict_1_of_32k", 1, 8, 32768, 32768, 2048),
        # a window's end in a batch of 64: up to 2,176 rows become 2,048, in place, in pages
        _evict("evict_b64_in_place", 64, 8, 2049, 2176, 2048, page=16, in_place=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "read", "attend", "attend", "evict"))
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 12, 16))
    page = rng.choice((0, 16, 32, 48, 64))
    seqs = _log_int(rng, 1, 64)
    if op == "append":
        rows = 16384 * 20 // (kv_heads * (4 + group))              # no more than the largest listed one
        tokens = _log_int(rng, 1, min(8192, max(1, rows // seqs)))
        lo = rng.randint(0, 1000)
        c = _append("", seqs, tokens, kv_heads, group, page=page, len_lo=lo, len_hi=lo + rng.randint(0, 3000),
                    ragged_new=rng.random() < 0.5, half_split=rng.random() < 0.5, theta=rng.choice((1e4, 5e5, 1e6)),
                    pos_hi=_log_int(rng, 16384, 1 << 20))
    elif op == "read":
        hi = _log_int(rng, 1, min(32768, 500000 // (seqs * kv_heads)))
        c = _read("", seqs, kv_heads, rng.randint(0, hi), hi, page=page)
    elif op == "attend":
        hi = _log_int(rng, 1, min(65536, 4000000 // (seqs * kv_heads)))
        c = _attend("", seqs, kv_heads, group, rng.randint(0, hi), hi, page=page, per_head=rng.random() < 0.4)
    else:
        hi = _log_int(rng, 32, min(32768, 900000 // (seqs * kv_heads)))
        budget = max(16, _log_int(rng, 16, hi))
        c = _evict("", seqs, kv_heads, rng.randint(0, hi), hi, budget, page=page, in_place=rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _spread(n, lo, hi, salt=0):
    """n lengths spread evenly over [lo, hi] in no particular order; the first is the largest."""
    xs = [lo + int((hi - lo + 1) * (((i + 1 + salt) * GOLDEN) % 1.0)) for i in range(n)]
    xs[0] = hi
    return xs


def _lens(case):
    S, H = case["seqs"], case["kv_heads"]
    if case.get("per_head"):
        return [_spread(S, case["len_lo"], case["len_hi"], 17 * h) for h in range(H)]          # [H][S]
    return [_spread(S, case["len_lo"], case["len_hi"])] * H


def _new_counts(case):
    T = case["tokens"]
    return _spread(case["seqs"], 0, T, 5) if case["ragged_new"] else [T] * case["seqs"]


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _up_to_bf16(x):
    """The smallest bf16 that is not below x (x >= 0)."""
    b = x.to(torch.bfloat16)
    return torch.where(b.to(x.dtype) < x, (b.view(torch.int16) + 1).view(torch.bfloat16), b)


def _quantise(x):
    """Rows [..., 128] as codes [..., 4, 32] (floating), scales and centres [..., 4, 1] (bf16)."""
    x = x.unflatten(-1, (4, 32))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    c = ((8 * hi + 7 * lo) / 15).to(torch.bfloat16)
    cw = c.to(x.dtype)
    s = _up_to_bf16(torch.maximum((hi - cw) / 7, (cw - lo) / 8))
    sw = s.to(x.dtype)
    n = torch.round((x - cw) / torch.where(sw > 0, sw, torch.ones_like(sw))).clamp(-8, 7)
    return n + 8, s, c


def _rows_of(x):
    """Rows [..., 128] as they are cached: bytes [..., 80]."""
    n, s, c = _quantise(x)
    n = n.to(torch.uint8).unflatten(-1, (4, 4, 2))                     # [g, t, i, h]
    d = n.dim()
    n = n.permute(*range(d - 4), d - 3, d - 4, d - 1, d - 2).flatten(-4).unflatten(-1, (64, 2))       # [t, g, h, i]
    par = torch.cat((s, c), -2).squeeze(-1).contiguous().view(torch.uint8)
    return torch.cat((n[..., 0] | (n[..., 1] << 4), par), -1)


def _values_of(rows):
    """Bytes [..., 80] as the values they stand for, in 32 bits (the product is exact, the sum rounded once)."""
    b = rows[..., :64]
    n = torch.stack((b & 15, b >> 4), -1).flatten(-2).unflatten(-1, (4, 4, 2, 4))                     # [t, g, h, i]
    d = n.dim()
    n = n.permute(*range(d - 4), d - 3, d - 4, d - 1, d - 2).flatten(-3)                              # [g, 8 t + 2 i + h]
    par = rows[..., 64:].contiguous().view(torch.bfloat16).float().unflatten(-1, (2, 4))
    return ((n.float() - 8) * par[..., 0, :, None] + par[..., 1, :, None]).flatten(-2)


def _cache(g, case, rows, fill=True):
    """K and V of one layer with room for `rows` rows per sequence, and the page table (None: contiguous).
    contiguous [1, S, H, N, 80]; paged [1, pages, H, page, 80] with the pages in random order."""
    S, H, page = case["seqs"], case["kv_heads"], case["page"]
    rows = max(rows, 1)
    table = None
    if page:
        per = -(-rows // page)
        table = torch.randperm(S * per, generator=g, device="cuda").to(torch.int32).view(S, per)
        shape = (1, S * per, H, page, ROW)
    else:
        shape = (1, S, H, rows, ROW)
    k, v = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
    if fill:
        kc, vc = _randn(g, H, D), 0.5 * _randn(g, H, D)                # rows lie around a centre of their head
        step = max(1, (1 << 26) // (shape[3] * D))
        for h in range(H):
            for a in range(0, shape[1], step):
                b = min(shape[1], a + step)
                k[0, a:b, h] = _rows_of(kc[h] + 0.5 * _randn(g, b - a, shape[3], D))
                v[0, a:b, h] = _rows_of(vc[h] + _randn(g, b - a, shape[3], D))
    return k, v, table


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    S, H, G = case["seqs"], case["kv_heads"], case["group"]
    st = {"op": case["op"], "case": case}
    lens = _lens(case)
    most = max(max(x) for x in lens)
    st["lens"] = _int32(lens[0])
    if case["op"] == "append":
        T = case["tokens"]
        st["k"], st["v"], st["table"] = _cache(g, case, most + T, fill=False)
        st["n_new"] = _int32(_new_counts(case)) if case["ragged_new"] else None
        st["pos"] = torch.randint(most, max(most + 1, case["pos_hi"]), (S,), generator=g, device="cuda")
        qkv = _randn(g, S, T, (G + 2) * H, D)                         # the output of a fused projection
        qkv[:, :, G * H:] += _randn(g, 2 * H, D)                      # keys and values around a centre of their head
        qkv = qkv.to(torch.bfloat16)
        st["q_in"], st["k_in"], st["v_in"] = qkv[:, :, :G * H], qkv[:, :, G * H:(G + 1) * H], qkv[:, :, (G + 1) * H:]
        st["q_out"] = torch.zeros(S, T, G * H, D, dtype=torch.bfloat16, device="cuda")
        st["new_lens"] = torch.zeros(S, dtype=torch.int32, device="cuda")
        st["k_back"], st["v_back"] = (torch.zeros(S, T, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        f = torch.arange(D // 2, dtype=torch.float64, device="cuda")
        st["omega"] = torch.exp(-(2.0 * f / D) * math.log(case["theta"]))
    else:
        st["k"], st["v"], st["table"] = _cache(g, case, most)
    if case["op"] == "read":
        st["k_back"], st["v_back"] = (torch.zeros(S, H, max(most, 1), D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    elif case["op"] == "attend":
        st["unit_lens"] = _int32(lens).t().contiguous() if case["per_head"] else None           # [S, H]
        st["q"] = (2.0 * _randn(g, S, G * H, D)).to(torch.bfloat16)
        st["out"] = torch.zeros(S, G * H, D, dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "evict":
        B = case["budget"]
        st["cnt"] = st["lens"].clamp(max=B)[:, None].expand(S, H).contiguous()                   # [S, H]
        score = torch.rand(S, H, max(most, B), generator=g, device="cuda")
        score -= 2.0 * (torch.arange(score.shape[2], device="cuda") >= st["lens"][:, None, None])
        best = score.topk(B, -1).indices                                                         # the rows that exist come first
        best += score.shape[2] * (torch.arange(B, device="cuda") >= st["cnt"][..., None])
        st["idx"] = (best.sort(-1).values % score.shape[2]).to(torch.int32)                      # ascending, [S, H, B]
        N = st["table"].shape[1] * case["page"] if case["page"] else st["k"].shape[3]
        st["pos"] = torch.arange(N, dtype=torch.int32, device="cuda").add(7).expand(1, S, H, N).contiguous()
        st["new_lens"] = torch.zeros(S, dtype=torch.int32, device="cuda")
        if case["in_place"]:
            st["k_to"], st["v_to"], st["pos_to"] = st["k"], st["v"], st["pos"]
        else:
            st["k_to"], st["v_to"] = (torch.zeros(1, S, H, B, ROW, dtype=torch.uint8, device="cuda") for _ in range(2))
            st["pos_to"] = torch.zeros(1, S, H, B, dtype=torch.int32, device="cuda")
    if own:
        _handles(st)
    return st


# ------------------------------------------------------------------------------------------------
# the framework's calls
# ------------------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _context(kv_heads, group, theta, half_split):
    """One context per model, as a program keeps it (its statistics serve the compression round, not these calls)."""
    from paper_2604_04921_b200 import binding as tb
    return tb.TriContext(1, kv_heads, group, torch.zeros(1, kv_heads * group, D), torch.ones(1, kv_heads * group, D // 2),
                         rope_theta=theta, pair_layout=int(half_split))


def _handles(st):
    from paper_2604_04921_b200 import binding as tb
    case = st["case"]
    st["ctx"] = _context(case["kv_heads"], case["group"], case.get("theta", 1e6), case.get("half_split", False))
    view = tb.CacheView(st["k"], st["v"], seq_lens=st["lens"], positions=st.get("pos") if st["op"] == "evict" else None,
                        page_table=st["table"])
    if st["op"] == "evict":
        st["from"], st["to"] = view, view if case["in_place"] else tb.CacheView(st["k_to"], st["v_to"], positions=st["pos_to"])
        return
    st["cache"] = tb.LayerCache(view, 0, unit_lens=st.get("unit_lens"))
    if st["op"] == "append":
        st["after"] = tb.LayerCache(tb.CacheView(st["k"], st["v"], seq_lens=st["new_lens"], page_table=st["table"]), 0)
    if st["op"] == "attend":
        st["ws"] = st["ctx"].attend_workspace(case["seqs"])


def run(st):
    if st["op"] == "append":
        if own:
            st["ctx"].append(st["cache"], st["k_in"], st["v_in"], st["pos"], q=st["q_in"], q_out=st["q_out"],
                             n_new=st["n_new"], new_lens=st["new_lens"])
            st["ctx"].read(st["after"], st["k_back"], st["v_back"], first=st["lens"])
        else:
            _plain_append(st)
        # (a row behind a sequence's new tokens is not read back and stays zero)
        return {"k": st["k_back"], "v": st["v_back"], "q": st["q_out"], "lens": st["new_lens"]}
    if st["op"] == "read":
        if own:
            st["ctx"].read(st["cache"], st["k_back"].transpose(1, 2), st["v_back"].transpose(1, 2))
        else:
            _plain_read(st)
        return {"k": st["k_back"], "v": st["v_back"]}
    if st["op"] == "attend":
        if own:
            st["ctx"].attend(st["cache"], st["q"], st["out"], st["ws"])
            return {"out": st["out"]}
        return {"out": _plain_attend(st)}
    if own:
        case = st["case"]
        st["ctx"].compact(st["from"], st["idx"], st["cnt"], case["seqs"], case["budget"], st["to"], st["new_lens"])
    else:
        _plain_evict(st)
    # rows are moved bit for bit: their bytes are whole numbers
    return {"k": st["k_to"], "v": st["v_to"], "positions": st["pos_to"], "lens": st["new_lens"]}


# ------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------
def _rotate(x, c, s, half_split):
    """x [S, T, heads, 128] in 64 bits (values next to the border of two codes), c and s [S, T, 1, 64]."""
    a, b = (x[..., :D // 2], x[..., D // 2:]) if half_split else (x[..., 0::2], x[..., 1::2])
    a, b = c * a - s * b, s * a + c * b
    return torch.cat((a, b), -1) if half_split else torch.stack((a, b), -1).flatten(-2)


def _at(st, slot):
    """Where rows `slot` [S, n] of a cache lie: an index of [1, S | pages, H, N | page, ..]."""
    seq = torch.arange(slot.shape[0], device="cuda")[:, None].expand_as(slot)
    if st["table"] is None:
        return torch.zeros_like(seq), seq, slice(None), slot
    page = st["case"]["page"]
    return torch.zeros_like(seq), st["table"].long().gather(1, slot // page), slice(None), slot % page


def _plain_append(st):
    T = st["k_in"].shape[1]
    t = torch.arange(T, device="cuda")
    n_new = st["n_new"] if st["n_new"] is not None else torch.full_like(st["lens"], T)
    keep = (t < n_new[:, None])[..., None, None]                                         # [S, T, 1, 1]
    where = (st["pos"][:, None] + t).double()
    ang = (where[..., None] * st["omega"])[:, :, None]
    c, s = torch.cos(ang), torch.sin(ang)
    k = _rows_of(_rotate(st["k_in"].double(), c, s, st["case"]["half_split"]))
    v = _rows_of(st["v_in"].double())
    q = _rotate(st["q_in"].double(), c, s, st["case"]["half_split"]).to(torch.bfloat16)
    at = _at(st, st["lens"].long()[:, None] + t)
    st["k"][at], st["v"][at] = torch.where(keep, k, st["k"][at]), torch.where(keep, v, st["v"][at])
    st["q_out"].copy_(torch.where(keep, q, st["q_out"]))
    st["k_back"].copy_(torch.where(keep, _values_of(st["k"][at]).to(torch.bfloat16), st["k_back"]))
    st["v_back"].copy_(torch.where(keep, _values_of(st["v"][at]).to(torch.bfloat16), st["v_back"]))
    torch.add(st["lens"], n_new, out=st["new_lens"])


def _rows(cache, table, n):
    """The first n cached rows of every unit, [S, H, n, 80]."""
    x = cache[0] if table is None else cache[0][table.long()].transpose(1, 2).flatten(2, 3)
    return x[:, :, :n]


def _plain_read(st):
    n = st["k_back"].shape[2]
    there = (torch.arange(n, device="cuda") < st["lens"][:, None])[:, None, :, None]
    for cache, back in ((st["k"], st["k_back"]), (st["v"], st["v_back"])):
        back.copy_(torch.where(there, _values_of(_rows(cache, st["table"], n)).to(torch.bfloat16), back))


def _plain_attend(st):
    S, H, G = st["case"]["seqs"], st["case"]["kv_heads"], st["case"]["group"]
    lens = st["unit_lens"] if st["unit_lens"] is not None else st["lens"][:, None]
    n = st["k"].shape[3] if st["table"] is None else st["table"].shape[1] * st["case"]["page"]
    there = torch.arange(n, device="cuda") < lens[:, :, None]                            # [S, H or 1, n]
    x = st["q"].float().view(S, H, G, D) @ _values_of(_rows(st["k"], st["table"], n)).transpose(-1, -2) / math.sqrt(D)
    x = torch.where(there[:, :, None], x, torch.full_like(x, -math.inf))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    l = p.sum(-1, keepdim=True)
    o = p @ _values_of(_rows(st["v"], st["table"], n))
    return torch.where(l > 0, o / l, torch.zeros_like(o)).reshape(S, H * G, D).to(torch.bfloat16)


def _plain_evict(st):
    case = st["case"]
    S, H, B = case["seqs"], case["kv_heads"], case["budget"]
    idx = st["idx"].long()
    seq, head = torch.arange(S, device="cuda")[:, None, None], torch.arange(H, device="cuda")[None, :, None]
    slot = torch.arange(B, device="cuda").expand(S, H, B)
    there = slot < st["cnt"][..., None]
    page = case["page"]
    src = (0, seq, head, idx) if not page else (0, st["table"].long()[seq, idx // page], head, idx % page)
    rows = [st[x][src] for x in ("k", "v")]                                              # all are read before one is written
    pos = st["pos"][0].gather(2, idx)
    n = min(B, st["pos_to"].shape[3])
    slot, there = slot[..., :n], there[..., :n]
    if not (page and case["in_place"]):
        dst = (0, seq, head, slot)
    else:
        dst = (0, st["table"].long()[seq, slot // page], head, slot % page)
    for x, r in zip(("k_to", "v_to"), rows):
        st[x][dst] = torch.where(there[..., None], r[:, :, :n], st[x][dst])
    st["pos_to"][0, :, :, :n] = torch.where(there, pos[..., :n], st["pos_to"][0, :, :, :n])
    st["new_lens"].copy_(st["cnt"][:, 0])


# ------------------------------------------------------------------------------------------------
# what one pass cannot do without, and its outputs in 64 bits
# ------------------------------------------------------------------------------------------------
def work(case):
    S, H, G = case["seqs"], case["kv_heads"], case["group"]
    if case["op"] == "append":
        n = sum(_new_counts(case))
        # queries in and out, keys and values in, their rows out (what the read back takes of them is then on the chip), values out
        return {"bytes": n * H * ((2 * G + 2) * D * 2 + 2 * ROW + 2 * D * 2) + S * 16, "flops": n * H * ((G + 1) * D * 3 + 2 * D * 8)}
    rows = sum(sum(x) for x in _lens(case))
    if case["op"] == "read":
        return {"bytes": 2 * rows * (ROW + 2 * D), "flops": 4 * rows * D}
    if case["op"] == "attend":
        return {"bytes": 2 * rows * ROW + 2 * S * G * H * D * 2, "flops": 4 * rows * G * D + 4 * rows * D}
    kept = sum(min(n, case["budget"]) for n in _lens(case)[0]) * H
    return {"bytes": kept * (4 * ROW + 12), "flops": 0}


def _decoder():
    """Byte and shift of every component of a cached row."""
    d = torch.arange(D, device="cuda")
    g, t, i, h = d // 32, d % 32 // 8, d % 8 // 2, d % 2
    bit = 32 * (4 * t + g) + 4 * (i + 4 * h)
    return bit // 8, bit % 8


def _exact_values(rows):
    """Rows [n, 80] as the values they stand for, in 64 bits."""
    byte, shift = _decoder()
    code = (rows[:, byte].long() >> shift) & 15
    words = rows[:, 64:].long()
    par = ((words[:, 0::2] | (words[:, 1::2] << 8)) << 16).to(torch.int32).view(torch.float32).double()       # bf16 bits
    group = torch.arange(D, device="cuda") // 32
    return (code - 8).double() * par[:, group] + par[:, 4 + group]


def _exact_quantised(x):
    """Rows [n, 128] (64 bits) as the values that a cache which has taken them holds."""
    out = torch.empty_like(x)
    for a in range(0, D, 32):
        y = x[:, a:a + 32]
        top, low = y.max(1).values, y.min(1).values
        c = ((8.0 * top + 7.0 * low) / 15.0).bfloat16().double()
        need = torch.maximum((top - c) / 7.0, (c - low) / 8.0)
        e = torch.floor(torch.log2(need.clamp(min=1e-300))) - 7                          # bf16 has 8 bits
        s = torch.ceil(need / torch.exp2(e)) * torch.exp2(e)
        steps = torch.where(s[:, None] > 0, (y - c[:, None]) / s[:, None].clamp(min=1e-300), torch.zeros_like(y))
        out[:, a:a + 32] = torch.round(steps).clamp(-8, 7) * s[:, None] + c[:, None]
    return out


def _unit(cache, table, seq, head, idx):
    """Rows idx of one sequence and head, [n, 80]."""
    if table is None:
        return cache[0, seq, head, idx]
    page = cache.shape[3]
    return cache[0, table[seq].long()[idx // page], head, idx % page]


def _exact_append(case, st):
    H, G = case["kv_heads"], case["group"]
    k, v, q = st["k_back"].double(), st["v_back"].double(), st["q_out"].double()
    counts, lens = _new_counts(case), _lens(case)[0]
    band = torch.arange(D // 2, device="cuda")
    re, im = (band, band + D // 2) if case["half_split"] else (2 * band, 2 * band + 1)
    for s in range(case["seqs"]):
        n = counts[s]
        if n == 0:
            continue
        p = int(st["pos"][s]) + torch.arange(n, device="cuda", dtype=torch.float64)
        turn = torch.polar(torch.ones(n, D // 2, dtype=torch.float64, device="cuda"),
                           p[:, None] * case["theta"] ** (-2.0 * band.double() / D))
        for h in range(H * (G + 1)):
            src = st["q_in"][s, :n, h] if h < H * G else st["k_in"][s, :n, h - H * G]
            z = torch.complex(src[:, re].double(), src[:, im].double()) * turn
            row = torch.empty(n, D, dtype=torch.float64, device="cuda")
            row[:, re], row[:, im] = z.real, z.imag
            if h < H * G:
                q[s, :n, h] = row
            else:
                k[s, :n, h - H * G] = _exact_quantised(row)
                v[s, :n, h - H * G] = _exact_quantised(st["v_in"][s, :n, h - H * G].double())
    return {"k": k, "v": v, "q": q, "lens": _int32([a + b for a, b in zip(lens, counts)])}


def _exact_read(case, st):
    k, v = st["k_back"].double(), st["v_back"].double()
    lens = _lens(case)[0]
    for s in range(case["seqs"]):
        at = torch.arange(lens[s], device="cuda")
        for h in range(case["kv_heads"]):
            k[s, h, :lens[s]] = _exact_values(_unit(st["k"], st["table"], s, h, at))
            v[s, h, :lens[s]] = _exact_values(_unit(st["v"], st["table"], s, h, at))
    return {"k": k, "v": v}


def _exact_attend(case, st):
    H, G, S = case["kv_heads"], case["group"], case["seqs"]
    lens = _lens(case)
    out = torch.zeros(S, H * G, D, dtype=torch.float64, device="cuda")
    for h in range(H):
        for s in range(S):
            at = torch.arange(lens[h][s], device="cuda")
            k, v = (_exact_values(_unit(st[x], st["table"], s, h, at)) for x in ("k", "v"))
            if len(k):
                logits = st["q"][s, h * G:(h + 1) * G].double() @ k.t() / math.sqrt(D)
                out[s, h * G:(h + 1) * G] = torch.softmax(logits, -1) @ v
    return {"out": out}


def _exact_evict(case, st):
    rows = {x: [] for x in ("k", "v")}
    units = [(s, h) for s in range(case["seqs"]) for h in range(case["kv_heads"])]
    kept = [min(n, case["budget"]) for n in _lens(case)[0]]
    for x in rows:
        for s, h in units:
            rows[x].append(_unit(st[x], st["table"], s, h, st["idx"][s, h, :kept[s]].long()).clone())
    pos = [st["pos"][0, s, h, st["idx"][s, h, :kept[s]].long()].clone() for s, h in units]
    for i, (s, h) in enumerate(units):
        at = torch.arange(kept[s], device="cuda")
        table = st["table"] if case["in_place"] else None
        for x in rows:
            to = st[x + "_to"]
            if table is None:
                to[0, s, h, at] = rows[x][i]
            else:
                to[0, table[s].long()[at // case["page"]], h, at % case["page"]] = rows[x][i]
        st["pos_to"][0, s, h, at] = pos[i]
    return {"k": st["k_to"], "v": st["v_to"], "positions": st["pos_to"], "lens": _int32(kept)}


def exact(case, seed):
    return {"append": _exact_append, "read": _exact_read, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](
        case, prepare(case, seed))
