"""Cases of the three decode-side operators of a KV cache, and their plain forms.

    append   new keys and values of one layer go into a contiguous or paged cache at each sequence's length, the keys
             (and the step's queries) rotated to their positions on the way
    attend   one query token per sequence attends over its cached rows (a cache that compression may have shortened,
             for each head by another amount)
    shared   the same where groups of sequences continue one long prompt: the prompt's rows are cached once, every
             sequence adds its own rows behind them

Head dimension 128 throughout.  ``run`` computes the plain form in torch, or makes the framework's calls where ``own``
is true.  Lengths follow from the case alone; the seed makes the contents, the page order and the positions.
"""
import functools
import math

import torch

own = False

D = 128
GOLDEN = 0.6180339887498949
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------------
def _append(name, seqs, tokens, kv_heads, group, **kw):
    return dict({"name": name, "op": "append", "seqs": seqs, "tokens": tokens, "kv_heads": kv_heads, "group": group,
                 "dtype": "bf16", "page": 0, "len_lo": 0, "len_hi": 0, "ragged_new": False, "positions": False,
                 "half_split": False, "theta": 1e6, "pos_hi": 32768}, **kw)


def _attend(name, seqs, kv_heads, group, len_lo, len_hi, **kw):
    return dict({"name": name, "op": "attend", "seqs": seqs, "kv_heads": kv_heads, "group": group, "dtype": "bf16",
                 "page": 0, "len_lo": len_lo, "len_hi": len_hi, "per_head": False}, **kw)


def _shared(name, prefixes, seqs, kv_heads, group, prefix_lo, prefix_hi, len_lo, len_hi, **kw):
    return dict({"name": name, "op": "shared", "prefixes": prefixes, "seqs": seqs, "kv_heads": kv_heads, "group": group,
                 "dtype": "bf16", "page": 0, "prefix_lo": prefix_lo, "prefix_hi": prefix_hi, "len_lo": len_lo,
                 "len_hi": len_hi}, **kw)


def listed():
    return [
        # one sequence decodes one token far into its text: latency is all there is
        _append("append_1x1", 1, 1, 8, 4, len_lo=2100, len_hi=2100, pos_hi=131072),
        # a batch of 64 decodes a token each into an 8-bit paged cache
        _append("append_b64_paged_e4m3", 64, 1, 8, 8, dtype="e4m3", page=16, len_lo=1, len_hi=2175),
        # a mixed step of a paged server: prompt pieces of any length from nothing to 517 tokens, original positions kept
        _append("append_ragged_pieces", 16, 517, 8, 8, page=16, len_lo=0, len_hi=4000, ragged_new=True, half_split=True),
        # a whole prompt of 32,768 tokens fills an empty contiguous cache
        _append("append_prompt_32k", 1, 32768, 8, 4, positions=True),
        # one sequence, a short cache
        _attend("attend_1x600", 1, 8, 4, 600, 600),
        # 64 sequences between two compression rounds: 2,048 kept rows and up to 128 new ones
        _attend("attend_steady_b64", 64, 8, 4, 2049, 2176),
        # one sequence of 131,072 tokens that was never compressed
        _attend("attend_long_128k", 1, 8, 4, 131072, 131072),
        # 16 sequences of 8K to 64K tokens in 16-token pages, eight query heads per KV head
        _attend("attend_ragged_paged", 16, 8, 8, 8192, 65536, page=16),
        # an 8-bit paged cache after compression with a budget of its own for each head
        _attend("attend_b64_e4m3_heads", 64, 8, 4, 1024, 4096, dtype="e4m3", page=32, per_head=True),
        # two samples of one short prompt
        _shared("shared_2_of_700", 1, 2, 8, 4, 700, 700, 3, 40),
        # 32 samples of one prompt of 32,768 tokens
        _shared("shared_32_of_32k", 1, 32, 8, 4, 32768, 32768, 1, 2176),
        # six prompts with 64 samples between them, paged, eight query heads per KV head
        _shared("shared_64_of_6_paged", 6, 64, 8, 8, 2048, 16384, 1, 2176, page=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("append", "attend", "shared"))
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 12, 16))
    dtype = rng.choice(("bf16", "bf16", "e4m3"))
    page = rng.choice((0, 16, 32, 48, 64))
    seqs = _log_int(rng, 1, 64)
    if op == "append":
        rows = 32768 * 20 // (kv_heads * (4 + group))              # no more than the largest listed one
        tokens = _log_int(rng, 1, min(8192, max(1, rows // seqs)))
        lo = rng.randint(0, 1000)
        c = _append("", seqs, tokens, kv_heads, group, dtype=dtype, page=page, len_lo=lo, len_hi=lo + rng.randint(0, 3000),
                    ragged_new=rng.random() < 0.5, positions=rng.random() < 0.5, half_split=rng.random() < 0.5,
                    theta=rng.choice((1e4, 5e5, 1e6)), pos_hi=_log_int(rng, 16384, 1 << 20))
    elif op == "attend":
        hi = _log_int(rng, 1, min(65536, 4000000 // (seqs * kv_heads)))
        c = _attend("", seqs, kv_heads, group, rng.randint(0, hi), hi, dtype=dtype, page=page, per_head=rng.random() < 0.4)
    else:
        prefixes = rng.randint(1, min(8, seqs))
        phi = _log_int(rng, 1, min(32768, 2000000 // (prefixes * kv_heads), (1 << 27) // (seqs * kv_heads)))
        hi = _log_int(rng, 1, min(4096, 2000000 // (seqs * kv_heads)))
        c = _shared("", prefixes, seqs, kv_heads, group, rng.randint(0, phi), phi, rng.randint(0, hi), hi, dtype=dtype,
                    page=page)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _spread(n, lo, hi, salt=0):
    """n lengths spread evenly over [lo, hi] in no particular order; the first is the largest."""
    if n == 0:
        return []
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


def _group_starts(case):
    """[P + 1]: prefix p belongs to the sequences [start[p], start[p + 1]); every group is a different size."""
    P, S = case["prefixes"], case["seqs"]
    w = [1.0 + (i * GOLDEN) % 1.0 for i in range(P)]
    acc, out = 0.0, [0]
    for i in range(P):
        acc += w[i]
        out.append(S if i == P - 1 else min(S, int(round(S * acc / sum(w)))))
    return out


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _to_cache(x, dtype):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn) if dtype == "e4m3" else x.to(torch.bfloat16)


def _cache(g, case, n_seqs, rows):
    """K and V of one layer with room for `rows` rows per sequence, and the page table (None: contiguous).
    contiguous [1, S, H, N, 128]; paged [1, pages, H, page, 128] with the pages in random order."""
    H, page = case["kv_heads"], case["page"]
    rows = max(rows, 1)
    table = None
    if page:
        per = -(-rows // page)
        table = torch.randperm(n_seqs * per, generator=g, device="cuda").to(torch.int32).view(n_seqs, per)
        shape = (1, n_seqs * per, H, page, D)
    else:
        shape = (1, n_seqs, H, rows, D)
    dt = torch.float8_e4m3fn if case["dtype"] == "e4m3" else torch.bfloat16
    k, v = torch.empty(shape, dtype=dt, device="cuda"), torch.empty(shape, dtype=dt, device="cuda")
    kc, vc = _randn(g, H, 1, D), 0.5 * _randn(g, H, 1, D)            # rows lie around a centre of their head
    step = max(1, (1 << 28) // (H * shape[3] * D))
    for a in range(0, shape[1], step):
        b = min(shape[1], a + step)
        for h in range(H):
            k[0, a:b, h] = _to_cache(kc[h] + 0.5 * _randn(g, b - a, shape[3], D), case["dtype"])
            v[0, a:b, h] = _to_cache(vc[h] + _randn(g, b - a, shape[3], D), case["dtype"])
    return k, v, table


def _scales(g, case):
    if case["dtype"] != "e4m3":
        return None, None
    H = case["kv_heads"]
    return tuple(0.25 + torch.rand(1, H, generator=g, device="cuda") for _ in range(2))


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    S, H, G = case["seqs"], case["kv_heads"], case["group"]
    st = {"op": case["op"], "case": case}
    lens = _lens(case)
    if case["op"] == "append":
        T = case["tokens"]
        st["k"], st["v"], st["table"] = _cache(g, case, S, max(lens[0]) + T)
        st["lens"] = _int32(lens[0])
        st["n_new"] = _int32(_new_counts(case)) if case["ragged_new"] else None
        lo = max(lens[0])                                             # compressed caches hold fewer rows than the text
        st["pos"] = torch.randint(lo, max(lo + 1, case["pos_hi"]), (S,), generator=g, device="cuda")
        qkv = _randn(g, S, T, (G + 2) * H, D).to(torch.bfloat16)      # the output of a fused projection
        st["q_in"], st["k_in"], st["v_in"] = qkv[:, :, :G * H], qkv[:, :, G * H:(G + 1) * H], qkv[:, :, (G + 1) * H:]
        st["q_out"] = torch.zeros(S, T, G * H, D, dtype=torch.bfloat16, device="cuda")
        rows = st["table"].shape[1] * case["page"] if case["page"] else st["k"].shape[3]
        st["positions"] = torch.zeros(1, S, H, rows, dtype=torch.int32, device="cuda") if case["positions"] else None
        st["new_lens"] = torch.zeros(S, dtype=torch.int32, device="cuda")
        f = torch.arange(D // 2, dtype=torch.float64, device="cuda")
        st["omega"] = torch.exp(-(2.0 * f / D) * math.log(case["theta"]))
    else:
        st["k"], st["v"], st["table"] = _cache(g, case, S, max(max(x) for x in lens))
        st["lens"] = _int32(lens[0])
        st["unit_lens"] = _int32(lens).t().contiguous() if case.get("per_head") else None      # [S, H]
        st["q"] = (2.0 * _randn(g, S, G * H, D)).to(torch.bfloat16)
        st["out"] = torch.zeros(S, G * H, D, dtype=torch.bfloat16, device="cuda")
        if case["op"] == "shared":
            plens = _spread(case["prefixes"], case["prefix_lo"], case["prefix_hi"], 3)
            st["pk"], st["pv"], st["ptable"] = _cache(g, case, case["prefixes"], max(plens))
            st["plens"] = _int32(plens)
            st["starts"] = _int32(_group_starts(case))
    st["ks"], st["vs"] = _scales(g, case)
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
    view = tb.CacheView(st["k"], st["v"], seq_lens=st["lens"], positions=st.get("positions"), page_table=st["table"])
    st["cache"] = tb.LayerCache(view, 0, unit_lens=st.get("unit_lens"), k_scale=st["ks"], v_scale=st["vs"])
    if case["op"] == "shared":
        pview = tb.CacheView(st["pk"], st["pv"], seq_lens=st["plens"], page_table=st["ptable"])
        st["prefix"] = tb.LayerCache(pview, 0, k_scale=st["ks"], v_scale=st["vs"])
    if case["op"] != "append":
        st["ws"] = st["ctx"].attend_workspace(case["seqs"], case.get("prefixes", 0))


def run(st):
    if st["op"] == "append":
        if own:
            st["ctx"].append(st["cache"], st["k_in"], st["v_in"], st["pos"], q=st["q_in"], q_out=st["q_out"],
                             n_new=st["n_new"], new_lens=st["new_lens"])
        else:
            _plain_append(st)
        out = {"k": st["k"], "v": st["v"], "q": st["q_out"], "lens": st["new_lens"]}
        return out if st["positions"] is None else dict(out, positions=st["positions"])
    if own:
        if st["op"] == "attend":
            st["ctx"].attend(st["cache"], st["q"], st["out"], st["ws"])
        else:
            st["ctx"].attend_shared(st["prefix"], st["starts"], st["cache"], st["q"], st["out"], st["ws"])
        return {"out": st["out"]}
    return {"out": _plain_attend(st)}


# ------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------
def _rotate(x, c, s, half_split):
    """x [S, T, heads, 128] in 64 bits (the rounding to the cache's type is the only one), c and s [S, T, 1, 64]."""
    a, b = (x[..., :D // 2], x[..., D // 2:]) if half_split else (x[..., 0::2], x[..., 1::2])
    a, b = c * a - s * b, s * a + c * b
    return torch.cat((a, b), -1) if half_split else torch.stack((a, b), -1).flatten(-2)


def _plain_append(st):
    case, T = st["case"], st["k_in"].shape[1]
    t = torch.arange(T, device="cuda")
    n_new = st["n_new"] if st["n_new"] is not None else torch.full_like(st["lens"], T)
    valid = t < n_new[:, None]                                                           # [S, T]
    slot = st["lens"].long()[:, None] + t
    where = (st["pos"][:, None] + t).double()
    ang = (where[..., None] * st["omega"])[:, :, None]                                   # far positions need 64 bits
    c, s = torch.cos(ang), torch.sin(ang)
    q = _rotate(st["q_in"].double(), c, s, case["half_split"])
    k = _rotate(st["k_in"].double(), c, s, case["half_split"])
    v = st["v_in"].double()
    if case["dtype"] == "e4m3":
        k, v = k / st["ks"][0].double()[:, None], v / st["vs"][0].double()[:, None]
    seq = torch.arange(slot.shape[0], device="cuda")[:, None].expand_as(slot)
    if st["table"] is None:
        at = (torch.zeros_like(seq), seq, slice(None), slot)
    else:
        page = case["page"]
        at = (torch.zeros_like(seq), st["table"].long().gather(1, slot // page), slice(None), slot % page)
    keep = valid[..., None, None]
    for cache, x in ((st["k"], k), (st["v"], v)):                                        # [S, T, H, 128] rows
        as_is = cache.view(torch.uint8 if case["dtype"] == "e4m3" else torch.int16)      # moved bit for bit
        new = _to_cache(x, case["dtype"]).view(as_is.dtype)
        as_is[at] = torch.where(keep, new, as_is[at])
    st["q_out"].copy_(torch.where(keep, q.to(torch.bfloat16), st["q_out"]))
    if st["positions"] is not None:
        old = st["positions"][0].transpose(1, 2)[seq, slot]                              # [S, T, H]
        st["positions"][0].transpose(1, 2)[seq, slot] = torch.where(valid[..., None], where.to(torch.int32)[..., None], old)
    torch.add(st["lens"], n_new, out=st["new_lens"])


def _rows(cache, table):
    """The cached rows as [S, H, N, 128] in 32 bits."""
    x = cache[0] if table is None else cache[0][table.long()].transpose(1, 2).flatten(2, 3)
    return x.float()


def _logits(q, k, mask):
    """Logits of q [B, H, R, 128] against k [B, H, N, 128], minus infinity outside mask [B, H or 1, R or 1, N]."""
    s = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    return torch.where(mask, s, torch.full_like(s, -math.inf))


def _plain_attend(st):
    S, H, G = st["case"]["seqs"], st["case"]["kv_heads"], st["case"]["group"]
    ks = 1.0 if st["ks"] is None else st["ks"][0].view(H, 1, 1)
    vs = 1.0 if st["vs"] is None else st["vs"][0].view(H, 1, 1)
    q = st["q"].float().view(S, H, G, D)
    k, v = _rows(st["k"], st["table"]), _rows(st["v"], st["table"])
    lens = st["unit_lens"] if st["unit_lens"] is not None else st["lens"][:, None]
    there = torch.arange(k.shape[2], device="cuda") < lens[:, :, None]                   # [S, H or 1, N]
    s = _logits(q, k, there[:, :, None]) * ks
    v = torch.where(there[..., None], v * vs, torch.zeros_like(v))
    m = s.amax(-1, keepdim=True)
    if st["op"] == "shared":
        pk, pv = _rows(st["pk"], st["ptable"]), _rows(st["pv"], st["ptable"])            # [P, H, Np, 128]
        P = pk.shape[0]
        seq = torch.arange(S, device="cuda")
        mine = (seq >= st["starts"][:-1, None]) & (seq < st["starts"][1:, None])         # [P, S]
        pthere = torch.arange(pk.shape[2], device="cuda") < st["plens"][:, None]         # [P, Np]
        allq = q.transpose(0, 1).reshape(1, H, S * G, D)
        mask = mine.repeat_interleave(G, 1)[:, None, :, None] & pthere[:, None, None]
        ps = _logits(allq, pk, mask) * ks                                              # [P, H, S * G, Np]
        pv = torch.where(pthere[:, None, :, None], pv * vs, torch.zeros_like(pv))
        pm = ps.amax(-1).amax(0).view(H, S, G).transpose(0, 1)[..., None]
        m = torch.maximum(m, pm)
    safe = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(s - safe)
    l, o = p.sum(-1, keepdim=True), p @ v
    if st["op"] == "shared":
        pp = torch.exp(ps - safe.transpose(0, 1).reshape(1, H, S * G, 1))
        l = l + pp.sum(-1).sum(0).view(H, S, G).transpose(0, 1)[..., None]
        o = o + (pp @ pv).sum(0).view(H, S, G, D).transpose(0, 1)
    o = torch.where(l > 0, o / l, torch.zeros_like(o))
    return o.reshape(S, H * G, D).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------
# what one pass cannot do without, and its outputs in 64 bits
# ------------------------------------------------------------------------------------------------
def work(case):
    S, H, G = case["seqs"], case["kv_heads"], case["group"]
    row = D * (1 if case["dtype"] == "e4m3" else 2)                                      # bytes of a cached row
    if case["op"] == "append":
        n = sum(_new_counts(case))
        per = (2 * G + 2) * H * D * 2 + 2 * H * row + (4 * H if case["positions"] else 0)
        return {"bytes": n * per + S * 16, "flops": n * (G + 1) * H * (D // 2) * 6}
    keys = sum(sum(x) for x in _lens(case))
    read, flops = 2 * keys * row, 4 * keys * G * D
    if case["op"] == "shared":
        starts = _group_starts(case)
        plens = _spread(case["prefixes"], case["prefix_lo"], case["prefix_hi"], 3)
        used = [n if starts[p + 1] > starts[p] else 0 for p, n in enumerate(plens)]
        read += 2 * sum(used) * H * row
        flops += sum(4 * n * H * G * D * (starts[p + 1] - starts[p]) for p, n in enumerate(plens))
    return {"bytes": read + 2 * S * G * H * D * 2, "flops": flops}


def _unit_rows(cache, table, seq, head, n):
    """The first n cached rows of one sequence and head, in 64 bits."""
    if table is None:
        return cache[0, seq, head, :n].double()
    page = cache.shape[3]
    idx = torch.arange(n, device="cuda")
    return cache[0, table[seq].long()[idx // page], head, idx % page].double()


def _exact_append(case, st):
    H, G = case["kv_heads"], case["group"]
    k, v = st["k"].double(), st["v"].double()
    q = st["q_out"].double()
    pos_out = st["positions"]
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
        slots = lens[s] + torch.arange(n, device="cuda")
        for h in range(H * (G + 1)):
            src = st["q_in"][s, :n, h] if h < H * G else st["k_in"][s, :n, h - H * G]
            z = torch.complex(src[:, re].double(), src[:, im].double()) * turn
            row = torch.empty(n, D, dtype=torch.float64, device="cuda")
            row[:, re], row[:, im] = z.real, z.imag
            if h < H * G:
                q[s, :n, h] = row
                continue
            h -= H * G
            val = st["v_in"][s, :n, h].double()
            if case["dtype"] == "e4m3":
                row = (row / st["ks"][0, h].double()).clamp(-E4M3_MAX, E4M3_MAX)
                val = (val / st["vs"][0, h].double()).clamp(-E4M3_MAX, E4M3_MAX)
            if case["page"]:
                pages, off = st["table"][s].long()[slots // case["page"]], slots % case["page"]
                k[0, pages, h, off], v[0, pages, h, off] = row, val
            else:
                k[0, s, h, slots], v[0, s, h, slots] = row, val
            if pos_out is not None:
                pos_out[0, s, h, slots] = p.to(torch.int32)
    out = {"k": k, "v": v, "q": q, "lens": st["lens"] + _int32(counts)}
    return out if pos_out is None else dict(out, positions=pos_out)


def _exact_attend(case, st):
    H, G, S = case["kv_heads"], case["group"], case["seqs"]
    lens = _lens(case)
    out = torch.zeros(S, H * G, D, dtype=torch.float64, device="cuda")
    starts = _group_starts(case) if case["op"] == "shared" else []
    plens = _spread(case["prefixes"], case["prefix_lo"], case["prefix_hi"], 3) if starts else []
    for h in range(H):
        ks = 1.0 if st["ks"] is None else float(st["ks"][0, h])
        vs = 1.0 if st["vs"] is None else float(st["vs"][0, h])
        shared = [(_unit_rows(st["pk"], st["ptable"], p, h, n), _unit_rows(st["pv"], st["ptable"], p, h, n))
                  for p, n in enumerate(plens)]
        for s in range(S):
            k, v = (_unit_rows(st[x], st["table"], s, h, lens[h][s]) for x in ("k", "v"))
            for p in range(len(plens)):
                if starts[p] <= s < starts[p + 1]:
                    k, v = torch.cat((shared[p][0], k)), torch.cat((shared[p][1], v))
            if len(k):
                logits = st["q"][s, h * G:(h + 1) * G].double() @ k.t() * (ks / math.sqrt(D))
                out[s, h * G:(h + 1) * G] = torch.softmax(logits, -1) @ v * vs
    return {"out": out}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_append(case, st) if case["op"] == "append" else _exact_attend(case, st)
