"""The operators of a 4-bit cache: append (rotation and quantisation), read back, attention, moving kept rows; against the 64-bit forms
of row4_reference.py, whose header derives the bounds."""
import ctypes
import math

import pytest
import torch

import row4_reference as R
from paper_2604_04921_b200 import binding as tb
from row4_reference import Cache4, D, ROW, U_BF16, as_rows, parts, values
from step_reference import Cache, pair_magnitude, rope

pytestmark = pytest.mark.gpu
DEV = "cuda"


def context(L, H, G, theta=1e6, half_split=False):
    return tb.TriContext(L, H, G, torch.zeros(L, H * G, D), torch.ones(L, H * G, D // 2), rope_theta=theta,
                         pair_layout=int(half_split))


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# ------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------
def check_row(row, x, e):
    """A stored row [80] against what went into it: x [128] float64, off by e [128] before it was quantised."""
    code, s, c = parts(row)
    y, eg = x.view(4, 32), e.view(4, 32).amax(1)
    lo, hi = y.amin(1), y.amax(1)
    span = hi.abs().maximum(lo.abs())
    exact_c = (8 * hi + 7 * lo) / 15
    assert bool(((c - exact_c).abs() <= U_BF16 * exact_c.abs() + eg + 2.0 ** -22 * span).all())
    need = torch.maximum((hi - c) / 7, (c - lo) / 8)
    slack = eg / 7 + 2.0 ** -22 * span
    assert bool((s >= need - slack).all())
    assert bool((s <= R.bf16_not_below((need + slack).clamp(min=0)) + 0 * s).all())
    off = ((code - 8) * s.repeat_interleave(32) + c.repeat_interleave(32) - x).abs()
    assert bool((off <= s.repeat_interleave(32) * (0.5 + 2.0 ** -20) + e + 2.0 ** -22 * span.repeat_interleave(32)).all())


def check_append(kind, half_split, page, order, H, G, lens, n_new, T, pos, per_head=False, positions=True, in_place_lens=False, seed=0,
                 theta=1e6, layer=1):
    """One append into layer `layer` of two; everything it may write is compared with the definition, everything else with what was
    there, byte for byte.  Padding tokens hold NaN."""
    S, L = len(n_new), 2
    g = gen(seed)
    unit = lens if per_head else [[n] * H for n in lens]
    c = Cache4(L, S, H, max(max(r) + n for r, n in zip(unit, n_new)), page, order, seed=seed)
    ctx = context(L, H, G, theta, half_split)
    x = (torch.randn(S, T, (G + 2) * H, D, generator=g, device=DEV) + torch.randn(1, 1, (G + 2) * H, D, generator=g, device=DEV))
    x = x.to(torch.bfloat16 if kind == 0 else torch.float32)
    for s in range(S):
        x[s, n_new[s]:] = float("nan")
    q, k, v = x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]
    q_out = torch.full((S, T, G * H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    pos_t = torch.full((L, S, H, c.rows), -7, dtype=torch.int32, device=DEV) if positions else None
    seq_lens = int32([r[0] for r in unit])
    unit_lens = int32([unit, unit]).contiguous() if per_head else None
    old = unit_lens if per_head else seq_lens
    new = old if in_place_lens else torch.full_like(old, -5)
    before = old.clone()
    status = int32([0])
    k0, v0 = c.k.clone(), c.v.clone()
    dst = tb.LayerCache(c.view(tb, seq_lens=seq_lens, positions=pos_t), layer, unit_lens=unit_lens)
    ragged = any(n != T for n in n_new)
    ctx.append(dst, k, v, None if pos is None else torch.tensor(pos, device=DEV), q=q, q_out=q_out,
               n_new=int32(n_new) if ragged else None, new_lens=new, device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    kk, vv = c.k.clone(), c.v.clone()
    for s in range(S):
        for t in range(n_new[s]):
            p = (pos[s] if pos is not None else unit[s][0]) + t
            want_q = rope(q[s, t].double(), p, theta, half_split)
            rot = 2.0 ** -21 + p * 2.0 ** -51
            assert bool(((q_out[s, t].double() - want_q).abs() <= U_BF16 * want_q.abs() + rot * pair_magnitude(want_q, half_split)).all())
            for h in range(H):
                n = unit[s][h] + t
                wk = rope(k[s, t, h].double(), p, theta, half_split)
                check_row(c.at(c.k, layer, s, h, n), wk, rot * pair_magnitude(wk, half_split))
                wv = v[s, t, h].double()
                check_row(c.at(c.v, layer, s, h, n), wv, torch.zeros_like(wv))
                if positions:
                    assert int(pos_t[layer, s, h, n]) == p
                    pos_t[layer, s, h, n] = -7
                c.at(kk, layer, s, h, n).copy_(c.at(k0, layer, s, h, n))
                c.at(vv, layer, s, h, n).copy_(c.at(v0, layer, s, h, n))
        assert bool(q_out[s, n_new[s]:].isnan().all())
    assert torch.equal(kk, k0) and torch.equal(vv, v0)               # nothing else was written
    if positions:
        assert bool((pos_t == -7).all())
    want = before.clone()
    if per_head:
        want[layer] += int32(n_new)[:, None]
        if not in_place_lens:
            want[1 - layer] = -5
    else:
        want += int32(n_new)
    assert torch.equal(new, want)


@pytest.mark.parametrize("half_split", [False, True])
@pytest.mark.parametrize("kind", [0, 1])
def test_append_types_and_layouts_of_bands(kind, half_split):
    check_append(kind, half_split, 16, "heads", 3, 2, [5, 0, 30], [3, 1, 2], 3, [70, 131071, 30])


@pytest.mark.parametrize("page,order", [(0, "heads"), (0, "tokens"), (0, "padded"), (48, "tokens"), (32, "padded"), (16, "heads")])
@pytest.mark.parametrize("T,n_new", [(1, [1, 1]), (1, [0, 1]), (9, [9, 9]), (20, [0, 17]), (8, [8, 3])])
def test_append_layouts_and_counts(page, order, T, n_new):
    check_append(0, True, page, order, 2, 3, [13, 33], n_new, T, [1000, 40000], seed=T)


@pytest.mark.parametrize("T", [1, 8, 17])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_lengths_of_heads_and_in_place(T, in_place):
    check_append(0, False, 16, "heads", 2, 1, [[4, 7], [0, 3], [9, 9]], [T, 0, T], T, [50, 60, 70], per_head=True, in_place_lens=in_place)


def test_append_positions():
    check_append(0, False, 16, "heads", 2, 2, [0, 21], [5, 5], 5, None, positions=False)
    check_append(1, False, 0, "heads", 1, 1, [3], [2], 2, [2 ** 31 - 4], theta=5e5)
    check_append(0, True, 16, "heads", 8, 16, [3 * s for s in range(9)], [1] * 9, 1, [1000 + s for s in range(9)], layer=0)


def stored(x):
    """Values x [n, 128] (fp32) appended to an empty cache, as rows [n, 80]."""
    ctx, c = context(1, 1, 1), Cache4(1, 1, 1, x.shape[0])
    v = x.view(1, -1, 1, D).contiguous()
    ctx.append(tb.LayerCache(c.view(tb, seq_lens=int32([0])), 0), torch.zeros_like(v), v, torch.tensor([0], device=DEV))
    torch.cuda.synchronize()
    assert bool((c.k[0, 0, 0, :, :64] == 0x88).all()) and bool((c.k[0, 0, 0, :, 64:] == 0).all())      # zero keys
    return c.v[0, 0, 0]


def test_append_bf16_values_as_the_definition_has_them():
    """Values that are bf16 leave nothing to the rounding of the kernel's fp32: rows are the reference's byte for byte.  Sixteenths
    give many (x - c) / s that lie halfway between two codes."""
    g = gen(5)
    x = torch.cat((torch.randn(300, D, generator=g, device=DEV), torch.randint(-40, 41, (300, D), generator=g, device=DEV) / 16,
                   torch.randint(-7, 8, (50, D), generator=g, device=DEV) * 0.5)).to(torch.bfloat16)
    x[300:].view(-1, 4, 32)[:, :, :2] = torch.tensor([-4.0, 3.5], dtype=torch.bfloat16, device=DEV)    # s = 1/2, c = 0 and 1/32
    got, want = stored(x.float()), as_rows(x.double())
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 520])
def test_append_groups_whose_scale_lies_behind_a_border(T, dtype):
    """A group from -t to hi with t tiny: (c - lo) / 8 is just above c / 8, itself a bf16 number, so that the smallest bf16 not below it
    is the next one; likewise (hi - c) / 7 with hi tiny.  Values and the keys of position 0 are the reference's byte for byte."""
    hi = torch.cat((1 + torch.arange(128, device=DEV) / 128, 0.7 * torch.exp2(torch.arange(-1, 1, device=DEV))))
    rows = []
    for t in (1e-9, 1e-8, 1e-7, 3e-11):
        x = hi[:, None] * torch.rand(len(hi), D, generator=gen(7), device=DEV)
        x[:, 5], x[:, 6] = hi, -t                                                # group 0
        x[:, 40], x[:, 41] = 256 * hi, -t                                        # group 1: not above 256
        x[:, 64:96] *= -1
        x[:, 70], x[:, 71] = -hi * 15 / 8, t                                     # group 2: hi - c = -c, for hi = 1: 7 / 8
        rows.append(x)
    x = torch.cat(rows).to(torch.bfloat16)
    want = as_rows(x.double())
    assert float((parts(want)[1][:, 0] * 8 > parts(want)[2][:, 0]).double().mean()) > 0.2                # what the case is about
    n = x.shape[0]
    assert n == 520
    ctx = context(1, 1, 1)
    S = n // T
    cache = Cache4(1, S, 1, T)
    v = x.to(dtype).view(S, T, 1, D)
    if T == 1:
        ctx.append(tb.LayerCache(cache.view(tb, seq_lens=int32([0] * S)), 0), v, v.clone(), torch.zeros(S, dtype=torch.int64, device=DEV))
        torch.cuda.synchronize()
        assert torch.equal(cache.k[0, :, 0, 0], want)
        got = cache.v[0, :, 0, 0]
    else:
        ctx.append(tb.LayerCache(cache.view(tb, seq_lens=int32([0])), 0), torch.zeros_like(v), v, torch.zeros(1, dtype=torch.int64, device=DEV))
        torch.cuda.synchronize()
        got = cache.v[0, 0, 0]
        for i in range(0, n, 40):                                                # tokens at position 0
            one = Cache4(1, 1, 1, 16)
            k = v[:, i:i + 1].expand(1, 2, 1, D).contiguous()
            ctx.append(tb.LayerCache(one.view(tb, seq_lens=int32([0])), 0), k, k.clone(), torch.zeros(1, dtype=torch.int64, device=DEV),
                       n_new=int32([1]))
            torch.cuda.synchronize()
            assert torch.equal(one.k[0, 0, 0, 0], want[i]) and torch.equal(one.v[0, 0, 0, 0], want[i])
    assert torch.equal(got, want)


def test_append_unusual_groups():
    """Constants, zeros, one outlier, values far from zero, tiny and huge ones, NaN and infinities."""
    x = torch.zeros(13, D, device=DEV)
    x[0] = 0.1
    x[1, 5] = 1e4
    x[2] = 100 + torch.arange(D, device=DEV) / D
    x[3] = torch.linspace(-1, 1, D, device=DEV) * 1e-38
    x[4] = torch.linspace(-3.2e38, 3.2e38, D, device=DEV)            # (its step is infinite in fp32, and every group has infinities)
    x[12] = torch.linspace(-3.2e38, 3.2e38, D, dtype=torch.float64, device=DEV).float()
    x[5] = -0.0
    x[6] = torch.linspace(1e-30, 2e-30, D, device=DEV)
    x[7, 3], x[7, 40] = float("nan"), float("inf")
    x[8, 64], x[8, 100], x[8, 101] = -float("inf"), float("inf"), -float("inf")
    x[9] = 3.4e38                                                    # above the largest bf16: its centre would be infinite
    x[10] = torch.randn(D, generator=gen(1), device=DEV)
    x[10, 31] = float("nan")
    rows = stored(x)
    got = values(rows)
    for r in (0, 1, 2, 6, 12):
        check_row(rows[r], x[r].double(), torch.zeros(D, dtype=torch.float64, device=DEV))
    assert bool((got[5] == 0).all()) and bool((got[11] == 0).all())
    assert float((got[3] - x[3].double()).abs().max()) <= 2.0 ** -127        # the smallest scale is 2^-126
    bad = got.isnan().view(13, 4, 32)
    assert bool((bad.any(-1) == bad.all(-1)).all())
    want = torch.zeros(13, 4, dtype=torch.bool, device=DEV)
    want[4] = want[7, :2] = want[8, 2:] = want[9] = want[10, 0] = True
    assert torch.equal(bad.any(-1), want)


def test_append_groups_as_wide_as_fp32():
    """A group from -m to n has c - lo = 8 (m + n) / 15: up to fp32's range it is quantised, beyond that it becomes NaN, on every
    path that keys and values take."""
    x = torch.randn(D, generator=gen(3), device=DEV)
    x[0:32:2], x[1:32:2] = 3.1e38, -3.1e38
    x[32:64:2], x[33:64:2] = 3.38e38, -3.38e38
    x[64:80], x[80:96] = -3.38e38, 2.9e38
    x = x.to(torch.bfloat16)
    ctx = context(1, 1, 1)
    code, s, c = R.quantised(x.double())
    for T in (1, 3):
        for dtype in (torch.bfloat16, torch.float32):
            cache = Cache4(1, 1, 1, 16)
            rows = x.to(dtype).expand(1, T, 1, D).contiguous()
            ctx.append(tb.LayerCache(cache.view(tb, seq_lens=int32([0])), 0), rows, rows.clone(), torch.zeros(1, dtype=torch.int64, device=DEV),
                       n_new=int32([1]))
            torch.cuda.synchronize()
            for got in (cache.at(cache.k, 0, 0, 0, 0), cache.at(cache.v, 0, 0, 0, 0)):
                got_code, got_s, got_c = parts(got)
                assert torch.equal(got_c.isnan(), torch.tensor([False, True, False, False], device=DEV)) and float(got_s[1]) == 0
                for g in (0, 2, 3):
                    assert torch.equal(got_code[32 * g:32 * g + 32], code[32 * g:32 * g + 32]), (T, dtype, g)
                    assert float(got_s[g]) == float(s[g]) and float(got_c[g]) == float(c[g])


@pytest.mark.parametrize("H", [1, 8, 40])
def test_append_keys_that_are_all_in_doubt(H):
    """Keys at position 0 stay as they are, and sixteenths put many (x - c) / s halfway between two codes: each row is done again, and
    is what the definition says byte for byte; so are more rows than a block lists, and the rows of the other tokens stay right."""
    T = 9
    x = (torch.randint(-40, 41, (1, T, H, D), generator=gen(6), device=DEV) / 16).to(torch.bfloat16)
    ctx = context(1, H, 1)
    cache = Cache4(1, 1, H, 16)
    status = int32([0])
    ctx.append(tb.LayerCache(cache.view(tb, seq_lens=int32([0])), 0), x, x.clone(), torch.zeros(1, dtype=torch.int64, device=DEV), device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    want = as_rows(x[0].double())
    for t in range(T):
        for h in range(H):
            assert torch.equal(cache.at(cache.v, 0, 0, h, t), want[t, h])
            wk = rope(x[0, t, h].double(), t, 1e6, False)
            check_row(cache.at(cache.k, 0, 0, h, t), wk, 2.0 ** -21 * pair_magnitude(wk, False))
            if t == 0:
                assert torch.equal(cache.at(cache.k, 0, 0, h, t), want[t, h])


@pytest.mark.parametrize("T", [1, 9])
@pytest.mark.parametrize("half_split", [False, True])
def test_append_queries_in_place(T, half_split):
    S, H, G = 3, 2, 5
    ctx = context(1, H, G, half_split=half_split)
    g = gen(T)
    q, k = (torch.randn(S, T, n, D, generator=g, device=DEV).to(torch.bfloat16) for n in (G * H, H))
    pos = torch.tensor([0, 7, 1000], device=DEV)
    want = torch.empty_like(q)
    for to in (want, q):
        cache = Cache4(1, S, H, 16)
        ctx.append(tb.LayerCache(cache.view(tb, seq_lens=int32([0, 3, 5])), 0), k, k.clone(), pos, q=q, q_out=to)
    torch.cuda.synchronize()
    assert torch.equal(q, want)


def test_append_without_values_and_rows_without_a_place():
    ctx, S = context(1, 1, 1), 1
    k = torch.randn(1, 4, 1, D, generator=gen(0), device=DEV)
    for lens, n_new, pos, table, want in ((28, 4, 0, None, (0, 4)), (30, 4, 0, None, (5, 2)), (-3, 4, 0, None, (0, 4)),
                                          (0, 4, 2 ** 31 - 2, None, (5, 2)), (14, 4, 0, [0, 99], (5, 2)), (14, 4, 0, [-1, 1], (5, 2)),
                                          (0, 9, 0, None, (5, 4))):
        c = Cache4(1, S, 1, 32, page=16)
        if table is not None:
            c.table.copy_(int32([table]))
        status = int32([0])
        view = tb.CacheView(c.k, None, seq_lens=int32([lens]), page_table=c.table)
        ctx.append(tb.LayerCache(view, 0), k, None, torch.tensor([pos], device=DEV), n_new=int32([n_new]), device_status=status)
        torch.cuda.synchronize()
        assert (int(status), int((c.k != 255).any(-1).sum())) == want and bool((c.v == 255).all())


# ------------------------------------------------------------------------------------------------
# read
# ------------------------------------------------------------------------------------------------
def check_read(fmt, kind, page, order, H, lens, T, first=None, per_head=False, token_major=True, scales=False, seed=0):
    S, L, layer = len(lens), 2, 1
    unit = lens if per_head else [[n] * H for n in lens]
    rows = max(max(max(r) for r in unit), 1)
    c = Cache4(L, S, H, rows, page, order, seed=seed) if fmt == "row4" else Cache(L, S, H, rows, fmt, page, order, seed=seed)
    g = gen(seed)
    for s in range(S):
        for h in range(H):
            if unit[s][h] > 0:
                c.fill(layer, s, h, unit[s][h], g)
    dt = torch.bfloat16 if kind == 0 else torch.float32
    mark = 7.0

    def make():
        t = torch.full((S, T, H, 136) if token_major else (S, H, T, D), mark, dtype=dt, device=DEV)
        return t[..., :D] if token_major else t.transpose(1, 2)
    ko, vo = make(), make()
    ks = 0.25 + torch.rand(L, H, generator=g, device=DEV) if scales else None
    vs = 0.25 + torch.rand(L, H, generator=g, device=DEV) if scales else None
    src = tb.LayerCache(c.view(tb, seq_lens=int32([r[0] for r in unit])), layer, unit_lens=int32([unit, unit]).contiguous() if per_head else None,
                        k_scale=ks, v_scale=vs)
    status = int32([0])
    context(L, H, 1).read(src, ko, vo, first=None if first is None else int32(first), device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    u = 2.0 ** -24 + (U_BF16 if kind == 0 else 0.0)
    for s in range(S):
        f = max(first[s], 0) if first is not None else 0
        for h in range(H):
            n = max(0, min(unit[s][h] - f, T))
            for t, out, sc in ((c.k, ko, ks), (c.v, vo, vs)):
                if n:
                    r = c.unit(t, layer, s, h, f + n)[f:]
                    want = (values(r) if fmt == "row4" else r) * (1.0 if sc is None else float(sc[layer, h]))
                    got = out[s, :n, h].double()
                    if fmt in ("row4", "e4m3") or (kind == 0 and fmt == "f32"):
                        assert bool(((got - want).abs() <= u * want.abs() * 1.0001).all())
                    else:
                        assert torch.equal(got, want)
                assert bool((out[s, n:, h] == mark).all())
    # between the rows nothing was written
    if token_major:
        for t in (ko, vo):
            assert bool((t.as_strided((S, T, H, 8), t.stride(), D) == mark).all())


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("fmt", ["row4", "bf16", "pre16", "e4m3", "f32"])
def test_read_formats(fmt, kind):
    check_read(fmt, kind, 16, "heads", 3, [5, 0, 37], 40, scales=fmt == "e4m3")


@pytest.mark.parametrize("page,order", [(0, "heads"), (0, "tokens"), (0, "padded"), (48, "tokens"), (32, "padded")])
@pytest.mark.parametrize("T,lens,first", [(1, [1, 30], [0, 29]), (7, [3, 20, 0], None), (33, [40, 12, 200], [7, 20, 190]), (300, [300, 129], None),
                                          (130, [140, 5], [-3, 2])])
def test_read_layouts_and_ranges(page, order, T, lens, first):
    check_read("row4", 0, page, order, 2, lens, T, first, token_major=order != "tokens", seed=T)


def test_read_lengths_of_heads_and_many_heads():
    check_read("row4", 0, 16, "heads", 2, [[4, 70], [0, 3]], 64, per_head=True)
    for T in (1, 2, 5):
        check_read("row4", 1, 16, "heads", 37, [9, 2], T, first=[6, 1])


def test_read_keys_or_values_alone_and_bad_pages():
    c = Cache4(1, 1, 1, 48, page=16)
    c.fill(0, 0, 0, 48, gen(0))
    want = values(c.unit(c.v, 0, 0, 0, 48))
    c.table[0, 1] = 77
    ctx, status = context(1, 1, 1), int32([0])
    lc = tb.LayerCache(c.view(tb, seq_lens=int32([48])), 0)
    v = torch.full((1, 48, 1, D), 7.0, device=DEV)
    ctx.read(lc, None, v, device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 5 and bool((v[0, 16:32] == 7).all())
    keep = torch.tensor([*range(16), *range(32, 48)], device=DEV)
    assert torch.allclose(v[0, keep, 0].double(), want[keep], rtol=2.0 ** -23, atol=0)
    k = torch.full_like(v, 7.0)
    keys = tb.LayerCache(tb.CacheView(c.k, None, seq_lens=int32([5]), page_table=c.table), 0)
    ctx.read(keys, k)
    torch.cuda.synchronize()
    assert bool((k[0, 5:] == 7).all()) and bool((k[0, :5] != 7).any(-1).all())


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------
def check_attend(G, H, lens, page=0, order="heads", per_head=False, scale=None, rows=None, seed=0, q_spread=2.0, k_spread=0.5, v_spread=1.0, layer=1,
                 fill=None, status=0, spot=1):
    S, L = len(lens), 2
    unit = lens if per_head else [[n] * H for n in lens]
    N = rows or max(max(max(r) for r in unit), 1)
    c = Cache4(L, S, H, N, page, order, seed=seed)
    g = gen(seed)
    have = [[min(max(n, 0), c.rows) for n in r] for r in unit]
    for s in range(S):
        for h in range(H):
            if have[s][h]:
                c.fill(layer, s, h, have[s][h], g, k_spread, v_spread)
                if fill:
                    fill(c, layer, s, h, have[s][h])
    q = (q_spread * torch.randn(S, H * G + 1, D, generator=g, device=DEV)).to(torch.bfloat16)[:, 1:]
    out = torch.full((S, H * G, 136), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((S, H * G), 7.0, device=DEV)
    ctx = context(L, H, G)
    src = tb.LayerCache(c.view(tb, seq_lens=int32([r[0] for r in unit])), layer, unit_lens=int32([unit, unit]).contiguous() if per_head else None)
    st = int32([0])
    ws = ctx.attend_workspace(S)
    ws.fill_(255)
    ctx.attend(src, q, out[..., :D], ws, scale=scale, lse=lse, device_status=st)
    torch.cuda.synchronize()
    assert int(st) == status
    assert bool((out[..., D:] == 7).all())
    again = torch.empty_like(out)
    ctx.attend(src, q, again[..., :D], ws, scale=scale, lse=lse)
    assert torch.equal(out[..., :D].contiguous().view(torch.int16), again[..., :D].contiguous().view(torch.int16))
    sc = D ** -0.5 if scale is None else scale
    for s in range(0, S, spot):                                      # (each spot-th sequence, and the head that goes with it)
        for h in range(H) if spot == 1 else (s % H,):
            n = have[s][h]
            k, v = c.unit(c.k, layer, s, h, n), c.unit(c.v, layer, s, h, n)
            for i in range(G):
                want, wl, tol, tl = R.attention(q[s, h * G + i].double(), k, v, sc)
                got = out[s, h * G + i, :D].double()
                off = (got - want).abs() - tol - U_BF16 * want.abs()
                assert bool((off <= 0).all()), (s, h, i, n, float(off.max()))
                if n:
                    assert abs(float(lse[s, h * G + i]) - wl) <= tl + 2.0 ** -22 * abs(wl)
                else:
                    assert float(lse[s, h * G + i]) == -math.inf


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 9, 12, 16])
def test_attend_groups(G):
    check_attend(G, 2, [1, 16, 47, 130, 0, 555], seed=G)                     # a cluster for each unit
    check_attend(G, 8, [3, 700, 129, 31, 0, 1, 64, 2000], page=16, seed=G)   # shares of the line


@pytest.mark.parametrize("page,order", [(0, "heads"), (0, "tokens"), (0, "padded"), (16, "heads"), (16, "tokens"), (32, "padded"), (48, "heads"), (64, "heads")])
def test_attend_layouts(page, order):
    check_attend(4, 3, [15, 16, 17, 33, 400, 127, 128, 129, 1, 0, 32, 31, 600], page, order, seed=page)
    check_attend(9, 2, [50, 300], page, order, seed=page + 1)


def test_attend_lengths():
    check_attend(4, 2, [5, -3, 900, 64], rows=80, page=16)                   # below 0: 0; above the capacity: the capacity
    check_attend(4, 3, [[5, 0, 300], [0, 0, 0], [129, 1, 64]] * 5, per_head=True, page=16)
    check_attend(5, 1, [4352]), check_attend(4, 1, [4353]), check_attend(16, 1, [9000], page=48)
    check_attend(4, 2, [8192, 8100]), check_attend(8, 1, [8193], page=16), check_attend(12, 1, [3584, 100]), check_attend(9, 1, [3585])
    check_attend(4, 8, [20000], page=16, seed=3), check_attend(8, 1, [20000, 3])
    check_attend(2, 1, [1]), check_attend(8, 1, [1], page=16)


def test_attend_many_short_units():
    check_attend(4, 8, [1 + 3 * (i % 7) for i in range(48)], page=16)
    check_attend(16, 8, [0] * 40 + [2])


@pytest.mark.parametrize("scale", [0.0, -0.1, 0.5])
def test_attend_scales(scale):
    check_attend(4, 2, [130, 700], scale=scale)


def test_attend_logits_far_apart():
    """One row that outweighs all others, wherever it lies; rows that go on passing the bound."""
    def spike(at, by):
        def fill(c, l, s, h, n):
            if n:
                c.put(c.k, l, s, h, torch.cat((c.unit(c.k, l, s, h, n)[:at % n], as_rows(by * torch.randn(1, D, generator=gen(9), device=DEV)),
                                               c.unit(c.k, l, s, h, n)[at % n + 1:])))
        return fill
    for at in (0, 17, 699):
        check_attend(4, 2, [700, 60], fill=spike(at, 12.0), q_spread=4.0)

    def rising(c, l, s, h, n):
        x = torch.randn(1, D, generator=gen(3), device=DEV) * torch.linspace(0, 3, n, device=DEV)[:, None]
        c.put(c.k, l, s, h, as_rows(x))
    check_attend(8, 2, [900, 60], fill=rising, q_spread=3.0)


@pytest.mark.parametrize("G", [4, 8, 16])
def test_attend_bounds_raised_before_and_behind_the_sums_of_16_steps(G):
    """Logits, or the sizes of values, that go on growing or falling along rows that one block walks past multiples of 16 steps of 128
    rows: in a cluster, and (many units of other lengths) in shares of the line."""
    def grows(keys, first, last):
        def fill(c, l, s, h, n):
            by = torch.linspace(first, last, max(n, 1), device=DEV)[:n, None]
            if keys and n:
                c.put(c.k, l, s, h, as_rows(by * torch.randn(1, D, generator=gen(3), device=DEV)))
            elif n:
                c.put(c.v, l, s, h, as_rows(torch.exp2(by) * torch.randn(n, D, generator=gen(n), device=DEV)))
        return fill
    for i, fill in enumerate((grows(True, 0, 3), grows(True, -3, 0), grows(False, -12, 12), grows(False, 12, -12))):
        check_attend(G, 1, [4480 if G <= 8 else 3500, 2100], fill=fill, q_spread=3.0 if i < 2 else 0.5, seed=i)
        if i in (0, 2):
            check_attend(G, 16, [2300] * 30 + [2100, 1], fill=fill, q_spread=3.0 if i < 2 else 0.5, seed=i, page=16, spot=3)


def test_attend_scales_of_values_far_apart():
    """Rows whose values differ by orders of magnitude, in both orders; constant rows, whose scale is 0; all of them constant."""
    for sign in (1, -1):
        n = 800
        spread = torch.exp2(sign * torch.linspace(-12, 12, n, device=DEV))[:, None]

        def fill(c, l, s, h, m):
            c.put(c.v, l, s, h, as_rows(spread[:m] * torch.randn(m, D, generator=gen(m), device=DEV)))
        check_attend(4, 2, [n, n - 77], fill=fill, q_spread=0.5)

    def constant(c, l, s, h, m):
        x = torch.randn(m, D, generator=gen(m), device=DEV)
        x[:, 32:64] = x[:, 32:33]
        x[::3] = x[::3, :1]
        c.put(c.v, l, s, h, as_rows(x))
    check_attend(4, 2, [300, 41], fill=constant)
    check_attend(4, 2, [300, 41], fill=lambda c, l, s, h, m: c.put(c.v, l, s, h, as_rows(torch.full((m, D), 0.75, device=DEV))))
    check_attend(4, 2, [300, 41], fill=lambda c, l, s, h, m: c.put(c.v, l, s, h, as_rows(1e-30 * torch.randn(m, D, generator=gen(m), device=DEV))))
    check_attend(4, 2, [300, 41], fill=lambda c, l, s, h, m: c.put(c.v, l, s, h, as_rows(1e20 * torch.randn(m, D, generator=gen(m), device=DEV))))


@pytest.mark.parametrize("sizes", [(None, 50), (None, 99), (-100, 90)])
@pytest.mark.parametrize("constant", [False, True])
def test_attend_rows_of_no_size_beside_huge_ones(sizes, constant):
    """All rows weigh about the same, and some hold values of size 2^50 to 2^99, others zeros or values down to 2^-100: before and
    behind one another in one warp, row by row, in warps, in blocks of a cluster and in shares of the line.  None drops out of the
    softmax.  `constant`: the huge groups have scale 0 and a huge centre."""
    small, big = sizes

    def rows_of(n, e, g):
        x = torch.zeros(n, D, dtype=torch.float64, device=DEV)
        if e is not None:
            x = 2.0 ** e * (1 + (0.0 if constant and e == big else 0.25) * torch.randn(n, D, generator=g, device=DEV).double())
        return as_rows(x)

    def fill(is_big):
        def put(c, l, s, h, n):
            g = gen(n)
            big_rows = is_big(torch.arange(n, device=DEV), n)
            c.put(c.v, l, s, h, torch.where(big_rows[:, None], rows_of(n, big, g), rows_of(n, small, g)))
        return put
    where = [lambda i, n: i >= n // 2, lambda i, n: i < (n + 1) // 2, lambda i, n: i % 2 == 1, lambda i, n: i % 64 >= 32,
             lambda i, n: i % 64 < 32, lambda i, n: i % 256 >= 128, lambda i, n: i == n - 1, lambda i, n: i == 0]
    for j, is_big in enumerate(where):
        G = (4, 8, 4, 16, 4, 1, 4, 8)[j]
        check_attend(G, 1, [2, 300, 2600], fill=fill(is_big), q_spread=0.25, seed=j)                          # clusters
        check_attend(G, 1, [9000, 33], fill=fill(is_big), q_spread=0.25, seed=j, page=16)                     # the whole GPU
        if j == 3:
            check_attend(G, 3, [130 + i for i in range(20)], fill=fill(is_big), q_spread=0.25, seed=j, spot=7)   # units cut between blocks


def test_attend_centres_far_from_zero():
    def fill(c, l, s, h, m):
        c.put(c.k, l, s, h, as_rows(20 + 0.1 * torch.randn(m, D, generator=gen(m), device=DEV)))
        c.put(c.v, l, s, h, as_rows(-50 + 0.1 * torch.randn(m, D, generator=gen(m + 1), device=DEV)))
    check_attend(4, 2, [300, 41], fill=fill, q_spread=0.5)


def test_attend_not_a_number():
    """A NaN among a unit's keys makes the unit's outputs NaN; one among its values those of its group of 32 components; none behind
    the length reaches anything (every unused row of these caches holds NaN)."""
    G, H = 4, 2
    for N in (100, 9000):
        ctx, c = context(1, H, G), Cache4(1, 2, H, N)
        for s in range(2):
            for h in range(H):
                c.fill(0, s, h, 70, gen(h))
        x = torch.randn(70, D, generator=gen(8), device=DEV)
        x[40, 33] = float("nan")
        ctx2 = context(1, 1, 1)
        one = Cache4(1, 1, 1, 70)
        ctx2.append(tb.LayerCache(one.view(tb, seq_lens=int32([0])), 0), x.view(1, 70, 1, D), x.view(1, 70, 1, D), torch.tensor([0], device=DEV))
        c.put(c.k, 0, 0, 1, one.k[0, 0, 0])
        c.put(c.v, 0, 1, 0, one.v[0, 0, 0])
        q = torch.randn(2, H * G, D, generator=gen(1), device=DEV).to(torch.bfloat16)
        out, lse = torch.empty_like(q), torch.zeros(2, H * G, device=DEV)
        ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([70, 70])), 0), q, out, ctx.attend_workspace(2), lse=lse)
        torch.cuda.synchronize()
        bad = out.isnan().view(2, H, G, 4, 32)
        want = torch.zeros_like(bad)
        want[0, 1] = True
        want[1, 0, :, 1] = True
        assert torch.equal(bad, want)
        assert torch.equal(lse.isnan().view(2, H, G), want[..., 0, 0] & want[..., 3, 0])


@pytest.mark.parametrize("rows", [200, 6000])
def test_attend_bad_pages(rows):
    """Rows of pages outside the pool count as absent, whatever their neighbours are."""
    G, H, n = 4, 2, 200
    c = Cache4(1, 1, H, rows, page=16)
    for h in range(H):
        c.fill(0, 0, h, n, gen(h))
    keep = [i for i in range(n) if i // 16 not in (0, 5, 12)]
    k = [c.unit(c.k, 0, 0, h, n)[keep] for h in range(H)]
    v = [c.unit(c.v, 0, 0, h, n)[keep] for h in range(H)]
    c.table[0, 0], c.table[0, 5], c.table[0, 12] = -1, 1 << 30, c.k.shape[1]
    ctx, st = context(1, H, G), int32([0])
    q = torch.randn(1, H * G, D, generator=gen(1), device=DEV).to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([n])), 0), q, out, ctx.attend_workspace(1), device_status=st)
    torch.cuda.synchronize()
    assert int(st) == 5
    for h in range(H):
        for i in range(G):
            want, _, tol, _ = R.attention(q[0, h * G + i].double(), k[h], v[h], D ** -0.5)
            assert bool(((out[0, h * G + i].double() - want).abs() <= tol + U_BF16 * want.abs()).all())


# ------------------------------------------------------------------------------------------------
# moving kept rows
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page,order", [(0, "heads"), (0, "tokens"), (0, "padded"), (16, "heads"), (48, "padded")])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("keep", ["random", "front", "back"])
def test_compact(page, order, in_place, keep):
    L, S, H, N, B = 2, 3, 2, 1500, 900
    lens = [1500, 700, 901]
    g = torch.Generator().manual_seed(page)
    c = Cache4(L, S, H, N, page, order)
    c.k.copy_(torch.randint(0, 256, c.k.shape, dtype=torch.uint8, generator=g))
    c.v.copy_(torch.randint(0, 256, c.v.shape, dtype=torch.uint8, generator=g))
    pos = torch.randint(0, 10 ** 6, (L, S, H, c.rows), dtype=torch.int32, generator=g).to(DEV)
    idx = torch.full((L, S, H, B), 1 << 29, dtype=torch.int32)
    cnt = torch.zeros(L, S, H, dtype=torch.int32)
    for l in range(L):
        for s in range(S):
            for h in range(H):
                n = min(B, lens[s])
                if keep == "random":
                    sel = torch.randperm(lens[s], generator=g)[:n].sort().values
                elif keep == "front":
                    sel = torch.arange(n)
                    sel[n // 2:] += lens[s] - n
                else:
                    sel = torch.arange(lens[s] - n, lens[s])
                idx[l, s, h, :n], cnt[l, s, h] = sel.to(torch.int32), n
    d = c if in_place else Cache4(L, S, H, B, 32, "padded", seed=1)
    dpos = pos if in_place else torch.full((L, S, H, d.rows), -1, dtype=torch.int32, device=DEV)
    wk, wv, wp = d.k.clone(), d.v.clone(), dpos.clone()
    for l in range(L):
        for s in range(S):
            for h in range(H):
                n = int(cnt[l, s, h])
                sel = idx[l, s, h, :n].long().to(DEV)
                for t, w in ((c.k, wk), (c.v, wv)):
                    d.put(w, l, s, h, c.unit(t, l, s, h, lens[s])[sel])
                wp[l, s, h, :n] = pos[l, s, h, sel]
    ctx, new = context(L, H, 2), int32([0] * S)
    src = c.view(tb, seq_lens=int32(lens), positions=pos)
    ctx.compact(src, idx.to(DEV), cnt.to(DEV), S, B, src if in_place else d.view(tb, positions=dpos), new)
    torch.cuda.synchronize()
    assert torch.equal(d.k, wk) and torch.equal(d.v, wv) and torch.equal(dpos, wp)
    assert new.tolist() == [min(B, n) for n in lens]


def test_compact_many_units_in_place():
    """Units enough to fill the GPU: one launch moves all of their rows, whatever part lies behind the kept count."""
    S, H, N, B = 40, 8, 400, 200
    g = gen(0)
    c = Cache4(1, S, H, N, page=16)
    c.k.copy_(torch.randint(0, 256, c.k.shape, dtype=torch.uint8, device=DEV, generator=g))
    c.v.copy_(torch.randint(0, 256, c.v.shape, dtype=torch.uint8, device=DEV, generator=g))
    lens = [N if s % 3 else 10 * (s % 7) for s in range(S)]
    cnt = int32([[min(B, n)] * H for n in lens])
    score = torch.rand(S, H, N, generator=g, device=DEV) - 2.0 * (torch.arange(N, device=DEV) >= int32(lens)[:, None, None])
    idx = score.topk(B, -1).indices
    idx = (idx + N * (torch.arange(B, device=DEV) >= cnt[..., None])).sort(-1).values % N
    want_k, want_v = c.k.clone(), c.v.clone()
    for s in range(S):
        n = min(B, lens[s])
        for h in range(H):
            for t, w in ((c.k, want_k), (c.v, want_v)):
                c.put(w, 0, s, h, c.unit(t, 0, s, h, N)[idx[s, h, :n]])
    new = int32([0] * S)
    view = c.view(tb, seq_lens=int32(lens))
    context(1, H, 1).compact(view, idx.to(torch.int32).contiguous(), cnt.contiguous(), S, B, view, new)
    torch.cuda.synchronize()
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v) and new.tolist() == [min(B, n) for n in lens]


@pytest.mark.parametrize("page", [0, 16])
def test_compact_few_units_of_many_rows_in_place(page):
    """Few units that keep less than half of their rows: a first launch for the rows from within the kept count, a second for the rest."""
    H, N, B = 6, 3000, 1200
    g = torch.Generator().manual_seed(page)
    c = Cache4(1, 1, H, N, page)
    c.k.copy_(torch.randint(0, 256, c.k.shape, dtype=torch.uint8, generator=g))
    c.v.copy_(torch.randint(0, 256, c.v.shape, dtype=torch.uint8, generator=g))
    pos = torch.randint(0, 10 ** 6, (1, 1, H, c.rows), dtype=torch.int32, generator=g).to(DEV)
    keep = [torch.randperm(N, generator=g)[:B].sort().values, torch.arange(N - B, N), torch.arange(B),
            torch.cat((torch.arange(1, 401), torch.arange(N - 800, N))), torch.cat((torch.arange(0, 2 * 500, 2), torch.arange(2000, 2100))), torch.arange(0)]
    idx = torch.full((1, 1, H, B), 1 << 29, dtype=torch.int32)
    cnt = int32([[[len(x) for x in keep]]])
    want_k, want_v, want_p = c.k.clone(), c.v.clone(), pos.clone()
    for h, sel in enumerate(keep):
        idx[0, 0, h, :len(sel)] = sel.to(torch.int32)
        for t, w in ((c.k, want_k), (c.v, want_v)):
            c.put(w, 0, 0, h, c.unit(t, 0, 0, h, N)[sel.to(DEV)])
        want_p[0, 0, h, :len(sel)] = pos[0, 0, h, sel.to(DEV)]
    view = c.view(tb, seq_lens=int32([N]), positions=pos)
    context(1, H, 1).compact(view, idx.to(DEV), cnt, 1, B, view)
    torch.cuda.synchronize()
    assert torch.equal(c.k, want_k) and torch.equal(c.v, want_v) and torch.equal(pos, want_p)


def test_compact_keys_alone_and_indices_outside():
    """Without values the keys move alone; indices outside the unit move nothing."""
    for in_place in (False, True):
        c = Cache4(1, 1, 1, 64)
        c.fill(0, 0, 0, 64, gen(0))
        k0 = c.k.clone()
        d = c if in_place else Cache4(1, 1, 1, 64)
        idx = int32([[[[1, 3, 40, 64, 1 << 30]]]])
        want = d.k.clone()
        want[0, 0, 0, :3] = k0[0, 0, 0, [1, 3, 40]]
        v0 = d.v.clone()
        context(1, 1, 1).compact(tb.CacheView(c.k, None), idx, int32([[[5]]]), 1, 5, tb.CacheView(d.k, None))
        torch.cuda.synchronize()
        assert torch.equal(d.k, want) and torch.equal(d.v, v0)


# ------------------------------------------------------------------------------------------------
# together, on streams, in graphs, and refused
# ------------------------------------------------------------------------------------------------
def test_prompt_round_and_decode_steps_together():
    """A prompt goes into the cache, a round keeps some of its rows (scored on what tri_read makes of the keys), decode steps go on
    behind them: the attention of the last step is that of a 64-bit computation over the rows that the cache holds, and every kept
    row is one that was appended, with its position."""
    H, G, S, T, B = 2, 4, 3, 300, 96
    g = gen(4)
    ctx = tb.TriContext(1, H, G, torch.randn(1, H * G, D, generator=torch.Generator().manual_seed(0)), torch.ones(1, H * G, D // 2))
    c = Cache4(1, S, H, T + 16, page=16)
    lens, after = int32([0] * S), int32([0] * S)
    pos_t = torch.zeros(1, S, H, c.rows, dtype=torch.int32, device=DEV)
    view = c.view(tb, seq_lens=lens, positions=pos_t)
    cache, then = tb.LayerCache(view, 0), tb.LayerCache(c.view(tb, seq_lens=after, positions=pos_t), 0)
    k, v = (torch.randn(S, T, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    counts = int32([300, 41, 255])
    pos = torch.tensor([0, 7, 1000], device=DEV)
    ctx.append(cache, k, v, pos, n_new=counts, new_lens=lens)
    keys = torch.zeros(1, S, H, c.rows, D, dtype=torch.bfloat16, device=DEV)
    ctx.read(cache, keys[0].transpose(1, 2))
    U = S * H
    idx, cnt = torch.zeros(U, B, dtype=torch.int32, device=DEV), torch.zeros(U, dtype=torch.int32, device=DEV)
    scores = torch.zeros(U, c.rows, device=DEV)
    cur = pos + counts
    ctx.score(tb.CacheView(keys, None, seq_lens=lens, positions=pos_t), cur, scores, ctx.workspace(S, c.rows, B))
    ctx.select(scores, lens, c.rows, B, idx, cnt)
    all_k, all_v = c.k.clone(), c.v.clone()
    ctx.compact(view, idx, cnt, S, B, view, lens)
    torch.cuda.synchronize()
    assert lens.tolist() == [96, 41, 96]
    for s in range(S):
        for h in range(H):
            n = int(lens[s])
            sel = idx[s * H + h, :n].long()
            assert torch.equal(c.unit(c.k, 0, s, h, n), c.unit(all_k, 0, s, h, 300)[sel])
            assert torch.equal(c.unit(c.v, 0, s, h, n), c.unit(all_v, 0, s, h, 300)[sel])
            assert torch.equal(pos_t[0, s, h, :n].long(), sel + pos[s])
    ws, status = ctx.attend_workspace(S), int32([0])
    for step in range(3):
        k1, v1 = (torch.randn(S, 1, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        q1 = torch.randn(S, 1, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
        q_rot, out = torch.empty_like(q1), torch.empty(S, H * G, D, dtype=torch.bfloat16, device=DEV)
        ctx.append(cache, k1, v1, cur + step, q=q1, q_out=q_rot, new_lens=after, device_status=status)
        ctx.attend(then, q_rot[:, 0], out, ws, device_status=status)
        lens.copy_(after)
    torch.cuda.synchronize()
    assert int(status) == 0 and lens.tolist() == [99, 44, 99]
    for s in range(S):
        for h in range(H):
            n = int(lens[s])
            assert int(pos_t[0, s, h, n - 1]) == int(cur[s]) + 2
            for i in range(G):
                want, _, tol, _ = R.attention(q_rot[s, 0, h * G + i].double(), c.unit(c.k, 0, s, h, n), c.unit(c.v, 0, s, h, n), D ** -0.5)
                assert bool(((out[s, h * G + i].double() - want).abs() <= tol + U_BF16 * want.abs()).all())


def test_rows_beyond_32_bits_of_offset():
    """A unit whose last rows lie 2^31 bytes behind its first: append, read back, attention and a move, in the second of two layers that
    lie 2^32 bytes apart.  The rows between are zeros (logit 0, value 0)."""
    N, G, L = 28_000_000, 2, 2                                        # 2.24e9 bytes of keys and of values per layer
    k, v = (torch.zeros(L, 1, 1, N, ROW, dtype=torch.uint8, device=DEV) for _ in range(2))
    for t in (k, v):
        t[1, ..., :64] = 0x88
    ctx = context(L, 1, G)
    lens, after = int32([N - 3]), int32([0])
    g = gen(3)
    x = torch.randn(1, 3, 1, D, generator=g, device=DEV).to(torch.bfloat16)
    view = tb.CacheView(k, v, seq_lens=lens)
    ctx.append(tb.LayerCache(view, 1), x, x, torch.tensor([5], device=DEV), new_lens=after)
    then = tb.LayerCache(tb.CacheView(k, v, seq_lens=after), 1)
    kb, vb = (torch.zeros(1, 3, 1, D, device=DEV) for _ in range(2))
    ctx.read(then, kb, vb, first=lens)
    torch.cuda.synchronize()
    assert int(after) == N
    for t in range(3):
        row = k[1, 0, 0, N - 3 + t]
        want = rope(x[0, t, 0].double(), 5 + t, 1e6, False)
        check_row(row, want, (2.0 ** -21 + 2.0 ** -48) * pair_magnitude(want, False))
        assert torch.allclose(kb[0, t, 0].double(), values(row), rtol=2.0 ** -23, atol=0)
        assert torch.allclose(vb[0, t, 0].double(), values(v[1, 0, 0, N - 3 + t]), rtol=2.0 ** -23, atol=0)
    assert not k[0].any() and not v[0].any() and bool((k[1, 0, 0, :N - 3, 64:] == 0).all())
    q = (6 * kb[0, 1:2, 0].expand(1, G, D)).to(torch.bfloat16).contiguous()       # a logit that outweighs 28 million zeros
    out, lse = torch.zeros(1, G, D, dtype=torch.bfloat16, device=DEV), torch.zeros(1, G, device=DEV)
    ctx.attend(then, q, out, ctx.attend_workspace(1), lse=lse)
    torch.cuda.synchronize()
    rows_k, rows_v = k[1, 0, 0, N - 3:], v[1, 0, 0, N - 3:]
    for i in range(G):
        qi = q[0, i].double()
        logit = values(rows_k) @ qi * D ** -0.5
        top = max(float(logit.max()), 0.0)
        p = torch.exp(logit - top)
        total = float(p.sum()) + (N - 3) * math.exp(-top)
        want = p @ values(rows_v) / total
        _, _, tol, tl = R.attention(qi, rows_k, rows_v, D ** -0.5)
        # (zero rows: their logits are off by d, too, and N weights, each rounded, are summed: 2^-15 of the sum as for all)
        assert bool(((out[0, i].double() - want).abs() <= 2 * tol + U_BF16 * want.abs() + 2.0 ** -14 * values(rows_v).abs().amax(0)).all())
        assert abs(float(lse[0, i]) - (top + math.log(total))) <= 2 * tl + 2.0 ** -14
    # the three rows to the front of the unit
    idx, cnt, new = int32([[0, 0, 0], [N - 3, N - 2, N - 1]]), int32([0, 3]), int32([0])
    want_k, want_v = rows_k.clone(), rows_v.clone()
    ctx.compact(view, idx, cnt, 1, 3, view, new)
    torch.cuda.synchronize()
    assert torch.equal(k[1, 0, 0, :3], want_k) and torch.equal(v[1, 0, 0, :3], want_v)


def step_inputs(S, H, G, N, seed):
    c = Cache4(1, S, H, N, page=16, seed=seed)
    for s in range(S):
        for h in range(H):
            c.fill(0, s, h, 1 + (37 * s + N // 2) % (N - 8), gen(seed + s))
    lens = int32([1 + (37 * s + N // 2) % (N - 8) for s in range(S)])
    g = gen(seed + 100)
    x = torch.randn(S, 1, (G + 2) * H, D, generator=g, device=DEV).to(torch.bfloat16)
    return c, lens, x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]


@pytest.mark.parametrize("N", [400, 6000])
def test_steps_on_two_streams_and_in_two_graphs(N):
    """Append, attention and read back of two batches, first one after the other, then on two streams at once, then captured into two
    graphs that share one workspace and are replayed in turn: the same bits."""
    S, H, G = 5, 2, 4
    ctx = context(1, H, G)
    runs = []
    for seed in (0, 10):
        c, lens, q, k, v = step_inputs(S, H, G, N, seed)
        after = torch.zeros_like(lens)
        q_rot, out = torch.zeros(S, 1, G * H, D, dtype=torch.bfloat16, device=DEV), torch.zeros(S, G * H, D, dtype=torch.bfloat16, device=DEV)
        back = torch.zeros(S, 1, H, D, device=DEV)
        cache, then = tb.LayerCache(c.view(tb, seq_lens=lens), 0), tb.LayerCache(c.view(tb, seq_lens=after), 0)
        pos = lens.long() + 1000

        def step(ws, cache=cache, then=then, lens=lens, after=after, q=q, k=k, v=v, q_rot=q_rot, out=out, back=back, pos=pos, c=c):
            ctx.append(cache, k, v, pos, q=q, q_out=q_rot, new_lens=after)
            ctx.attend(then, q_rot[:, 0], out, ws)
            ctx.read(then, back, first=lens)
        runs.append((step, (out, back, after, q_rot, c.k, c.v)))
    ws = [ctx.attend_workspace(S), ctx.attend_workspace(S)]
    for (step, _), w in zip(runs, ws):
        step(w)
    torch.cuda.synchronize()
    want = [[t.clone() for t in outs] for _, outs in runs]

    def wipe():
        for _, outs in runs:
            for t in outs[:4]:
                t.zero_()
        torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        return all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for w, (_, outs) in zip(want, runs) for a, b in zip(w, outs))
    wipe()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (step, _), w, st in zip(runs, ws, streams):
            with torch.cuda.stream(st):
                step(w)
    assert same()
    graphs = []
    for step, _ in runs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(ws[0])
        graphs.append(gr)
    wipe()
    for _ in range(3):
        for gr in graphs:
            gr.replay()
    assert same()


def test_refusals():
    L, S, H, G = 2, 2, 2, 4
    ctx, lib = context(L, H, G), tb.lib()
    c = Cache4(L, S, H, 32)
    lens, f32 = int32([3, 5]), torch.ones(L, H, device=DEV)
    out = torch.zeros(S, 4, H, D, dtype=torch.bfloat16, device=DEV)
    out2 = torch.zeros_like(out)

    def layer_cache(layer=0, unit_lens=None, k_scale=None, v_scale=None, **kw):
        cv = c.view(tb, seq_lens=lens).c_view()
        for name, val in kw.items():
            setattr(cv, name, val)
        lc = tb._LayerCache(ctypes.pointer(cv), layer, unit_lens, k_scale, v_scale)
        lc.keep = cv
        return lc

    def read(lc=None, S=S, h=ctx._h, **kw):
        r = tb._ReadRows(k=out.data_ptr(), v=out2.data_ptr(), kind=0, T=4)
        for p in ("k", "v"):
            for n, st in zip(("seq", "tok", "head"), out.stride()):
                setattr(r, f"{p}_stride_{n}", st)
        for name, val in kw.items():
            setattr(r, name, val)
        return lib.tri_read(h, ctypes.byref(lc or layer_cache()), S, ctypes.byref(r), None, None)

    assert read() == 0 and read(k=None) == 0 and read(v=None) == 0
    torch.cuda.synchronize()
    assert lib.tri_read(ctx._h, None, 1, None, None, None) == 1 and read(h=None) == 1
    assert lib.tri_read(ctx._h, ctypes.byref(layer_cache()), S, None, None, None) == 1
    assert read(S=0) == 1 and read(T=0) == 1 and read(kind=2) == 1 and read(k=None, v=None) == 1 and read(v=out.data_ptr()) == 1
    assert read(k=out.data_ptr() + 8) == 1 and read(k_stride_tok=260) == 1 and read(v_stride_head=4) == 1
    assert read(k_stride_seq=0) == 1 and read(k_stride_tok=0) == 1 and read(v_stride_head=64) == 1      # destinations that meet
    assert read(layer_cache(layer=2)) == 1 and read(layer_cache(v=None)) == 1 and read(layer_cache(seq_lens=None)) == 1
    assert read(layer_cache(k_kind=4)) == 1 and read(layer_cache(k_kind=6)) == 1
    assert read(layer_cache(k_scale=f32.data_ptr())) == 1 and read(layer_cache(v_scale=f32.data_ptr())) == 1
    assert read(layer_cache(stride_tok=64)) == 1 and read(layer_cache(stride_tok=88)) == 1 and read(layer_cache(stride_head=8)) == 1
    # attention: rows too far apart, prefixes; the calls that score keys
    q = torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
    ws = ctx.attend_workspace(S, 1)
    with pytest.raises(tb.TriError) as e:
        ctx.attend_shared(tb.LayerCache(c.view(tb, seq_lens=lens), 0), int32([0, 1, 2]), tb.LayerCache(c.view(tb, seq_lens=lens), 0), q, q.clone(),
                          ctx.attend_workspace(S, 2))
    assert e.value.code == 2
    io = tb._AttendIo(q.data_ptr(), *q.stride()[:2], out.data_ptr(), *q.stride()[:2], None, 0.1)

    def attend(lc):
        return lib.tri_attend(ctx._h, ctypes.byref(lc), S, ctypes.byref(io), None, ws.data_ptr(), ws.numel(), None)
    assert attend(layer_cache()) == 0
    torch.cuda.synchronize()
    assert attend(layer_cache(v=None)) == 1 and attend(layer_cache(stride_tok=1 << 31)) == 2
    view = c.view(tb, seq_lens=lens)
    cur = torch.zeros(S, dtype=torch.int64, device=DEV)
    big = torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)
    scores = torch.zeros(L * S * H * 32, device=DEV)
    for call in (lambda: ctx.score(view, cur, scores, big), lambda: ctx.score_static(view, cur, scores),
                 lambda: ctx.compress(view, cur, 8, view, big),
                 lambda: ctx.compress(view, cur, 8, view, big, unit_budgets=int32([8] * (L * S * H))),
                 lambda: ctx.compress_windowed(view, cur, 8, int32([0] * S), 1, 128, view, big)):
        with pytest.raises(tb.TriError) as e:
            call()
        assert e.value.code == 2
    # formats do not mix
    other = tb.CacheView(torch.zeros(L, S, H, 32, D, dtype=torch.bfloat16, device=DEV), None)
    with pytest.raises(tb.TriError) as e:
        ctx.compact(tb.CacheView(c.k, None), torch.zeros(L * S * H, 8, dtype=torch.int32, device=DEV), int32([0] * (L * S * H)), S, 8, other)
    assert e.value.code == 1
    x = torch.zeros(S, 1, H, D, dtype=torch.bfloat16, device=DEV)
    wide = tb.LayerCache(tb.CacheView(c.k[:, :, :1].expand(L, S, H, 32, ROW), None, seq_lens=lens), 0)
    with pytest.raises(tb.TriError) as e:                             # heads that are one head
        ctx.append(wide, x, None, torch.zeros(S, dtype=torch.int64, device=DEV))
    assert e.value.code == 1


def test_another_current_device_and_host_pointers_are_refused_by_the_binding():
    ctx, c = context(1, 2, 1), Cache4(1, 1, 2, 16)
    lc = tb.LayerCache(c.view(tb, seq_lens=int32([3])), 0)
    x = torch.zeros(1, 3, 2, D, dtype=torch.bfloat16)
    for bad in (lambda: ctx.read(lc, x), lambda: ctx.read(lc, x.to(DEV), x), lambda: ctx.read(lc, x.to(DEV), first=torch.zeros(1, dtype=torch.int32)),
                lambda: ctx.read(lc, x.to(DEV), device_status=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(AssertionError):
            bad()


def test_rows_that_meet_under_their_strides_together_are_refused():
    """Strides that are each as long as a row, but bring two rows to one place; layouts that are unusual and sound are taken."""
    S, H, G, T = 2, 2, 3, 2
    ctx = context(1, H, G)
    c = Cache4(1, S, H, 32)
    lens = int32([3, 5])
    for s in range(S):
        for h in range(H):
            c.fill(0, s, h, 5, gen(2 * s + h))
    lc = tb.LayerCache(c.view(tb, seq_lens=lens), 0)
    room = torch.zeros(1 << 14, dtype=torch.bfloat16, device=DEV)

    def refused(call):
        with pytest.raises(tb.TriError) as e:
            call()
        assert e.value.code == 1

    def rows(*strides, n=(S, T, H)):
        return room.as_strided((*n, D), (*strides, 1))
    sound = torch.zeros(S, T, H, D, dtype=torch.bfloat16, device=DEV)
    for strides in ((512, 128, 128), (128, 256, 128), (128, 128, 512), (256, 384, 128), (1024, 200, 256)):
        refused(lambda: ctx.read(lc, rows(*strides)))
        refused(lambda: ctx.read(lc, None, rows(*strides)))
        refused(lambda: ctx.read(lc, sound, rows(*strides)))
    ctx.read(lc, sound)
    ctx.read(lc, rows(1024, 384, 256))                                   # not nested, and apart
    torch.cuda.synchronize()
    assert torch.equal(rows(1024, 384, 256), sound) and bool((sound != 0).any())
    # outputs of attention, rotated queries, a cache's heads among its slots
    q = torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
    refused(lambda: ctx.attend(lc, q, rows(256, 128, n=(S, H * G)), ctx.attend_workspace(S)))
    k, pos = torch.zeros(S, 1, H, D, dtype=torch.bfloat16, device=DEV), torch.zeros(S, dtype=torch.int64, device=DEV)
    q1, k2, q2 = q[:, None], k.expand(S, T, H, D).contiguous(), q[:, None].expand(S, T, H * G, D).contiguous()
    refused(lambda: ctx.append(lc, k, k.clone(), pos, q=q1, q_out=rows(256, 4096, 128, n=(S, 1, H * G))))
    refused(lambda: ctx.append(lc, k2, k2.clone(), pos, q=q2, q_out=rows(4096, 256, 128, n=(S, T, H * G))))
    pool = torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    for strides in ((1 << 13, 80, 80), (80, 80 * 32, 80), (80 * 32, 80 * 32, 80), (80 * 32, 80 * 16, 80)):
        heads = tb.LayerCache(tb.CacheView(pool.as_strided((1, S, H, 32, ROW), (1 << 15, *strides, 1)), None, seq_lens=lens), 0)
        refused(lambda: ctx.append(heads, k, None, pos))
    for strides in ((80 * 64, 80, 160), (80, 80 * 64, 160)):
        heads = tb.LayerCache(tb.CacheView(pool.as_strided((1, S, H, 32, ROW), (1 << 15, *strides, 1)), None, seq_lens=lens), 0)
        ctx.append(heads, k, None, pos)
    torch.cuda.synchronize()
