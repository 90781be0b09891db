"""The decode step around the compression round: appending rows to a cache with their rotation, attention of one query
token per sequence over the cache, and over prefixes that sequences share.  Against the 64-bit forms of
step_reference.py, whose header derives the bounds."""
import ctypes
import math

import pytest
import torch

from paper_2604_04921_b200 import binding as tb
from step_reference import Cache, D, E4M3_MAX, U_BF16, U_E4M3, attention, pair_magnitude, rope

pytestmark = pytest.mark.gpu
DEV = "cuda"


def context(L, H, G, theta=1e6, half_split=False):
    return tb.TriContext(L, H, G, torch.zeros(L, H * G, D), torch.ones(L, H * G, D // 2), rope_theta=theta,
                         pair_layout=int(half_split))


def raw(t):
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------
def check_append(fmt, kind, half_split, page, order, H, G, lens, n_new, T, pos, per_head=False, positions=True, layer=1,
                 in_place_lens=False, scales=False, rows=None, seed=0, theta=1e6):
    """One append into layer `layer` of two; everything it may write is compared with the definition, everything else
    with what was there, bit for bit.  Padding tokens hold NaN."""
    S, L = len(n_new), 2
    g = torch.Generator(device=DEV).manual_seed(seed)
    unit = lens if per_head else [[n] * H for n in lens]
    need = max(max(r) + c for r, c in zip(unit, n_new))
    c = Cache(L, S, H, rows or need, fmt, page, order, seed=seed)
    ctx = context(L, H, G, theta, half_split)
    dt = torch.bfloat16 if kind == 0 else torch.float32
    x = torch.randn(S, T, (G + 2) * H, D, generator=g, device=DEV).to(dt)
    for s in range(S):
        x[s, n_new[s]:] = float("nan")
    q, k, v = x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]
    q_out = torch.full((S, T, G * H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    pos_t = torch.full((L, S, H, c.rows), -7, dtype=torch.int32, device=DEV) if positions else None
    seq_lens = int32([r[0] for r in unit])
    unit_lens = int32([unit, unit]).contiguous() if per_head else None
    ks = 0.25 + torch.rand(L, H, generator=g, device=DEV) if scales else None
    vs = 0.25 + torch.rand(L, H, generator=g, device=DEV) if scales else None
    old = unit_lens if per_head else seq_lens
    new = old if in_place_lens else torch.full_like(old, -5)
    before = old.clone()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    k0, v0 = raw(c.k).clone(), raw(c.v).clone()
    dst = tb.LayerCache(c.view(tb, seq_lens=seq_lens, positions=pos_t), layer, unit_lens=unit_lens, k_scale=ks, v_scale=vs)
    ragged = any(n != T for n in n_new)
    ctx.append(dst, k, v, None if pos is None else torch.tensor(pos, device=DEV), q=q, q_out=q_out,
               n_new=int32(n_new) if ragged else None, new_lens=new, device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    kk, vv = raw(c.k).clone(), raw(c.v).clone()
    for s in range(S):
        for t in range(n_new[s]):
            p = (pos[s] if pos is not None else unit[s][0]) + t
            want_q = rope(q[s, t].double(), p, theta, half_split)
            rot = 2.0 ** -21 + p * 2.0 ** -51
            tol = U_BF16 * want_q.abs() + rot * pair_magnitude(want_q, half_split)
            assert bool(((q_out[s, t].double() - want_q).abs() <= tol).all()), ("q", s, t)
            for h in range(H):
                n = unit[s][h] + t
                wk = k[s, t, h].double() if fmt in ("pre16", "f32") else rope(k[s, t, h].double(), p, theta, half_split)
                wv = v[s, t, h].double()
                mag = pair_magnitude(wk, half_split)
                if ks is not None:
                    wk, mag, wv = wk / float(ks[layer, h]), mag / float(ks[layer, h]), wv / float(vs[layer, h])
                gk, gv = c.at(c.k, layer, s, h, n).double(), c.at(c.v, layer, s, h, n).double()
                if fmt == "e4m3":
                    tk = U_E4M3 * wk.abs() + 2.0 ** -10 + rot * mag
                    tv = U_E4M3 * wv.abs() + 2.0 ** -10
                else:
                    tk = U_BF16 * wk.abs() + rot * mag if fmt != "f32" else torch.zeros_like(wk)
                    tv = U_BF16 * wv.abs()
                assert bool(((gk - wk).abs() <= tk).all()), ("k", s, t, h)
                assert bool(((gv - wv).abs() <= tv).all()), ("v", s, t, h)
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
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "pre16", "f32"])
def test_append_formats(fmt, kind, half_split):
    check_append(fmt, kind, half_split, 16, "heads", 3, 2, [5, 0, 30], [3, 1, 2], 3, [70, 131071, 30], scales=fmt == "e4m3")


@pytest.mark.parametrize("fmt,page,order", [("bf16", 0, "heads"), ("bf16", 0, "tokens"), ("bf16", 0, "padded"),
                                            ("bf16", 48, "tokens"), ("e4m3", 0, "tokens"), ("e4m3", 32, "padded"),
                                            ("bf16", 16, "padded")])
@pytest.mark.parametrize("T,n_new", [(1, [1, 1]), (1, [0, 1]), (9, [9, 9]), (20, [0, 17]), (8, [8, 3])])
def test_append_layouts_and_counts(fmt, page, order, T, n_new):
    check_append(fmt, 0, True, page, order, 2, 3, [13, 33], n_new, T, [1000, 40000], seed=T)


@pytest.mark.parametrize("T", [1, 2, 8, 9, 16, 17])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_lengths_in_place(T, in_place):
    check_append("bf16", 0, False, 0, "heads", 1, 1, [4, 0, 9], [T, max(T - 1, 0), T], T, [4, 0, 9], in_place_lens=in_place)
    check_append("bf16", 0, False, 16, "heads", 2, 1, [[4, 7], [0, 3], [9, 9]], [T, 0, T], T, [50, 60, 70], per_head=True,
                 in_place_lens=in_place)


def test_append_position_is_the_slot_without_positions():
    check_append("bf16", 0, False, 16, "heads", 2, 2, [0, 21], [5, 5], 5, None, positions=False)


@pytest.mark.parametrize("theta,pos", [(1e4, 0), (1e6, 2 ** 20 + 3), (5e5, 2 ** 31 - 4), (1e6, 2 ** 31 - 2)])
def test_append_far_positions(theta, pos):
    check_append("bf16", 1, False, 0, "heads", 1, 1, [3], [2], 2, [pos], theta=theta)


def test_append_one_token_many_heads_and_sequences():
    check_append("bf16", 0, True, 16, "heads", 8, 16, [3 * s for s in range(33)], [1] * 33, 1, [1000 + s for s in range(33)])


def test_append_queries_in_place_and_values_kept_bit_for_bit():
    ctx, S, T, H, G = context(1, 2, 4), 2, 3, 2, 4
    c = Cache(1, S, H, 16)
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randn(S, T, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    k, v = (torch.randn(S, T, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    pos = torch.tensor([11, 5], device=DEV)
    a, b = torch.empty_like(q), q.clone()
    dst = tb.LayerCache(c.view(tb, seq_lens=int32([0, 4])), 0)
    ctx.append(dst, k, v, pos, q=q, q_out=a)
    ctx.append(dst, k, v, pos, q=b, q_out=b)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    assert torch.equal(c.v[0, 0, :, :T].transpose(0, 1), v[0]) and torch.equal(c.v[0, 1, :, 4:4 + T].transpose(0, 1), v[1])


def test_append_extreme_values_in_8_bits():
    """Beyond +-448 the nearest value, infinities too; NaN stays NaN; ties to even."""
    ctx, c = context(1, 1, 1), Cache(1, 1, 1, 16, "e4m3")
    row = torch.zeros(D, device=DEV)
    vals = [float("inf"), -float("inf"), 448.0, 464.0, 500.0, -1e30, float("nan"), 0.0, -0.0, 2.0 ** -9, 2.0 ** -10,
            3 * 2.0 ** -10, 1.0625, 1.1875, 17.0, 19.0]
    row[:len(vals)] = torch.tensor(vals)
    v = row.view(1, 1, 1, D)
    k = torch.zeros_like(v)
    ctx.append(tb.LayerCache(c.view(tb, seq_lens=int32([0])), 0), k, v, torch.tensor([0], device=DEV))
    got = c.v[0, 0, 0, 0].float()[:len(vals)].cpu()
    want = [448.0, -448.0, 448.0, 448.0, 448.0, -448.0, float("nan"), 0.0, 0.0, 2.0 ** -9, 0.0, 2.0 ** -8, 1.0, 1.25, 16.0, 20.0]
    assert torch.equal(torch.nan_to_num(got, nan=-1.0), torch.nan_to_num(torch.tensor(want), nan=-1.0))


def test_append_reports_rows_without_a_place():
    """No slot left, a page id outside the pool, a position outside [0, 2^31), a count outside [0, T]: reported, skipped,
    and the rows that have a place are stored."""
    def run(lens, n_new, pos, table=None, T=4, page=16):
        ctx, c = context(1, 1, 1), Cache(1, 1, 1, 32, page=page)
        if table is not None:
            c.table.copy_(int32([table]))
        k = torch.ones(1, T, 1, D, dtype=torch.bfloat16, device=DEV)
        status, new = torch.zeros(1, dtype=torch.int32, device=DEV), int32([0])
        ctx.append(tb.LayerCache(c.view(tb, seq_lens=int32([lens])), 0), k, k, torch.tensor([pos], device=DEV),
                   n_new=int32([n_new]), new_lens=new, device_status=status)
        torch.cuda.synchronize()
        stored = int((~c.v.float().isnan()).any(-1).sum())
        return int(status), stored, int(new)
    assert run(28, 4, 0) == (0, 4, 32)
    assert run(30, 4, 0) == (5, 2, 32)
    assert run(40, 4, 0) == (5, 0, 32)
    assert run(-3, 4, 0) == (0, 4, 4)
    assert run(0, 4, 2 ** 31 - 2) == (5, 2, 4)
    assert run(0, 4, -2) == (5, 2, 4)
    assert run(14, 4, 0, table=[0, 99]) == (5, 2, 18)
    assert run(14, 4, 0, table=[-1, 1]) == (5, 2, 18)
    assert run(0, 9, 0) == (5, 4, 4)
    assert run(3, -1, 0) == (5, 0, 3)


# ------------------------------------------------------------------------------------------------
# attend
# ------------------------------------------------------------------------------------------------
def check_rows(out, lse, q, rows_of, S, H, G, scale, ks=None, vs=None, extra=0.0):
    """out, lse against the definition; rows_of(s, h) -> (k, v) float64."""
    for s in range(S):
        for h in range(H):
            k, v = rows_of(s, h)
            for g in range(G):
                hq = h * G + g
                want, wl, tol = attention(q[s, hq].double(), k, v, scale)
                if extra and k.shape[0]:
                    x = torch.softmax(k @ q[s, hq].double() * scale, 0)
                    tol = tol + extra * (x @ v.abs())
                err = (out[s, hq].double() - want).abs()
                assert bool((err <= U_BF16 * want.abs() + tol * (1 + U_BF16)).all()), (s, h, g, k.shape[0], float(err.max()))
                if lse is not None:
                    if k.shape[0] == 0:
                        assert float(lse[s, hq]) == -math.inf
                    else:
                        d = 2.0 ** -19 * abs(scale) * float((k.abs() @ q[s, hq].double().abs()).max())
                        assert abs(float(lse[s, hq]) - wl) <= d + 2.0 ** -15 + 2.0 ** -22 * abs(wl)


def check_attend(fmt, page, order, H, G, lens, per_head=False, scales=False, layer=1, scale=D ** -0.5, seed=0, spread=1.0,
                 rows=None):
    S, L = len(lens), 2
    g = torch.Generator(device=DEV).manual_seed(seed)
    unit = lens if per_head else [[n] * H for n in lens]
    c = Cache(L, S, H, rows or max(1, max(max(r) for r in unit)), fmt, page, order, seed=seed)
    for s in range(S):
        for h in range(H):
            c.fill(layer, s, h, unit[s][h], g, spread)
    ks = 0.25 + torch.rand(L, H, generator=g, device=DEV) if scales else None
    vs = 0.25 + torch.rand(L, H, generator=g, device=DEV) if scales else None
    ctx = context(L, H, G)
    wide = torch.randn(S, (G + 2) * H, D, generator=g, device=DEV).to(torch.bfloat16)
    q = wide[:, :G * H]                                              # a slice of a fused projection
    out = torch.full((S, G * H, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((S, G * H), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    unit_lens = int32([unit, unit]) if per_head else None
    src = tb.LayerCache(c.view(tb, seq_lens=None if per_head else int32([r[0] for r in unit])), layer, unit_lens=unit_lens,
                        k_scale=ks, v_scale=vs)
    ws = ctx.attend_workspace(S)
    ws.fill_(255)                                                    # NaN patterns: nothing in it may be relied on
    ctx.attend(src, q, out, ws, scale=scale, lse=lse, device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0

    def rows_of(s, h):
        a, b = c.unit(c.k, layer, s, h, unit[s][h]), c.unit(c.v, layer, s, h, unit[s][h])
        return (a * float(ks[layer, h]), b * float(vs[layer, h])) if scales else (a, b)
    check_rows(out, lse, q, rows_of, S, H, G, scale)
    again = torch.empty_like(out)
    ctx.attend(src, q, again, ws, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(raw(again), raw(out))
    return out


EDGES = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 9, 16])
def test_attend_group_sizes_and_edge_lengths(fmt, G):
    check_attend(fmt, 16, "heads", 2, G, EDGES, scales=fmt == "e4m3", seed=G)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("G", [1, 4, 7, 8, 16])
@pytest.mark.parametrize("S,rows", [(40, None), (5, 6000)])
def test_attend_edge_lengths_where_units_are_cut_over_the_gpu(fmt, G, S, rows):
    """More units than clusters of blocks hold at a time, or room for more rows than they take."""
    check_attend(fmt, 16, "heads", 2, G, [EDGES[(5 * s) % len(EDGES)] for s in range(S)], scales=fmt == "e4m3", seed=G, rows=rows)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [63, 64, 65, 511, 512, 513, 1024, 2176, 4351, 4352, 4353])
def test_attend_few_units_around_the_cluster_limits(fmt, n):
    check_attend(fmt, 0, "tokens", 1, 4, [n], seed=n)
    check_attend(fmt, 16, "heads", 2, 12, [n // 2, n, 0], per_head=False, seed=n)


@pytest.mark.parametrize("fmt,page,order", [("bf16", 0, "heads"), ("bf16", 0, "tokens"), ("bf16", 0, "padded"),
                                            ("bf16", 48, "heads"), ("bf16", 64, "tokens"), ("bf16", 32, "padded"),
                                            ("e4m3", 0, "heads"), ("e4m3", 0, "tokens"), ("e4m3", 48, "padded")])
def test_attend_layouts(fmt, page, order):
    check_attend(fmt, page, order, 3, 4, [333, 0, 50, 1000], seed=3)


@pytest.mark.parametrize("fmt,G", [("bf16", 4), ("bf16", 16), ("e4m3", 4), ("e4m3", 12)])
def test_attend_lengths_per_head(fmt, G):
    check_attend(fmt, 16, "heads", 3, G, [[0, 77, 300], [1, 0, 0], [600, 5, 64]], per_head=True, scales=fmt == "e4m3")


@pytest.mark.parametrize("fmt,G,n", [("bf16", 4, 40000), ("bf16", 16, 20000), ("e4m3", 8, 30011)])
def test_attend_long_units_are_cut_over_the_gpu(fmt, G, n):
    check_attend(fmt, 0, "heads", 1, G, [n], seed=n)
    check_attend(fmt, 16, "heads", 2, G, [n // 3, 1, n // 2, 0], seed=n + 1)


def test_attend_many_units_more_than_blocks():
    check_attend("bf16", 0, "heads", 8, 1, [(37 * s) % 90 for s in range(64)], seed=5)


def test_attend_all_empty():
    out = check_attend("bf16", 0, "heads", 2, 4, [0, 0, 0], rows=8)
    assert bool((out == 0).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attend_peaked_weights(fmt):
    """Logits tens of units apart, the running bound is raised many times."""
    check_attend(fmt, 0, "heads", 1, 4, [777], scale=1.0, spread=2.0, seed=8)
    check_attend(fmt, 0, "heads", 1, 4, [777], scale=-1.0, seed=9)
    check_attend(fmt, 0, "heads", 1, 4, [300], scale=0.0, seed=10)


def test_attend_ascending_and_descending_logits():
    """Keys ordered by their logit: every subtile raises the bound, or none after the first."""
    ctx, n = context(1, 1, 4), 512
    for sign in (1.0, -1.0):
        c = Cache(1, 1, 1, n)
        g = torch.Generator(device=DEV).manual_seed(2)
        c.fill(0, 0, 0, n, g)
        q = torch.zeros(1, 4, D, dtype=torch.bfloat16, device=DEV)
        q[..., 0] = 1.0
        c.k[0, 0, 0, :, 0] = (sign * torch.linspace(-60, 60, n, device=DEV)).to(torch.bfloat16)
        out, lse = torch.empty_like(q), torch.empty(1, 4, device=DEV)
        ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([n])), 0), q, out, ctx.attend_workspace(1), scale=1.0, lse=lse)
        torch.cuda.synchronize()
        check_rows(out, lse, q, lambda s, h: (c.unit(c.k, 0, 0, 0, n), c.unit(c.v, 0, 0, 0, n)), 1, 1, 4, 1.0)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attend_non_finite_rows_stay_in_their_unit(fmt):
    """A NaN key makes its own unit's outputs NaN and no others; an 8-bit cache has no infinities, a bf16 one has."""
    ctx, S, H, G, n = context(1, 2, 4), 3, 2, 4, 100
    g = torch.Generator(device=DEV).manual_seed(4)
    c = Cache(1, S, H, 128, fmt)
    for s in range(S):
        for h in range(H):
            c.fill(0, s, h, n, g)
    c.k[0, 1, 0, 40, 3] = float("nan")
    c.v[0, 2, 1, 10, 5] = float("nan")
    if fmt == "bf16":
        c.v[0, 0, 1, 99, 7] = float("inf")
    q = torch.randn(S, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([n] * S)), 0), q, out, ctx.attend_workspace(S))
    torch.cuda.synchronize()
    o = out.float().view(S, H, G, D)
    assert bool(o[1, 0].isnan().all())
    assert bool(o[2, 1, :, 5].isnan().all()) and bool(o[2, 1, :, :5].isfinite().all())
    if fmt == "bf16":
        # (the rest of a rounded weight may be zero or negative: an infinite value gives infinity or NaN)
        assert not bool(o[0, 1, :, 7].isfinite().any()) and bool(o[0, 1, :, 8:].isfinite().all())
    assert bool(o[0, 0].isfinite().all()) and bool(o[1, 1].isfinite().all()) and bool(o[2, 0].isfinite().all())


def test_attend_queries_of_any_magnitude_in_8_bits():
    """The 8-bit path holds queries in f16: rows far outside f16's range must come out as in the definition."""
    ctx, n = context(1, 1, 6), 90
    g = torch.Generator(device=DEV).manual_seed(6)
    c = Cache(1, 1, 1, n, "e4m3")
    c.fill(0, 0, 0, n, g)
    q = torch.randn(1, 6, D, generator=g, device=DEV)
    q[0] *= torch.tensor([1e-30, 1e-8, 1.0, 300.0, 1e5, 0.0], device=DEV)[:, None]
    q = q.to(torch.bfloat16)
    for i, scale in enumerate([1e28, 1e7, 0.1, 3e-4, 1e-6, 1.0]):
        out = torch.empty_like(q)
        ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([n])), 0), q, out, ctx.attend_workspace(1), scale=scale)
        torch.cuda.synchronize()
        k, v = c.unit(c.k, 0, 0, 0, n), c.unit(c.v, 0, 0, 0, n)
        want, _, tol = attention(q[0, i].double(), k, v, scale)
        assert bool(((out[0, i].double() - want).abs() <= U_BF16 * want.abs() + 1.01 * tol).all()), i


def test_attend_reports_bad_pages_and_leaves_their_rows_out():
    ctx, c = context(1, 1, 2), Cache(1, 2, 1, 64, page=16)
    g = torch.Generator(device=DEV).manual_seed(7)
    for s in range(2):
        c.fill(0, s, 0, 60, g)
    good = c.table.clone()
    k = [c.unit(c.k, 0, s, 0, 60) for s in range(2)]
    v = [c.unit(c.v, 0, s, 0, 60) for s in range(2)]
    c.table[0, 1], c.table[1, 3] = -1, c.k.shape[1]
    q = torch.randn(2, 2, D, generator=g, device=DEV).to(torch.bfloat16)
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device=DEV)
    ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([60, 60])), 0), q, out, ctx.attend_workspace(2), device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 5
    keep = [torch.cat((torch.arange(16), torch.arange(32, 60))).to(DEV), torch.arange(48).to(DEV)]
    check_rows(out, None, q, lambda s, h: (k[s][keep[s]], v[s][keep[s]]), 2, 1, 2, D ** -0.5)
    # entries behind the last row are not looked at
    c.table.copy_(good)
    c.table[0, 3] = -1
    status.zero_()
    ctx.attend(tb.LayerCache(c.view(tb, seq_lens=int32([48, 60])), 0), q, out, ctx.attend_workspace(2), device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0


def test_attend_and_append_past_32_bit_offsets():
    """The last layer of a cache whose element offsets pass 2^31 and byte offsets 2^32."""
    L, H, G, N = 33, 1, 4, 1 << 19
    free = torch.cuda.mem_get_info()[0]
    if free < 14 << 30:
        pytest.skip("needs 10 GB of device memory")
    k = torch.empty(L, 1, H, N, D, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    g = torch.Generator(device=DEV).manual_seed(11)
    n = 3001
    a, b = (torch.randn(n, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    # the rows end at the very end of the memory: a view of the last layer's last rows as slots 0..
    k[L - 1, 0, 0, N - n - 1:N - 1], v[L - 1, 0, 0, N - n - 1:N - 1] = a, b
    kk, vv = k[:, :, :, N - n - 1:], v[:, :, :, N - n - 1:]
    ctx = context(L, H, G)
    lens = int32([n])
    lc = tb.LayerCache(tb.CacheView(kk, vv, seq_lens=lens), L - 1)
    row = torch.randn(1, 1, H, D, generator=g, device=DEV).to(torch.bfloat16)
    ctx.append(lc, row, row, torch.tensor([0], device=DEV), new_lens=lens)
    q = torch.randn(1, G, D, generator=g, device=DEV).to(torch.bfloat16)
    out = torch.empty_like(q)
    ctx.attend(lc, q, out, ctx.attend_workspace(1))
    torch.cuda.synchronize()
    assert torch.equal(k[L - 1, 0, 0, N - 1], row.view(-1)) and torch.equal(v[L - 1, 0, 0, N - 1], row.view(-1))
    kd, vd = (torch.cat((x, row.view(1, D))).double() for x in (a, b))
    check_rows(out, None, q, lambda s, h: (kd, vd), 1, 1, G, D ** -0.5)


# ------------------------------------------------------------------------------------------------
# shared prefixes
# ------------------------------------------------------------------------------------------------
def check_shared(fmt, page, H, G, starts, plens, lens, pfmt=None, ppage=None, per_head=False, seed=0, order="heads",
                 rows=None):
    S, P, L, layer = len(lens), len(plens), 2, 1
    g = torch.Generator(device=DEV).manual_seed(seed)
    pfmt, ppage = pfmt or fmt, page if ppage is None else ppage
    pu = plens if per_head else [[n] * H for n in plens]
    c = Cache(L, S, H, max(1, max(lens)), fmt, page, order, seed=seed)
    pc = Cache(L, P, H, rows or max(1, max(max(r) for r in pu)), pfmt, ppage, order, seed=seed + 1)
    for h in range(H):
        for s in range(S):
            c.fill(layer, s, h, lens[s], g)
        for p in range(P):
            pc.fill(layer, p, h, pu[p][h], g)
    sc = {}
    for name, f in (("c", fmt), ("p", pfmt)):
        sc[name] = [0.25 + torch.rand(L, H, generator=g, device=DEV) if f == "e4m3" else None for _ in range(2)]
    ctx = context(L, H, G)
    q = torch.randn(S, G * H, D, generator=g, device=DEV).to(torch.bfloat16)
    out, lse = torch.full_like(q, float("nan")), torch.full((S, G * H), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    src = tb.LayerCache(c.view(tb, seq_lens=int32(lens)), layer, k_scale=sc["c"][0], v_scale=sc["c"][1])
    pre = tb.LayerCache(pc.view(tb, seq_lens=None if per_head else int32(plens)), layer,
                        unit_lens=int32([pu, pu]) if per_head else None, k_scale=sc["p"][0], v_scale=sc["p"][1])
    ws = ctx.attend_workspace(S, P)
    ws.fill_(255)
    ctx.attend_shared(pre, int32(starts), src, q, out, ws, lse=lse, device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0

    def rows_of(s, h):
        parts = [(c.unit(c.k, layer, s, h, lens[s]), c.unit(c.v, layer, s, h, lens[s]), sc["c"])]
        for p in range(P):
            if starts[p] <= s < starts[p + 1]:
                parts.append((pc.unit(pc.k, layer, p, h, pu[p][h]), pc.unit(pc.v, layer, p, h, pu[p][h]), sc["p"]))
        ks = torch.cat([k if x[0] is None else k * float(x[0][layer, h]) for k, _, x in parts])
        vs = torch.cat([v if x[1] is None else v * float(x[1][layer, h]) for _, v, x in parts])
        return ks, vs
    check_rows(out, lse, q, rows_of, S, H, G, D ** -0.5, extra=U_BF16)
    again = torch.empty_like(out)
    ctx.attend_shared(pre, int32(starts), src, q, again, ws)
    torch.cuda.synchronize()
    assert torch.equal(raw(again), raw(out))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("G", [1, 3, 4, 5, 8, 16])
def test_shared_group_sizes(fmt, G):
    check_shared(fmt, 16, 2, G, [0, 1, 6, 6, 9], [300, 65, 40, 128], [0, 5, 17, 64, 1, 0, 130, 2, 33], seed=G)


@pytest.mark.parametrize("fmt,page,order", [("bf16", 0, "heads"), ("bf16", 0, "tokens"), ("bf16", 48, "padded"),
                                            ("e4m3", 0, "heads"), ("e4m3", 64, "tokens")])
def test_shared_layouts(fmt, page, order):
    check_shared(fmt, page, 2, 4, [0, 7], [1000], [3 * s for s in range(7)], order=order)


@pytest.mark.parametrize("G,S", [(4, 40), (8, 33), (16, 20), (1, 140), (5, 60)])
def test_shared_many_sequences(G, S):
    check_shared("bf16", 16, 2, G, [0, S - 3, S], [517, 129], [(7 * s) % 40 for s in range(S)], seed=S)
    check_shared("e4m3", 16, 1, G, [0, S - 3, S], [517, 129], [(7 * s) % 40 for s in range(S)], seed=S)


def test_shared_sequences_without_a_prefix_and_empty_parts():
    # sequences 0, 1 and 6, 7 belong to no prefix; prefix 1 has no rows, prefix 2 no sequences
    check_shared("bf16", 16, 2, 4, [2, 4, 6, 6], [100, 0, 30], [5, 0, 9, 0, 0, 7, 3, 0])
    check_shared("bf16", 16, 1, 4, [0, 0], [50], [5, 0])


@pytest.mark.parametrize("a,b", [("bf16", "e4m3"), ("e4m3", "bf16")])
def test_shared_formats_may_differ(a, b):
    check_shared(a, 16, 2, 4, [0, 3, 5], [200, 77], [10, 0, 65, 3, 20], pfmt=b, ppage=0)


def test_shared_prefix_lengths_per_head():
    check_shared("bf16", 16, 3, 4, [0, 3, 5], [[200, 0, 77], [1, 64, 129]], [10, 0, 65, 3, 20], per_head=True)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_shared_long_prefix(fmt):
    check_shared(fmt, 16, 1, 4, [0, 5], [20000], [100, 0, 3000, 1, 64], seed=20)
    check_shared(fmt, 0, 1, 8, [0, 24], [9001], [10 * s for s in range(24)], seed=21)


# The same with room for more rows than clusters of blocks take: passes over prefixes and own rows, then joined.
ROOM = 6000


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("G", [1, 3, 4, 5, 8, 16])
def test_shared_in_passes_group_sizes(fmt, G):
    check_shared(fmt, 16, 2, G, [0, 1, 6, 6, 9], [300, 65, 40, 128], [0, 5, 17, 64, 1, 0, 130, 2, 33], seed=G, rows=ROOM)
    check_shared(fmt, 16, 1, G, [0, 24, 25], [300, 140], [(7 * s) % 30 for s in range(25)], seed=G, rows=ROOM)


@pytest.mark.parametrize("fmt,page,order", [("bf16", 0, "heads"), ("bf16", 0, "tokens"), ("bf16", 48, "padded"), ("bf16", 128, "heads"),
                                            ("e4m3", 0, "heads"), ("e4m3", 64, "tokens"), ("e4m3", 48, "padded")])
@pytest.mark.parametrize("S", [3, 30])
def test_shared_in_passes_layouts(fmt, page, order, S):
    check_shared(fmt, page, 2, 4, [0, S], [1000], [3 * s for s in range(S)], order=order, rows=ROOM)


@pytest.mark.parametrize("fmt,page", [("bf16", 0), ("bf16", 16), ("e4m3", 0), ("e4m3", 16)])
@pytest.mark.parametrize("n", [1, 15, 50, 127, 128])
def test_shared_in_passes_prefixes_shorter_than_a_tile(fmt, page, n):
    check_shared(fmt, page, 2, 4, [0, 30, 31], [n, n], [1 + s % 3 for s in range(31)], seed=n)
    check_shared(fmt, page, 2, 16, [0, 31], [n], [s % 3 for s in range(31)], seed=n)


@pytest.mark.parametrize("a,b", [("bf16", "e4m3"), ("e4m3", "bf16")])
@pytest.mark.parametrize("S", [5, 40])
def test_shared_in_passes_formats_lengths_per_head_and_empty_parts(a, b, S):
    lens = [(7 * s) % 40 for s in range(S)]
    check_shared(a, 16, 2, 4, [0, S - 2, S], [200, 77], lens, pfmt=b, ppage=0, rows=ROOM)
    check_shared(a, 16, 3, 4, [0, S - 2, S], [[200, 0, 77], [1, 64, 129]], lens, per_head=True, rows=ROOM)
    check_shared(a, 16, 2, 4, [1, S - 2, S - 2, S - 1], [100, 0, 30], lens, rows=ROOM)
    check_shared(a, 16, 1, 4, [0, S], [0], [0] * S, rows=ROOM)


@pytest.mark.parametrize("rows", [32, ROOM])
def test_shared_reports_descending_groups(rows):
    ctx, S, P = context(1, 1, 4), 4, 3
    c, pc = Cache(1, S, 1, 16), Cache(1, P, 1, rows)
    g = torch.Generator(device=DEV).manual_seed(1)
    for s in range(S):
        c.fill(0, s, 0, 16, g)
    for p in range(P):
        pc.fill(0, p, 0, 32, g)
    q = torch.randn(S, 4, D, generator=g, device=DEV).to(torch.bfloat16)
    out = torch.empty_like(q)
    src, pre = tb.LayerCache(c.view(tb, seq_lens=int32([16] * S)), 0), tb.LayerCache(pc.view(tb, seq_lens=int32([32] * P)), 0)
    for starts, want in (([0, 4, 1, 4], 5), ([-3, 1, 2, 99], 0), ([4, 0, 4, 0], 5), ([0, 0, 0, 0], 0)):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        ctx.attend_shared(pre, int32(starts), src, q, out, ctx.attend_workspace(S, P), device_status=status)
        torch.cuda.synchronize()
        assert int(status) == want, starts


@pytest.mark.parametrize("S,P", [(4096, 512), (64, 2048)])
def test_shared_descending_groups_of_long_prefixes_take_no_work(S, P):
    # all even groups are the whole batch: (4096, 512) would be 2^31 steps and more, which no unit's place may wrap around
    ctx, H, n = context(1, 8, 4), 8, 2 ** 20
    page = torch.zeros(1, 1, H, 1024, D, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(P, n // 1024, dtype=torch.int32, device=DEV)
    pre = tb.LayerCache(tb.CacheView(page, page, page_table=table, n_max=n, seq_lens=int32([n] * P)), 0)
    c = Cache(1, S, H, 16)
    g = torch.Generator(device=DEV).manual_seed(1)
    for s in (0, S - 1):
        for h in range(H):
            c.fill(0, s, h, 16, g)
    src = tb.LayerCache(c.view(tb, seq_lens=int32([16] + [0] * (S - 2) + [16])), 0)
    q = torch.randn(S, 4 * H, D, generator=g, device=DEV).to(torch.bfloat16)
    out, status = torch.empty_like(q), int32([0])
    ws = ctx.attend_workspace(S, P)
    for fill in (0, 1, 127, 255):
        ws.fill_(fill)
        status.zero_()
        ctx.attend_shared(pre, int32([0, S] * (P // 2) + [S]), src, q, out, ws, device_status=status)
        torch.cuda.synchronize()
        assert int(status) == 5
    # the context goes on: the same call without prefixes of any sequence
    status.zero_()
    ctx.attend_shared(pre, int32([0] * (P + 1)), src, q, out, ws, device_status=status)
    alone = torch.empty_like(q)
    ctx.attend(src, q, alone, ws)
    torch.cuda.synchronize()
    # (the same sums; divided before or after the join, so that a rounding to bf16 may fall to the neighbour, 2 U apart)
    assert int(status) == 0 and bool(((out.float() - alone.float()).abs() <= 2 * U_BF16 * alone.float().abs()).all())


@pytest.mark.parametrize("rows", [1000, ROOM])
@pytest.mark.parametrize("scale", [1.0, -1.0, 0.0])
@pytest.mark.parametrize("fmt,S", [("bf16", 20), ("e4m3", 20), ("bf16", 3)])
def test_shared_ascending_and_descending_logits(fmt, S, scale, rows):
    """Keys ordered by their logit, 60 units apart over the prefix: the bound is raised tile after tile, or never again."""
    H, G, n = 1, 4, 1000
    for sign in (1.0, -1.0):
        g = torch.Generator(device=DEV).manual_seed(2)
        pc, c = Cache(1, 1, H, rows, fmt), Cache(1, S, H, 4, fmt)
        pc.fill(0, 0, 0, n, g)
        for s in range(S):
            c.fill(0, s, 0, s % 3, g)
        pc.k.view({1: torch.uint8, 2: torch.int16}[pc.k.element_size()])[0, 0, 0, :n, 0] = raw(
            (sign * torch.linspace(-60, 60, n, device=DEV)).to(pc.k.dtype))
        q = torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
        q[..., 0], q[..., 1] = 1.0, torch.linspace(-1, 1, S, device=DEV)[:, None]
        out, lse = torch.empty_like(q), torch.empty(S, H * G, device=DEV)
        ctx, lens = context(1, H, G), int32([s % 3 for s in range(S)])
        ctx.attend_shared(tb.LayerCache(pc.view(tb, seq_lens=int32([n])), 0), int32([0, S]), tb.LayerCache(c.view(tb, seq_lens=lens), 0),
                          q, out, ctx.attend_workspace(S, 1), scale=scale, lse=lse)
        torch.cuda.synchronize()
        check_rows(out, lse, q, lambda s, h: tuple(torch.cat((pc.unit(a, 0, 0, 0, n), c.unit(b, 0, s, 0, s % 3)))
                                                   for a, b in ((pc.k, c.k), (pc.v, c.v))), S, H, G, scale, extra=U_BF16)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("S", [1, 24])
def test_many_small_weights_beside_a_large_one(fmt, S):
    """60,000 rows whose weight is 2^-25.5 of one row's: together 0.13 % of the sum, below what an f16 resolves beside 1."""
    H, G, n = 1, 4, 60000
    c = Cache(1, S, H, 1, fmt)
    pc = Cache(1, 1, H, n, fmt)
    pc.k.zero_()
    pc.v.copy_(torch.ones(1, device=DEV).to(pc.v.dtype).expand_as(pc.v))
    pc.k[0, 0, 0, 7, 0] = 1.0
    pc.v[0, 0, 0, 7] = 0.0
    q = torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 16.0
    scale = 25.5 * math.log(2.0) / 16.0
    ctx, out = context(1, H, G), torch.empty_like(q)
    pre = tb.LayerCache(pc.view(tb, seq_lens=int32([n])), 0)
    src = tb.LayerCache(c.view(tb, seq_lens=int32([0] * S)), 0)
    ctx.attend_shared(pre, int32([0, S]), src, q, out, ctx.attend_workspace(S, 1), scale=scale)
    torch.cuda.synchronize()
    rows = (pc.unit(pc.k, 0, 0, 0, n), pc.unit(pc.v, 0, 0, 0, n))
    check_rows(out, None, q, lambda s, h: rows, S, H, G, scale, extra=U_BF16)
    if S == 1:
        ctx.attend(pre, q, out, ctx.attend_workspace(1), scale=scale)
        torch.cuda.synchronize()
        check_rows(out, None, q, lambda s, h: rows, 1, H, G, scale)


def test_shared_more_prefixes_than_a_warp():
    P = 70
    starts, s = [0], 0
    for p in range(P):
        s += p % 3
        starts.append(s)
    check_shared("bf16", 16, 1, 4, starts, [(11 * p) % 50 for p in range(P)], [(5 * i) % 9 for i in range(s + 2)])
    check_shared("bf16", 16, 1, 16, starts, [(11 * p) % 50 for p in range(P)], [(5 * i) % 9 for i in range(s + 2)])


@pytest.mark.parametrize("rows", [300, ROOM])
@pytest.mark.parametrize("fmt,S", [("bf16", 3), ("bf16", 30), ("e4m3", 3), ("e4m3", 30)])
def test_shared_reports_bad_pages_of_a_prefix(fmt, S, rows):
    H, G, n, page = 2, 4, 300, 32
    g = torch.Generator(device=DEV).manual_seed(7)
    pc, c = Cache(1, 1, H, rows, fmt, page), Cache(1, S, H, 16, fmt, 16)
    for h in range(H):
        pc.fill(0, 0, h, n, g)
        for s in range(S):
            c.fill(0, s, h, 5, g)
    rows = [(pc.unit(pc.k, 0, 0, h, n), pc.unit(pc.v, 0, 0, h, n)) for h in range(H)]
    keep = torch.tensor([i for i in range(n) if i // page not in (0, 4, 9)], device=DEV)
    pc.table[0, 0], pc.table[0, 4], pc.table[0, 9] = -1, pc.k.shape[1], 1 << 30
    q = torch.randn(S, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device=DEV)
    ctx = context(1, H, G)
    ctx.attend_shared(tb.LayerCache(pc.view(tb, seq_lens=int32([n])), 0), int32([0, S]),
                      tb.LayerCache(c.view(tb, seq_lens=int32([5] * S)), 0), q, out, ctx.attend_workspace(S, 1), device_status=status)
    torch.cuda.synchronize()
    assert int(status) == 5
    check_rows(out, None, q, lambda s, h: tuple(torch.cat((x[keep], c.unit(t, 0, s, h, 5))) for x, t in zip(rows[h], (c.k, c.v))),
               S, H, G, D ** -0.5, extra=U_BF16)


@pytest.mark.parametrize("H,rows", [(2, 150), (1, 150), (2, ROOM)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_shared_non_finite_queries_and_rows_stay_in_their_group(fmt, H, rows):
    G, S, n = 4, 24, 150
    g = torch.Generator(device=DEV).manual_seed(5)
    pc, c = Cache(1, 2, H, rows, fmt), Cache(1, S, H, 8, fmt)
    for h in range(H):
        for p in range(2):
            pc.fill(0, p, h, n, g)
        for s in range(S):
            c.fill(0, s, h, 3, g)
    pc.k[0, 1, 0, 70, 3] = float("nan")
    q = torch.randn(S, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    q[4, H * G - 3, 9] = float("nan")
    out = torch.empty_like(q)
    ctx = context(1, H, G)
    ctx.attend_shared(tb.LayerCache(pc.view(tb, seq_lens=int32([n, n])), 0), int32([0, 13, S]),
                      tb.LayerCache(c.view(tb, seq_lens=int32([3] * S)), 0), q, out, ctx.attend_workspace(S, 2))
    torch.cuda.synchronize()
    nan = out.isnan().any(-1)
    want = torch.zeros_like(nan)
    want[13:, :G] = True
    want[4, H * G - 3] = True
    assert torch.equal(nan, want) and bool(out[want].isnan().all())


def test_heads_that_share_one_cache_by_a_stride_of_zero():
    """Multi-query layouts as an expanded head: prefix and own rows, against the same rows copied out."""
    H, G, S, n = 4, 4, 10, 200
    g = torch.Generator(device=DEV).manual_seed(6)
    k, v = (torch.randn(1, S, 1, n, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    pk, pv = (torch.randn(1, 1, 1, n, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(S, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    ctx, lens, plens, starts = context(1, H, G), int32([20 * s for s in range(S)]), int32([n]), int32([0, S])
    outs = []
    for f in (lambda x: x.expand(-1, -1, H, -1, -1), lambda x: x.expand(-1, -1, H, -1, -1).contiguous()):
        src, pre = tb.LayerCache(tb.CacheView(f(k), f(v), seq_lens=lens), 0), tb.LayerCache(tb.CacheView(f(pk), f(pv), seq_lens=plens), 0)
        a, b = torch.empty_like(q), torch.empty_like(q)
        ctx.attend(src, q, a, ctx.attend_workspace(S))
        ctx.attend_shared(pre, starts, src, q, b, ctx.attend_workspace(S, 1))
        outs.append((a, b))
    torch.cuda.synchronize()
    assert torch.equal(raw(outs[0][0]), raw(outs[1][0]))
    check_rows(outs[0][1], None, q, lambda s, h: tuple(torch.cat((a[0, 0, 0].double(), b[0, s, 0, :20 * s].double()))
                                                       for a, b in ((pk, k), (pv, v))), S, H, G, D ** -0.5, extra=U_BF16)


def test_strides_of_single_dimensions_do_not_matter():
    ctx, H, G = context(1, 1, 1), 1, 1
    c = Cache(1, 1, 1, 8)
    odd = torch.randn(D, device=DEV).to(torch.bfloat16)
    x = odd.as_strided((1, 1, 1, D), (3, 5, 7, 1))
    lens = int32([0])
    lc = tb.LayerCache(c.view(tb, seq_lens=lens), 0)
    qo = torch.empty_like(odd).as_strided((1, 1, 1, D), (1, 3, 5, 1))
    ctx.append(lc, x, x, torch.tensor([0], device=DEV), q=x, q_out=qo, new_lens=lens)
    out = torch.empty(D, dtype=torch.bfloat16, device=DEV).as_strided((1, 1, D), (3, 5, 1))
    ctx.attend(lc, qo.as_strided((1, 1, D), (9, 11, 1)), out, ctx.attend_workspace(1))
    torch.cuda.synchronize()
    assert torch.equal(out.view(-1), odd) and torch.equal(c.k[0, 0, 0, 0], odd)


# ------------------------------------------------------------------------------------------------
# together, on streams, in graphs
# ------------------------------------------------------------------------------------------------
def test_decode_loop_with_windowed_compression_eager_and_captured():
    """Append, attend, compress behind the window trigger, step after step: the eager loop's attention against the
    definition on the rows its cache holds at that step; the loop replayed from one captured graph gives the same bits."""
    L, S, H, G, B, beta, steps = 2, 3, 2, 4, 32, 8, 20
    ctx = tb.TriContext(L, H, G, torch.randn(L, H * G, D, generator=torch.Generator().manual_seed(0)),
                        1.0 + torch.rand(L, H * G, D // 2, generator=torch.Generator().manual_seed(1)), rope_theta=1e4)
    n_max = 64
    g = torch.Generator(device=DEV).manual_seed(3)
    steps_q = torch.randn(steps, L, S, 1, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    steps_k, steps_v = (torch.randn(steps, L, S, 1, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    start = [30, 5, 33]

    class Loop:
        def __init__(self):
            gg = torch.Generator(device=DEV).manual_seed(4)
            self.k, self.v = (torch.randn(L, S, H, n_max, D, generator=gg, device=DEV).to(torch.bfloat16) for _ in range(2))
            self.lens, self.decoded = int32(start), torch.zeros(S, dtype=torch.int32, device=DEV)
            self.pos = torch.tensor([x + 100 for x in start], device=DEV)
            self.positions = torch.arange(n_max, device=DEV, dtype=torch.int32).expand(L, S, H, n_max).contiguous()
            self.next = torch.zeros(S, dtype=torch.int32, device=DEV)
            self.view = tb.CacheView(self.k, self.v, seq_lens=self.lens, positions=self.positions)
            # the appended row counts for this step's attention, so that one reads the lengths behind the append
            self.after = [tb.LayerCache(tb.CacheView(self.k, self.v, seq_lens=self.next), l) for l in range(L)]
            self.cache = [tb.LayerCache(self.view, l) for l in range(L)]
            self.q = torch.empty(L, S, 1, H * G, D, dtype=torch.bfloat16, device=DEV)
            self.kin, self.vin, self.qin = steps_k[0].clone(), steps_v[0].clone(), steps_q[0].clone()
            self.out = torch.empty(L, S, H * G, D, dtype=torch.bfloat16, device=DEV)
            self.ws, self.aws = ctx.workspace(S, n_max, B), ctx.attend_workspace(S)

        def load(self, i):
            self.kin.copy_(steps_k[i]); self.vin.copy_(steps_v[i]); self.qin.copy_(steps_q[i])

        def attend_all(self):
            for l in range(L):
                ctx.append(self.cache[l], self.kin[l], self.vin[l], self.pos, q=self.qin[l], q_out=self.q[l], new_lens=self.next)
                ctx.attend(self.after[l], self.q[l, :, 0], self.out[l], self.aws)

        def finish(self):
            self.lens.copy_(self.next)
            self.pos.add_(1)
            ctx.compress_windowed(self.view, self.pos, B, self.decoded, 1, beta, self.view, self.ws, new_seq_lens=self.lens)

    a = Loop()
    outs = []
    for i in range(steps):
        a.load(i)
        a.attend_all()
        torch.cuda.synchronize()
        n = [int(x) for x in a.next]
        for l in range(L):
            check_rows(a.out[l], None, a.q[l, :, 0], lambda s, h: (a.k[l, s, h, :n[s]].double(), a.v[l, s, h, :n[s]].double()),
                       S, H, G, D ** -0.5)
        a.finish()
        outs.append(a.out.clone())
    assert int(a.lens.max()) <= B + beta
    b = Loop()
    b.load(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            b.attend_all()
            b.finish()
    torch.cuda.current_stream().wait_stream(s)
    for i in range(steps):
        b.load(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(raw(b.out), raw(outs[i])), i
    assert torch.equal(raw(a.k), raw(b.k)) and torch.equal(a.positions, b.positions) and torch.equal(a.lens, b.lens)


FIRST_CALL = """
import torch
from paper_2604_04921_b200 import binding as tb
ctx = tb.TriContext(1, 2, 4, torch.zeros(1, 8, 128), torch.ones(1, 8, 64))
g = torch.Generator(device="cuda").manual_seed(0)
k, v = (torch.randn(1, 20, 2, 64, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
x = torch.randn(20, 1, 12, 128, generator=g, device="cuda").to(torch.bfloat16)
lens, pos = torch.full((20,), 5, dtype=torch.int32, device="cuda"), torch.arange(20, device="cuda")
q, out, both = torch.empty(20, 1, 8, 128, dtype=torch.bfloat16, device="cuda"), *(torch.empty(20, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
lc = tb.LayerCache(tb.CacheView(k, v, seq_lens=lens), 0)
ws, starts = ctx.attend_workspace(20, 20), torch.zeros(21, dtype=torch.int32, device="cuda")
starts[1:] = 20
x2 = x.clone()
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    x2.copy_(x)                                  # a memory copy before the first kernel, and one in between
    ctx.append(lc, x2[:, :, 8:10], x2[:, :, 10:], pos, q=x2[:, :, :8], q_out=q, new_lens=lens)
    x2.copy_(x)
    ctx.attend(lc, q[:, 0], out, ws)
    ctx.attend_shared(lc, starts, lc, q[:, 0], both, ws)
graph.replay()
torch.cuda.synchronize()
a, b = out.clone(), both.clone()
lens.fill_(5)
ctx.append(lc, x[:, :, 8:10], x[:, :, 10:], pos, q=x[:, :, :8], q_out=q, new_lens=lens)
ctx.attend(lc, q[:, 0], out, ws)
ctx.attend_shared(lc, starts, lc, q[:, 0], both, ws)
torch.cuda.synchronize()
assert torch.equal(a, out) and torch.equal(b, both) and bool((lens == 6).all()) and bool(a.isfinite().all())
print("same")
"""


def test_first_calls_of_a_process_inside_a_capture():
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], capture_output=True, text=True, timeout=300, cwd=str(tb._ROOT))
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_two_streams_with_a_workspace_each():
    ctx, H, G, n = context(1, 2, 4), 2, 4, 5000
    g = torch.Generator(device=DEV).manual_seed(5)
    jobs = []
    for i in range(2):
        c = Cache(1, 2, H, n)
        for s in range(2):
            for h in range(H):
                c.fill(0, s, h, n - 100 * i - s, g)
        q = torch.randn(2, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
        src = tb.LayerCache(c.view(tb, seq_lens=int32([n - 100 * i, n - 100 * i - 1])), 0)
        jobs.append((c, q, src, torch.empty_like(q), torch.empty_like(q), ctx.attend_workspace(2), torch.cuda.Stream()))
    for _, q, src, alone, _, ws, _ in jobs:
        ctx.attend(src, q, alone, ws)
    torch.cuda.synchronize()
    for r in range(20):
        for _, q, src, _, out, ws, st in jobs:
            with torch.cuda.stream(st):
                ctx.attend(src, q, out, ws)
    torch.cuda.synchronize()
    for _, _, _, alone, out, _, _ in jobs:
        assert torch.equal(raw(alone), raw(out))


def test_attend_after_compression_with_budgets_per_head():
    """compress(..., unit_budgets) leaves a length per head in kept_cnt; attention and a further append take it as it is."""
    L, S, H, G, n, B = 2, 2, 3, 4, 200, 64
    ctx = tb.TriContext(L, H, G, torch.randn(L, H * G, D, generator=torch.Generator().manual_seed(0)),
                        1.0 + torch.rand(L, H * G, D // 2, generator=torch.Generator().manual_seed(1)))
    g = torch.Generator(device=DEV).manual_seed(9)
    k, v = (torch.randn(L, S, H, n, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    view = tb.CacheView(k, v, seq_lens=int32([n, 150]))
    budgets = torch.randint(1, B + 1, (L * S * H,), generator=g, device=DEV, dtype=torch.int32)
    kept = torch.zeros(L * S * H, dtype=torch.int32, device=DEV)
    ctx.compress(view, torch.tensor([n, 150], device=DEV), B, view, ctx.workspace(S, n, B), kept_cnt=kept, unit_budgets=budgets)
    caches = [tb.LayerCache(view, l, unit_lens=kept) for l in range(L)]
    row = torch.randn(S, 1, H, D, generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn(S, H * G, D, generator=g, device=DEV).to(torch.bfloat16)
    before = kept.clone()
    for l in range(L):
        ctx.append(caches[l], row, row, torch.tensor([n, 150], device=DEV), new_lens=kept)
        out = torch.empty_like(q)
        ctx.attend(caches[l], q, out, ctx.attend_workspace(S))
        torch.cuda.synchronize()
        cnt = (before + 1).view(L, S, H)[l]
        check_rows(out, None, q, lambda s, h: (k[l, s, h, :int(cnt[s, h])].double(), v[l, s, h, :int(cnt[s, h])].double()),
                   S, H, G, D ** -0.5)
    assert torch.equal(kept, before + 1)


# ------------------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------------------
def test_refusals_of_the_c_interface():
    lib, ctx = tb.lib(), context(2, 2, 4)
    S, H, G, T = 2, 2, 4, 3
    c = Cache(2, S, H, 32)
    lens = int32([0, 0])
    x = torch.zeros(S, T, H, D, dtype=torch.bfloat16, device=DEV)
    xq = torch.zeros(S, T, H * G, D, dtype=torch.bfloat16, device=DEV)
    q, out = xq[:, 0], torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
    f32 = torch.zeros(2 * H, device=DEV)
    pos = torch.zeros(S, dtype=torch.int64, device=DEV)
    ws = ctx.attend_workspace(S, 1)

    def layer_cache(fmt_cache=None, layer=0, unit_lens=None, k_scale=None, **kw):
        cv = (fmt_cache or c).view(tb, seq_lens=lens).c_view()
        for name, val in kw.items():
            setattr(cv, name, val)
        lc = tb._LayerCache(ctypes.pointer(cv), layer, unit_lens, k_scale, None)
        lc.keep = cv
        return lc

    def append(lc=None, S=S, **kw):
        r = tb._AppendRows(k=x.data_ptr(), v=x.data_ptr(), kind=0, T=T, pos=pos.data_ptr())
        for p in ("k", "v"):
            for n, st in zip(("seq", "tok", "head"), x.stride()):
                setattr(r, f"{p}_stride_{n}", st)
        for name, val in kw.items():
            setattr(r, name, val)
        return lib.tri_append(ctx._h, ctypes.byref(lc or layer_cache()), S, ctypes.byref(r), None, None, None)

    assert append() == 0
    torch.cuda.synchronize()
    assert lib.tri_append(None, None, 1, None, None, None, None) == 1
    assert lib.tri_append(ctx._h, None, 1, None, None, None, None) == 1
    assert append(S=0) == 1 and append(T=0) == 1 and append(kind=2) == 1 and append(k=None) == 1 and append(v=None) == 1
    assert append(k=x.data_ptr() + 8) == 1 and append(k_stride_tok=260) == 1 and append(v_stride_head=4) == 1
    assert append(q=xq.data_ptr()) == 1 and append(q_out=xq.data_ptr()) == 1
    assert append(q=xq.data_ptr(), q_out=xq.data_ptr(), q_stride_tok=128, qo_stride_tok=256) == 1   # in place needs equal strides
    assert append(layer_cache(layer=2)) == 1 and append(layer_cache(layer=-1)) == 1
    assert append(layer_cache(k_scale=f32.data_ptr())) == 1                                         # scales belong to 8 bits
    assert append(layer_cache(v=None)) == 1 and append(layer_cache(k=None)) == 1
    assert append(layer_cache(seq_lens=None)) == 1 and append(layer_cache(n_max=0)) == 1 and append(layer_cache(k_kind=4)) == 1
    assert append(layer_cache(stride_tok=100)) == 1
    assert append(layer_cache(unit_lens=lens.data_ptr()), pos=None) == 1
    assert append(layer_cache(Cache(2, S, H, 32, page=16), page_size=8)) == 2
    r = tb._AppendRows(k=x.data_ptr(), v=x.data_ptr(), kind=0, T=T, pos=pos.data_ptr(), n_new=lens.data_ptr())
    for p in ("k", "v"):
        for n, st in zip(("seq", "tok", "head"), x.stride()):
            setattr(r, f"{p}_stride_{n}", st)
    assert lib.tri_append(ctx._h, ctypes.byref(layer_cache()), S, ctypes.byref(r), lens.data_ptr(), None, None) == 1

    def attend(lc=None, S=S, bytes=None, w=None, h=ctx._h, **kw):
        io = tb._AttendIo(q.data_ptr(), *q.stride()[:2], out.data_ptr(), *out.stride()[:2], None, 0.1)
        for name, val in kw.items():
            setattr(io, name, val)
        return lib.tri_attend(h, ctypes.byref(lc or layer_cache()), S, ctypes.byref(io), None, w or ws.data_ptr(),
                              ws.numel() if bytes is None else bytes, None)

    need = ctx.attend_workspace_bytes(S)
    assert attend() == 0 and attend(bytes=need) == 0 and attend(bytes=need - 1) == 3
    torch.cuda.synchronize()
    assert attend(h=None) == 1 and attend(S=0) == 1 and attend(w=ws.data_ptr() + 8) == 1
    assert attend(q=None) == 1 and attend(out=None) == 1 and attend(q=q.data_ptr() + 2) == 1 and attend(q_stride_head=4) == 1
    assert attend(scale=float("nan")) == 1 and attend(scale=float("inf")) == 1
    assert attend(layer_cache(v=None)) == 1 and attend(layer_cache(seq_lens=None)) == 1 and attend(layer_cache(layer=2)) == 1
    assert attend(scale=3e38) == 1                                              # times log2 e: beyond fp32
    assert attend(out=q.data_ptr()) == 1
    assert attend(layer_cache(n_max=2 ** 31 - 1), S=64) == 2                    # the line of steps would pass 2^31
    assert attend(layer_cache(k_kind=2)) == 2 and attend(layer_cache(Cache(2, S, H, 32, "f32"))) == 2
    assert lib.tri_attend_workspace_bytes(None, 1, 0) == 0 and lib.tri_attend_workspace_bytes(ctx._h, 0, 0) == 0
    assert lib.tri_attend_workspace_bytes(ctx._h, 1, -1) == 0

    def shared(P=1, starts=None, pre=None, bytes=None):
        io = tb._AttendIo(q.data_ptr(), *q.stride()[:2], out.data_ptr(), *out.stride()[:2], None, 0.1)
        st = int32([0, S, S]) if starts is None else starts
        return lib.tri_attend_shared(ctx._h, pre if pre is not None else ctypes.byref(layer_cache()), P,
                                     None if st is False else st.data_ptr(), ctypes.byref(layer_cache()), S, ctypes.byref(io),
                                     None, ws.data_ptr(), ws.numel() if bytes is None else bytes, None)

    assert shared() == 0
    torch.cuda.synchronize()
    assert shared(P=0) == 1 and shared(starts=False) == 1 and shared(bytes=ctx.attend_workspace_bytes(S, 1) - 1) == 3
    assert shared(pre=ctypes.byref(layer_cache(k_kind=2))) == 2
    torch.cuda.synchronize()


def test_refusals_of_the_binding():
    ctx, S, H, G = context(1, 2, 4), 2, 2, 4
    c = Cache(1, S, H, 32)
    lc = tb.LayerCache(c.view(tb, seq_lens=int32([0, 0])), 0)
    x = torch.zeros(S, 1, H, D, dtype=torch.bfloat16, device=DEV)
    q = torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(S, dtype=torch.int64, device=DEV)
    ws = ctx.attend_workspace(S)
    for bad in (lambda: ctx.append(lc, x[:1], x[:1], pos), lambda: ctx.append(lc, x.half(), x.half(), pos),
                lambda: ctx.append(lc, x, None, pos), lambda: ctx.append(lc, x, x, pos.int()), lambda: ctx.append(lc, x.cpu(), x, pos),
                lambda: ctx.append(lc, x, x, pos, q=x), lambda: ctx.append(lc, x, x, pos, n_new=pos),
                lambda: ctx.append(lc, x, x, pos, new_lens=int32([0])), lambda: ctx.attend(lc, q[:1], q[:1], ws),
                lambda: ctx.attend(lc, q.float(), q, ws), lambda: ctx.attend(lc, q.cpu(), q, ws),
                lambda: ctx.attend(lc, q, q.clone(), ws.cpu()), lambda: ctx.attend(lc, q, q.clone(), ws, lse=q),
                lambda: tb.LayerCache(c.view(tb), 0), lambda: tb.LayerCache(c.view(tb, seq_lens=int32([0, 0]), n_max=33), 0), lambda: tb.LayerCache(c.view(tb, seq_lens=int32([0, 0])), 1),
                lambda: tb.LayerCache(c.view(tb, seq_lens=torch.zeros(2, dtype=torch.int32)), 0),
                lambda: ctx.attend_shared(lc, int32([0, 1]), lc, q, q.clone(), ws)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(tb.TriError) as e:
        ctx.attend(lc, q, q.clone(), ws[:256])
    assert e.value.code == 3
