"""64-bit forms of the operators of a 4-bit cache, written row by row from the format's definition, and the caches the tests run
them on.

Error bounds used by the tests (half a step relative to the value: bf16 2^-8, f16 2^-11, fp32 2^-24):
  append   keys are rotated before they are quantised, in fp32 (fp64 for rows that fp32 leaves in doubt): a component x is off by e =
           (2^-21 + p 2^-51) |z|, |z| the pair's magnitude (see step_reference.py); values are quantised as they come (e = 0).  From
           the stored s and c: c is off by one rounding to bf16 of its formula, whose inputs are off by e, and fp32 roundings
           (2^-22); s is not below the formula's bound, taken with the stored c, by more than those, and the bf16 number below s
           is not above it by more; a component is off by s / 2, e, and what the fp32 quotient, off by 2^-20 at most (8 in
           magnitude, two roundings), moves over a border
  read     fp32: one rounding of the sum (2^-24 of the value, the product is exact); bf16: one more, 2^-8
  attend   d, what a logit is off by: per group of 32, with |q| the sum of the queries' magnitudes: two matrix instructions over u q, u <=
           15, some 8 truncations of 2^-23 of at most 15 |q|: 2^-16 |q|; Q and -8 Q, |Q| <= |q|, in two bf16 parts: 2^-16 of 8 |q|;
           together below 2^-12 |q|, times s; the centres likewise 2^-16 |c| |q|, and 2^-19 for the instruction's truncations, below
           2^-15 |c| |q|; a query in f16 beside one 2^28 times as large, 2^-24 of that one, is far below; the sum of all below 2^-19
           sum |q k|; all times the scale.
           A weight: the factor e^d, 2^-20 of it (exponential, products).  Values are summed as p s u and p (c - 8 s), the weights p s
           of the former with one rounding to f16: 2^-11 of p s u, or, where f16 ends, 2^-25 steps of weights of which the largest is at least 2^11 and of scales that are below
           2 s_max: 2^-35 s_max 8 for each row.  Sums: 2^-15 of all that is summed, as in step_reference.py: sum
           p (s u + |c| + 8 s).  One rounding to bf16.
"""
from __future__ import annotations

import math

import torch

D, ROW = 128, 80
U_BF16 = 2.0 ** -8


def position(d: int):
    """(byte, shift) of component d in a row."""
    g, t, i, h = d // 32, d % 32 // 8, d % 8 // 2, d % 2
    bit = 32 * (4 * t + g) + 4 * (i + 4 * h)
    return bit // 8, bit % 8


BYTE, SHIFT = (torch.tensor([position(d)[x] for d in range(D)]) for x in (0, 1))


def parts(rows: torch.Tensor):
    """Rows [..., 80] as codes [..., 128], scales and centres [..., 4], all in float64."""
    byte, shift = BYTE.to(rows.device), SHIFT.to(rows.device)
    code = (rows[..., byte].to(torch.int64) >> shift) & 15
    par = rows[..., 64:].contiguous().view(torch.bfloat16).double()
    return code.double(), par[..., :4], par[..., 4:]


def values(rows: torch.Tensor) -> torch.Tensor:
    """What rows [..., 80] stand for, [..., 128] in float64."""
    code, s, c = parts(rows)
    return (code - 8) * s.repeat_interleave(32, -1) + c.repeat_interleave(32, -1)


def bf16_not_below(x: torch.Tensor) -> torch.Tensor:
    """The smallest bf16 >= x > 0, at least 2^-126; 0 for 0 (float64 in and out)."""
    e = torch.floor(torch.log2(x.clamp(min=2.0 ** -126)))
    step = torch.exp2(e - 7)
    return torch.where(x > 0, torch.ceil(x / step).mul(step).clamp(min=2.0 ** -126), torch.zeros_like(x))


def quantised(x: torch.Tensor):
    """Codes [..., 128], scales and centres [..., 4] that rows x [..., 128] (float64) get."""
    y = x.unflatten(-1, (4, 32))
    lo, hi = y.amin(-1), y.amax(-1)
    c = ((8 * hi + 7 * lo) / 15).float().bfloat16().double()
    s = bf16_not_below(torch.maximum((hi - c) / 7, (c - lo) / 8))
    n = torch.where(s[..., None] > 0, (y - c[..., None]) / s.clamp(min=2.0 ** -130)[..., None], torch.zeros_like(y))
    code = torch.round(n).clamp(-8, 7) + 8
    return code.flatten(-2), s, c


def packed(code: torch.Tensor, s: torch.Tensor, c: torch.Tensor) -> torch.Tensor:
    """Rows [..., 80] of codes [..., 128], scales and centres [..., 4]."""
    rows = torch.zeros(*code.shape[:-1], ROW, dtype=torch.int64, device=code.device)
    for d in range(D):
        byte, shift = position(d)
        rows[..., byte] |= code[..., d].to(torch.int64) << shift
    par = torch.cat((s, c), -1).to(torch.bfloat16).contiguous().view(torch.uint8)
    return torch.cat((rows[..., :64].to(torch.uint8), par), -1)


def as_rows(x: torch.Tensor) -> torch.Tensor:
    return packed(*quantised(x.double()))


class Cache4:
    """One multi-layer 4-bit cache in some layout, every byte 0xff except where rows are put: scales and centres of other rows are
    NaN."""

    def __init__(self, L, S, H, rows, page=0, order="heads", seed=0, device="cuda", spare_pages=1):
        self.L, self.S, self.H, self.page = L, S, H, page
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.table = None
        if page:
            per = -(-rows // page)
            n = S * per + spare_pages
            self.table = torch.randperm(n, generator=g)[:S * per].to(torch.int32).view(S, per).to(device)
            rows, shape = per * page, (L, n, H, page)
        else:
            shape = (L, S, H, rows)
        self.rows = rows

        def make():
            if order == "tokens":                                    # token-major memory: [.., row, head, 80]
                return torch.full((shape[0], shape[1], shape[3], shape[2], ROW), 255, dtype=torch.uint8, device=device).transpose(2, 3)
            pitch = {"heads": ROW, "padded": 112}[order]
            return torch.full((*shape, pitch), 255, dtype=torch.uint8, device=device)[..., :ROW]
        self.k, self.v = make(), make()

    def at(self, t, l, s, h, n):
        if self.page:
            return t[l, int(self.table[s, n // self.page]), h, n % self.page]
        return t[l, s, h, n]

    def unit(self, t, l, s, h, n):
        """The first n rows of a unit, [n, 80]."""
        idx = torch.arange(n, device=t.device)
        if self.page:
            return t[l, self.table[s].long()[idx // self.page], h, idx % self.page]
        return t[l, s, h, idx]

    def put(self, t, l, s, h, x):
        """Rows x [n, 80] into the first slots of a unit."""
        idx = torch.arange(x.shape[0], device=t.device)
        if self.page:
            t[l, self.table[s].long()[idx // self.page], h, idx % self.page] = x
        else:
            t[l, s, h, idx] = x

    def fill(self, l, s, h, n, g, k_spread=0.5, v_spread=1.0):
        """Random rows in the first n slots of a unit; v_spread may be a tensor [n, 1]."""
        for t, c in ((self.k, k_spread), (self.v, v_spread)):
            x = c * torch.randn(n, D, generator=g, device=t.device) + 0.5 * torch.randn(1, D, generator=g, device=t.device)
            self.put(t, l, s, h, as_rows(x))

    def view(self, tb, **kw):
        return tb.CacheView(self.k, self.v, page_table=self.table, **kw)


def attention(q, krows, vrows, scale):
    """q [128] float64, rows [n, 80] -> (out [128], lse, error bound [128] without the last rounding, bound of the lse)."""
    n = krows.shape[0]
    if n == 0:
        z = torch.zeros(D, dtype=torch.float64, device=q.device)
        return z, -math.inf, z, 0.0
    k, v = values(krows), values(vrows)
    x = k @ q * scale
    _, ks, kc = parts(krows)
    aq = q.abs()
    qg = aq.unflatten(-1, (4, 32)).sum(-1)
    d = abs(scale) * float((2.0 ** -12 * (ks @ qg) + 2.0 ** -15 * (kc.abs() @ qg) + 2.0 ** -19 * (k.abs() @ aq)).max())
    m = x.max()
    p = torch.exp(x - m)
    l = p.sum()
    p = p / l
    _, vs, vc = parts(vrows)
    coded = p @ (v - (vc - 8 * vs).repeat_interleave(32, -1))         # s u >= 0
    tol = 2 * d * (p @ v.abs()) + 2.0 ** -15 * (p @ (vc.abs() + 8 * vs).repeat_interleave(32, -1)) + (2.0 ** -11 + 2.0 ** -15) * coded
    return p @ v, float(m + torch.log(l)), tol + n * 2.0 ** -32 * float(vs.max()), d + 2.0 ** -18
