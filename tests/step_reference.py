"""Plain 64-bit forms of the decode step's operators (append with rotation, attention over a cache, attention with shared
prefixes), written row by row from their definitions, and the caches the tests run them on.

Error bounds used by the tests (u = half a step of a format relative to the value: bf16 2^-8, e4m3 2^-4):
  append   the rotation is fp32 (cos and sin to 2^-23, three roundings): off by less than 2^-21 |z| before the one rounding
           to the cache's format, |z| the pair's magnitude; the reference's own angle, p times a double, by p 2^-51 more; e4m3 steps below 2^-6 are 2^-9 wide, half of that 2^-10
  attend   a logit is off by at most d = 2^-19 scale sum_i |q_i k_i| (128 products in fp32 with truncating adders, < 16
           truncations of 2^-23 each on a path), a weight by the factor e^d (1 + 2^-20) (base-2 exponential 2^-22, and the
           16 + 16 bits it is split into), so a normalised sum by (2 d + 2^-15) sum_n p_n |v_n|, rounded once to bf16
  shared   where many sequences share a prefix the prefix's weights are rounded to bf16: 2^-8 sum_n p_n |v_n| more
"""
from __future__ import annotations

import math

import torch

D = 128
U_BF16, U_E4M3 = 2.0 ** -8, 2.0 ** -4
E4M3_MAX = 448.0


def rope(x: torch.Tensor, pos: int, theta: float, half_split: bool) -> torch.Tensor:
    """One row [128] in float64 rotated to `pos`."""
    f = torch.arange(64, dtype=torch.float64, device=x.device)
    ang = pos * theta ** (-2.0 * f / D)
    c, s = torch.cos(ang), torch.sin(ang)
    y = torch.empty_like(x)
    re, im = (slice(0, 64), slice(64, 128)) if half_split else (slice(0, 128, 2), slice(1, 128, 2))
    y[..., re] = c * x[..., re] - s * x[..., im]
    y[..., im] = s * x[..., re] + c * x[..., im]
    return y


def pair_magnitude(x: torch.Tensor, half_split: bool) -> torch.Tensor:
    """|z| of the pair every component belongs to, same shape."""
    a, b = (x[..., :64], x[..., 64:]) if half_split else (x[..., 0::2], x[..., 1::2])
    m = torch.sqrt(a * a + b * b)
    return torch.cat((m, m), -1) if half_split else m.repeat_interleave(2, -1)


class Cache:
    """One multi-layer cache in some layout, filled with NaN except where rows are put."""

    def __init__(self, L, S, H, rows, fmt="bf16", page=0, order="heads", seed=0, device="cuda", spare_pages=1):
        self.L, self.S, self.H, self.rows, self.fmt, self.page = L, S, H, rows, fmt, page
        g = torch.Generator(device="cpu").manual_seed(seed)
        kd = {"bf16": torch.bfloat16, "pre16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[fmt]
        vd = torch.float8_e4m3fn if fmt == "e4m3" else torch.bfloat16
        self.table = None
        if page:
            per = -(-rows // page)
            n = S * per + spare_pages
            perm = torch.randperm(n, generator=g)[:S * per]
            self.table = perm.to(torch.int32).view(S, per).to(device)
            self.rows = per * page
            shape = (L, n, H, page, D)
        else:
            shape = (L, S, H, rows, D)

        def make(dt):
            if order == "tokens":                                    # token-major memory: [.., row, head, 128]
                t = torch.empty(shape[0], shape[1], shape[3], shape[2], D, dtype=dt, device=device).transpose(2, 3)
            elif order == "padded":                                  # rows 144 elements apart
                t = torch.empty(*shape[:4], 144, dtype=dt, device=device)[..., :D]
            else:
                t = torch.empty(shape, dtype=dt, device=device)
            t.copy_(torch.full((1,), float("nan"), device=device).to(dt).expand(shape))
            return t
        self.k, self.v = make(kd), make(vd)
        if kd != vd and order != "heads":
            raise ValueError("K and V of different widths share their strides only in plain layouts")

    def at(self, t, l, s, h, n):
        if self.page:
            return t[l, int(self.table[s, n // self.page]), h, n % self.page]
        return t[l, s, h, n]

    def unit(self, t, l, s, h, n):
        """The first n rows of a unit, float64 [n, 128]."""
        if n == 0:
            return torch.zeros(0, D, dtype=torch.float64, device=t.device)
        if self.page:
            idx = torch.arange(n, device=t.device)
            return t[l, self.table[s].long()[idx // self.page], h, idx % self.page].double()
        return t[l, s, h, :n].double()

    def fill(self, l, s, h, n, g, spread=1.0):
        """Random rows in the first n slots of a unit."""
        for t, c in ((self.k, spread), (self.v, 1.0)):
            x = c * torch.randn(n, D, generator=g, device=t.device) + torch.randn(1, D, generator=g, device=t.device)
            x = (x.clamp(-E4M3_MAX, E4M3_MAX)).to(t.dtype)
            raw = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]
            if self.page:
                idx = torch.arange(n, device=t.device)
                t.view(raw)[l, self.table[s].long()[idx // self.page], h, idx % self.page] = x.view(raw)
            else:
                t.view(raw)[l, s, h, :n] = x.view(raw)

    def view(self, tb, **kw):
        return tb.CacheView(self.k, self.v, page_table=self.table, pre_rope=self.fmt == "pre16", **kw)


def attention(q, k, v, scale, kscale=1.0, vscale=1.0):
    """q [128], k, v [n, 128] float64 -> (out [128], lse, error bound [128] without the last rounding)."""
    if k.shape[0] == 0:
        z = torch.zeros(D, dtype=torch.float64, device=q.device)
        return z, -math.inf, z
    x = k @ q * (scale * kscale)
    d = 2.0 ** -19 * abs(scale) * kscale * float((k.abs() @ q.abs()).max())
    m = x.max()
    p = torch.exp(x - m)
    l = p.sum()
    out = (p / l) @ v * vscale
    return out, float(m + torch.log(l)), (2 * d + 2.0 ** -15) * ((p / l) @ v.abs() * vscale)
