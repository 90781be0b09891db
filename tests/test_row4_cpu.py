"""Host-only checks of the 4-bit cache: structure layouts, the binding's own checks, and the 64-bit forms the GPU tests compare with."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2604_04921_b200 import binding as tb
from row4_reference import Cache4, D, ROW, as_rows, bf16_not_below, packed, parts, position, quantised, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layout_matches_the_header(tmp_path):
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "tri_attention.h"', 'int main(void){',
           'printf("row %d\\n", TRI_ROW4_BYTES);', 'printf("tri_read_rows %zu\\n", sizeof(tri_read_rows));']
    src += [f'printf("{f} %zu\\n", offsetof(tri_read_rows, {f}));' for f, _ in tb._ReadRows._fields_]
    (tmp_path / "l.c").write_text("\n".join(src + ['return 0;}']))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "l"), str(tmp_path / "l.c")], check=True)
    out = dict(x.split() for x in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(out["row"]) == ROW == tb.ROW4_BYTES and int(out["tri_read_rows"]) == ctypes.sizeof(tb._ReadRows)
    for f, _ in tb._ReadRows._fields_:
        assert int(out[f]) == getattr(tb._ReadRows, f).offset, f
    assert len(tb._pack_read(1, 2, 0, 3, 4, 5, 6, 7, 8, 9, 10)) == ctypes.sizeof(tb._ReadRows)


def test_null_arguments_are_rejected():
    tb.build()
    assert tb.lib().tri_read(None, None, 1, None, None, None) == 1


def test_views_of_4_bit_rows():
    c = Cache4(2, 3, 2, 16, page=16, device="cpu")
    cv = c.view(tb).c_view()
    assert cv.k_kind == 5 and (cv.stride_slot, cv.stride_head, cv.page_size) == (80, 80 * 16, 16)
    plain = Cache4(1, 3, 2, 16, order="tokens", device="cpu").view(tb).c_view()
    assert (plain.stride_tok, plain.stride_head, plain.n_max) == (160, 80, 16)
    k = torch.zeros(1, 1, 1, 16, 80, dtype=torch.uint8)
    for bad in (tb.CacheView(k[..., :64], None), tb.CacheView(torch.zeros(1, 1, 1, 16, 128, dtype=torch.uint8), None),
                tb.CacheView(k, k.to(torch.bfloat16)), tb.CacheView(k, None, pre_rope=True),
                tb.CacheView(torch.zeros(1, 1, 1, 16, 128, dtype=torch.bfloat16), k)):
        with pytest.raises(AssertionError):
            bad.c_view()


def test_positions_fill_a_row():
    seen = {(8 * position(d)[0] + position(d)[1]) // 4 for d in range(D)}
    assert seen == set(range(D))
    assert position(0) == (0, 0) and position(1) == (2, 0) and position(2) == (0, 4) and position(8) == (16, 0) and position(32) == (4, 0)


def test_quantised_rows_come_back_within_half_a_step():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(200, D, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(200, 1, generator=g, dtype=torch.float64)) + 2
    x[7, :32] = 3.0
    x[8, :64] = 0.0
    code, s, c = quantised(x)
    rows = packed(code, s, c)
    code2, s2, c2 = parts(rows)
    assert torch.equal(code, code2) and torch.equal(s, s2) and torch.equal(c, c2)
    err = (values(rows) - x).abs()
    assert bool((err <= s.repeat_interleave(32, -1) / 2 * (1 + 1e-12)).all())
    assert bool((code >= 0).all()) and bool((code <= 15).all())
    assert float(s[7, 0]) == 0 and bool((values(rows)[7, :32] == 3).all()) and bool((values(rows)[8, :64] == 0).all())
    # the ends of the range are used: 15 steps span a group but for the rounding up of s and of c
    span = x.unflatten(-1, (4, 32)).amax(-1) - x.unflatten(-1, (4, 32)).amin(-1)
    assert bool((15 * s <= span * (1 + 2 ** -6) + 16 * 2.0 ** -8 * c.abs()).all())


def test_bf16_not_below():
    for x, want in ((1.0, 1.0), (1.0 + 2 ** -30, 1.0 + 2 ** -7), (0.0, 0.0), (1e-45, 2.0 ** -126), (255.5, 256.0)):
        assert float(bf16_not_below(torch.tensor(x, dtype=torch.float64))) == want


def test_rows_hold_what_was_put_there():
    c = Cache4(1, 2, 2, 20, page=16, device="cpu")
    x = torch.randn(20, D, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    c.put(c.k, 0, 1, 1, as_rows(x))
    assert torch.equal(c.unit(c.k, 0, 1, 1, 20), as_rows(x))
    assert torch.equal(c.at(c.k, 0, 1, 1, 17), as_rows(x)[17]) and bool((c.unit(c.k, 0, 0, 1, 20) == 255).all())


def test_kernels_read_nothing_through_the_read_only_path():
    """They begin while their predecessor still runs; a read-only load may be moved before the wait for it."""
    for name in ("tri_row4.cuh", "tri_append4.cuh", "tri_read.cuh", "tri_attend4.cuh"):
        with open(os.path.join(ROOT, "paper_2604_04921_b200", "csrc", name)) as f:
            code = [line.split("//")[0] for line in f]
        assert not [line for line in code if "__ldg" in line or ".nc." in line or " row_offset(" in line], name


def test_caches_and_rows_of_another_device_never_reach_the_library(monkeypatch):
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0
    monkeypatch.setattr(tb, "lib", Library)
    monkeypatch.setattr(tb, "_stream_on", lambda device: 0)
    ctx = tb.TriContext.__new__(tb.TriContext)
    ctx.n_layers, ctx.n_kv_heads, ctx.group_size, ctx._h, ctx._dev = 1, 2, 4, None, 0
    c, lens = Cache4(1, 3, 2, 16, device="cpu"), torch.zeros(3, dtype=torch.int32)
    lc = tb.LayerCache(c.view(tb, seq_lens=lens), 0)
    x = torch.zeros(3, 5, 2, 128, dtype=torch.bfloat16)
    for dev in (-1, 0):                                              # (0: as if the cache were there: the rows are not)
        lc._dev = dev
        with pytest.raises(AssertionError):
            ctx.read(lc, x, x.clone())
    lc._dev = ctx._dev = -1                                          # all of it on one device: the other checks
    keyless = tb.LayerCache(tb.CacheView(c.k, None, seq_lens=lens), 0)
    keyless._dev = -1
    for bad in (lambda: ctx.read(lc, None, None), lambda: ctx.read(lc, x[:2], None), lambda: ctx.read(lc, x, x[:, :4].clone()),
                lambda: ctx.read(lc, x, x.float()), lambda: ctx.read(lc, x.half(), None), lambda: ctx.read(lc, x.transpose(2, 3), None),
                lambda: ctx.read(lc, x, None, first=lens.long()), lambda: ctx.read(lc, x, None, first=lens[:2]),
                lambda: ctx.read(keyless, x, x.clone())):
        with pytest.raises(AssertionError):
            bad()
    assert not reached
    ctx.read(lc, x, x.clone(), first=lens)
    assert reached == ["tri_read"]


def test_strides_under_which_rows_meet(tmp_path):
    """tri_rows.h against all pairs of rows, for random strides, nested ones and ones that only interleave."""
    src = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "tri_rows.h"
using tri::RowDim;
static bool brute(const RowDim *d, int64_t row)
{
    std::vector<int64_t> at;
    for (int64_t i = 0; i < d[0].n; ++i) for (int64_t j = 0; j < d[1].n; ++j) for (int64_t k = 0; k < d[2].n; ++k)
        at.push_back(i * d[0].stride + j * d[1].stride + k * d[2].stride);
    std::sort(at.begin(), at.end());
    for (size_t i = 1; i < at.size(); ++i) if (at[i] - at[i - 1] < row) return false;
    return true;
}
int main()
{
    srand(1);
    int apart = 0, meet = 0, woven = 0, wrong = 0;
    for (int t = 0; t < 300000; ++t) {
        RowDim d[3];
        const int64_t row = t % 2 ? 128 : 80;
        for (RowDim &x : d) x = {1 + rand() % 5, (rand() % 2 ? 8 * (rand() % 130) : row * (rand() % 9)) * (rand() % 4 ? 1 : -1)};
        const bool want = brute(d, row), got = tri::rows_apart(d[0], d[1], d[2], row);
        wrong += want != got;
        (want ? apart : meet)++;
        if (want) {                                          // apart although no order of the strides nests
            std::sort(d, d + 3, [](RowDim a, RowDim b) { return llabs(a.n > 1 ? a.stride : 0) < llabs(b.n > 1 ? b.stride : 0); });
            int64_t extent = row;
            bool nested = true;
            for (RowDim &x : d) if (x.n > 1) { nested = nested && llabs(x.stride) >= extent; extent += (x.n - 1) * llabs(x.stride); }
            woven += !nested;
        }
    }
    const int64_t far = INT64_MAX / 4, h = 128;
    const bool edges = tri::rows_apart({4, far}, {2, h}, {1, 0}, h) && !tri::rows_apart({2, INT64_MIN}, {2, INT64_MIN}, {1, 7}, h) &&
        tri::rows_apart({2, INT64_MIN}, {1, 0}, {1, 0}, h) && tri::rows_apart({1, 0}, {1, 0}, {1, 0}, h) &&
        tri::rows_apart({1 << 20, 1 << 20}, {64, 128}, {128, 64 * 128}, h) && !tri::rows_apart({2, h}, {2, h}, {1, 0}, h) &&
        !tri::rows_apart({1000000, 256}, {8, 384}, {4, 768}, h);
    printf("%d %d %d %d %d\n", wrong, apart, meet, woven, edges);
}
"""
    (tmp_path / "r.cpp").write_text(src)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2604_04921_b200", "csrc"), "-o", str(tmp_path / "r"),
                    str(tmp_path / "r.cpp")], check=True)
    wrong, apart, meet, woven, edges = map(int, subprocess.run([str(tmp_path / "r")], check=True, capture_output=True, text=True).stdout.split())
    assert wrong == 0 and edges and min(apart, meet, woven) > 500
