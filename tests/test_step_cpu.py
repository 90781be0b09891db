"""Host-only checks of the decode step's entry points: structure layouts, null arguments, the binding's own checks, and the
64-bit forms the GPU tests compare with."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2604_04921_b200 import binding as tb
from step_reference import Cache, attention, pair_magnitude, rope

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_the_header(tmp_path):
    mirrors = {"tri_layer_cache": tb._LayerCache, "tri_append_rows": tb._AppendRows, "tri_attend_io": tb._AttendIo}
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "tri_attention.h"', 'int main(void){']
    for st, cls in mirrors.items():
        src.append(f'printf("{st} %zu\\n", sizeof({st}));')
        src += [f'printf("{st}.{f} %zu\\n", offsetof({st}, {f}));' for f, _ in cls._fields_]
    (tmp_path / "l.c").write_text("\n".join(src + ['return 0;}']))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "l"), str(tmp_path / "l.c")], check=True)
    out = dict(x.split() for x in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    for st, cls in mirrors.items():
        assert int(out[st]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(out[f"{st}.{f}"]) == getattr(cls, f).offset, (st, f)


def test_null_arguments_are_rejected():
    tb.build()
    lib = tb.lib()
    assert lib.tri_append(None, None, 1, None, None, None, None) == 1
    assert lib.tri_attend(None, None, 1, None, None, None, 0, None) == 1
    assert lib.tri_attend_shared(None, None, 1, None, None, 1, None, None, None, 0, None) == 1
    assert lib.tri_attend_workspace_bytes(None, 1, 1) == 0


def test_layer_cache_checks_its_parts():
    c = Cache(2, 3, 2, 16, page=16, device="cpu")
    lens = torch.zeros(3, dtype=torch.int32)
    view = c.view(tb, seq_lens=lens)
    lc = tb.LayerCache(view, 1)
    assert (lc.n_layers, lc.n_seqs, lc.n_kv_heads) == (2, 3, 2)
    assert lc._c.view.contents.page_size == 16 and lc._c.layer == 1 and lc._c.unit_lens is None
    tb.LayerCache(c.view(tb), 0, unit_lens=torch.zeros(2, 3, 2, dtype=torch.int32))
    for bad in (lambda: tb.LayerCache(view, 2), lambda: tb.LayerCache(c.view(tb), 0),
                lambda: tb.LayerCache(view, 0, unit_lens=torch.zeros(2, 3, dtype=torch.int32)),
                lambda: tb.LayerCache(view, 0, unit_lens=torch.zeros(2, 3, 2, dtype=torch.int64)),
                lambda: tb.LayerCache(view, 0, k_scale=torch.zeros(2, 2, dtype=torch.float64)),
                lambda: tb.LayerCache(view, 0, k_scale=torch.zeros(3)),
                lambda: tb.LayerCache(c.view(tb, seq_lens=lens, positions=torch.zeros(1, 3, 2, 16, dtype=torch.int32)), 0)):
        with pytest.raises(AssertionError):
            bad()


@pytest.mark.parametrize("half_split", [False, True])
def test_reference_rotation(half_split):
    """Keeps magnitudes, composes, and leaves position 0 alone."""
    x = torch.randn(128, dtype=torch.float64, generator=torch.Generator().manual_seed(0))
    assert torch.equal(rope(x, 0, 1e6, half_split), x)
    y = rope(x, 1234, 1e6, half_split)
    assert torch.allclose(pair_magnitude(x, half_split), pair_magnitude(y, half_split), atol=1e-12)
    assert torch.allclose(rope(y, 766, 1e6, half_split), rope(x, 2000, 1e6, half_split), atol=1e-9)


def test_reference_attention_merges_over_cuts():
    """The identity every split of the kernels rests on: parts joined by their lse give the whole."""
    g = torch.Generator().manual_seed(1)
    q, k, v = torch.randn(128, generator=g).double(), torch.randn(50, 128, generator=g).double(), torch.randn(50, 128, generator=g).double()
    whole, lse, _ = attention(q, k, v, 0.1)
    a, la, _ = attention(q, k[:17], v[:17], 0.1)
    b, lb, _ = attention(q, k[17:], v[17:], 0.1)
    m = max(la, lb)
    wa, wb = math.exp(la - m), math.exp(lb - m)
    assert torch.allclose((wa * a + wb * b) / (wa + wb), whole, atol=1e-12)
    assert abs(m + math.log(wa + wb) - lse) < 1e-12


def test_step_kernels_read_nothing_through_the_read_only_path():
    """They begin while their predecessor still runs; a read-only load may be moved before the wait for it."""
    for name in ("tri_step.cuh", "tri_append.cuh", "tri_attend.cuh", "tri_attend_umma.cuh"):
        with open(os.path.join(ROOT, "paper_2604_04921_b200", "csrc", name)) as f:
            code = [line.split("//")[0] for line in f]
        assert not [line for line in code if "__ldg" in line or ".nc." in line or " row_offset(" in line], name


@pytest.mark.parametrize("call", ["append", "attend", "attend_shared"])
def test_caches_of_another_device_never_reach_the_library(call, monkeypatch):
    """A cache in host memory is consistent in itself; only the context knows that its kernels could not read it."""
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0
    monkeypatch.setattr(tb, "lib", Library)
    monkeypatch.setattr(tb, "_stream_on", lambda device: 0)
    ctx = tb.TriContext.__new__(tb.TriContext)
    ctx.n_layers, ctx.n_kv_heads, ctx.group_size, ctx._h, ctx._dev = 1, 2, 4, None, 0
    c, lens = Cache(1, 3, 2, 16, device="cpu"), torch.zeros(3, dtype=torch.int32)
    lc = tb.LayerCache(c.view(tb, seq_lens=lens), 0)
    x, q = torch.zeros(3, 1, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    run = {"append": lambda: ctx.append(lc, x, x, torch.zeros(3, dtype=torch.int64)),
           "attend": lambda: ctx.attend(lc, q, q.clone(), ws),
           "attend_shared": lambda: ctx.attend_shared(lc, torch.tensor([0, 3, 3, 3], dtype=torch.int32), lc, q, q.clone(), ws)}[call]
    with pytest.raises(AssertionError):
        run()
    assert not reached
    lc._dev = 0                                                       # (as if it were there: the rest of the arguments is not)
    with pytest.raises(AssertionError):
        run()
    assert not reached


def test_the_documented_decode_step_attends_over_the_new_token():
    """The README's decode step, run with a context that only keeps lengths: every layer's attention counts the appended row,
    in the first step and in one behind it."""
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = [b.split("```")[0] for b in f.read().split("```python\n")[1:]]
    code, = [b for b in blocks if "ctx.append(" in b]
    L, S, H, G = 3, 2, 2, 4
    c = Cache(L, S, H, 16, device="cpu")
    seq_lens = torch.tensor([3, 9], dtype=torch.int32)
    src = c.view(tb, seq_lens=seq_lens)
    other = [tb.LayerCache(c.view(tb, seq_lens=torch.zeros(S, dtype=torch.int32)), l) for l in range(L)]
    attended = []

    class Lengths:
        def append(self, cache, k, v, pos, q=None, q_out=None, n_new=None, new_lens=None):
            if new_lens is not None:
                new_lens.copy_(cache.view.seq_lens + 1)

        def attend(self, cache, q, out, ws):
            attended.append((cache.layer, cache.view.seq_lens.tolist()))

        def attend_shared(self, prefix, starts, cache, q, out, ws):
            self.attend(cache, q, out, ws)

        def attend_workspace(self, S, n_prefixes=0):
            return None
    new = torch.zeros(S, 1, H, 128)
    names = dict(tb=tb, torch=torch, ctx=Lengths(), src=src, seq_lens=seq_lens, k=c.k, v=c.v, q=new, k_new=new, v_new=new, q_new=new,
                 q_rot=new, pos=torch.zeros(S), out=None, n_layers=L, S=S, after=other, prefix=other, starts=None, n_prefixes=1)
    for step in range(2):
        attended.clear()
        exec(code, dict(names))
        want = [4 + step, 10 + step]
        assert {l for l, _ in attended} == set(range(L)) and all(n == want for _, n in attended), attended
        assert seq_lens.tolist() == want
