"""Calls of the decode step that follow each other in a stream with nothing in between: each reads what the one before it
wrote (lengths, rotated queries, cached rows), although its launch begins while that one still runs."""
import pytest
import torch

from paper_2604_04921_b200 import binding as tb
from step_reference import Cache, D, U_BF16
from test_gpu_step import DEV, check_rows, context, int32, raw

pytestmark = pytest.mark.gpu

ROOM = 6000          # more rows than clusters of blocks take: passes over prefixes and own rows, then joined


class Step:
    """One layer that appends T tokens per sequence and attends for the last of them, `steps` times."""

    def __init__(self, S, fmt, page, T, steps, G=4, H=2, n=700):
        self.S, self.G, self.H, self.T, self.n, self.steps, self.fmt = S, G, H, T, n, steps, fmt
        g = torch.Generator(device=DEV).manual_seed(S + T)
        self.start = [(5 * s) % 40 for s in range(S)]
        self.c = Cache(1, S, H, max(self.start) + T * steps, fmt, page)
        self.pc = Cache(1, 1, H, ROOM, fmt, page, seed=1)
        for h in range(H):
            self.pc.fill(0, 0, h, n, g)
            for s in range(S):
                self.c.fill(0, s, h, self.start[s], g)
        self.lens, self.first = int32(self.start), int32(self.start)
        self.pos = torch.tensor([1000 + s for s in self.start], device=DEV)
        self.x = torch.randn(steps, S, T, (G + 2) * H, D, generator=g, device=DEV).to(torch.bfloat16)
        self.q = torch.zeros(steps, S, T, G * H, D, dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros(steps, S, G * H, D, dtype=torch.bfloat16, device=DEV)
        self.ctx = context(1, H, G)
        self.cache = tb.LayerCache(self.c.view(tb, seq_lens=self.lens), 0)
        self.prefix = tb.LayerCache(self.pc.view(tb, seq_lens=int32([n])), 0)
        self.groups = int32([0, S])
        self.ws = self.ctx.attend_workspace(S, 1)

    def run(self):
        GH = self.G * self.H
        self.lens.copy_(self.first)
        for i in range(self.steps):
            x = self.x[i]
            self.ctx.append(self.cache, x[:, :, GH:GH + self.H], x[:, :, GH + self.H:], self.pos, q=x[:, :, :GH], q_out=self.q[i],
                            new_lens=self.lens)
            self.ctx.attend_shared(self.prefix, self.groups, self.cache, self.q[i, :, -1], self.out[i], self.ws)


@pytest.mark.parametrize("fmt,page", [("bf16", 0), ("bf16", 16), ("e4m3", 16)])
@pytest.mark.parametrize("S", [3, 20])                               # the 16-row and the 128-row pass over the prefix
@pytest.mark.parametrize("T", [1, 9])                                # lengths in place: by the append's launch, by one behind it
def test_append_then_attend_shared_back_to_back(fmt, page, S, T):
    st = Step(S, fmt, page, T, 24)
    st.run()
    torch.cuda.synchronize()
    for i in range(0, st.steps, 5):
        check_rows(st.out[i], None, st.q[i, :, -1],
                   lambda s, h: tuple(torch.cat((st.pc.unit(a, 0, 0, h, st.n), st.c.unit(b, 0, s, h, st.start[s] + (i + 1) * T)))
                                      for a, b in ((st.pc.k, st.c.k), (st.pc.v, st.c.v))),
                   S, st.H, st.G, D ** -0.5, extra=2 * U_BF16 if S == 20 else 0.0)
    want = st.out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.run()
    for r in range(3):
        st.q.zero_()
        st.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(raw(st.out), raw(want)), r


def test_three_streams_append_and_attend_shared_at_once():
    """Each with a cache and a workspace of its own, through the 16-row and the 128-row pass: the bits of each alone."""
    jobs = [Step(S, "bf16", 16, 1, 12) for S in (3, 20, 33)]
    want = []
    for st in jobs:
        st.run()
        torch.cuda.synchronize()
        want.append(st.out.clone())
    streams = [torch.cuda.Stream() for _ in jobs]
    for r in range(4):
        for st in jobs:
            st.out.zero_()
        torch.cuda.synchronize()
        for st, stream in zip(jobs, streams):
            with torch.cuda.stream(stream):
                st.run()
        torch.cuda.synchronize()
        for st, out in zip(jobs, want):
            assert torch.equal(raw(st.out), raw(out)), (r, st.S)
