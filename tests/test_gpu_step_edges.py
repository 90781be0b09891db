"""Calls of the decode step that its documentation allows or refuses at the edges: group boundaries outside the batch,
destinations that meet, tensors of another device."""
import pytest
import torch

from paper_2604_04921_b200 import binding as tb
from step_reference import Cache, D
from test_gpu_step import DEV, check_shared, context, int32

pytestmark = pytest.mark.gpu

ROOM = 6000          # more rows than clusters of blocks take


@pytest.mark.parametrize("rows", [None, ROOM])
@pytest.mark.parametrize("S", [4, 30])
def test_group_boundaries_outside_the_batch_count_as_the_nearest_bound(S, rows):
    """Entries that descend only outside [0, S] are no descending groups: the prefixes between them have no sequences, and
    the others keep theirs."""
    lens = [(7 * s) % 30 for s in range(S)]
    check_shared("bf16", 16, 2, 4, [-1, -5, S], [50, 70], lens, rows=rows)
    check_shared("e4m3", 16, 2, 4, [0, 2, S + 5, S + 2], [150, 70, 9], lens, rows=rows)


def test_destinations_that_meet_are_refused():
    """Lengths stored over others that are still to be read, rows of several heads, sequences or tokens in one place."""
    S, T, H, G = 3, 20, 2, 4
    ctx, c = context(1, H, G), Cache(1, S, H, 64)
    x = torch.zeros(S, T, H, D, dtype=torch.bfloat16, device=DEV)
    xq = torch.zeros(S, T, H * G, D, dtype=torch.bfloat16, device=DEV)
    many = int32([1] * 16)
    lens, pos = many[:S], torch.zeros(8, dtype=torch.int64, device=DEV)
    lc = tb.LayerCache(c.view(tb, seq_lens=lens), 0)

    def refused(lc, code=1, pos=pos[:S], **kw):
        with pytest.raises(tb.TriError) as e:
            ctx.append(lc, x, x, pos, **kw)
        assert e.value.code == code

    refused(lc, new_lens=many[1:1 + S])                               # another sequence's length
    refused(lc, new_lens=many[2:2 + S])
    refused(lc, new_lens=many[6:6 + S], n_new=many[8:8 + S])
    refused(lc, new_lens=pos.view(torch.int32)[1:1 + S])
    heads = int32([1] * (2 * S * H))
    refused(tb.LayerCache(c.view(tb), 0, unit_lens=heads[:S * H]), new_lens=heads[H:H + S * H])
    wide = c.k[:, :, :1].expand(-1, -1, H, -1, -1)
    refused(tb.LayerCache(tb.CacheView(wide, wide, seq_lens=lens), 0))
    wide = c.k[:, :1].expand(-1, S, -1, -1, -1)
    refused(tb.LayerCache(tb.CacheView(wide, wide, seq_lens=lens), 0))
    for q_out in (xq[:, :, :1].expand(-1, -1, H * G, -1), xq[:, :1].expand(-1, T, -1, -1), xq[:1].expand(S, -1, -1, -1)):
        refused(lc, q=xq, q_out=q_out)
    q, ws = xq[:, 0], ctx.attend_workspace(S)
    out = torch.zeros(S, H * G, D, dtype=torch.bfloat16, device=DEV)
    for o in (out[:1].expand(S, -1, -1), out[:, :1].expand(-1, H * G, -1)):
        with pytest.raises(tb.TriError) as e:
            ctx.attend(lc, q, o, ws)
        assert e.value.code == 1
    torch.cuda.synchronize()
    assert bool((many == 1).all()) and bool((heads == 1).all()) and bool(c.k.isnan().all())      # nothing ran
    # apart from the lengths, right behind them, or the lengths themselves
    ctx.append(lc, x, x, pos[:S], new_lens=many[S:2 * S])
    ctx.append(lc, x, x, pos[:S], new_lens=lens)
    torch.cuda.synchronize()
    assert many.tolist() == [1 + T] * (2 * S) + [1] * 10
