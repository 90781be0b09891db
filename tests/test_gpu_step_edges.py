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
