"""Attention with shared prefixes held to the bound of the path a call takes.

Only the 128-row pass over a prefix rounds weights once, so only there is more allowed than step_reference.py derives for
weights of 16 + 16 bits:
  clusters, 16-row pass   nothing more, whatever the prefix's format and scales (sums that go on from a prefix of other scales
                          are multiplied by their ratio: 2^-24, inside the 2^-15 that stand there)
  128-row pass, 8 bits    weights are f16 values of [2^-14, 2^15], off by 2^-11 of themselves: 2^-11 sum p_n |v_n|; smaller ones by
                          2^-25 where the largest is 2^11 at least, 2^-36 of the sum for a row, inside the 2^-15 for 2^21 rows
"""
import pytest
import torch

import test_gpu_step as step

pytestmark = pytest.mark.gpu

ROOM = 6000          # more rows than clusters of blocks take
PLACES = 8           # blocks of a cluster


@pytest.fixture
def check(monkeypatch):
    plain = step.check_rows

    def run(fmt, page, H, G, starts, plens, lens, extra=0.0, **kw):
        monkeypatch.setattr(step, "check_rows", lambda *a, **k: plain(*a, **dict(k, extra=extra)))
        step.check_shared(fmt, page, H, G, starts, plens, lens, **kw)
    return run


GROUPS = {1: [0, 1, 6, 6, 9], 3: [0, 1, 6, 6, 9], 4: [0, 1, 6, 6, 9], 5: [0, 1, 6, 6, 9], 8: [0, 1, 5, 5, 7], 16: [0, 2, 3, 3, 4]}


@pytest.mark.parametrize("rows", [None, ROOM])                        # clusters; the 16-row pass
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("G", sorted(GROUPS))
def test_up_to_16_query_rows_per_prefix(check, fmt, G, rows):
    starts = GROUPS[G]
    S = starts[-1]
    assert S * 2 * PLACES <= 2 * torch.cuda.get_device_properties(0).multi_processor_count and S * G <= 16 * 4
    check(fmt, 16, 2, G, starts, [300, 65, 40, 128], [0, 5, 17, 64, 1, 0, 130, 2, 33][:S], seed=40 + G, rows=rows)


@pytest.mark.parametrize("a,b", [("bf16", "e4m3"), ("e4m3", "bf16")])
def test_prefixes_of_another_format(check, a, b):
    check(a, 16, 2, 4, [0, 3, 5], [200, 77], [10, 0, 65, 3, 20], pfmt=b, ppage=0, rows=ROOM, seed=50)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_long_prefixes_of_few_sequences(check, fmt):
    check(fmt, 16, 1, 4, [0, 3], [20000], [100, 0, 3000], seed=51)
    check(fmt, 0, 2, 1, [0, 13], [5000], [10 * s for s in range(13)], seed=52)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("G,S", [(1, 140), (4, 40), (5, 60), (8, 33), (16, 20)])
def test_8_bit_prefixes_of_many_sequences(check, G, S, page):
    check("e4m3", page, 2, G, [0, S - 3, S], [1517, 129], [(7 * s) % 40 for s in range(S)], extra=2.0 ** -11, rows=ROOM, seed=60 + G)
