"""Which launch attention over the paged key/value cache takes (host arithmetic; no GPU): the rules that stand beside attention_plan with both sides
measured, away from the sizes that they were measured at."""
import ctypes

import pytest

from paper_2410_09426_amd import binding as fq


class Plan(ctypes.Structure):
    _fields_ = [("tile_rows", ctypes.c_int), ("waves", ctypes.c_int), ("workgroups", ctypes.c_int), ("chunk", ctypes.c_int), ("splits", ctypes.c_int),
                ("stats_at", ctypes.c_int64), ("workspace", ctypes.c_int64)]


def plan(B, rows, length, H=8, G=4, seen=None):
    fn = getattr(fq.lib(), "_ZN2fq14attention_planElliilll")
    fn.restype, fn.argtypes = Plan, [ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int] + [ctypes.c_int64] * 3
    p = fn(B, B * rows, H, H * G, rows, length, length if seen is None else seen)
    cache = fq.KvCache(*[4096 * k for k in range(1, 5)], 8, 16, H, 4, 4)
    batch = fq.KvBatch(4096, 4096, 4096, B, B * rows, 1, 1, rows, length)
    assert seen is not None or p.workspace == fq.fq_cache_attention_workspace(cache, batch, H * G)
    return p


@pytest.mark.parametrize("B,rows,length,waves", [
    (64, 10, 2800, 4), (40, 30, 6000, 4), (33, 15, 1400, 4),      # rows for a quarter or half of the eight waves
    (32, 26, 1400, 8), (32, 26, 7000, 4), (32, 12, 1400, 4),      # one workgroup for each CU
    (32, 45, 5000, 8), (45, 36, 5000, 4), (64, 63, 5000, 8),
    (64, 70, 7000, 4), (64, 128, 7000, 8), (2, 4000, 7000, 8),
    (2, 4000, 1200, 4), (1, 200, 7000, 4), (7, 256, 7000, 4),     # few tokens, workgroups for some of the CUs
])
def test_eight_waves_have_rows(B, rows, length, waves):
    p = plan(B, rows, length)
    assert p.waves == waves and p.tile_rows == (256 if waves == 8 else 128)


@pytest.mark.parametrize("B,rows,length,balanced", [
    (1, 5, 900, False), (1, 6, 4500, True), (1, 8, 2500, True),   # a few pairs: from about 2000 tokens on
    (16, 7, 1800, False), (16, 5, 6000, True), (30, 8, 3000, False), (30, 5, 10000, True),
    (45, 6, 3000, False), (40, 6, 16000, True), (64, 7, 9000, False),      # more than one a CU
    (300, 5, 100, False),                                         # more sequences than that launch holds
])
def test_tiles_of_32_rows_are_balanced_by_what_they_take(B, rows, length, balanced):
    p = plan(B, rows, length)
    assert p.tile_rows == 32 and p.waves == 4 and (p.workgroups > 0) == balanced


@pytest.mark.parametrize("B,rows,length,waves", [(1, 1, 900, 8), (1, 3, 20000, 0), (16, 2, 3500, 16), (16, 1, 20000, 0), (50, 1, 6000, 8), (64, 4, 3000, 8),
                                               (70, 1, 5000, 8), (70, 1, 2000, 4), (300, 2, 9000, 8), (300, 2, 100, 4)])
def test_tiles_of_16_rows(B, rows, length, waves):
    p = plan(B, rows, length)
    assert p.tile_rows == 16 and ((p.workgroups > 0) if waves == 0 else (p.workgroups == 0 and p.waves == waves))
