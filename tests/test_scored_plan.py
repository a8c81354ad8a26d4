"""Which launch a window gets, alone and beside a prefix (host arithmetic), and what such launches answer where the prefix is most of what is seen."""
import ctypes

import numpy as np
import pytest

from paper_2410_09426_amd import binding as fq
from test_cache_plan import Plan, plan


def windowed(B, rows, length, window, prefix, H=8, G=4, sinks=0):
    fn = getattr(fq.lib(), "_ZN2fq21attention_plan_windowElliilliib")
    i64 = ctypes.c_int64
    fn.restype, fn.argtypes = Plan, [i64, i64, ctypes.c_int, ctypes.c_int, i64, i64, ctypes.c_int, ctypes.c_int, ctypes.c_bool]
    return fn(B, B * rows, H, H * G, rows, length, window, sinks, prefix)


def _fields(p, but=()):
    return {n: getattr(p, n) for n, _ in Plan._fields_ if n not in but}


SIZES = [(1, 1, 131072), (1, 64, 131072), (4, 8, 16384), (16, 1, 8192), (64, 1, 4096), (16, 13, 3000), (1, 2048, 8192), (300, 2, 500), (2, 100, 700), (3, 1, 0)]


@pytest.mark.parametrize("window,sinks", [(1, 0), (512, 4), (100000, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("B,rows,length", SIZES)
def test_a_prefix_is_planned_for(B, rows, length, window, sinks):
    """As the whole length, split finer (the kernels lengthen the splits); without a prefix, by what the window shows."""
    whole, p, alone = plan(B, rows, length), windowed(B, rows, length, window, True, sinks=sinks), windowed(B, rows, length, window, False, sinks=sinks)
    assert _fields(p, ("chunk",)) == _fields(whole, ("chunk",))
    assert p.chunk == (min(whole.chunk, 256) if whole.splits > 1 else whole.chunk)
    fewer = plan(B, rows, length, seen=window + sinks + rows + 64)
    assert _fields(alone) == _fields(fewer if fewer.workspace <= whole.workspace else whole)
    assert _fields(windowed(B, rows, length, 0, True)) == _fields(windowed(B, rows, length, 0, False)) == _fields(whole)


@pytest.mark.gpu
@pytest.mark.parametrize("hint", ["length", "less"])
@pytest.mark.parametrize("rows,lengths,prefix", [([1, 1], [20000, 9000], [15000, 3]), ([5, 2], [16000, 12000], [9999, 12000]), ([64], [20000], [15001]), ([64, 33], [9000, 20000], [0, 17000]),
                                                 ([300, 1], [6000, 12000], [5600, 11000])])
def test_long_prefixes_beside_short_windows(rows, lengths, prefix, hint):
    from cache_util import D, Batch
    from oracle import step_oracle as so
    from test_gpu_scored import expect, run_scored
    print(f"[case] {rows} of {lengths}, prefixes {prefix}, hint {hint}", flush=True)
    H, G, heads = 2, 4, [0, 7]
    c = Batch(52, rows, lengths, H, page=64).upload()
    q = c.row_tensor(H * G)
    how = dict(cap=30.0, prefix=prefix, window=70, sinks=2)
    got = run_scored(c, q, G, 0.09, batch=c.batch(max_length=max(lengths) if hint == "length" else 200), **how)
    sequences = None
    if max(rows) > 64:                                                         # (the oracle goes through rows: some of the first sequence's)
        sequences, L, keep = [1], lengths[0], np.r_[0:3, 150, rows[0] - 2:rows[0]]
        pos = L - rows[0] + keep
        seen = (np.arange(L) <= pos[:, None]) & ((np.arange(L) > pos[:, None] - 70) | (np.arange(L) < 2)) | (np.arange(L) < prefix[0])
        k, v = (x.values(c.table[0, :c.width], np.arange(L)) for x in c.host)
        ks, vs = (x.steps(c.table[0, :c.width], np.arange(L)) for x in c.host)
        for h in heads:
            o, A, S, E = so.scored64(q.reshape(c.T, H * G, D)[keep, h], k[h // G], v[h // G], seen, 0.09, pos, 30.0, 0.0, ks[h // G], vs[h // G])
            assert (np.abs(got[keep, h] - o) <= so.scored_bound(o, A, S, E, L)).all()
    want, tol = expect(c, q.reshape(c.T, H * G, D), G, 0.09, heads=heads, sequences=sequences, **how)
    looked = ~np.isnan(want)
    assert looked.any() and (np.abs(got.astype(np.float64) - want)[looked] <= tol[looked]).all()
