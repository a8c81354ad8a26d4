"""Queries that are no numbers in attention with other scores (flatquant_cache_scored_attention): NaN wherever such a row sees a token, in every launch, though a cap would make
a number of an infinite score; other rows as they are."""
import numpy as np
import pytest

from cache_util import D, Batch
from oracle import cache_oracle as co
from test_gpu_scored import expect, kind_of, run_scored

pytestmark = pytest.mark.gpu
# rows, lengths, query heads a head: few rows in whole tiles, 17 to 32, many (whole, with an odd half, split)
SIZES = {"few": ([3, 1, 2], [3, 40, 1], 2), "tile of 32": ([9, 4], [9, 300], 3), "prompt": ([100, 33], [100, 31], 2), "half": ([40], [40], 1), "split": ([50, 40], [50, 1500], 4)}


def _channel(c, b, h, tokens):
    """A channel in which the first `tokens` tokens of head h have codes that are not the zero point, so that no product is infinity times zero."""
    p = [c.host[0].place(c.table[b, :c.width], j) for j in range(tokens)]
    q = np.stack([co.unpack(c.host[0].codes[x[0], h, x[1]][None], c.bits[0])[0].astype(int) for x in p])
    z = np.array([int(c.host[0].params[x[0], h, x[1]]) >> 16 for x in p])
    return int(np.flatnonzero((q != z[:, None]).all(0))[0])


@pytest.mark.parametrize("waves", [None, 4])
@pytest.mark.parametrize("kind", ["cap", "small cap", "large cap", "slopes", "prefix", "all"])
@pytest.mark.parametrize("size", SIZES)
def test_rows_of_infinities(size, kind, waves, tuning):
    rows, lengths, G = SIZES[size]
    print(f"[case] {size} {kind} waves={waves}", flush=True)
    if waves:
        tuning("FLATQUANT_ATT_WAVES", waves)
    H = 2
    c = Batch(41, rows, lengths, H).upload()
    how = kind_of(kind, c, G)
    q = c.row_tensor(H * G)
    bad = np.zeros((c.T, H * G), dtype=bool)
    n = c.starts[-1]
    # the first row of the first sequence sees one token (or what the prefix has), the others more
    for t, h, value in ((0, 0, np.inf), (0, G, -np.inf), (1, G, np.inf), (2, 0, -np.inf), (n - 1, H * G - 1, np.nan), (n - 2, 0, np.inf)):
        q[t, h * D + (_channel(c, 0, h // G, t + 1) if t < 3 else 77)] = value
        bad[t, h] = True
    got = run_scored(c, q, G, 0.09, **how)
    fine = np.where(np.repeat(bad, D, axis=1), np.float16(0), q).reshape(c.T, H * G, D)
    want, tol = expect(c, fine, G, 0.09, **how)
    seen = np.zeros(c.T, dtype=bool)
    for b in range(c.B):
        first = 0 if "prefix" not in how else how["prefix"][b]
        seen[c.starts[b]:c.starts[b + 1]] = c.visible(b).any(1) | (first > 0)
    none = bad & seen[:, None]
    assert none.sum() >= 4 and np.isnan(got[none]).all()
    ok = ~none[:n]
    assert np.isfinite(got[:n][ok]).all() and (np.abs(got[:n].astype(np.float64) - want[:n])[ok] <= tol[:n][ok]).all()
