"""Attention over the paged key/value cache at the ends of what scores can be: the largest scales, rows whose queries are no numbers beside rows whose are,
groups whose steps are none, and long contexts."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from cache_util import D, Batch, check_attention, run_attention

pytestmark = pytest.mark.gpu
LAUNCHES = {"chosen": {}, "balanced": {"FLATQUANT_ATT_WAVES": 0, "FLATQUANT_ATT_CHUNK": 128}, "4 waves": {"FLATQUANT_ATT_WAVES": 4},
            "8 waves": {"FLATQUANT_ATT_WAVES": 8}, "16 waves": {"FLATQUANT_ATT_WAVES": 16}}
SIZES = [((1, 2), (300, 45), 3), ((9, 4), (70, 300), 3), ((100,), (260,), 2)]      # rows, lengths, query heads a head


@pytest.fixture
def launched(tuning, request):
    for name, value in LAUNCHES[request.param].items():
        tuning(name, value)
    return request.param


def _of_sequence(c, b):
    L = c.lengths[b]
    return [f(c.table[b, :c.width], np.arange(L)) for f in (c.host[0].values, c.host[1].values, c.host[1].steps)]


@pytest.mark.parametrize("launched", LAUNCHES, indirect=True)
@pytest.mark.parametrize("scale", [1e25, 1e30, -1e30, 3.4e38, -3.4e38])
@pytest.mark.parametrize("rows,lengths,G", SIZES)
def test_the_largest_score_has_it_all(rows, lengths, G, scale, launched):
    """One value, but where scores are equal: rows of zeros get the mean of what they see.  Rows whose two largest scores lie within the rounding of a score
    of each other are not looked at."""
    print(f"[case] scale {scale}, {rows} of {lengths}, {launched}", flush=True)
    H = 2
    c = Batch(81, rows, lengths, H, 16, 4, 4).upload()
    q = c.row_tensor(H * G)
    q[::5, :D] = 0
    got = run_attention(c, q, G, scale).astype(np.float64)
    looked = 0
    for b in range(c.B):
        k, v, step = _of_sequence(c, b)
        seen = c.visible(b)
        for i in range(rows[b]):
            t, j = c.starts[b] + i, np.flatnonzero(seen[i])
            for h in range(H * G):
                y = q[t, h * D:(h + 1) * D].astype(np.float64)
                s = np.sign(scale) * (k[h // G][j] @ y)
                if y.any():
                    top = np.argsort(s)[::-1][:2]
                    # a score: 280 roundings of fp32 over its products, and 132 * 2^-18 max |q| code units (co.attention64), twice
                    off = 2 * (280 * 2.0 ** -24 * (np.abs(k[h // G][j]) @ np.abs(y)).max() * 16 + 132 * 2.0 ** -18 * np.abs(y).max())
                    if len(j) > 1 and s[top[0]] - s[top[1]] <= off:
                        continue
                    w = np.zeros(len(j))
                    w[top[0]] = 1.0
                else:
                    w = np.full(len(j), 1.0 / len(j))
                vj, sj = v[h // G][j], step[h // G][j]
                tol = co.attention_bound((w @ vj)[None], (w @ np.abs(vj))[None], np.array([w @ sj]), np.zeros(1), lengths[b])[0]
                assert np.all(np.abs(got[t, h] - w @ vj) <= tol), (t, h)
                looked += 1
    assert looked > c.starts[-1] * H * G // 2


@pytest.mark.parametrize("launched", LAUNCHES, indirect=True)
@pytest.mark.parametrize("rows,lengths,G", SIZES)
def test_queries_that_are_no_numbers_leave_the_other_rows_alone(rows, lengths, G, launched):
    print(f"[case] queries of infinity and NaN, {rows} of {lengths}, {launched}", flush=True)
    H = 2
    c = Batch(82, rows, lengths, H, 16, 4, 3).upload()
    q = c.row_tensor(H * G)
    bad = np.zeros((c.T, H * G), dtype=bool)
    for n, value in enumerate((np.inf, -np.inf, np.nan, 65504.0)):
        t, h = (n * 7) % c.T, (n * 5 + 1) % (H * G)
        q[t, h * D + 11 * n] = value
        bad[t, h] = True
    got = run_attention(c, q, G, 0.09)
    fine = np.where(np.repeat(bad, D, axis=1), np.float16(0), q)
    want, tol = c.attention(fine.reshape(c.T, H * G, D), G, 0.09)
    n = c.starts[-1]
    err = np.abs(got[:n].astype(np.float64) - want[:n])
    assert np.all(err[~bad[:n]] <= tol[:n][~bad[:n]])


@pytest.mark.parametrize("launched", LAUNCHES, indirect=True)
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("rows,lengths,G,at", [((1, 2), (300, 45), 3, (299, 43)), ((1, 2), (300, 45), 3, (100, 44)), ((9, 4), (70, 300), 3, (66, 298)), ((9, 4), (70, 300), 3, (3, 64)),
                                               ((100,), (260,), 2, (190,)), ((100,), (260,), 2, (50,))])
def test_groups_whose_step_is_no_number(rows, lengths, G, at, which, launched):
    """A key or a value that overflowed when it was written (an infinite step, zero codes): NaN for the rows of its head that see it, whether the other rows
    of the step do or not, and nothing for the others."""
    print(f"[case] {('key', 'value')[which]} {at} of {rows} of {lengths}, {launched}", flush=True)
    H = 2
    c = Batch(84, rows, lengths, H, 16, 4, 3)
    x = c.host[which]
    for b, j in enumerate(at):
        page, slot = x.place(c.table[b, :c.width], j)
        x.codes[page, 0, slot], x.params[page, 0, slot] = 0, 0x7C00
    c.upload()
    q = c.row_tensor(H * G)
    got = run_attention(c, q, G, 0.09)
    sees = np.zeros(c.T, dtype=bool)
    for b, j in enumerate(at):
        sees[c.starts[b]:c.starts[b + 1]] = c.visible(b)[:, j]
    assert sees.any() and np.isnan(got[sees][:, :G]).all()
    for x in c.host:
        x.params[(x.params & 0xFFFF) == 0x7C00] = 0                 # as zeros, for the rows that do not see them
    want, tol = c.attention(q.reshape(c.T, H * G, D), G, 0.09)
    err = np.abs(got.astype(np.float64) - want)
    assert np.all(err[:, G:] <= tol[:, G:]) and np.all(err[~sees] <= tol[~sees])


@pytest.mark.parametrize("rows,lengths,H,G,bits,window,sinks", [
    ((1, 1), (20000, 9000), 1, 4, (4, 4), 0, 0),
    ((2, 6), (9001, 17000), 1, 5, (2, 4), 0, 0),
    ((3, 1), (12000, 30), 1, 4, (3, 3), 5000, 9),
    ((40, 3), (12000, 7000), 1, 2, (4, 3), 0, 0),
    ((40, 3), (12000, 7000), 1, 2, (2, 2), 4100, 70),
])
def test_long_contexts(rows, lengths, H, G, bits, window, sinks):
    print(f"[case] {rows} of {lengths}, {H} x {G} heads, {bits} bits, window {window} + {sinks}", flush=True)
    c = Batch(83, rows, lengths, H, 64, *bits).upload()
    q = c.row_tensor(H * G, gain=2.0)
    check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, window, sinks), window=window, sinks=sinks)
    if not window and max(rows) <= 64:
        masks = c.r.integers(0, 2 ** 63, c.T).astype(np.uint64)
        check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, masks=masks), masks=masks)
