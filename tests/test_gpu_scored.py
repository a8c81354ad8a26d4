"""Attention over the paged cache with capped scores, slopes and prefixes (flatquant_cache_scored_attention) against fp64."""
import numpy as np
import pytest
import torch

from cache_util import D, Batch, run_attention
from oracle import step_oracle as so
from paper_2410_09426_amd import binding as fq

pytestmark = pytest.mark.gpu


def run_scored(c, q, G, scale, cap=0.0, slopes=None, prefix=None, window=0, sinks=0, masks=None, pad=0, batch=None, stream=None):
    """q: numpy [T, H G 128 + pad]; returns fp16 [T, H G, 128].  The output's padding and the rows of no sequence keep what they held."""
    cache, batch = c.cache(), batch or c.batch()
    Hq = c.H * G
    dq = torch.from_numpy(q.view(np.uint16).copy()).view(torch.float16).cuda()
    out = torch.full((c.T, Hq * D + pad), -7.25, dtype=torch.float16, device="cuda")
    size = fq.fq_cache_attention_workspace(cache, batch, Hq)
    work = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    ds = None if slopes is None else torch.from_numpy(np.asarray(slopes, dtype=np.float32)).cuda()
    dp = None if prefix is None else torch.from_numpy(np.asarray(prefix, dtype=np.int32)).cuda()
    dm = None if masks is None else torch.from_numpy(np.asarray(masks, dtype=np.uint64).view(np.int64)).cuda()
    fq.flatquant_cache_scored_attention(cache, batch, dq, q.shape[1], Hq, scale, cap, ds, dp, window, sinks, dm, out, Hq * D + pad, work, size,
                                        stream=stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool((work[size:] == 0xFF).all()), "written behind the workspace"
    got = out.cpu().view(torch.int16).numpy().view(np.float16)
    assert np.all(got[:, Hq * D:] == np.float16(-7.25)), "padding of the rows overwritten"
    assert np.all(got[c.starts[-1]:] == np.float16(-7.25)), "rows behind the last sequence overwritten"
    return got[:, :Hq * D].reshape(c.T, Hq, D)


def expect(c, q, G, scale, cap=0.0, slopes=None, prefix=None, window=0, sinks=0, masks=None, heads=None, sequences=None):
    out = np.full((c.T, c.H * G, D), np.nan)
    tol = np.ones_like(out)
    for b in range(c.B) if sequences is None else sequences:
        n, L = c.rows[b], max(0, c.lengths[b])
        if n == 0:
            continue
        k, v = (np.nan_to_num(x.values(c.table[b, :c.width], np.arange(L))) for x in c.host)
        ks, vs = (np.nan_to_num(x.steps(c.table[b, :c.width], np.arange(L))) for x in c.host)
        seen = c.visible(b, window, sinks, masks)
        if prefix is not None:
            held = np.array([c.host[0].place(c.table[b, :c.width], t) is not None for t in range(L)], dtype=bool)
            seen = seen | ((np.arange(L) < prefix[b]) & held)[None]
        t = slice(c.starts[b], c.starts[b + 1])
        pos = c.lengths[b] - n + np.arange(n)
        for h in range(c.H * G) if heads is None else heads:
            o, A, S, E = so.scored64(q[t, h], k[h // G], v[h // G], seen, scale, pos, cap, 0.0 if slopes is None else float(slopes[h]), ks[h // G], vs[h // G], c.bits[0])
            out[t, h] = o
            tol[t, h] = so.scored_bound(o, A, S, E, L, c.bits[1])
    return out, tol


def check(c, G, scale=0.09, gain=1.0, pad=0, heads=None, sequences=None, **how):
    q = c.row_tensor(c.H * G, pad=pad, gain=gain)
    got = run_scored(c, q, G, scale, pad=pad, **how)
    want, tol = expect(c, q[:, :c.H * G * D].reshape(c.T, c.H * G, D), G, scale, heads=heads, sequences=sequences, **how)
    n = c.starts[-1]
    looked = ~np.isnan(want[:n])
    assert np.all(np.isfinite(got[:n])), "not finite"
    err = np.abs(got[:n].astype(np.float64) - want[:n])[looked] / tol[:n][looked]
    worst = float(err.max()) if err.size else 0.0
    print(f"[case] worst error {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0
    return q, got


KINDS = {"cap": dict(cap=30.0), "small cap": dict(cap=0.7), "large cap": dict(cap=300.0), "slopes": dict(slopes=True), "prefix": dict(prefix=True),
         "all": dict(cap=30.0, slopes=True, prefix=True), "nothing": dict()}


def kind_of(name, c, G, seed=0):
    how = dict(KINDS[name])
    r = np.random.default_rng(seed)
    if how.get("slopes"):
        how["slopes"] = so.slopes(c.H * G)
    if how.get("prefix"):
        how["prefix"] = [int(r.integers(-2, max(1, n) + 3)) for n in c.lengths]
    return how


# a launch form each: few rows in 8 or 4 waves, 17 to 32 rows, balanced, many rows in four waves, split
SHAPES = {"one row": ([1, 1, 1, 0], [700, 33, 1, 50], 2, 4), "few": ([3, 1, 4], [300, 1, 45], 2, 4), "tile of 32": ([5, 2], [400, 90], 2, 5),
          "prompt": ([130, 31, 1], [130, 200, 5], 1, 4), "split": ([40, 9], [1500, 700], 1, 4), "mha": ([70, 1], [70, 400], 3, 1)}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", KINDS)
def test_scores_of_every_kind(shape, kind):
    rows, lengths, H, G = SHAPES[shape]
    print(f"[case] {shape} {kind}", flush=True)
    c = Batch(len(shape), rows, lengths, H, pad=2).upload()
    check(c, G, gain=3.0 if "cap" in kind else 1.0, pad=8, **kind_of(kind, c, G))


@pytest.mark.parametrize("waves", [0, 4, 8, 16])
@pytest.mark.parametrize("shape", ["one row", "few", "tile of 32", "prompt"])
def test_forced_launches(tuning, waves, shape):
    rows, lengths, H, G = SHAPES[shape]
    print(f"[case] waves={waves} {shape}", flush=True)
    tuning("FLATQUANT_ATT_WAVES", waves)
    c = Batch(31 + waves, rows, lengths, H).upload()
    check(c, G, gain=2.0, **kind_of("all", c, G, waves))


@pytest.mark.parametrize("k_bits", [2, 3, 4])
@pytest.mark.parametrize("v_bits", [2, 3, 4])
@pytest.mark.parametrize("shape", ["one row", "prompt"])
def test_code_widths(k_bits, v_bits, shape):
    rows, lengths, H, G = SHAPES[shape]
    print(f"[case] bits {k_bits} {v_bits} {shape}", flush=True)
    c = Batch(k_bits * 8 + v_bits, rows, lengths, H, k_bits=k_bits, v_bits=v_bits).upload()
    check(c, G, gain=2.0, **kind_of("all", c, G))


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (64, 1), (100, 200), (5000, 2)])
@pytest.mark.parametrize("shape", ["one row", "few", "prompt", "split"])
def test_windows_with_prefixes(window, sinks, shape):
    rows, lengths, H, G = SHAPES[shape]
    print(f"[case] window={window} sinks={sinks} {shape}", flush=True)
    c = Batch(window + sinks, rows, lengths, H).upload()
    check(c, G, window=window, sinks=sinks, **kind_of("all", c, G, window))


@pytest.mark.parametrize("page", [16, 32, 128])
def test_pages(page):
    print(f"[case] page={page}", flush=True)
    c = Batch(page, [2, 90, 1], [333, 150, 17], 2, page=page, no_page=[(0, 1), (1, 0)]).upload()
    check(c, 4, **kind_of("all", c, 4))


@pytest.mark.parametrize("rows,H,G", [([13, 1, 5], 2, 4), ([64, 30], 1, 8), ([2, 3], 2, 2)])
def test_trees_with_a_cap(rows, H, G):
    print(f"[case] tree {rows}", flush=True)
    c = Batch(sum(rows), rows, [n + 200 - 30 * k for k, n in enumerate(rows)], H).upload()
    masks = [int(c.r.integers(0, 2 ** 63)) for _ in range(c.T)]
    check(c, G, gain=3.0, cap=20.0, masks=masks)


def test_rows_that_see_nothing():
    """Lengths below the rows' number: rows of negative positions see the prefix alone, or nothing and get zeros."""
    print("[case] nothing seen", flush=True)
    c = Batch(3, [6, 4, 3], [3, 0, -5], 2).upload()
    _, got = check(c, 2, cap=5.0, slopes=so.slopes(4))
    assert not got[:3].any() and got[3:6].any() and not got[6:13].any()
    _, got = check(c, 2, cap=5.0, slopes=so.slopes(4), prefix=[2, 9, 4])
    assert got[:6].any(axis=(1, 2)).all() and not got[6:13].any()


def test_plain_scores_are_those_of_the_plain_call():
    """No cap, no slopes, no prefix: the same bits; a prefix of nothing: weights within a rounding of the factor."""
    print("[case] plain", flush=True)
    for shape in ("one row", "tile of 32", "prompt", "split"):
        rows, lengths, H, G = SHAPES[shape]
        c = Batch(77, rows, lengths, H).upload()
        q, got = check(c, G)
        plain = run_attention(c, q, G, 0.09)
        assert np.array_equal(got, plain)
        got, n = run_scored(c, q, G, 0.09, prefix=[0] * c.B), c.starts[-1]
        assert np.abs(got[:n].astype(float) - plain[:n]).max() <= 2.0 ** -9 * np.abs(plain[:n].astype(float)).max()


def test_what_a_row_does_not_see_does_not_change_it():
    """Steps that are infinities and NaN of both signs, wherever no row of the prefix's sequence sees a token; a NaN step that is seen makes its rows NaN."""
    print("[case] hidden", flush=True)
    rows, lengths, H, G = [2, 40], [300, 200], 2, 4
    for window, prefix in ((50, [20, 0]), (30, [0, 64])):
        clean, dirty = (Batch(5, rows, lengths, H) for _ in range(2))
        for b in range(2):
            first = lengths[b] - rows[b] - window + 1
            for j in range(lengths[b]):
                if prefix[b] <= j < first:
                    p, s = int(dirty.table[b, j // 16]), j % 16
                    for x, w in zip(dirty.host, (0x7C00, 0xFC00, 0x7E00)[j % 3:] + (0x7C00,)):
                        x.params[p, :, s] = w | 0x000F0000
        how = dict(cap=10.0, slopes=so.slopes(H * G), prefix=prefix, window=window)
        q = clean.row_tensor(H * G)
        a, b = (run_scored(c.upload(), q, G, 0.09, **how) for c in (clean, dirty))
        assert np.array_equal(a, b)
    for which, word in ((0, 0x7C00), (0, 0x7E00), (1, 0x7C00), (1, 0xFC00)):
        c = Batch(6, rows, lengths, H)
        p = int(c.table[0, 100 // 16])
        c.host[which].params[p, 1, 100 % 16] = word | 0x00030000
        got = run_scored(c.upload(), c.row_tensor(H * G), G, 0.09, cap=10.0)
        assert np.isnan(got[:2, G:]).all() and np.isfinite(got[:2, :G]).all() and np.isfinite(got[2:42]).all()


@pytest.mark.parametrize("scale", [1e-30, 1.0, 1e4, 1e30, -1.0, 0.0])
def test_scales_of_all_sizes(scale):
    """Saturated caps share the weight among all tokens on the cap's side."""
    print(f"[case] scale={scale}", flush=True)
    c = Batch(8, [2, 40], [200, 90], 1).upload()
    check(c, 4, scale=scale, cap=12.0) if abs(scale) <= 1 else run_and_compare_signs(c, scale)


def run_and_compare_signs(c, scale):
    q = c.row_tensor(4)
    got = run_scored(c, q, 4, scale, cap=3.0)
    for b in range(2):
        L = c.lengths[b]
        k, v = (x.values(c.table[b, :c.width], np.arange(L))[0] for x in c.host)
        for t in range(c.starts[b], c.starts[b + 1]):
            n = c.lengths[b] - c.starts[b + 1] + t + 1
            for h in range(4):
                dot = k[:n] @ q[t, h * D:(h + 1) * D].astype(np.float64)
                w = np.where(np.abs(dot) * scale > 100, np.exp(3.0 * np.sign(dot)), np.nan)
                if not np.isnan(w).any():
                    want = w @ v[:n] / w.sum()
                    assert np.abs(got[t, h] - want).max() <= 2.0 ** -8 * np.abs(v).max()


@pytest.mark.parametrize("cap", [1e-30, 1e-5, 63.0, 65.0, 1e6, 3e38])
def test_caps_of_all_sizes(cap):
    print(f"[case] cap={cap}", flush=True)
    c = Batch(9, [2, 40], [200, 90], 1).upload()
    check(c, 4, gain=4.0, cap=cap)


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_steep_slopes(sign):
    """Far tokens without weight, or near ones."""
    print(f"[case] steep {sign}", flush=True)
    c = Batch(10, [3, 50], [900, 300], 1).upload()
    check(c, 4, slopes=[sign * 0.5, sign * 4.0, sign * 100.0, 0.0])
    got = run_scored(c, c.row_tensor(4), 4, 0.09, slopes=[3e38, -3e38, 1e20, -1e20])
    assert np.isfinite(got).all()


def test_long_axes():
    print("[case] long", flush=True)
    c = Batch(11, [1, 1, 20], [9000, 500, 7000], 2, page=64).upload()
    check(c, 4, heads=[0, 5], slopes=so.slopes(8), cap=40.0, gain=2.0)


def test_hints_that_are_wrong():
    print("[case] hints", flush=True)
    c = Batch(12, [40, 3], [500, 700], 2).upload()
    how = kind_of("all", c, 4)
    q = c.row_tensor(8)
    want, tol = expect(c, q.reshape(c.T, 8, D), 4, 0.09, **how)
    for rows, length in ((0, 0), (1, 100), (40, 0), (3, 10 ** 6), (10 ** 6, 10 ** 9)):
        got = run_scored(c, q, 4, 0.09, batch=c.batch(max_rows=rows, max_length=length), **how)
        assert (np.abs(got - want) / tol).max() <= 1, (rows, length)


@pytest.mark.parametrize("B,H,G,length", [(20, 8, 2, 300), (70, 8, 4, 200), (300, 2, 8, 90)])
def test_launches_of_many_pairs(B, H, G, length):
    """160 to 600 pairs, more sequences than the balanced launch holds; some sequences and heads against fp64."""
    print(f"[case] pairs {B} x {H}", flush=True)
    r = np.random.default_rng(B)
    c = Batch(B, [1] * B, [int(n) for n in r.integers(1, length, B)], H, k_bits=3, v_bits=4).upload()
    check(c, G, heads=[0, H * G - 1], sequences=sorted(set(r.integers(0, B, 12).tolist())), **kind_of("all", c, G))


def test_trees_without_a_cap_are_those_of_the_tree_call():
    print("[case] plain tree", flush=True)
    c = Batch(17, [13, 1, 30], [300, 40, 90], 2).upload()
    masks = [int(c.r.integers(0, 2 ** 63)) for _ in range(c.T)]
    q = c.row_tensor(8)
    assert np.array_equal(run_scored(c, q, 4, 0.09, masks=masks), run_attention(c, q, 4, 0.09, masks=masks))
