"""The operators of the paged key/value cache as they are used together: prompts, decode steps in a replayed graph, drafted tokens, other
streams, and what a batch may hold besides ordinary sequences."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2410_09426_amd import binding as fq
from cache_util import D, Batch, check_attention, run_attention

pytestmark = pytest.mark.gpu
LAUNCHES = {"chosen": {}, "balanced": {"FLATQUANT_ATT_WAVES": 0}, "4 waves": {"FLATQUANT_ATT_WAVES": 4}, "8 waves": {"FLATQUANT_ATT_WAVES": 8}}


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.uint16).copy()).view(torch.float16).cuda()


def _set(c, rows, lengths):
    """Other rows and lengths on the same pages."""
    c.rows, c.lengths = list(rows), list(lengths)
    c.starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    c.T = int(c.starts[-1])
    c.d["starts"], c.d["lengths"] = torch.from_numpy(c.starts).cuda(), torch.tensor(c.lengths, dtype=torch.int32, device="cuda")


def _write(c, k, v, batch=None, stream=None):
    """On the device and on the host by the oracle."""
    fq.flatquant_cache_write(c.cache(), batch or c.batch(), _dev(k), k.shape[1], _dev(v), v.shape[1], None, None, 1, 0.95, 0.95,
                             stream=stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    for b in range(c.B):
        for i in range(c.rows[b]):
            for x, rows in zip(c.host, (k, v)):
                x.write(c.table[b, :c.width], c.lengths[b] - c.rows[b] + i, rows[c.starts[b] + i, :c.H * D].reshape(c.H, D), 0.95)


def _same_pages(c):
    for name, x in zip("kv", c.host):
        assert np.array_equal(c.d[name + "c"].cpu().numpy(), x.codes) and np.array_equal(c.d[name + "p"].cpu().numpy().view(np.uint32), x.params), name


@pytest.mark.parametrize("H,G,bits,window,sinks", [(2, 4, (4, 4), 0, 0), (3, 1, (4, 3), 40, 4)])
def test_prompts_then_decode_in_a_graph_then_drafts(H, G, bits, window, sinks):
    """Ragged prompts; decode steps of all sequences, write and attention in one graph that is replayed as lengths grow over page ends; a tree of
    drafted tokens, part of which is kept; all of it read back."""
    B, steps, prompts = 5, 6, [30, 1, 129, 64, 77]
    c = Batch(60, [0] * B, [n + 24 for n in prompts], H, 16, *bits, filled=False).upload()
    Hq, st = H * G, torch.cuda.current_stream()
    _set(c, prompts, prompts)
    print(f"[case] prompts {prompts}, {H} x {G} heads", flush=True)
    k, v, q = c.row_tensor(H), c.row_tensor(H), c.row_tensor(Hq)
    _write(c, k, v)
    check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, window, sinks), window=window, sinks=sinks)

    # decode: the graph's tensors stay, their contents change
    _set(c, [1] * B, [n + 1 for n in prompts])
    gk, gv = (torch.zeros((B, H * D), dtype=torch.float16, device="cuda") for _ in range(2))
    gq, gout = (torch.zeros((B, Hq * D), dtype=torch.float16, device="cuda") for _ in range(2))
    cache = c.cache()
    batch = fq.KvBatch(c.d["starts"], c.d["lengths"], c.d["table"], B, B, c.width, c.table.shape[1], 1, max(prompts) + 24)
    size = fq.fq_cache_attention_workspace(cache, batch, Hq)
    work = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

    def step(stream):
        fq.flatquant_cache_write(cache, batch, gk, H * D, gv, H * D, None, None, 1, 0.95, 0.95, stream=stream)
        fq.flatquant_cache_attention(cache, batch, gq, Hq * D, Hq, 0.09, window, sinks, gout, Hq * D, work, size, stream=stream)

    saved = [c.d[n].clone() for n in ("kc", "kp", "vc", "vp")]
    side = torch.cuda.Stream()
    side.wait_stream(st)
    with torch.cuda.stream(side):
        step(side)                                               # warm-up, undone below
    st.wait_stream(side)
    for n, x in zip(("kc", "kp", "vc", "vp"), saved):
        c.d[n].copy_(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    for s in range(steps):
        print(f"[case] decode step {s}", flush=True)
        c.lengths = [n + 1 + s for n in prompts]
        c.d["lengths"].copy_(torch.tensor(c.lengths, dtype=torch.int32))
        k, v, q = c.row_tensor(H), c.row_tensor(H), c.row_tensor(Hq)
        for dst, src in ((gk, k), (gv, v), (gq, q)):
            dst.copy_(_dev(src))
        gout.fill_(-3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = gout.cpu()
        _write(c, k, v)                                          # eagerly, the same again
        _same_pages(c)
        eager = run_attention(c, q, G, 0.09, window, sinks, batch=batch)
        assert np.array_equal(got.view(torch.int16).numpy().view(np.float16).reshape(B, Hq, D), eager)
        check_attention(c, q, G, 0.09, eager, window=window, sinks=sinks)

    # drafted tokens: chains of two from a root
    n = 7
    at = list(c.lengths)
    _set(c, [n, 0, n, n, 1], [a + m for a, m in zip(at, (n, 0, n, n, 1))])
    masks = np.zeros(c.T, dtype=np.uint64)
    for b in range(B):
        for i in range(c.rows[b]):
            masks[c.starts[b] + i] = 1 | 1 << i | (1 << (i - 1) if i and i % 2 == 0 else 0)
    k, v, q = c.row_tensor(H), c.row_tensor(H), c.row_tensor(Hq)
    _write(c, k, v)
    check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, masks=masks), masks=masks)

    # the first two are kept: everything held is read back, and a later token takes a dropped one's place
    kept = [a + min(2, m) for a, m in zip(at, c.rows)]
    _set(c, [1] * B, [a + 1 for a in kept])
    k, v, q = c.row_tensor(H), c.row_tensor(H), c.row_tensor(Hq)
    _write(c, k, v)
    check_attention(c, q, G, 0.09, run_attention(c, q, G, 0.09, window, sinks), window=window, sinks=sinks)
    _set(c, [a + 1 for a in kept], [a + 1 for a in kept])
    rk, rv = (torch.empty((c.T, H * D), dtype=torch.float16, device="cuda") for _ in range(2))
    fq.flatquant_cache_read(cache, c.batch(), rk, H * D, rv, H * D, stream=st)
    torch.cuda.synchronize()
    for x, got in zip(c.host, (rk, rv)):
        got = got.cpu().view(torch.int16).numpy().view(np.float16)
        for b in range(B):
            y = x.values(c.table[b, :c.width], np.arange(c.lengths[b])).transpose(1, 0, 2).reshape(-1, H * D)
            assert np.array_equal(got[c.starts[b]:c.starts[b + 1]], y.astype(np.float16))


@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("rows,lengths", [((1, 1), (900, 20)), ((20, 1), (300, 700)), ((150, 3), (500, 3))])
def test_hints_do_not_change_results(rows, lengths, launch, tuning):
    """max_rows and max_length too small, too large and zero."""
    for name, value in LAUNCHES[launch].items():
        tuning(name, value)
    c = Batch(71, rows, lengths, 2, 16, 4, 4).upload()
    q = c.row_tensor(4)
    masks = c.r.integers(0, 2 ** 63, c.T).astype(np.uint64)
    for max_rows, max_length in ((0, 0), (1, 1), (8, 10 ** 6), (40, 64), (10 ** 6, 300), (0, 2 ** 40)):
        print(f"[case] {rows} of {lengths} as at most {max_rows} of {max_length}", flush=True)
        hints = c.batch(max_rows, max_length)
        check_attention(c, q, 2, 0.1, run_attention(c, q, 2, 0.1, batch=hints))
        check_attention(c, q, 2, 0.1, run_attention(c, q, 2, 0.1, 50, 7, batch=hints), window=50, sinks=7)
        if max_rows <= 64:
            check_attention(c, q, 2, 0.1, run_attention(c, q, 2, 0.1, masks=masks, batch=hints), masks=masks)


@pytest.mark.parametrize("launch", LAUNCHES)
def test_rows_and_tokens_without_a_place(launch, tuning):
    """Rows at negative positions, sequences of no length, pages that are none, lengths behind the table: nothing is written or seen there, zeros are
    read, and a row that sees nothing has zeros."""
    for name, value in LAUNCHES[launch].items():
        tuning(name, value)
    rows, lengths = (5, 3, 1, 40, 1, 2), (2, 0, 70, 100, 33, 40)
    c = Batch(72, rows, lengths, 2, 16, 3, 4, no_page=((2, 1), (2, 4), (3, 0), (3, 6), (5, 0), (5, 1), (5, 2)), pad=2, extra_width=0).upload()
    print(f"[case] {rows} of {lengths}", flush=True)
    q = c.row_tensor(4, 8)
    for how in ({}, {"window": 20, "sinks": 3}, {"masks": np.full(c.T, 0b1011, dtype=np.uint64)}):
        got = run_attention(c, q, 2, 0.1, pad=8, **how)
        check_attention(c, q, 2, 0.1, got, **how)
        assert not got[c.starts[5]:c.starts[6]].any()
        assert "masks" in how or not got[:3].any()               # (in the tree bit 3 is the token at position 0)
    # a table that is narrower than the lengths, and one of no width
    for width in (2, 0):
        narrow = fq.KvBatch(c.d["starts"], c.d["lengths"], c.d["table"], c.B, c.T, width, c.table.shape[1], max(rows), max(lengths))
        old, c.width = c.width, width
        got = run_attention(c, q, 2, 0.1, batch=narrow)
        check_attention(c, q, 2, 0.1, got)
        c.width = old
        if width == 0:
            assert not got[:c.starts[-1]].any()
    k, v = c.row_tensor(2), c.row_tensor(2)
    _write(c, k, v)
    _same_pages(c)
    out = torch.full((c.T, 2 * D), 9.0, dtype=torch.float16, device="cuda")
    fq.flatquant_cache_read(c.cache(), c.batch(), out, 2 * D, None, 0, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    out = out.cpu().numpy().reshape(c.T, 2, D)
    for b in range(c.B):
        for i in range(rows[b]):
            pos = lengths[b] - rows[b] + i
            held = c.host[0].place(c.table[b, :c.width], pos) is not None
            want = c.host[0].values(c.table[b, :c.width], np.array([pos]))[:, 0] if held else np.zeros((2, D))
            assert np.array_equal(out[c.starts[b] + i], want.astype(np.float16)), (b, i)
    assert np.all(out[c.starts[-1]:] == 9.0)


@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("scale,q_gain,k_gain,v_gain", [(0.0, 1.0, 1.0, 1.0), (-0.1, 1.0, 1.0, 1.0), (0.09, 40.0, 20.0, 1.0), (1e-5, 1.0, 1.0, 1e-4), (0.09, 1e-3, 1.0, 3000.0),
                                                     (1e30, 1.0, 1.0, 1.0)])
def test_scales_and_magnitudes(scale, q_gain, k_gain, v_gain, launch, tuning):
    for name, value in LAUNCHES[launch].items():
        tuning(name, value)
    for rows, lengths in (((1, 2), (300, 45)), ((100,), (260,))):
        print(f"[case] scale {scale}, gains {q_gain} {k_gain} {v_gain}, {rows} of {lengths}", flush=True)
        c = Batch(73, rows, lengths, 2, 16, 4, 4, k_gain=k_gain, v_gain=v_gain).upload()
        q = c.row_tensor(4, gain=q_gain)
        q[0, :D] = 0
        got = run_attention(c, q, 2, scale)
        if scale < 1e10:
            check_attention(c, q, 2, scale, got)
        else:                                                    # the largest score has it all
            assert np.all(np.isfinite(got[:c.starts[-1]]))


def test_many_sequences_and_streams():
    """More sequences than the balanced launch holds, and two calls at the same time on streams of their own."""
    rows, lengths = [1] * 300, [1 + 7 * b % 200 for b in range(300)]
    c = Batch(74, rows, lengths, 2, 16, 4, 2).upload()
    q = [c.row_tensor(8), c.row_tensor(8)]
    want = [run_attention(c, x, 4, 0.1) for x in q]
    check_attention(c, q[0], 4, 0.1, want[0])
    few = Batch(75, [1, 3], [3000, 2000], 2, 16, 4, 4).upload()
    q2 = [few.row_tensor(4), few.row_tensor(4)]
    want2 = [run_attention(few, x, 2, 0.1) for x in q2]
    check_attention(few, q2[0], 2, 0.1, want2[0])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    size = fq.fq_cache_attention_workspace(few.cache(), few.batch(), 4)
    assert size > 0
    cache, batch = few.cache(), few.batch()
    work = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in streams]
    dq = [_dev(x) for x in q2]
    outs = [[torch.empty((few.T, 4 * D), dtype=torch.float16, device="cuda") for _ in range(8)] for _ in streams]
    torch.cuda.synchronize()
    for k in range(8):
        for s, w, x, out in zip(streams, work, dq, outs):
            fq.flatquant_cache_attention(cache, batch, x, 4 * D, 4, 0.1, 0, 0, out[k], 4 * D, w, size, stream=s)
    torch.cuda.synchronize()
    for out, w in zip(outs, want2):
        for o in out:
            assert np.array_equal(o.cpu().view(torch.int16).numpy().view(np.float16).reshape(few.T, 4, D), w)


def test_offsets_beyond_32_bits():
    """Pages whose codes and parameters lie more than 2^32 bytes into their arrays, rows far apart."""
    H, page, pages = 8, 128, 1100000 // 8
    c = Batch(76, [3, 130], [400, 200], H, page, 4, 4, filled=True)
    c.upload()
    print(f"[case] {pages} pages of {page} tokens of {H} heads", flush=True)
    shift = pages - c.pages
    big = {}
    for n in ("kc", "kp", "vc", "vp"):
        big[n] = torch.zeros((pages, *c.d[n].shape[1:]), dtype=c.d[n].dtype, device="cuda")
        big[n][shift:] = c.d[n]
    assert big["kc"].numel() > 2 ** 33
    table = torch.from_numpy(np.where((c.table >= 0) & (c.table < c.pages), c.table + shift, c.table).astype(np.int32)).cuda()
    cache = fq.KvCache(big["kc"], big["kp"], big["vc"], big["vp"], pages, page, H, 4, 4)
    batch = fq.KvBatch(c.d["starts"], c.d["lengths"], table, c.B, c.T, c.width, c.table.shape[1], 130, 400)
    st, far = torch.cuda.current_stream(), 2 ** 25              # T * far halves: 2^33 bytes and more
    rows = torch.zeros((c.T, far), dtype=torch.float16, device="cuda")
    k = c.row_tensor(H)
    rows[:, :H * D] = _dev(k)
    fq.flatquant_cache_write(cache, batch, rows, far, rows, far, None, None, 1, 0.95, 0.95, stream=st)
    torch.cuda.synchronize()
    for b in range(c.B):
        for i in range(c.rows[b]):
            for x in c.host:
                x.write(c.table[b, :c.width], c.lengths[b] - c.rows[b] + i, k[c.starts[b] + i].reshape(H, D), 0.95)
    for n, x in zip("kv", c.host):
        assert np.array_equal(big[n + "c"][shift:].cpu().numpy(), x.codes) and np.array_equal(big[n + "p"][shift:].cpu().numpy().view(np.uint32), x.params)
    q = c.row_tensor(H)
    rows[:, :H * D] = _dev(q)
    size = fq.fq_cache_attention_workspace(cache, batch, H)
    work = torch.empty(max(16, size), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(rows)
    fq.flatquant_cache_attention(cache, batch, rows, far, H, 0.09, 0, 0, out, far, work, size, stream=st)
    torch.cuda.synchronize()
    check_attention(c, q, 1, 0.09, out[:, :H * D].cpu().view(torch.int16).numpy().view(np.float16).reshape(c.T, H, D))
    assert not bool(out[:, H * D:2 * H * D].any())
