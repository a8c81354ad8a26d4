"""The paged key/value cache on the GPU: write and read bit by bit against the oracle, attention against fp64 within the bound of its
arithmetic (oracle.cache_oracle.attention_bound)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2410_09426_amd import binding as fq
from cache_util import Batch, check_attention, run_attention

pytestmark = pytest.mark.gpu
D = 128


def _dev(a):
    return torch.from_numpy(a.view(np.uint16).copy()).view(torch.float16).cuda()


def _host(t):
    return t.cpu().view(torch.int16).numpy().view(np.float16)


def _write(c, k, v, k_clip=0.95, v_clip=0.9):
    """On the device, and on the host by the oracle."""
    dk, dv = (None if x is None else _dev(x) for x in (k, v))
    fq.flatquant_cache_write(c.cache(), c.batch(), dk, 0 if k is None else k.shape[1], dv, 0 if v is None else v.shape[1], None, None, 1, k_clip, v_clip,
                             stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for b in range(c.B):
        for i in range(c.rows[b]):
            t = c.starts[b] + i
            for x, rows, clip in zip(c.host, (k, v), (k_clip, v_clip)):
                if rows is not None:
                    x.write(c.table[b, :c.width], c.lengths[b] - c.rows[b] + i, rows[t, :c.H * D].reshape(c.H, D), clip)


def _same_pages(c):
    for name, x in zip("kv", c.host):
        assert np.array_equal(c.d[name + "c"].cpu().numpy(), x.codes), f"{name} codes"
        assert np.array_equal(c.d[name + "p"].cpu().numpy().view(np.uint32), x.params), f"{name} parameters"


def _read(c, pad=(0, 0), which="kv"):
    out = [torch.full((c.T, c.H * D + p), -3.5, dtype=torch.float16, device="cuda") for p in pad]
    a, b = (o if n in which else None for o, n in zip(out, "kv"))
    fq.flatquant_cache_read(c.cache(), c.batch(), a, c.H * D + pad[0], b, c.H * D + pad[1], stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    return [_host(o) for o in out]


SHAPES = [  # rows, lengths, H, page
    ((1,), (1,), 1, 16),
    ((1,), (33,), 3, 16),
    ((1, 1, 1, 1, 1), (7, 64, 65, 128, 1), 8, 64),
    ((5, 0, 17, 1, 0), (5, 9, 100, 40, 0), 2, 32),
    ((300, 1, 77), (300, 300, 513), 5, 128),
    ((1100,), (1500,), 4, 1024),
]


@pytest.mark.parametrize("k_bits,v_bits", [(4, 4), (3, 2), (2, 3)])
@pytest.mark.parametrize("rows,lengths,H,page", SHAPES)
def test_write_and_read_bit_by_bit(rows, lengths, H, page, k_bits, v_bits):
    print(f"[case] write {rows} of {lengths}, {H} heads, pages of {page}, {k_bits}/{v_bits} bits", flush=True)
    c = Batch(11 + len(rows), rows, lengths, H, page, k_bits, v_bits, pad=3, filled=False).upload()
    k, v = c.row_tensor(H, 8), c.row_tensor(H, 0, gain=3.0)
    k[0, :D] = 0                                             # a group of zeros: step 0
    if c.T > 2:
        k[1, :D] = np.float16(6e-8)                          # a step that rounds to zero
        v[1, :D] = np.arange(D) - 3.0                        # whole numbers
        k[c.T - 4, -D - 8:-8] = 65504.0                      # one sign only, the largest number
    _write(c, k, v)
    _same_pages(c)
    pk, pv = _read(c, (0, 16))
    for x, got in zip(c.host, (pk, pv)):
        for b in range(c.B):
            n = rows[b]
            if n:
                y = x.values(c.table[b, :c.width], np.arange(lengths[b] - n, lengths[b])).transpose(1, 0, 2)
                with np.errstate(over="ignore"):
                    assert np.array_equal(got[c.starts[b]:c.starts[b] + n, :H * D].reshape(n, H, D), y.astype(np.float16))
    assert np.all(pk[c.starts[-1]:] == -3.5) and np.all(pv[c.starts[-1]:] == -3.5) and np.all(pv[:, H * D:] == -3.5)


@pytest.mark.parametrize("bits", [2, 3, 4])
def test_steps_next_to_fp16_midpoints(bits):
    """Many groups, so that some fp32 steps are fp16 midpoints that the unrounded quotient is not."""
    rows, H = 1200, 32
    print(f"[case] write {rows} rows of {H} heads, {bits} bits", flush=True)
    c = Batch(77, (rows,), (rows,), H, 64, bits, bits, filled=False).upload()
    k, v = c.row_tensor(H), c.row_tensor(H, gain=7.0)
    k[0, 0], k[0, 1:D] = -7.6796875, 2.505859375          # 0.95 * 10.185546875 / 7 is one in fp32 and just below it
    dk, dv = _dev(k), _dev(v)
    fq.flatquant_cache_write(c.cache(), c.batch(), dk, H * D, dv, H * D, None, None, 1, 0.95, 0.95, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    pos = np.arange(rows)
    for name, y in zip("kv", (k, v)):
        q, s, z = co.grid32(y.reshape(rows, H, D), 0.95, bits)
        at = (c.table[0, pos // 64], slice(None), pos % 64)
        assert np.array_equal(c.d[name + "p"].cpu().numpy().view(np.uint32)[at], co.parameters(s, z))
        assert np.array_equal(c.d[name + "c"].cpu().numpy()[at], co.pack(q, bits))


ATTEND = [  # rows, lengths, H, G, page, bits, window, sinks
    ((1,), (1,), 1, 1, 16, (4, 4), 0, 0),
    ((1,), (31,), 2, 1, 16, (4, 4), 0, 0),
    ((1,), (32,), 1, 4, 32, (4, 4), 0, 0),
    ((1,), (33,), 1, 8, 16, (3, 3), 0, 0),
    ((1, 1, 1), (129, 1, 700), 2, 4, 64, (4, 4), 0, 0),
    ((1, 1), (1500, 1027), 1, 5, 16, (2, 4), 0, 0),
    ((1, 1), (1500, 40), 3, 16, 128, (4, 2), 0, 0),
    ((1, 0, 1), (1000, 300, 900), 2, 7, 16, (3, 4), 100, 0),
    ((1, 1), (1000, 70), 2, 4, 16, (4, 3), 64, 4),
    ((3, 1), (1000, 70), 2, 4, 16, (2, 2), 33, 40),
    ((7, 2), (300, 2), 2, 4, 16, (4, 4), 0, 0),
    ((64, 5), (64, 200), 2, 1, 16, (4, 4), 0, 0),
    ((130, 33), (130, 400), 1, 3, 32, (3, 4), 0, 0),
    ((200,), (777,), 1, 2, 64, (4, 2), 90, 5),
    ((40,), (40,), 1, 32, 16, (2, 3), 1, 0),
]


LAUNCHES = {"chosen": {}, "balanced": {"FLATQUANT_ATT_WAVES": 0, "FLATQUANT_ATT_CHUNK": 128}, "balanced, few": {"FLATQUANT_ATT_WAVES": 0, "FLATQUANT_ATT_WG_PER_CU": 1},
            "4 waves": {"FLATQUANT_ATT_WAVES": 4}, "8 waves": {"FLATQUANT_ATT_WAVES": 8}, "16 waves": {"FLATQUANT_ATT_WAVES": 16}}


@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("rows,lengths,H,G,page,bits,window,sinks", ATTEND)
def test_attention(rows, lengths, H, G, page, bits, window, sinks, launch, tuning):
    for name, value in LAUNCHES[launch].items():
        tuning(name, value)
    print(f"[case] attention {rows} of {lengths}, {H} x {G} heads, pages of {page}, {bits} bits, window {window} + {sinks}", flush=True)
    c = Batch(500 + sum(lengths), rows, lengths, H, page, *bits, pad=2).upload()
    q = c.row_tensor(H * G, 8, gain=2.0)
    got = run_attention(c, q, G, 0.09, window, sinks, pad=16)
    check_attention(c, q, G, 0.09, got, window=window, sinks=sinks)


TREES = [((1,), (1,), 1, 1, 16, (4, 4)), ((13, 5), (400, 5), 2, 4, 16, (4, 4)), ((64,), (1000,), 1, 8, 64, (4, 3)), ((64, 1, 33), (64, 90, 600), 2, 2, 32, (2, 2)),
         ((9, 20), (50, 320), 2, 1, 16, (3, 4))]


@pytest.mark.parametrize("launch", LAUNCHES)
@pytest.mark.parametrize("rows,lengths,H,G,page,bits", TREES)
def test_tree_attention(rows, lengths, H, G, page, bits, launch, tuning):
    for name, value in LAUNCHES[launch].items():
        tuning(name, value)
    print(f"[case] tree {rows} of {lengths}, {H} x {G} heads", flush=True)
    c = Batch(900 + sum(lengths), rows, lengths, H, page, *bits, pad=1).upload()
    masks = np.zeros(c.T, dtype=np.uint64)
    for b in range(c.B):
        for i in range(c.rows[b]):
            up = int(masks[c.starts[b] + c.r.integers(0, i)]) if i else 0
            masks[c.starts[b] + i] = up | 1 << i
    masks[c.T - 1] = 0xFFFFFFFFFFFFFFFF
    if c.rows[0] > 4:
        masks[3] = 0                                          # sees the prefix alone, or nothing
    q = c.row_tensor(H * G)
    got = run_attention(c, q, G, 0.088, masks=masks)
    check_attention(c, q, G, 0.088, got, masks=masks)


@pytest.mark.parametrize("bits", [(4, 4), (3, 2), (2, 3)])
@pytest.mark.parametrize("rows,lengths,H,Hp,page", [((1, 1, 1), (7, 65, 1), 4, 4, 64), ((40, 0, 33, 1), (50, 3, 33, 200), 3, 1, 16), ((2500, 700), (2500, 900), 5, 5, 32)])
@pytest.mark.parametrize("few", [0, 1])
def test_write_through_matrices(rows, lengths, H, Hp, page, bits, few, tuning):
    """The codes, steps and zero points of flatquant_kv_transform_quant_bits on the same rows, in their tokens' places and nowhere else."""
    print(f"[case] write {rows} of {lengths} through {Hp} matrices, {H} heads, {bits} bits, few {few}", flush=True)
    tuning("FLATQUANT_KV_FEW", few)
    c = Batch(31, rows, lengths, H, page, *bits, pad=2, filled=False, no_page=((0, 0),)).upload()
    st = torch.cuda.current_stream()
    P = [_dev((c.r.standard_normal((Hp, D, D)) * 0.1).astype(np.float16)) for _ in "kv"]
    x = [_dev(c.row_tensor(H, 8 * n)) for n in (1, 0)]
    before = {n: c.d[n].clone() for n in ("kc", "kp", "vc", "vp")}
    fq.flatquant_cache_write(c.cache(), c.batch(), x[0], x[0].shape[1], x[1], x[1].shape[1], P[0], None, Hp, 0.95, 0.9, stream=st)
    torch.cuda.synchronize()
    half = Batch(31, rows, lengths, H, page, *bits, pad=2, filled=False, no_page=((0, 0),)).upload()      # the values' half without a matrix
    fq.flatquant_cache_write(half.cache(), half.batch(), None, 0, x[1], x[1].shape[1], None, None, 1, 0.95, 0.9, stream=st)
    assert torch.equal(half.d["vc"], c.d["vc"]) and torch.equal(half.d["vp"], c.d["vp"])
    fq.flatquant_cache_write(c.cache(), c.batch(), None, 0, x[1], x[1].shape[1], None, P[1], Hp, 0.95, 0.9, stream=st)
    for name, m, y, qb, clip in zip("kv", P, x, bits, (0.95, 0.9)):
        flat = y[:, :H * D].contiguous()
        codes = torch.empty((c.T, H, 16 * qb), dtype=torch.uint8, device="cuda")
        steps, zeros = (torch.empty((c.T, H), dtype=torch.float16, device="cuda") for _ in range(2))
        fq.flatquant_kv_transform_quant_bits(flat, m, Hp, clip, qb, c.T, H, D, codes, steps, zeros, stream=st)
        torch.cuda.synchronize()
        word = _host(steps).view(np.uint16).astype(np.uint32) | _host(zeros).astype(np.uint32) << 16
        want_c, want_p = before[name + "c"].cpu().numpy(), before[name + "p"].cpu().numpy().view(np.uint32)
        for b in range(c.B):
            for i in range(rows[b]):
                at = c.host[0].place(c.table[b, :c.width], lengths[b] - rows[b] + i)
                if at is not None:
                    want_c[at[0], :, at[1]] = codes[c.starts[b] + i].cpu().numpy()
                    want_p[at[0], :, at[1]] = word[c.starts[b] + i]
        assert np.array_equal(c.d[name + "c"].cpu().numpy(), want_c) and np.array_equal(c.d[name + "p"].cpu().numpy().view(np.uint32), want_p)


def test_groups_that_hold_no_numbers_leave_the_others_alone():
    """Infinities and NaN in a group: its step overflows or ignores them; its neighbours in the row, the wave and the page are as without."""
    c = Batch(5, (70,), (70,), 3, 16, 4, 3, filled=False).upload()
    k, v = c.row_tensor(3), c.row_tensor(3)
    print("[case] write 70 rows, some without numbers", flush=True)
    _write(c, k, v)
    _same_pages(c)
    for t, h, value in ((0, 0, np.inf), (1, 1, -np.inf), (2, 2, np.nan), (66, 0, np.nan)):
        for x in (k, v):
            x[t, h * D + 5] = value
    dk, dv = _dev(k), _dev(v)
    fq.flatquant_cache_write(c.cache(), c.batch(), dk, 3 * D, dv, 3 * D, None, None, 1, 0.95, 0.9, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for name, x in zip("kv", c.host):
        codes, params = c.d[name + "c"].cpu().numpy(), c.d[name + "p"].cpu().numpy().view(np.uint32)
        for t, h in ((0, 0), (1, 1), (2, 2), (66, 0)):
            page, slot = x.place(c.table[0, :c.width], t)
            if t < 2:                                             # a step that overflows has zero codes
                assert not codes[page, h, slot].any() and params[page, h, slot] == 0x7C00
            x.codes[page, h, slot], x.params[page, h, slot] = codes[page, h, slot], params[page, h, slot]
    _same_pages(c)


@pytest.mark.parametrize("bits", [(4, 3), (2, 4)])
def test_many_rows_are_written_like_few(bits):
    """One call of 134400 (row, head) groups and the same rows in calls of 130 rows each; keys and values alone."""
    rows, H = 4200, 32
    print(f"[case] write {rows} rows of {H} heads, {bits} bits, whole and in parts", flush=True)
    c = Batch(78, (rows,), (rows,), H, 64, *bits, filled=False).upload()
    st = torch.cuda.current_stream()
    k, v = (torch.randn((rows, H * D), device="cuda", generator=torch.Generator("cuda").manual_seed(n)).half() for n in (1, 2))
    fq.flatquant_cache_write(c.cache(), c.batch(), k, H * D, v, H * D, None, None, 1, 0.95, 0.9, stream=st)
    whole = [c.d[n].clone() for n in ("kc", "kp", "vc", "vp")]
    for alone in (True, False):
        for n in ("kc", "kp", "vc", "vp"):
            c.d[n].copy_(torch.from_numpy(c.host["kv".index(n[0])].codes if n[1] == "c" else c.host["kv".index(n[0])].params.view(np.int32)))
        if alone:
            fq.flatquant_cache_write(c.cache(), c.batch(), k, H * D, None, 0, None, None, 1, 0.95, 0.9, stream=st)
            fq.flatquant_cache_write(c.cache(), c.batch(), None, 0, v, H * D, None, None, 1, 0.95, 0.9, stream=st)
        else:
            for t in range(0, rows, 130):
                n = min(130, rows - t)
                starts, lengths = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [t + n]))
                part = fq.KvBatch(starts, lengths, c.d["table"], 1, n, c.width, c.table.shape[1], n, t + n)
                fq.flatquant_cache_write(c.cache(), part, k[t:t + n], H * D, v[t:t + n], H * D, None, None, 1, 0.95, 0.9, stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, c.d[n]) for a, n in zip(whole, ("kc", "kp", "vc", "vp"))), alone
    pos = np.arange(0, rows, 97)
    for x, y, name, clip in zip(c.host, (k, v), "kv", (0.95, 0.9)):
        q, s, z = co.grid32(_host(y).reshape(rows, H, D)[pos], clip, x.bits)
        at = (c.table[0, pos // 64], slice(None), pos % 64)
        assert np.array_equal(c.d[name + "c"].cpu().numpy()[at], co.pack(q, x.bits)) and np.array_equal(c.d[name + "p"].cpu().numpy().view(np.uint32)[at], co.parameters(s, z))
    out = torch.empty_like(k)
    fq.flatquant_cache_read(c.cache(), c.batch(), None, 0, out, H * D, stream=st)
    torch.cuda.synchronize()
    codes, params = c.d["vc"].cpu().numpy(), c.d["vp"].cpu().numpy().view(np.uint32)
    host = co.Pages(c.pages, H, 64, bits[1])
    host.codes[:], host.params[:] = codes, params
    assert np.array_equal(_host(out)[pos].reshape(-1, H, D), host.values(c.table[0, :c.width], pos).transpose(1, 0, 2).astype(np.float16))
