"""The calls of a step around the paged key/value cache without a GPU: refusals that return before a device is touched, marshalling, the turns of
frequencies, and the oracle's own pins."""
import ctypes
import importlib
import inspect

import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import step_oracle as so
from paper_2410_09426_amd import binding as fq

A = 0x10000000          # addresses that are never followed
FAR = A + 0x10000000
CACHE = dict(k_codes=A, k_params=A + 0x1000000, v_codes=A + 0x2000000, v_params=A + 0x3000000, pages=8, page_tokens=16, H=4, k_bits=4, v_bits=3)
BATCH = dict(row_starts=A + 0x4000000, lengths=A + 0x4001000, page_table=A + 0x4002000, B=2, T=0, table_width=4, table_stride=4, max_rows=1, max_length=64)
POOL = dict(ring=A + 0x5000000, state=A + 0x5100000, next=A + 0x5200000, capacity=8)


def _advance(batch=None, pool=None, **k):
    return fq.flatquant_cache_advance(**{**dict(batch=fq.KvBatch(**{**BATCH, "T": 5, **(batch or {})}), pool=fq.PagePool(**{**POOL, **(pool or {})}), page_tokens=16,
                                                pages=8, held=FAR, keep=FAR + 0x1000, rows=FAR + 0x2000, positions=FAR + 0x3000, slots=FAR + 0x4000,
                                                check=False), **k})


ROPE = dict(q=FAR, q_stride=1024, Hq=8, k=FAR + 0x100000, k_stride=512, H=4, T=5, positions=FAR + 0x200000, turns=FAR + 0x210000, rotary=128, interleaved=0,
            w_q=FAR + 0x220000, w_k=FAR + 0x221000, eps=1e-6, P_q=FAR + 0x300000, P_k=FAR + 0x400000, per_head=0, q_out=FAR + 0x500000, q_out_stride=1024,
            k_out=FAR + 0x600000, k_out_stride=512)


def _rope(**k):
    return fq.flatquant_head_rope(**{**ROPE, "check": False, **k})


def _scored(cache=None, batch=None, **k):
    return fq.flatquant_cache_scored_attention(**{**dict(cache=fq.KvCache(**{**CACHE, **(cache or {})}), batch=fq.KvBatch(**{**BATCH, "T": 3, **(batch or {})}), q=FAR,
                                                         q_stride=1024, Hq=8, scale=0.1, cap=30.0, slopes=FAR + 0x200000, prefix=FAR + 0x201000, window=0, sinks=0,
                                                         visible=None, out=FAR + 0x100000, out_stride=1024, workspace=None, workspace_bytes=0, check=False), **k})


def test_advance_refuses():
    # what is refused is refused before the alignment, which every call here gets wrong at the end
    wrong = dict(rows=FAR + 0x2001)
    assert _advance(**wrong) == fq.FQ_MISALIGNED
    assert _advance(batch=dict(B=0)) == fq.FQ_OK
    for bad in (dict(batch=dict(B=-1)), dict(batch=dict(T=-1)), dict(batch=dict(table_width=-1)), dict(batch=dict(table_stride=3)), dict(pool=dict(capacity=0)),
                dict(page_tokens=0), dict(pages=0), dict(held=None), dict(keep=None), dict(rows=None), dict(pool=dict(ring=None)), dict(pool=dict(state=None)),
                dict(pool=dict(next=None)), dict(batch=dict(row_starts=None)), dict(batch=dict(lengths=None)), dict(batch=dict(page_table=None))):
        assert _advance(**{**wrong, **bad}) == fq.FQ_INVALID_ARG, bad
    assert fq.flatquant_cache_advance(None, fq.PagePool(**POOL), 16, 8, FAR, FAR, FAR, None, None, check=False) == fq.FQ_INVALID_ARG
    assert fq.flatquant_cache_advance(fq.KvBatch(**BATCH), None, 16, 8, FAR, FAR, FAR, None, None, check=False) == fq.FQ_INVALID_ARG
    for bad in (dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048), dict(pages=2 ** 31), dict(pool=dict(capacity=2 ** 31)), dict(batch=dict(T=2 ** 29 + 1)),
                dict(batch=dict(B=2 ** 24)), dict(batch=dict(table_width=2 ** 20 + 1, table_stride=2 ** 21)), dict(batch=dict(table_stride=2 ** 48))):
        assert _advance(**{**wrong, **bad}) == fq.FQ_UNSUPPORTED_SHAPE, bad
    for bad in (dict(held=FAR + 2), dict(keep=FAR + 0x1001), dict(positions=FAR + 0x3002), dict(slots=FAR + 0x4004), dict(pool=dict(ring=A + 0x5000001)),
                dict(pool=dict(state=A + 0x5100004)), dict(pool=dict(next=A + 0x5200004)), dict(batch=dict(lengths=A + 0x4001002)),
                dict(batch=dict(row_starts=A + 0x4000001)), dict(batch=dict(page_table=A + 0x4002001))):
        assert _advance(**bad) == fq.FQ_MISALIGNED, bad
    for bad in (dict(positions=FAR), dict(slots=FAR), dict(slots=FAR + 0x1000), dict(positions=FAR + 0x2004), dict(held=A + 0x4000000), dict(rows=A + 0x4001000),
                dict(held=A + 0x4001004), dict(keep=A + 0x5000000), dict(positions=A + 0x4002010), dict(slots=FAR + 0x3000), dict(pool=dict(next=A + 0x5000008)),
                dict(pool=dict(next=A + 0x5100008)), dict(batch=dict(lengths=A + 0x4000008)), dict(rows=A + 0x4002004)):
        assert _advance(**bad) == fq.FQ_INVALID_ARG, bad


def test_rope_refuses():
    wrong = dict(turns=FAR + 0x210008)
    assert _rope(**wrong) == fq.FQ_MISALIGNED
    assert _rope(T=0) == fq.FQ_OK and _rope(q=None, k=None) == fq.FQ_OK
    assert _rope(T=0, q=None, Hq=-5, k=None) == fq.FQ_OK
    for bad in (dict(T=-1), dict(rotary=-32), dict(interleaved=2), dict(per_head=-1), dict(Hq=0), dict(H=-1), dict(q_stride=1016), dict(k_stride=504),
                dict(q_out_stride=1016), dict(k_out_stride=511), dict(eps=0.0), dict(eps=1e-40), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_out=None),
                dict(k_out=None), dict(positions=None), dict(turns=None)):
        assert _rope(**{**wrong, **bad}) == fq.FQ_INVALID_ARG, bad
    for bad in (dict(rotary=16), dict(rotary=100), dict(rotary=160), dict(T=2 ** 29 + 1), dict(Hq=65536, q_stride=2 ** 23, q_out_stride=2 ** 23),
                dict(H=32768, per_head=1, k_stride=2 ** 22, k_out_stride=2 ** 22), dict(q_stride=2 ** 48), dict(k_out_stride=2 ** 41),
                dict(T=2 ** 28, Hq=8)):
        assert _rope(**{**wrong, **bad}) == fq.FQ_UNSUPPORTED_SHAPE, bad
    for name in ("q", "k", "w_q", "w_k", "P_q", "P_k", "q_out", "k_out"):
        assert _rope(**{name: ROPE[name] + 8}) == fq.FQ_MISALIGNED, name
    for bad in (dict(q_stride=1028), dict(k_stride=514), dict(q_out_stride=1025), dict(k_out_stride=516), dict(positions=FAR + 0x200002)):
        assert _rope(**bad) == fq.FQ_MISALIGNED, bad
    # outputs overlap nothing
    for bad in (dict(q_out=FAR), dict(k_out=FAR), dict(k_out=FAR + 0x100000), dict(q_out=FAR + 0x200000), dict(q_out=FAR + 0x210000), dict(k_out=FAR + 0x220000),
                dict(q_out=FAR + 0x300000), dict(k_out=FAR + 0x400000), dict(k_out=FAR + 0x500000), dict(q_out=FAR + 0x221000),
                dict(P_q=FAR + 0x500000 - 0x9000, per_head=1)):
        assert _rope(**bad) == fq.FQ_INVALID_ARG, bad
    # what is left out is not looked at
    assert _rope(q=None, Hq=0, q_stride=3, q_out=None, w_q=1, P_q=2, **wrong) == fq.FQ_MISALIGNED
    assert _rope(w_q=None, w_k=None, eps=-1.0, **wrong) == fq.FQ_MISALIGNED
    assert _rope(rotary=0, turns=None, positions=FAR + 0x200002) == fq.FQ_MISALIGNED


def test_scored_attention_refuses():
    wrong = dict(q=FAR + 8)
    work = dict(workspace=FAR + 0x800000, workspace_bytes=1 << 40)
    assert _scored(**wrong, **work) == fq.FQ_MISALIGNED
    assert _scored(batch=dict(T=0)) == fq.FQ_OK and _scored(batch=dict(B=0)) == fq.FQ_OK
    for bad in (dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(scale=float("inf")), dict(window=-1), dict(sinks=-1), dict(Hq=6), dict(q_stride=1016),
                dict(visible=FAR + 0x300000), dict(visible=FAR + 0x300000, slopes=None), dict(visible=FAR + 0x300000, prefix=None),
                dict(visible=FAR + 0x300000, prefix=None, slopes=None, window=3), dict(visible=FAR + 0x300000, prefix=None, slopes=None, sinks=3),
                dict(cache=dict(pages=0)), dict(batch=dict(B=-1)), dict(out=None), dict(workspace_bytes=-1)):
        assert _scored(**{**wrong, **work, **bad}) == fq.FQ_INVALID_ARG, bad
    assert _scored(visible=FAR + 0x300000, slopes=None, prefix=None, **wrong, **work) == fq.FQ_MISALIGNED
    assert _scored(batch=dict(max_rows=65), visible=FAR + 0x300000, slopes=None, prefix=None, **work) == fq.FQ_UNSUPPORTED_SHAPE
    for bad in (dict(slopes=FAR + 0x200002), dict(prefix=FAR + 0x201001), dict(visible=FAR + 0x300004, slopes=None, prefix=None), dict(out=FAR + 0x100008)):
        assert _scored(**{**work, **bad}) == fq.FQ_MISALIGNED, bad
    long = dict(batch=dict(T=16, max_rows=8, max_length=4000, table_width=256, table_stride=256))      # rows that need a workspace
    assert fq.fq_cache_attention_workspace(fq.KvCache(**CACHE), fq.KvBatch(**{**BATCH, **long["batch"]}), 8) > 4096
    for bad in (dict(slopes=FAR + 0x100010), dict(prefix=FAR + 0x100004), dict(slopes=FAR + 0x800000), dict(prefix=FAR + 0x800004), dict(out=FAR)):
        assert _scored(**{**work, **long, **bad}) == fq.FQ_INVALID_ARG, bad
    assert fq.flatquant_cache_scored_attention(None, fq.KvBatch(**{**BATCH, "T": 3}), FAR, 1024, 8, 0.1, 0.0, None, None, 0, 0, None, FAR, 1024, None, 0,
                                               check=False) == fq.FQ_INVALID_ARG
    assert fq.flatquant_cache_scored_attention(fq.KvCache(**CACHE), None, FAR, 1024, 8, 0.1, 0.0, None, None, 0, 0, None, FAR, 1024, None, 0,
                                               check=False) == fq.FQ_INVALID_ARG


class _Buffer:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


class _Stream:
    cuda_stream = 0


def _nothing_to_do(name):
    """Arguments of a call that launches nothing."""
    if name == "flatquant_cache_advance":
        return dict(batch=fq.KvBatch(**{**BATCH, "B": 0}), pool=fq.PagePool(**POOL), page_tokens=16, pages=8, held=FAR, keep=FAR, rows=FAR, positions=FAR, slots=FAR)
    if name == "flatquant_head_rope":
        return {**ROPE, "T": 0}
    return dict(cache=fq.KvCache(**CACHE), batch=fq.KvBatch(**BATCH), q=FAR, q_stride=1024, Hq=8, scale=0.1, cap=2.0, slopes=FAR, prefix=FAR, window=0, sinks=0, visible=None,
                out=FAR, out_stride=1024, workspace=FAR, workspace_bytes=0)


@pytest.mark.parametrize("through", ["extension", "ctypes"])
@pytest.mark.parametrize("name", fq.STEP_CALLS)
def test_calls_marshal_like_their_signatures(name, through):
    fn = getattr(fq, name) if through == "extension" else fq._ctypes_call(name)
    assert type(getattr(fq, name)) is type(len), "the extension is not built"
    assert str(inspect.signature(getattr(fq, name))) == str(inspect.signature(fq._ctypes_call(name)))
    names = list(inspect.signature(fn).parameters)
    good = _nothing_to_do(name)
    assert names[-2:] == ["stream", "check"] and names[:-2] == list(good)
    assert fn(*good.values()) == fq.FQ_OK and fn(**good, stream=None) == fq.FQ_OK and fn(*good.values(), _Stream(), False) == fq.FQ_OK
    as_objects = {n: _Buffer(v) if isinstance(v, int) and v >= FAR else np.int64(v) if isinstance(v, int) else np.float64(v) if isinstance(v, float) else v
                  for n, v in good.items()}
    assert fn(**as_objects, stream=_Stream(), check=True) == fq.FQ_OK
    bad = {"flatquant_cache_advance": dict(pages=0), "flatquant_head_rope": dict(T=-1), "flatquant_cache_scored_attention": dict(cap=-1.0)}[name]
    with pytest.raises(fq.FlatQuantError, match=name) as e:
        fn(**{**good, **bad})
    assert e.value.status == fq.FQ_INVALID_ARG
    for args, kw in (((), {}), (tuple(good.values())[:-1], {}), (tuple(good.values()), {"no_such": 1}), (tuple(good.values()) + (None, True, 1), {})):
        with pytest.raises(TypeError):
            fn(*args, **kw)


def test_calls_reach_the_c_function_of_their_name():
    """With a recording function in the place of each C function: every argument in its place and its C type."""
    calls = importlib.import_module("paper_2410_09426_amd._fqcall")
    seen, keep = [], []
    real = {n: ctypes.cast(getattr(fq.lib(), n), ctypes.c_void_p).value for n in fq.STEP_CALLS}
    fakes = {}
    for name in fq.STEP_CALLS:
        c = getattr(fq.lib(), name)
        keep.append(ctypes.CFUNCTYPE(c.restype, *c.argtypes)(lambda *a, name=name: seen.append((name, *a)) or fq.FQ_OK))
        fakes[name] = ctypes.cast(keep[-1], ctypes.c_void_p).value
    calls.bind(fakes)
    try:
        for name in fq.STEP_CALLS:
            types = getattr(fq.lib(), name).argtypes[:-1]
            args = [0.25 + k if t is ctypes.c_float else 2 ** 40 + k if t is ctypes.c_int64 else 100 + k if t is ctypes.c_int else 2 ** 45 + k
                    for k, t in enumerate(types)]
            assert getattr(fq, name)(*args, 2 ** 44) == fq.FQ_OK
            assert seen.pop() == (name, *args, 2 ** 44) and not seen
    finally:
        calls.bind(real)


def test_pool_holds_its_fields():
    buffers = [_Buffer(A + 0x1000 * k) for k in range(3)]
    p = fq.PagePool(*buffers, 77)
    assert list((ctypes.c_uint64 * 4).from_address(p.data_ptr())) == [b.address for b in buffers] + [77]
    assert all(b in p._kept for b in buffers)


def test_turns_of_frequencies():
    """Within 2^-53 of the turn that a double says, which long double holds to 2^-64: the angle at position 2^31 is within 2^-32 of a turn."""
    f = [10000.0 ** (-2 * i / 128) for i in range(64)] + [0.0, -1.0, 6.283185307179586, 1e-12, 123.456, -1e-30, 2.0 ** 40]
    got = fq.fq_rope_turns(np.array(f))
    assert got.dtype == np.uint64
    for x, t in zip(f, got.tolist()):
        off = (t - so.turns_exact(x)) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= 2 + 2 ** -63 * abs(x) * 2 ** 64, (x, off)
    assert len(fq.fq_rope_turns(np.zeros(0))) == 0
    for bad in (np.inf, -np.inf, np.nan):
        with pytest.raises(fq.FlatQuantError):
            fq.fq_rope_turns([1.0, bad])
    with pytest.raises(ValueError):
        fq.fq_rope_turns(np.zeros((2, 2)))
    lib = fq.lib()
    assert lib.fq_rope_turns(None, 1, got.ctypes.data) == fq.FQ_INVALID_ARG and lib.fq_rope_turns(got.ctypes.data, -1, got.ctypes.data) == fq.FQ_INVALID_ARG


# ---- the oracle

def test_oracle_advance_worked_by_hand():
    table = [[5, 6, -9, -9], [7, -1, 8, -9], [-9] * 4]
    ring = [0, 1, 2, 3, 4]
    got = so.advance([20, 40, 0], [20, 5, 0], [13, 2, 1], table, 4, 16, 9, ring, 13, 17, 20)
    # sequence 0: 33 tokens, a third page (ring[13 % 5]); 1: 7 tokens, entries 1 (no page) and 2 (page 8) go; 2: its first page
    assert got[0] == [0, 13, 15, 16] and got[1] == [33, 7, 1] and got[2] == (15, 18, 0)
    assert table == [[5, 6, 3, -9], [7, -1, 8, -9], [4, -9, -9, -9]] and ring == [0, 1, 8, 3, 4]
    assert got[3] == list(range(20, 33)) + [5, 6, 0] + [-1] * 4
    assert got[4] == [6 * 16 + p - 16 for p in range(20, 32)] + [3 * 16, 7 * 16 + 5, 7 * 16 + 6, 4 * 16] + [-1] * 4


def test_oracle_rotation_closed_forms():
    r = np.random.Generator(np.random.PCG64(3))
    x = r.standard_normal((3, 2, 128)).astype(np.float16)
    f = [np.pi / 2, np.pi, 0.0, 2 * np.pi] * 4
    for pairs in (False, True):
        y, size = so.turned64(x, None, 0.0, [0, 1, 2], f, pairs)
        assert np.array_equal(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
        a, b = (0, 1) if pairs else (0, 16)
        assert np.allclose(y[1, :, a], -x[1, :, b].astype(float)) and np.allclose(y[1, :, b], x[1, :, a].astype(float))
        assert np.allclose(y[2, :, a], -x[2, :, a].astype(float))
        assert np.allclose((y ** 2).sum(-1), (x.astype(float) ** 2).sum(-1))
    y, _ = so.turned64(x, np.full(128, 2.0), 0.0, [5, 6, 7], f, False)
    assert np.allclose((y ** 2).mean(-1), 4.0)


def test_oracle_bounds_reject_planted_mistakes():
    """A position more, sine's sign, the pairs of the other order, a weight left out, a row's norm over 127 channels; a cap of 1.92 for 2, a slope a tenth off, one
    token of the prefix: each is far outside the bound, and what rounding alone does is inside."""
    r = np.random.Generator(np.random.PCG64(4))
    x, w = r.standard_normal((4, 1, 128)).astype(np.float16), (1 + 0.2 * r.standard_normal(128)).astype(np.float16)
    f, pos = [100.0 ** (-2 * i / 128) for i in range(64)], np.array([3, 50, 1000, 7])
    y, tol = so.rope64(x, w, 1e-6, pos, f, False)
    assert (np.abs(y.astype(np.float16) - y) / tol).max() <= 1
    one = w.copy()
    one[5] *= np.float16(1.01)
    for z in (so.rope64(x, w, 1e-6, pos + 1, f, False), so.rope64(x, w, 1e-6, -pos, f, False), so.rope64(x, w, 1e-6, pos, f, True), so.rope64(x, one, 1e-6, pos, f, False),
              so.rope64(x, w, 1.0 / 128, pos, f, False)):
        assert (np.abs(z[0] - y) / tol).max() > 2
    L = 120
    grids = [co.grid32(r.standard_normal((L, 128)), 1.0, 4) for _ in range(2)]
    (k, v), (ks, vs) = [co.dequantize(*g) for g in grids], [g[1].astype(np.float64) for g in grids]
    q, seen = 2 * r.standard_normal((2, 128)), np.ones((2, L), dtype=bool)
    seen[0, 100:] = False
    how = dict(scale=0.09, positions=np.array([60, 119]), k_step=ks, v_step=vs)
    out, A_, S, E = so.scored64(q, k, v, seen, cap=2.0, slope=0.1, **how)
    tol = so.scored_bound(out, A_, S, E, L)
    fewer = seen.copy()
    fewer[0, 99] = False
    for z in (so.scored64(q, k, v, seen, cap=1.92, slope=0.1, **how), so.scored64(q, k, v, seen, cap=2.0, slope=0.11, **how),
              so.scored64(q, k, v, seen, cap=2.0, slope=0.1, **{**how, "positions": np.array([40, 119])}), so.scored64(q, k, v, fewer, cap=2.0, slope=0.1, **how)):
        assert (np.abs(z[0] - out) / tol).max() > 2
    plain, *size = co.attention64(q, k, v, seen, 0.09, ks, vs)
    assert np.allclose(so.scored64(q, k, v, seen, cap=0.0, slope=0.0, **how)[0], plain)
