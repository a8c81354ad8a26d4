"""The paged key/value cache without a GPU: refusals that return before a device is touched, marshalling, the workspace figure, and the
oracle's own pins."""
import ctypes
import inspect

import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import flatquant_oracle as fo
from paper_2410_09426_amd import binding as fq

A = 0x10000000          # addresses that are never followed
CACHE = dict(k_codes=A, k_params=A + 0x1000000, v_codes=A + 0x2000000, v_params=A + 0x3000000, pages=8, page_tokens=16, H=4, k_bits=4, v_bits=3)
BATCH = dict(row_starts=A + 0x4000000, lengths=A + 0x4001000, page_table=A + 0x4002000, B=2, T=0, table_width=4, table_stride=4, max_rows=1, max_length=64)
FAR = A + 0x8000000


def _cache(**k):
    return fq.KvCache(**{**CACHE, **k})


def _batch(**k):
    return fq.KvBatch(**{**BATCH, **k})


def _write(cache=None, batch=None, **k):
    return fq.flatquant_cache_write(**{**dict(cache=cache or _cache(), batch=batch or _batch(), k=FAR, k_stride=512, v=FAR + 0x100000, v_stride=512, P_k=None,
                                              P_v=None, Hp=1, k_clip=0.9, v_clip=0.9, check=False), **k})


def _read(cache=None, batch=None, **k):
    return fq.flatquant_cache_read(**{**dict(cache=cache or _cache(), batch=batch or _batch(), k=FAR, k_stride=512, v=FAR + 0x100000, v_stride=512,
                                             check=False), **k})


def _attend(cache=None, batch=None, **k):
    return fq.flatquant_cache_attention(**{**dict(cache=cache or _cache(), batch=batch or _batch(), q=FAR, q_stride=1024, Hq=8, scale=0.1, window=0, sinks=0,
                                                  out=FAR + 0x100000, out_stride=1024, workspace=None, workspace_bytes=0, check=False), **k})


def _tree(cache=None, batch=None, **k):
    return fq.flatquant_cache_tree_attention(**{**dict(cache=cache or _cache(), batch=batch or _batch(), q=FAR, q_stride=1024, Hq=8, scale=0.1,
                                                       visible=FAR + 0x200000, out=FAR + 0x100000, out_stride=1024, workspace=None, workspace_bytes=0,
                                                       check=False), **k})


CALLS = [_write, _read, _attend, _tree]


@pytest.mark.parametrize("call", CALLS)
def test_what_every_call_on_a_cache_refuses(call):
    some = dict(T=3)
    assert call() == fq.FQ_OK                                            # no rows: nothing launched
    assert call(batch=_batch(T=3, B=0)) == fq.FQ_OK
    for bad in (dict(pages=0), dict(pages=-1), dict(H=0), dict(k_bits=1), dict(v_bits=5), dict(k_bits=8), dict(page_tokens=0)):
        assert call(cache=_cache(**bad)) == fq.FQ_INVALID_ARG, bad
    for bad in (dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048), dict(H=65536), dict(pages=2 ** 31), dict(pages=2 ** 31 - 1, H=65535)):
        assert call(cache=_cache(**bad)) == fq.FQ_UNSUPPORTED_SHAPE, bad
    for bad in (dict(B=-1), dict(T=-1), dict(table_width=-1), dict(table_stride=3), dict(max_rows=-1), dict(max_length=-1)):
        assert call(batch=_batch(**bad)) == fq.FQ_INVALID_ARG, bad
    for bad in (dict(T=2 ** 29 + 1), dict(B=2 ** 22), dict(table_width=2 ** 31, table_stride=2 ** 31)):
        assert call(batch=_batch(**bad)) == fq.FQ_UNSUPPORTED_SHAPE, bad
    for name in ("k_codes", "k_params", "v_codes", "v_params"):
        assert call(cache=_cache(**{name: None}), batch=_batch(**some)) == fq.FQ_INVALID_ARG, name
        assert call(cache=_cache(**{name: CACHE[name] + 8}), batch=_batch(**some)) == fq.FQ_MISALIGNED, name
    for name in ("row_starts", "lengths", "page_table"):
        assert call(batch=_batch(**some, **{name: None})) == fq.FQ_INVALID_ARG, name
        assert call(batch=_batch(**some, **{name: BATCH[name] + 2})) == fq.FQ_MISALIGNED, name
    rest = dict(check=False)
    if call in (_attend, _tree):
        rest.update(q=FAR, q_stride=1024, Hq=8, scale=0.1, out=FAR, out_stride=1024, workspace=None, workspace_bytes=0)
        rest.update(dict(window=0, sinks=0) if call is _attend else dict(visible=FAR))
    else:
        rest.update(k=FAR, k_stride=512, v=FAR, v_stride=512)
        if call is _write:
            rest.update(P_k=None, P_v=None, Hp=1, k_clip=1.0, v_clip=1.0)
    fn = {_write: fq.flatquant_cache_write, _read: fq.flatquant_cache_read, _attend: fq.flatquant_cache_attention, _tree: fq.flatquant_cache_tree_attention}[call]
    assert fn(cache=None, batch=_batch(), **rest) == fq.FQ_INVALID_ARG
    assert fn(cache=_cache(), batch=None, **rest) == fq.FQ_INVALID_ARG


def test_row_tensors_that_write_and_read_refuse():
    b = _batch(T=3)
    for call in (_write, _read):
        assert call(batch=b, k=None, v=None) == fq.FQ_OK                  # nothing to do
        assert call(batch=b, k_stride=511) == fq.FQ_INVALID_ARG and call(batch=b, v_stride=504) == fq.FQ_INVALID_ARG
        assert call(batch=b, k_stride=516) == fq.FQ_MISALIGNED and call(batch=b, v=FAR + 0x100008) == fq.FQ_MISALIGNED
        assert call(batch=b, k_stride=2 ** 41) == fq.FQ_UNSUPPORTED_SHAPE
        for inside in (A, A + 0x1000000, A + 0x2000010, A + 0x3000000, A + 0x4000000, A + 0x4001000, A + 0x4002000):
            assert call(batch=b, v=inside) == fq.FQ_INVALID_ARG, hex(inside)
    assert _read(batch=b, v=FAR) == fq.FQ_INVALID_ARG                     # both into the same rows
    assert _write(batch=b, k_clip=0.0) == fq.FQ_INVALID_ARG and _write(batch=b, v_clip=float("nan")) == fq.FQ_INVALID_ARG
    assert _write(batch=b, Hp=2) == fq.FQ_INVALID_ARG and _write(batch=b, P_k=FAR + 8) == fq.FQ_MISALIGNED


@pytest.mark.parametrize("call", [_attend, _tree])
def test_what_attention_refuses(call):
    b = _batch(T=3)
    for bad in (dict(Hq=0), dict(Hq=6), dict(Hq=-4), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride=1016), dict(out_stride=1000),
                dict(q=None), dict(out=None), dict(workspace_bytes=-1), dict(out=FAR + 1024), dict(out=A), dict(out=A + 0x4002000)):
        assert call(batch=b, **bad) == fq.FQ_INVALID_ARG, bad
    for bad in (dict(q=FAR + 8), dict(out=FAR + 0x100008), dict(q_stride=1028), dict(out_stride=1028), dict(workspace=FAR + 0x300008, workspace_bytes=64)):
        assert call(batch=b, **bad) == fq.FQ_MISALIGNED, bad
    assert call(batch=b, q_stride=2 ** 41) == fq.FQ_UNSUPPORTED_SHAPE
    assert call(batch=_batch(T=2 ** 29), Hq=2 ** 22, q_stride=2 ** 29, out_stride=2 ** 29) == fq.FQ_UNSUPPORTED_SHAPE
    if call is _attend:
        assert call(batch=b, window=-1) == fq.FQ_INVALID_ARG and call(batch=b, sinks=-1) == fq.FQ_INVALID_ARG
    else:
        assert call(batch=b, visible=None) == fq.FQ_INVALID_ARG and call(batch=b, visible=FAR + 0x200004) == fq.FQ_MISALIGNED
        assert call(batch=b, visible=FAR + 0x100010) == fq.FQ_INVALID_ARG and call(batch=_batch(T=3, max_rows=65)) == fq.FQ_UNSUPPORTED_SHAPE
    long = _batch(T=1, B=1, max_rows=1, max_length=100000, table_width=8000, table_stride=8000)
    need = fq.fq_cache_attention_workspace(_cache(), long, 8)
    assert need > 0
    assert call(batch=long) == fq.FQ_INVALID_ARG                          # no workspace where one is needed
    assert call(batch=long, workspace=FAR + 0x1000000, workspace_bytes=need - 1) == fq.FQ_INVALID_ARG
    assert call(batch=long, workspace=FAR + 0x100000, workspace_bytes=need) == fq.FQ_INVALID_ARG      # the output lies in it
    assert call(batch=long, workspace=A, workspace_bytes=need) == fq.FQ_INVALID_ARG                   # the cache does


def test_workspace_follows_from_the_host_figures():
    size = lambda H=4, Hq=8, **b: fq.fq_cache_attention_workspace(_cache(H=H), _batch(**b), Hq)      # noqa: E731
    assert size(T=0) == 0 and size(T=5, B=0) == 0 and size(T=2, max_length=64) == 0
    assert size(T=1, B=1, max_length=131072) > 0 and size(T=1, B=1, max_length=131072) % 16 == 0
    assert size(T=300, B=3, max_rows=100, max_length=131072) > size(T=100, B=1, max_rows=100, max_length=1000)
    for bad in (dict(Hq=0), dict(Hq=6), dict(T=-1), dict(T=2 ** 29 + 1), dict(B=2 ** 22)):
        with pytest.raises(fq.FlatQuantError):
            size(**{**dict(T=1), **bad})
    for rows in (1, 3, 64, 5000):
        for length in (0, 1, 31, 4096, 10 ** 6, 2 ** 30):
            for B in (1, 7, 300):
                n = size(T=B * rows, B=B, max_rows=rows, max_length=length)
                assert 0 <= n <= max(2 * 4 * 256 * 32, B * rows * 8 * 128) * 130 * 4 and n % 16 == 0


class _Buffer:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


class _Stream:
    cuda_stream = 0


@pytest.mark.parametrize("name", fq.CACHE_CALLS)
def test_calls_marshal_like_their_signatures(name):
    """Positional and named arguments, addresses, buffers and numpy numbers, without a launch; wrong calls are errors of Python's own."""
    fn = getattr(fq, name)
    names = list(inspect.signature(fn).parameters)
    assert names[-2:] == ["stream", "check"] and names[:2] == ["cache", "batch"]
    numbers = dict(k_stride=512, v_stride=512, Hp=1, k_clip=0.9, v_clip=0.9, q_stride=1024, Hq=8, scale=0.1, window=0, sinks=0, out_stride=1024, workspace_bytes=0)
    good = {n: _cache() if n == "cache" else _batch() if n == "batch" else numbers.get(n, FAR + 0x100000 * k) for k, n in enumerate(names[:-2])}
    assert fn(*good.values()) == fq.FQ_OK and fn(**good, stream=None) == fq.FQ_OK and fn(*good.values(), _Stream(), False) == fq.FQ_OK
    as_objects = {n: v if n in ("cache", "batch") else _Buffer(v) if n not in numbers else np.float64(v) if isinstance(v, float) else np.int64(v) for n, v in good.items()}
    assert fn(**as_objects, stream=_Stream(), check=True) == fq.FQ_OK
    with pytest.raises(fq.FlatQuantError, match=name) as e:
        fn(**{**good, "cache": _cache(pages=0)})
    assert e.value.status == fq.FQ_INVALID_ARG
    for args, kw in (((), {}), (tuple(good.values())[:-1], {}), (tuple(good.values()), {"no_such": 1}), (tuple(good.values()) + (None, True, 1), {})):
        with pytest.raises(TypeError):
            fn(*args, **kw)


def test_structs_hold_their_fields_and_keep_their_tensors():
    buffers = [_Buffer(A + 0x1000 * k) for k in range(4)]
    c = fq.KvCache(*buffers, 2 ** 31 - 1, 64, 8, 4, 2)
    raw = (ctypes.c_uint64 * 5).from_address(c.data_ptr())
    assert list(raw) == [b.address for b in buffers] + [2 ** 31 - 1]
    assert list((ctypes.c_int32 * 4).from_address(c.data_ptr() + 40)) == [64, 8, 4, 2]
    b = fq.KvBatch(*buffers[:3], 1, 2, 3, 4, 5, 6)
    assert list((ctypes.c_int64 * 9).from_address(b.data_ptr())) == [x.address for x in buffers[:3]] + [1, 2, 3, 4, 5, 6]
    assert all(x in c._kept for x in buffers)


# ---- the oracle

@pytest.mark.parametrize("bits", [2, 3, 4])
def test_oracle_grid_against_the_fp64_one(bits):
    """The fp32 sequence and the fp64 definition give the same steps but for those that fp32 rounds onto an fp16 midpoint, and the same codes on
    the same steps (a quotient of two fp16 numbers is a tie exactly, or fp32 keeps it away from one)."""
    r = np.random.Generator(np.random.PCG64(bits))
    y = (r.standard_normal((3000, 128)) * 2.0 ** r.integers(-6, 7, size=(3000, 1))).astype(np.float16)
    for clip in (1.0, 0.95, 0.5):
        q, s, z = co.grid32(y, clip, bits)
        q64, s64, z64, _, _ = fo.kv_quantize_asym(y, np.float32(clip), bits)
        same = (s == s64) & (z == z64)
        assert same.mean() > 0.9 and np.array_equal(q[same], q64[same])
        assert np.abs(s.view(np.int16).astype(int) - s64.view(np.int16).astype(int)).max() <= 1
        assert np.array_equal(co.pack(q, bits), fo.pack_bits(q, bits)) and np.array_equal(co.unpack(co.pack(q, bits), bits), q)


def test_oracle_grid_on_zero_rows_ties_and_overflow():
    y = np.zeros((4, 128), dtype=np.float16)
    y[1, 0], y[1, 1:16] = 15.0, np.arange(15) + 0.5                       # step 1, zero point 0: ties go to even
    y[2, :] = np.float16(6e-8)
    y[3, 0] = 65504.0
    q, s, z = co.grid32(y, 1.0, 4)
    assert s[0] == 0 and s[1] == 1 and s[2] == 0 and not q[0].any() and not q[2].any()
    assert list(q[1, 1:16]) == [0, 2, 2, 4, 4, 6, 6, 8, 8, 10, 10, 12, 12, 14, 14]
    assert co.grid32(y, 100.0, 4)[1][3] == np.inf and not co.grid32(y, 100.0, 4)[0][3].any()


def test_oracle_attention_closed_forms():
    r = np.random.Generator(np.random.PCG64(9))
    k, v, q = r.standard_normal((7, 128)), r.standard_normal((7, 128)), r.standard_normal((3, 128))
    seen = np.array([[1, 0, 0, 0, 0, 0, 0], [0] * 7, [0, 1, 1, 0, 0, 0, 1]], dtype=bool)
    one = np.ones(7)
    out, A, S, delta = co.attention64(q, k, v, seen, 0.3, one, 2 * one)
    assert np.allclose(out[0], v[0]) and not out[1].any() and np.allclose(A[0], np.abs(v[0])) and S[1] == 0 and np.isclose(S[2], 2)
    assert delta[1] == 0 and np.isclose(delta[2], 0.3 * (280 * 15 * np.abs(q[2]).sum() / 2 ** 24 + 132 * np.abs(q[2]).max() / 2 ** 18))
    assert np.allclose(co.attention64(q, k, v, seen, 0.0, one, one)[0][2], v[[1, 2, 6]].mean(0))


def test_oracle_bound_rejects_planted_mistakes():
    """A token too many, a token too few, a token of every 32 left out, two query heads exchanged, a step halved: each is far outside the bound."""
    r = np.random.Generator(np.random.PCG64(10))
    L = 200
    grids = [co.grid32(r.standard_normal((L, 128)), 1.0, 4) for _ in range(2)]
    (k, v), (ks, vs) = [co.dequantize(*g) for g in grids], [g[1].astype(np.float64) for g in grids]
    q = r.standard_normal((2, 128))
    seen = np.ones((2, L), dtype=bool)
    seen[0, -1] = False
    out, *size = co.attention64(q, k, v, seen, 0.09, ks, vs)
    tol = co.attention_bound(out, *size, L)
    worse = [co.attention64(q, k, v, m, 0.09, ks, vs)[0] for m in (np.ones_like(seen), seen & (np.arange(L) > 0), seen & (np.arange(L) % 32 != 5))]
    worse += [out[::-1], co.attention64(q, k, v * np.where(np.arange(L) == 3, 0.5, 1.0)[:, None], seen, 0.09, ks, vs)[0], out * 1.02]
    for x in worse:
        assert (np.abs(x - out) / tol).max() > 1.0
    assert (np.abs(out.astype(np.float16) - out) / tol).max() < 1.0


def test_calls_reach_the_c_function_of_their_name():
    """With a recording function in the place of each C function, native or through ctypes: every argument in its place and its C type."""
    import importlib
    calls = importlib.import_module("paper_2410_09426_amd._fqcall")
    seen, keep = [], []
    real = {n: ctypes.cast(getattr(fq.lib(), n), ctypes.c_void_p).value for n in fq.NATIVE + fq.CACHE_CALLS}
    fakes = dict(real)
    for name in fq.CACHE_CALLS:
        c = getattr(fq.lib(), name)
        keep.append(ctypes.CFUNCTYPE(c.restype, *c.argtypes)(lambda *a, name=name: seen.append((name, *a)) or fq.FQ_OK))
        fakes[name] = ctypes.cast(keep[-1], ctypes.c_void_p).value
    calls.bind(fakes)
    try:
        calls.bind({n: real[n] for n in fq.NATIVE})                       # what is not named stays
        for name in fq.CACHE_CALLS:
            types = getattr(fq.lib(), name).argtypes[:-1]                 # without the stream
            args = [0.25 if t is ctypes.c_float else 2 ** 40 + k if t is ctypes.c_int64 else 100 + k if t is ctypes.c_int else 2 ** 45 + k for k, t in enumerate(types)]
            assert getattr(fq, name)(*args, 2 ** 44) == fq.FQ_OK
            assert seen.pop() == (name, *args, 2 ** 44) and not seen
    finally:
        calls.bind(real)
    for name in fq.CACHE_CALLS:                                           # the signature of the one is that of the other
        assert str(inspect.signature(getattr(fq, name))) == str(inspect.signature(fq._ctypes_call(name)))
