"""Which C functions the native calls go to."""
import ctypes
import importlib

import pytest

from paper_2410_09426_amd import binding as fq


@pytest.mark.parametrize("name", fq.NATIVE + fq.CACHE_CALLS)
def test_binding_one_entry_point_leaves_the_others(name):
    calls = importlib.import_module("paper_2410_09426_amd._fqcall")
    seen = []
    real = {n: ctypes.cast(getattr(fq.lib(), n), ctypes.c_void_p).value for n in fq.NATIVE + fq.CACHE_CALLS}
    keep = {}
    for n in real:
        c = getattr(fq.lib(), n)
        keep[n] = ctypes.CFUNCTYPE(c.restype, *c.argtypes)(lambda *a, n=n: seen.append(n) or fq.FQ_OK)
    fakes = {n: ctypes.cast(f, ctypes.c_void_p).value for n, f in keep.items()}

    def called(n):
        args = [0.25 if t is ctypes.c_float else 1 if t in (ctypes.c_int, ctypes.c_int64) else 4096 for t in getattr(fq.lib(), n).argtypes[:-1]]
        assert getattr(fq, n)(*args, 0) == fq.FQ_OK
        return seen.pop()
    try:
        calls.bind(fakes)
        calls.bind({name: fakes["flatquant_head_transform"] if name != "flatquant_head_transform" else fakes[name]})
        assert all(called(n) == n for n in real if n != name)
    finally:
        calls.bind(real)
    with pytest.raises(TypeError):
        calls.bind({name: "no address"})
    with pytest.raises(TypeError):
        calls.bind(4096)
    calls.bind({})
