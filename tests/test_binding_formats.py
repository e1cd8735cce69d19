"""Each call of the serving loop reaches its own entry point, by the module and by ctypes (no GPU): stand-ins for the library's functions say
which one was called and with what."""
import ctypes

import numpy as np
import pytest

from paper_2602_11530_amd import binding as pkv
from test_binding_calls import Buffer

T = [Buffer((i + 1) << 20, 1 << 30) for i in range(16)]
SHAPE = pkv.make_shape(4, 8, 2, 19, 128)
ROPE = pkv.make_rope(4, 128, 19 * 16)

CALLS = {
    "kv_append": (*T[:6], SHAPE), "kv_append_fp8": (*T[:6], 0.5, 0.25, SHAPE), "kv_append_fp4": (*T[:6], SHAPE),
    "paged_decode_attn": (*T[:5], 0.5, T[5], SHAPE, T[6]),
    "paged_decode_attn_fp8kv": (*T[:5], 0.5, 2.0, 4.0, T[5], SHAPE, T[6]),
    "paged_decode_attn_fp4kv": (*T[:5], 0.5, T[5], SHAPE, T[6]),
    "paged_decode_attn_static": (*T[:5], 0.5, T[5], SHAPE),
    "paged_decode_attn_window": (*T[:5], 0.5, 7, 3, T[5], SHAPE, T[6]),
    "paged_decode_attn_window_fp8kv": (*T[:5], 0.5, 2.0, 4.0, 7, 3, T[5], SHAPE, T[6]),
    "paged_decode_attn_window_fp4kv": (*T[:5], 0.5, 7, 3, T[5], SHAPE, T[6]),
    "kv_blocks_gather": (*T[:3], 1, 64, 9), "kv_blocks_scatter": (*T[:3], 1, 64, 9), "kv_blocks_move": (*T[:4], 1, 64, 9, 9),
    "kv_rope_append": (*T[:12], ROPE, SHAPE), "kv_rope_append_fp8": (*T[:12], 0.5, 0.25, ROPE, SHAPE),
    "kv_rope_append_fp4": (*T[:12], ROPE, SHAPE),
}


def as_c(x):
    return x.data_ptr() if isinstance(x, Buffer) else ctypes.addressof(x) if isinstance(x, ctypes.Structure) else x


@pytest.fixture(params=["module", "ctypes"])
def called(request, monkeypatch):
    """Names and arguments of the C functions that are called."""
    L, log = pkv.lib(), []
    if request.param == "ctypes":
        monkeypatch.setattr(pkv, "_call", pkv._ByCtypes())

        def record(name):
            return lambda *a: log.append((name, a)) or 0
        stand_in = type("Library", (), {name: staticmethod(record(name)) for name in CALLS})
        monkeypatch.setattr(pkv, "_lib", stand_in)
        yield log
        return
    if isinstance(pkv._call, pkv._ByCtypes):
        pytest.skip("the module is not built")
    keep, addresses = [], {}
    for name in CALLS:
        kinds = getattr(L, name).argtypes
        plain = [ctypes.c_void_p if hasattr(k, "_type_") and not isinstance(k._type_, str) else k for k in kinds]
        fn = ctypes.CFUNCTYPE(ctypes.c_int, *plain)(lambda *a, name=name: log.append((name, a)) or 0)
        keep.append(fn)
        addresses[name] = ctypes.cast(fn, ctypes.c_void_p).value
    pkv._call.setup(addresses, pkv.AttnShape, pkv.RopeShape, bool, None, None)
    yield log
    import torch
    pkv._setup_call(L, torch)


@pytest.mark.parametrize("name", CALLS)
def test_each_call_reaches_its_own_entry_point(called, name):
    getattr(pkv, name)(*CALLS[name], 48)
    (got, args), = called
    assert got == name
    want = [as_c(x) for x in CALLS[name]]
    if len(args) > len(want) + 1:      # the workspace's bytes
        want.append(1 << 30)
    plain = [a.value if hasattr(a, "value") else as_c(a._obj) if hasattr(a, "_obj") else a for a in args]
    assert plain == [*want, 48]


@pytest.mark.parametrize("module", [False, True])
@pytest.mark.parametrize("name", [n for n in CALLS if "window" in n])
@pytest.mark.parametrize("where", [0, 1])
def test_numbers_of_tokens_beyond_32_bits(monkeypatch, name, module, where):
    """Refused, not cut to their lower bits; whole numbers of another class are taken."""
    pkv.lib()
    if not module:
        monkeypatch.setattr(pkv, "_call", pkv._ByCtypes())
    args = list(CALLS[name])
    at = 8 if "fp8" in name else 6
    empty = pkv.make_shape(0, 8, 2, 19, 128)
    args = [empty if a is SHAPE else a for a in args]
    for bad in (2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 70, -1):
        args[at + where] = bad
        with pytest.raises(pkv.PkvError) as e:
            getattr(pkv, name)(*args, 0)
        assert e.value.status == pkv.PKV_ERR_SHAPE
    for good in (np.int64(5), np.int32(2 ** 31 - 1), 0):
        args[at + where] = good
        getattr(pkv, name)(*args, 0)
    args[at + where] = 5.0
    with pytest.raises(TypeError):
        getattr(pkv, name)(*args, 0)
