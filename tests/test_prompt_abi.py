"""Argument checks of prompt attention and of the calls for pools with a scale for each block and KV head: errors before anything is launched (no
GPU).  And that each call of the binding reaches its own entry point, by the module and by ctypes."""
import ctypes

import numpy as np
import pytest

from paper_2602_11530_amd import binding as pkv
from test_binding_calls import Buffer

SH = pkv.make_shape(4, 8, 2, 19, 128)
NONE = pkv.make_shape(0, 8, 2, 19, 128)
MIB = 1 << 20
BAD_SHAPES = (dict(head_dim=96), dict(block_size=48), dict(num_kv_heads=3), dict(head_dim=256, num_q_heads=32), dict(num_seqs=2049))
LONG = pkv.make_shape(4, 8, 2, 190, 128)     # contexts that are cut where tokens are few
FEW = 64     # new tokens


def bad_shape(**kw):
    return pkv.make_shape(**{**dict(num_seqs=4, num_q_heads=8, num_kv_heads=2, max_blocks_per_seq=19, num_pool_blocks=128), **kw})


def ref(shape):
    return ctypes.byref(shape) if shape is not None else None


def prompt(name, q=MIB, k=2 * MIB, v=3 * MIB, ks=4 * MIB, vs=5 * MIB, t=6 * MIB, l=7 * MIB, s=8 * MIB, n=FEW, k_scale=1.0, v_scale=1.0, o=9 * MIB,
           shape=LONG, ws=20 * MIB, nb=None):
    need = nb if nb is not None else pkv.pkv_prompt_workspace_bytes(LONG, FEW)
    arrays = (ks, vs) if name.endswith("blk") else ()
    scales = (k_scale, v_scale) if name.endswith("fp8kv") else ()
    return getattr(pkv.lib(), name)(q, k, v, *arrays, t, l, s, n, 1.0, *scales, o, ref(shape), ws, need, None)


@pytest.mark.parametrize("name", ["paged_prompt_attn", "paged_prompt_attn_fp8kv", "paged_prompt_attn_fp8blk"])
def test_prompt(name):
    f = lambda **kw: prompt(name, **kw)  # noqa: E731
    blk = ("ks", "vs") if name.endswith("blk") else ()
    need = pkv.pkv_prompt_workspace_bytes(LONG, FEW)
    assert need > 0
    for x in ("q", "k", "v", "t", "l", "o", "shape", *blk):
        assert f(**{x: None}) == pkv.PKV_ERR_NULL, x
    for x in ("q", "k", "v", "o", "ws", *blk):
        assert f(**{x: 40 * MIB + 8}) == pkv.PKV_ERR_ALIGN, x
    for x in ("t", "l", "s"):
        assert f(**{x: 40 * MIB + 2}) == pkv.PKV_ERR_ALIGN, x
    assert f(ws=None) == f(nb=need - 1) == pkv.PKV_ERR_WORKSPACE
    for bad in BAD_SHAPES:
        assert f(shape=bad_shape(**bad)) == pkv.PKV_ERR_SHAPE, bad
    assert f(n=-1) == f(n=1 << 24) == f(n=2 ** 62) == pkv.PKV_ERR_SHAPE
    assert f(s=None) == pkv.PKV_ERR_SHAPE                              # one token for each of four requests
    if name.endswith("fp8kv"):
        for a, b in ((0.0, 1.0), (1.0, -2.0), (float("nan"), 1.0), (1.0, float("inf"))):
            assert f(k_scale=a, v_scale=b) == pkv.PKV_ERR_SHAPE
    # rows written where something is still to be read
    rows = FEW * 8 * 128 * 2
    assert f(o=MIB + 16) == f(o=MIB - rows + 16) == f(o=2 * MIB) == f(o=3 * MIB) == f(o=6 * MIB) == f(o=7 * MIB) == f(o=8 * MIB) == pkv.PKV_ERR_SHAPE
    if blk:
        assert f(o=4 * MIB) == f(o=5 * MIB - rows + 16) == pkv.PKV_ERR_SHAPE
    nothing = dict(q=None, k=None, v=None, ks=None, vs=None, t=None, l=None, o=None, ws=None, nb=0)
    assert f(n=0, **nothing) == f(shape=NONE, **nothing) == pkv.PKV_OK
    assert f(n=0, s=None, **nothing) == pkv.PKV_ERR_SHAPE and f(n=0, s=None, shape=NONE, **nothing) == pkv.PKV_OK


def test_prompt_workspace():
    assert pkv.pkv_prompt_workspace_bytes(SH, 0) == pkv.pkv_prompt_workspace_bytes(NONE, 100) == 0
    assert pkv.lib().pkv_prompt_workspace_bytes(ref(SH), 4, None) == pkv.PKV_ERR_NULL
    long = pkv.make_shape(1, 40, 8, 4096, 4096)
    some = pkv.pkv_prompt_workspace_bytes(long, 64)
    assert some > 0 and some % (64 * 40 * 130 * 4) == 0                # rows and statistics of whole pieces
    assert pkv.pkv_prompt_workspace_bytes(pkv.make_shape(64, 40, 8, 4, 4096), 4096) == 0   # short contexts, many tokens
    for n in (-1, 1 << 24, 2 ** 63, 2 ** 80):
        with pytest.raises(pkv.PkvError) as e:
            pkv.pkv_prompt_workspace_bytes(SH, n)
        assert e.value.status == pkv.PKV_ERR_SHAPE
    for bad in BAD_SHAPES:
        with pytest.raises(pkv.PkvError):
            pkv.pkv_prompt_workspace_bytes(bad_shape(**bad), 4)
    with pytest.raises(pkv.PkvError):      # more workgroups than a launch numbers
        pkv.pkv_prompt_workspace_bytes(pkv.make_shape(4, 16384, 16384, 19, 128), 1 << 22)


@pytest.mark.parametrize("hkv,row", [(1, 16), (8, 16), (16, 16), (17, 32), (40, 48)])
def test_scale_rows(hkv, row):
    shape = pkv.make_shape(4, hkv, hkv, 19, 128)
    assert pkv.pkv_fp8blk_scale_bytes(shape) == row
    assert pkv.lib().pkv_fp8blk_scale_bytes(ref(shape), None) == pkv.PKV_ERR_NULL
    shape.head_dim = 8
    with pytest.raises(pkv.PkvError):
        pkv.pkv_fp8blk_scale_bytes(shape)


def test_step_attention():
    need = pkv.pkv_attn_workspace_bytes(SH)

    def f(q=MIB, k=2 * MIB, v=3 * MIB, ks=4 * MIB, vs=5 * MIB, t=6 * MIB, l=7 * MIB, o=9 * MIB, shape=SH, ws=20 * MIB, nb=need):
        return pkv.lib().paged_decode_attn_fp8blk(q, k, v, ks, vs, t, l, 1.0, o, ref(shape), ws, nb, None)
    for x in ("q", "k", "v", "ks", "vs", "t", "l", "o", "shape"):
        assert f(**{x: None}) == pkv.PKV_ERR_NULL, x
    for x in ("q", "k", "v", "ks", "vs", "o", "ws"):
        assert f(**{x: 40 * MIB + 8}) == pkv.PKV_ERR_ALIGN, x
    assert f(t=MIB + 2) == f(l=MIB + 2) == pkv.PKV_ERR_ALIGN
    assert f(ws=None) == f(nb=need - 1) == pkv.PKV_ERR_WORKSPACE
    assert f(o=4 * MIB) == f(o=5 * MIB + 128 * 16 - 16) == pkv.PKV_ERR_SHAPE
    for bad in BAD_SHAPES:
        assert f(shape=bad_shape(**bad)) == pkv.PKV_ERR_SHAPE
    assert f(q=None, k=None, v=None, ks=None, vs=None, t=None, l=None, o=None, shape=NONE, ws=None, nb=0) == pkv.PKV_OK


def test_append():
    def f(kn=MIB, vn=2 * MIB, k=3 * MIB, v=4 * MIB, ks=5 * MIB, vs=6 * MIB, t=7 * MIB, l=8 * MIB, shape=SH):
        return pkv.lib().kv_append_fp8blk(kn, vn, k, v, ks, vs, t, l, ref(shape), None)
    for x in ("kn", "vn", "k", "v", "ks", "vs", "t", "l", "shape"):
        assert f(**{x: None}) == pkv.PKV_ERR_NULL, x
    for x in ("kn", "vn", "k", "v", "ks", "vs"):
        assert f(**{x: MIB + 8}) == pkv.PKV_ERR_ALIGN, x
    assert f(t=MIB + 2) == f(l=MIB + 1) == pkv.PKV_ERR_ALIGN
    assert f(shape=bad_shape(head_dim=96)) == pkv.PKV_ERR_SHAPE
    assert f(kn=None, vn=None, k=None, v=None, ks=None, vs=None, t=None, l=None, shape=NONE) == pkv.PKV_OK


def test_rope_append():
    def f(q=MIB, k=2 * MIB, v=3 * MIB, qn=4 * MIB, kn=5 * MIB, cs=6 * MIB, qo=7 * MIB, kp=8 * MIB, vp=9 * MIB, ks=10 * MIB, vs=11 * MIB, t=12 * MIB,
          l=13 * MIB, starts=None, shape=SH, rope=None, **kw):
        rope = rope if rope is not None else pkv.make_rope(**{**dict(num_tokens=4, rotary_dim=128, num_positions=19 * 16), **kw})
        return pkv.lib().kv_rope_append_fp8blk(q, k, v, qn, kn, cs, qo, kp, vp, ks, vs, t, l, starts, ctypes.byref(rope) if rope != 0 else None,
                                               ref(shape), None)
    for x in ("q", "k", "v", "cs", "qo", "kp", "vp", "ks", "vs", "t", "l", "shape"):
        assert f(**{x: None}) == pkv.PKV_ERR_NULL, x              # q or q_out alone as well
    assert f(rope=0) == pkv.PKV_ERR_NULL
    for x in ("q", "k", "v", "qn", "kn", "cs", "qo", "kp", "vp", "ks", "vs"):
        assert f(**{x: 20 * MIB + 8}) == pkv.PKV_ERR_ALIGN, x
    assert f(t=MIB + 2) == f(l=MIB + 1) == f(starts=MIB + 2) == pkv.PKV_ERR_ALIGN
    for kw in (dict(num_tokens=-1), dict(num_tokens=1 << 24), dict(num_tokens=5), dict(rotary_dim=8), dict(num_positions=19 * 16 - 1),
               dict(norm_eps=float("nan")), dict(k_stride=2 * 128 - 8), dict(interleaved=2), dict(shape=bad_shape(head_dim=96))):
        assert f(**kw) == pkv.PKV_ERR_SHAPE, kw
    assert f(qo=2 * MIB) == f(qo=MIB + 16) == pkv.PKV_ERR_SHAPE
    nothing = dict(q=None, k=None, v=None, qn=None, kn=None, cs=None, qo=None, kp=None, vp=None, ks=None, vs=None, t=None, l=None)
    assert f(num_tokens=0, starts=MIB, **nothing) == f(num_tokens=0, shape=NONE, **nothing) == pkv.PKV_OK


T = [Buffer((i + 1) << 20, 1 << 30) for i in range(18)]
SHAPE = pkv.make_shape(4, 8, 2, 19, 128)
ROPE = pkv.make_rope(4, 128, 19 * 16)
CALLS = {
    "paged_decode_attn_fp8blk": (*T[:7], 0.5, T[7], SHAPE, T[8]), "kv_append_fp8blk": (*T[:8], SHAPE),
    "kv_rope_append_fp8blk": (*T[:14], ROPE, SHAPE), "paged_prompt_attn": (*T[:6], 77, 0.5, T[6], SHAPE, T[7]),
    "paged_prompt_attn_fp8kv": (*T[:6], 77, 0.5, 2.0, 4.0, T[6], SHAPE, T[7]),
    "paged_prompt_attn_fp8blk": (*T[:8], 77, 0.5, T[8], SHAPE, T[9]),
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
        monkeypatch.setattr(pkv, "_lib", type("Library", (), {name: staticmethod(record(name)) for name in CALLS}))
        yield log
        return
    if isinstance(pkv._call, pkv._ByCtypes):
        pytest.skip("the module is not built")
    keep, addresses = [], {}
    for name in CALLS:
        plain = [ctypes.c_void_p if hasattr(k, "_type_") and not isinstance(k._type_, str) else k for k in getattr(L, name).argtypes]
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
    assert [a.value if hasattr(a, "value") else as_c(a._obj) if hasattr(a, "_obj") else a for a in args] == [*want, 48]


@pytest.mark.parametrize("module", [False, True])
@pytest.mark.parametrize("name", [n for n in CALLS if "prompt" in n])
def test_numbers_of_tokens(monkeypatch, name, module):
    """Too large ones are refused, not cut to their lower bits; whole numbers of another class are taken."""
    pkv.lib()
    if not module:
        monkeypatch.setattr(pkv, "_call", pkv._ByCtypes())
    args = [NONE if a is SHAPE else a for a in CALLS[name]]
    at = args.index(77)
    for bad in (2 ** 24, 2 ** 63, 2 ** 64 + 5, -2 ** 63 - 1, -1):
        args[at] = bad
        with pytest.raises(pkv.PkvError) as e:
            getattr(pkv, name)(*args, 0)
        assert e.value.status == pkv.PKV_ERR_SHAPE
    for good in (np.int64(5), 0):
        args[at] = good
        getattr(pkv, name)(*args, 0)
    args[at] = 5.0
    with pytest.raises(TypeError):
        getattr(pkv, name)(*args, 0)


def test_longest_contexts():
    """Positions some tiles behind the end of a context are numbered in 32 bits."""
    def shape(most):
        return pkv.make_shape(1, 1, 1, 2 ** 27 - 1, 128, max_context_len=most)
    longest = 2 ** 31 - 4097
    assert pkv.pkv_prompt_workspace_bytes(shape(longest), 1) > 0
    for most in (longest + 1, 0):
        with pytest.raises(pkv.PkvError) as e:
            pkv.pkv_prompt_workspace_bytes(shape(most), 1)
        assert e.value.status == pkv.PKV_ERR_SHAPE
        for name in ("paged_prompt_attn", "paged_prompt_attn_fp8kv", "paged_prompt_attn_fp8blk"):
            assert prompt(name, shape=shape(most), n=1) == pkv.PKV_ERR_SHAPE
        assert pkv.lib().kv_append_fp8blk(MIB, 2 * MIB, 3 * MIB, 4 * MIB, 5 * MIB, 6 * MIB, 7 * MIB, 8 * MIB, ref(shape(most)), None) == pkv.PKV_ERR_SHAPE
        rope = pkv.make_rope(1, 0, 0)
        assert pkv.lib().kv_rope_append_fp8blk(None, MIB, 2 * MIB, None, None, None, None, 3 * MIB, 4 * MIB, 5 * MIB, 6 * MIB, 7 * MIB, 8 * MIB, 9 * MIB,
                                               ctypes.byref(rope), ref(shape(most)), None) == pkv.PKV_ERR_SHAPE
