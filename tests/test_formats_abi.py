"""Argument checks of the calls for windows, 4-bit pools and rotated appends: errors before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2602_11530_amd import binding as pkv

SH = pkv.make_shape(4, 8, 2, 19, 128)
NONE = pkv.make_shape(0, 8, 2, 19, 128)
MIB = 1 << 20


def attend(name, q=MIB, k=2 * MIB, v=3 * MIB, t=4 * MIB, l=5 * MIB, o=6 * MIB, window=5, sinks=1, ks=1.0, vs=1.0, shape=SH, ws=7 * MIB, nb=None):
    need = nb if nb is not None else pkv.pkv_attn_workspace_bytes(SH)
    scales = (ks, vs) if name.endswith("fp8kv") else ()
    span = (window, sinks) if "window" in name else ()
    return getattr(pkv.lib(), name)(q, k, v, t, l, 1.0, *scales, *span, o, ctypes.byref(shape) if shape is not None else None, ws, need, None)


@pytest.mark.parametrize("name", ["paged_decode_attn_window", "paged_decode_attn_window_fp8kv", "paged_decode_attn_window_fp4kv",
                                  "paged_decode_attn_fp4kv"])
def test_attention(name):
    need = pkv.pkv_attn_workspace_bytes(SH)
    for x in ("q", "k", "v", "t", "l", "o", "shape"):
        assert attend(name, **{x: None}) == pkv.PKV_ERR_NULL
    for x in ("q", "k", "v", "o", "ws"):
        assert attend(name, **{x: MIB + 8}) == pkv.PKV_ERR_ALIGN
    for x in ("t", "l"):
        assert attend(name, **{x: MIB + 2}) == pkv.PKV_ERR_ALIGN
    assert attend(name, ws=None) == pkv.PKV_ERR_WORKSPACE and attend(name, nb=need - 1) == pkv.PKV_ERR_WORKSPACE
    for bad in (dict(head_dim=96), dict(block_size=48), dict(num_kv_heads=3), dict(head_dim=256, num_q_heads=32), dict(num_seqs=2049)):
        assert attend(name, shape=pkv.make_shape(**{**dict(num_seqs=4, num_q_heads=8, num_kv_heads=2, max_blocks_per_seq=19,
                                                           num_pool_blocks=128), **bad})) == pkv.PKV_ERR_SHAPE
    if "window" in name:
        assert attend(name, window=-1) == attend(name, sinks=-1) == attend(name, window=-2 ** 31) == pkv.PKV_ERR_SHAPE
        assert attend(name, window=-1, shape=NONE) == pkv.PKV_ERR_SHAPE     # wrong for any batch
    if name.endswith("fp8kv"):
        for ks, vs in ((0.0, 1.0), (1.0, -2.0), (float("nan"), 1.0), (1.0, float("inf"))):
            assert attend(name, ks=ks, vs=vs) == pkv.PKV_ERR_SHAPE
    assert attend(name, q=None, k=None, v=None, t=None, l=None, o=None, shape=NONE, ws=None, nb=0) == pkv.PKV_OK


def test_append_fp4():
    f = lambda kn=MIB, vn=2 * MIB, k=3 * MIB, v=4 * MIB, t=5 * MIB, l=6 * MIB, shape=SH: pkv.lib().kv_append_fp4(  # noqa: E731
        kn, vn, k, v, t, l, ctypes.byref(shape) if shape is not None else None, None)
    for x in ("kn", "vn", "k", "v", "t", "l", "shape"):
        assert f(**{x: None}) == pkv.PKV_ERR_NULL
    for x in ("kn", "vn", "k", "v"):
        assert f(**{x: MIB + 8}) == pkv.PKV_ERR_ALIGN
    assert f(t=MIB + 2) == f(l=MIB + 1) == pkv.PKV_ERR_ALIGN
    assert f(shape=pkv.make_shape(4, 8, 2, 19, 128, head_dim=96)) == pkv.PKV_ERR_SHAPE
    assert f(kn=None, vn=None, k=None, v=None, t=None, l=None, shape=NONE) == pkv.PKV_OK


@pytest.mark.parametrize("dim,block,hkv", [(64, 16, 1), (128, 32, 8), (256, 64, 3)])
def test_block_bytes(dim, block, hkv):
    shape = pkv.make_shape(4, hkv, hkv, 19, 128, head_dim=dim, block_size=block)
    assert pkv.pkv_fp4_block_bytes(shape) == hkv * block * dim * 17 // 32
    assert pkv.pkv_fp4_block_bytes(shape) % 16 == 0          # as the copies take it
    assert pkv.lib().pkv_fp4_block_bytes(ctypes.byref(shape), None) == pkv.PKV_ERR_NULL
    shape.block_size = 8
    with pytest.raises(pkv.PkvError) as e:
        pkv.pkv_fp4_block_bytes(shape)
    assert e.value.status == pkv.PKV_ERR_SHAPE


def rope_call(name, q=MIB, k=2 * MIB, v=3 * MIB, qn=4 * MIB, kn=5 * MIB, cs=6 * MIB, qo=7 * MIB, kp=8 * MIB, vp=9 * MIB, t=10 * MIB, l=11 * MIB,
              starts=None, ks=1.0, vs=1.0, shape=SH, rope=None, **kw):
    rope = rope if rope is not None else pkv.make_rope(**{**dict(num_tokens=4, rotary_dim=128, num_positions=19 * 16), **kw})
    scales = (ks, vs) if name.endswith("fp8") else ()
    return getattr(pkv.lib(), name)(q, k, v, qn, kn, cs, qo, kp, vp, t, l, starts, *scales, ctypes.byref(rope) if rope != 0 else None,
                                    ctypes.byref(shape) if shape is not None else None, None)


@pytest.mark.parametrize("name", ["kv_rope_append", "kv_rope_append_fp8", "kv_rope_append_fp4"])
def test_rope_append(name):
    f = lambda **kw: rope_call(name, **kw)  # noqa: E731
    for x in ("q", "k", "v", "cs", "qo", "kp", "vp", "t", "l", "shape"):
        assert f(**{x: None}) == pkv.PKV_ERR_NULL, x
    assert f(rope=0) == pkv.PKV_ERR_NULL
    for x in ("q", "k", "v", "qn", "kn", "cs", "qo", "kp", "vp"):
        assert f(**{x: 20 * MIB + 8}) == pkv.PKV_ERR_ALIGN, x
    assert f(t=MIB + 2) == f(l=MIB + 1) == f(starts=MIB + 2) == pkv.PKV_ERR_ALIGN
    bad = [dict(num_tokens=-1), dict(num_tokens=1 << 24), dict(num_tokens=5), dict(rotary_dim=-16), dict(rotary_dim=8), dict(rotary_dim=144),
           dict(num_positions=19 * 16 - 1), dict(norm_eps=-1e-6), dict(norm_eps=float("nan")), dict(norm_eps=float("inf")),
           dict(q_stride=8 * 128 - 8), dict(k_stride=2 * 128 - 8), dict(v_stride=8), dict(q_stride=-1024), dict(k_stride=2 ** 31 + 8),
           dict(shape=pkv.make_shape(4, 8, 2, 19, 128, head_dim=96)), dict(interleaved=2)]
    for kw in bad:
        assert f(**kw) == pkv.PKV_ERR_SHAPE, kw
    assert f(q_stride=8 * 128 + 4) == pkv.PKV_ERR_ALIGN
    # queries written where rows are still to be read
    assert f(qo=MIB + 16) == f(qo=2 * MIB) == f(qo=3 * MIB - 16) == pkv.PKV_ERR_SHAPE
    assert f(qo=MIB, q_stride=8 * 128 + 8) == pkv.PKV_ERR_SHAPE      # in place only without gaps
    if name.endswith("fp8"):
        for ks, vs in ((0.0, 1.0), (1.0, -2.0), (float("nan"), 1.0), (1.0, float("inf"))):
            assert f(ks=ks, vs=vs) == pkv.PKV_ERR_SHAPE
    nothing = dict(q=None, k=None, v=None, qn=None, kn=None, cs=None, qo=None, kp=None, vp=None, t=None, l=None)
    assert f(num_tokens=0, starts=MIB, **nothing) == pkv.PKV_OK
    assert f(num_tokens=0, shape=NONE, **nothing) == pkv.PKV_OK
    assert f(num_tokens=0) == pkv.PKV_ERR_SHAPE                      # one token for each of four requests
    # a table of positions is only needed where something is rotated
    assert f(num_positions=0) == pkv.PKV_ERR_SHAPE and f(num_positions=0, rotary_dim=0, cs=None, q=None) == pkv.PKV_ERR_NULL
