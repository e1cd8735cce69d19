"""Batches, pools of the three kinds and the attention calls over them, for the GPU tests of windows, 4-bit pools and rotated appends."""
import types

import numpy as np
import torch

import plain
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl

KINDS = ["bf16", "fp8", "fp4"]
K_SCALE, V_SCALE = 0.0134, 0.0171


def make_batch(lens, hq, hkv, dim, block, seed, spare=0):
    """Lengths, tables over a shuffled pool that holds them (unused entries are -1), and queries."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    used = (lens + block - 1) // block
    b = types.SimpleNamespace(lens=lens, hq=hq, hkv=hkv, dim=dim, block=block, rng=rng, scale=1 / np.sqrt(dim),
                              num_blocks=max(int(used.sum()) + spare, 1))
    b.tables = wl.make_tables(lens, b.num_blocks, rng, block_size=block)
    b.q_bits = wl.normal_bf16(rng, (len(lens), hq, dim))
    b.q = wl.bf16_bits_to_f64(b.q_bits).reshape(len(lens), hq, dim)
    return b


def pools_of(b, kind):
    """K and V as the device holds them, and their values in 64 bits."""
    shape = (b.num_blocks, b.hkv, b.block, b.dim)
    p = types.SimpleNamespace(kind=kind)
    if kind == "bf16":
        p.k_bits, p.v_bits = wl.normal_bf16(b.rng, shape), wl.normal_bf16(b.rng, shape)
        p.k, p.v = (wl.bf16_bits_to_f64(x).reshape(shape) for x in (p.k_bits, p.v_bits))
    elif kind == "fp8":
        p.k_bits, p.v_bits = wl.normal_e4m3(b.rng, shape, K_SCALE), wl.normal_e4m3(b.rng, shape, V_SCALE)
        p.k, p.v = (e4m3(x) * float(np.float32(s)) for x, s in ((p.k_bits, K_SCALE), (p.v_bits, V_SCALE)))
    else:
        values = [b.rng.standard_normal(shape) * 2.0 ** b.rng.integers(-3, 4, (*shape[:3], 1)) for _ in range(2)]
        p.k_bits, p.v_bits = tiles(values[0], False), tiles(values[1], True)
        p.k, p.v = plain.decode(p.k_bits, b.dim, False), plain.decode(p.v_bits, b.dim, True)
    p.k_dev, p.v_dev = to_dev(p.k_bits), to_dev(p.v_bits)
    return p


def tiles(values, is_v):
    """plain.encode, all rows of a tile at once."""
    nb, hkv, block, dim = values.shape
    code, scale = plain.quantise(values.reshape(nb, hkv, block // 16, 16, dim))
    code_at, scale_at, _ = plain._places(dim, is_v)
    pool = np.zeros((nb, hkv, block // 16, plain.tile_bytes(dim)), np.uint8)
    pool[..., code_at[:, 0::2]] = code[..., 0::2] | code[..., 1::2] << 4
    pool[..., scale_at[:, ::32]] = scale
    return pool


def e4m3(x):
    return torch.from_numpy(np.ascontiguousarray(x)).view(torch.float8_e4m3fn).double().numpy()


def poison(p, kind, where):
    """NaN in all tokens [NB, B] of the device's pools where it says so; in tiles the bytes of a token are its own."""
    for name, is_v in (("k", False), ("v", True)):
        bits = getattr(p, name + "_bits").copy()
        if kind == "fp4":
            dim = bits.shape[-1] * 2 // 17
            code_at, scale_at, _ = plain._places(dim, is_v)
            for b, s in np.argwhere(where):
                bits[b, :, s // 16, code_at[s % 16]] = 0xff
                bits[b, :, s // 16, scale_at[s % 16]] = 0xff
        else:
            bits[np.broadcast_to(where[:, None, :, None], bits.shape)] = wl.BF16_NAN if kind == "bf16" else wl.E4M3_NAN
        setattr(p, name + "_dev", to_dev(bits))


def shape_of(b, max_context_len=0, partition_size=0, num_seqs=None):
    return pkv.make_shape(len(b.lens) if num_seqs is None else num_seqs, b.hq, b.hkv, b.tables.shape[1], b.num_blocks, b.dim, b.block, partition_size,
                          max_context_len)


def attend(b, p, window=None, sinks=None, max_context_len=0, partition_size=0, q=None, out=None, stream=None, wait=True):
    """Attention over the whole context, or what a window and sinks leave: bits on the host, or the device's tensor if it is not waited for."""
    shape = shape_of(b, max_context_len, partition_size)
    ws = torch.full((max(pkv.pkv_attn_workspace_bytes(shape), 16),), 0xa5, dtype=torch.uint8, device="cuda")
    q = to_dev(b.q_bits) if q is None else q
    if out is None:
        out = torch.full(b.q.shape, 0x7FC1, dtype=torch.int16, device="cuda")
    tables, lens = to_dev(b.tables), to_dev(b.lens)
    if stream is not None:
        torch.cuda.synchronize()     # what the call reads was made on another stream
    name = "paged_decode_attn" + ("" if window is None else "_window") + {"bf16": "", "fp8": "_fp8kv", "fp4": "_fp4kv"}[p.kind]
    scales = (K_SCALE, V_SCALE) if p.kind == "fp8" else ()
    span = () if window is None else (window, sinks)
    getattr(pkv, name)(q, p.k_dev, p.v_dev, tables, lens, float(b.scale), *scales, *span, out, shape, ws, stream)
    if not wait:
        out.kept = (q, tables, lens, ws)
        return out
    torch.cuda.synchronize()
    return to_bits(out)
