"""Plain implementations in 64 bits: pools held in 4 bits, attention over what a window and sinks leave, normalised and rotated rows.
Written from the definitions in include/pkv.h, for the tests alone."""
import numpy as np

from paper_2602_11530_amd import workloads as wl

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def tile_bytes(dim):
    return 8 * dim + dim // 2


def code_byte(dim, token, d, is_v):
    """Byte of a tile that holds dim d of a token's codes."""
    if not is_v:
        return (d // 32) * 256 + token * 16 + d % 32 // 2
    w = 4 if dim == 64 else 8
    return ((token // 4 * (dim // w) + d // w) * 4 + token % 4) * (w // 2) + d % w // 2


def _places(dim, is_v):
    d, t = np.meshgrid(np.arange(dim), np.arange(16))
    return np.vectorize(lambda t, d: code_byte(dim, t, d, is_v))(t, d), 8 * dim + d // 32 * 16 + t, d % 2 * 4


def decode(pool, dim, is_v):
    """Tiles [NB, Hkv, units, bytes] -> values [NB, Hkv, B, D]"""
    code_at, scale_at, shift = _places(dim, is_v)
    code, scale = (pool[..., code_at] >> shift) & 15, pool[..., scale_at].astype(np.int64)
    x = np.where(code >= 8, -1.0, 1.0) * E2M1[code & 7]
    x = np.where(scale == 255, np.nan, np.ldexp(x, scale - 127))
    return x.reshape(x.shape[0], x.shape[1], -1, dim)


def quantise(x):
    """Values [..., D] -> codes [..., D] and scale bytes [..., D / 32]"""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    bad = np.isnan(g).any(-1)
    size = np.where(np.isfinite(g), np.abs(g), 2.0 ** 128)
    most = size.max(-1)
    e = np.full(most.shape, -120)
    for k in range(-119, 126):      # as long as the largest is rounded past 6
        e = np.where(most >= 7 * 2.0 ** (k - 1), k, e)
    y = size / 2.0 ** e[..., None]
    middles = (E2M1[1:] + E2M1[:-1]) / 2
    code = np.zeros(y.shape, np.uint8)
    for i, m in enumerate(middles):   # between codes i and i + 1, a tie to the even one
        code = np.where((y > m) | ((y == m) & (i % 2 == 1)), i + 1, code)
    code = (code + 8 * np.signbit(g)).astype(np.uint8)
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def encode(values, is_v):
    """Values [NB, Hkv, B, D] -> tiles"""
    nb, hkv, block, dim = values.shape
    pool = np.zeros((nb, hkv, block // 16, tile_bytes(dim)), np.uint8)
    for t in range(block):
        put(pool, dim, np.arange(nb), np.full(nb, t), values[:, :, t], is_v)
    return pool


def put(pool, dim, ids, slots, rows, is_v):
    """Rows [N, Hkv, D] to slot slots[i] of block ids[i]"""
    code_at, scale_at, _ = _places(dim, is_v)
    code, scale = quantise(rows)
    packed = code[..., 0::2] | code[..., 1::2] << 4
    for i, (b, s) in enumerate(zip(ids, slots)):
        tile = pool[b, :, s // 16]
        tile[:, code_at[s % 16, 0::2]] = packed[i]
        tile[:, scale_at[s % 16, ::32]] = scale[i]


def attention(q, k, v, tables, lens, scale, window=None, sinks=0):
    """Rows in 64 bits and how far fp32 arithmetic and the rounding to bf16 may take a result from them, element by element.

    q [S, Hq, D], pools [NB, Hkv, B, D], all as values.  A score is a sum of D products in fp32, off by at most
    D * 2^-24 * sum |q k|; times the softmax scale, and with the base-2 exponential's own error (2^-22 of a weight and 2^-22 of the score), that is
    a relative error of a weight, twice that of its share; weights are held to 2^-16 as two bf16 numbers and rows are summed in fp32.
    The result is rounded to bf16: 2^-8 of it."""
    S, hq, dim = q.shape
    hkv, block = k.shape[1], k.shape[2]
    out, off = np.zeros(q.shape), np.zeros(q.shape)
    scale = float(np.float32(scale))
    for s in range(S):
        n = max(int(lens[s]), 0)
        t = np.arange(n)
        t = t if window is None else t[(t >= n - window) | (t < sinks)]
        ids = tables[s][t // block]
        t, ids = t[(ids >= 0) & (ids < len(k))], ids[(ids >= 0) & (ids < len(k))]   # ids outside the pool are left out
        if not len(t):
            continue
        rows_k, rows_v = k[ids, :, t % block], v[ids, :, t % block]     # [n, Hkv, D]
        for h in range(hq):
            kk, vv = rows_k[:, h // (hq // hkv)], rows_v[:, h // (hq // hkv)]
            score = kk @ q[s, h] * scale
            p = np.exp(score - score.max())
            p /= p.sum()
            out[s, h] = p @ vv
            d = dim * 2.0 ** -24 * (np.abs(kk) @ np.abs(q[s, h])).max() * scale + 2.0 ** -22 * (1 + np.abs(score).max())
            off[s, h] = (2 * d + 2.0 ** -15) * (p @ np.abs(vv))
    return out, off + 2.0 ** -8 * np.abs(out) + 2.0 ** -130


def within(got_bits, want, off):
    got = wl.bf16_bits_to_f64(np.asarray(got_bits)).reshape(want.shape)
    bad = ~(np.abs(got - want) <= off)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], off[bad][:3])


def turn(x, weight, cos_sin, interleaved, eps):
    """Rows x [T, H, D] with cos_sin [T, R] -> normalised and rotated rows, and the sizes that fp32 errors are relative to."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * weight
    half = cos_sin.shape[-1] // 2
    c, s = cos_sin[:, None, :half].astype(np.float64), cos_sin[:, None, half:].astype(np.float64)
    y, size = x.copy(), np.abs(x)
    one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    size[..., one] = size[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    return y, size


def positions(lens, starts, max_ctx, tokens):
    """(request, position) of each token, (-1, -1) for one that has none"""
    found = [(-1, -1)] * tokens
    for s, n in enumerate(lens):
        n = min(max(int(n), 0), max_ctx)
        a, b = (s, s + 1) if starts is None else (int(starts[s]), int(starts[s + 1]))
        for i in range(a, min(b, tokens)):
            if n - b + i >= 0:
                found[i] = (s, n - b + i)
    return found
