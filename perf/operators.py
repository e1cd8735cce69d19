"""Operators of a decode step around the paged KV cache, with the sizes that a serving program calls them at.

* ``window``  decode attention where each request sees its last ``window`` tokens and its first ``sinks`` ones
* ``fp4``     the cache held in 4 bits: the new token's rows are quantised and appended, then every request attends over its cache
* ``rope``    new tokens of a fused projection: queries and keys are normalised head by head and rotated to their positions, the
              queries go to the attention's input and keys and values into the cache

A case is one pass through one of them.  Lengths belong to the case (so its work is known); the values, the order of the requests
and the placement of their blocks come from the seed.

The 4-bit format: values of E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), 32 dims of a token and KV head with one scale
2^(byte - 127).  A pool holds 16 tokens of a KV head as one tile of 8.5 * D bytes, the codes and then a scale for each of the
D / 32 groups and 16 tokens:
    K codes [D / 32][16 tokens][16 bytes]
    V codes [4][D / w][4 tokens][w / 2 bytes], token t at [t / 4][.][t % 4], w = 4 dims at D = 64, 8 otherwise
"""
import math

import numpy as np
import torch

own = False

K_SCALE, V_SCALE = 0.0134, 0.0171   # 8-bit pools: 448 of them cover 6 and 7.7 sigma
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def _case(name, op, seqs, lo, hi, hq=40, hkv=8, dim=128, block=16, kv="bf16", lens_seed=1, **more):
    c = {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "hq": hq, "hkv": hkv, "dim": dim, "block": block, "kv": kv,
         "mix": "uniform", "lens_seed": lens_seed, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a handful of short requests of a small model shard: nothing but latency
        _case("window_tiny_b4", "window", 4, 17, 300, hq=8, hkv=2, window=64, sinks=4),
        # a layer with a window of a model that alternates them, ordinary full batch
        _case("window_b64", "window", 64, 1024, 8192, window=1024, sinks=4),
        # long reasoning on 8-bit pools, where a window bounds what a step reads
        _case("window_longcot_fp8", "window", 128, 512, 32768, kv="fp8", mix="lognormal", window=4096, sinks=64),
        # narrow heads, 4-bit pools, window and sinks that end inside blocks
        _case("window_d64_fp4", "window", 32, 500, 6000, hq=32, hkv=8, dim=64, block=32, kv="fp4", window=777, sinks=10),
        # one user, one long chain of thought (odd length): interactive latency
        _case("fp4_one_8k", "fp4", 1, 8191, 8191, kv="fp4"),
        # wide heads, 64-token blocks, a few requests
        _case("fp4_d256_b8", "fp4", 8, 1000, 3000, hq=16, hkv=8, dim=256, block=64, kv="fp4"),
        # the ordinary full batch
        _case("fp4_b64", "fp4", 64, 1024, 8192, kv="fp4"),
        # contexts for which a cache in 4 bits is kept
        _case("fp4_b32_long", "fp4", 32, 8192, 32768, kv="fp4"),
        # one new token for each of a handful of requests: latency
        _case("rope_tiny_b4", "rope", 4, 17, 300, hq=8, hkv=2, new_lo=1, new_hi=1, rotary=128, interleaved=False, norm=True),
        # the step of an ordinary full batch
        _case("rope_decode_b64", "rope", 64, 1024, 8192, new_lo=1, new_hi=1, rotary=128, interleaved=False, norm=True),
        # prompts of all lengths in one call
        _case("rope_prompts", "rope", 16, 0, 0, new_lo=100, new_hi=2000, rotary=128, interleaved=False, norm=True),
        # pieces of prompts behind what is cached, narrow heads of which half is rotated in pairs, 8-bit pools
        _case("rope_pieces_d64_fp8", "rope", 24, 0, 4096, hq=32, hkv=8, dim=64, block=32, kv="fp8", new_lo=1, new_hi=900, rotary=32,
              interleaved=True, norm=False),
    ]


_HEADS = [(40, 8), (32, 8), (16, 8), (28, 4), (10, 2), (8, 2), (8, 8), (8, 1)]   # whole models and their shards


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["window", "window", "fp4", "rope", "rope"])
    dim, block = rng.choice([128, 128, 64, 256]), rng.choice([16, 16, 32, 64])
    hq, hkv = rng.choice(_HEADS)
    kv = "fp4" if op == "fp4" else rng.choice(["bf16", "fp8", "fp4"] if op == "window" else ["bf16", "fp8"])
    base = dict(hq=hq, hkv=hkv, dim=dim, block=block, kv=kv, lens_seed=rng.randrange(1, 1 << 30))
    if op == "rope":
        rotary = rng.choice([dim, dim, dim // 2])
        more = dict(base, rotary=rotary, interleaved=rng.random() < 0.3, norm=rng.random() < 0.7)
        if rng.random() < 0.5:           # a step
            hi = _log_int(rng, 16, 8192)
            return _case(None, "rope", _log_int(rng, 1, 512), max(1, int(hi * rng.uniform(0.05, 1.0))), hi, new_lo=1, new_hi=1, **more)
        hi = _log_int(rng, 2, 4096)
        return _case(None, "rope", _log_int(rng, 1, max(1, min(64, (1 << 14) // hi))), 0, rng.choice([0, 1000]), new_lo=max(1, hi // 8), new_hi=hi,
                     **more)
    hi = _log_int(rng, 64, 16384)
    lo = max(1, int(hi * rng.uniform(0.05, 1.0)))
    seqs = _log_int(rng, 1, max(1, min(512, (1 << 29) // (hkv * dim * hi))))
    if op == "fp4":
        return _case(None, "fp4", seqs, lo, hi, **base)
    return _case(None, "window", seqs, lo, hi, window=_log_int(rng, 16, 4096), sinks=rng.choice([0, 1, 4, 4, 16, 70]), **base)


def _lengths(case):
    """Tokens in the cache before the call's own, and the call's own, of each request."""
    rng = np.random.default_rng(case["lens_seed"])
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    if case["mix"] == "lognormal":
        lens = np.clip(np.rint(np.exp(rng.normal(math.log(6000.0), 0.8, size=n))), lo, hi).astype(np.int64)
    else:
        lens = rng.integers(lo, hi + 1, size=n)
    if case["op"] != "rope":
        return lens, np.ones(n, dtype=np.int64)      # the last of them is the call's
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=n)
    return (lens, new) if case["new_hi"] == 1 else (lens + new, new)


def _visible(case, lens):
    w = case.get("window", 1 << 30)
    return np.minimum(lens, w) + np.minimum(case.get("sinks", 0), np.maximum(lens - w, 0))


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _tile_bytes(dim):
    return 8 * dim + dim // 2


def _quantise(x):
    """Values [..., D] in fp32 -> codes [..., D] and scale bytes [..., D / 32].  The scale is the smallest power of two with which no
    value is rounded past 6, codes are the nearest value's, ties to the even one."""
    groups = x.unflatten(-1, (-1, 32))
    most = groups.abs().amax(dim=-1)
    m, e = torch.frexp(most)
    e = (e - 3 + (m >= 0.875).int()).clamp(-120, 125)
    y = torch.ldexp(groups.abs(), -e[..., None])
    code = (y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
    code = code + 8 * torch.signbit(groups).to(torch.uint8)
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _pair(code):
    return code[..., 0::2] | code[..., 1::2] << 4


def _dims_together(dim):
    return 4 if dim == 64 else 8


def _tiles(x, is_v):
    """[..., 16 tokens, D] -> tiles [..., 8.5 D] of K or V."""
    dim = x.shape[-1]
    code, scale = _quantise(x)
    packed = _pair(code)
    if is_v:
        packed = packed.unflatten(-1, (-1, _dims_together(dim) // 2)).unflatten(-3, (4, 4))    # [..., 4, 4 tokens, D / w, w / 2]
        packed = packed.transpose(-3, -2).flatten(-4)
    else:
        packed = packed.unflatten(-1, (-1, 16)).transpose(-3, -2).flatten(-3)
    return torch.cat([packed, scale.transpose(-2, -1).flatten(-2)], dim=-1)


def _pool(case, blocks, g, is_v):
    """One pool of N(0, 1) values: bf16, e4m3 bytes of the values divided by the pool's scale, or tiles."""
    rows = (case["hkv"], case["block"], case["dim"])
    kv = case["kv"]
    if kv == "fp4":
        pool = torch.empty((blocks, case["hkv"], case["block"] // 16, _tile_bytes(case["dim"])), dtype=torch.uint8, device="cuda")
    else:
        pool = torch.empty((blocks,) + rows, dtype=torch.bfloat16 if kv == "bf16" else torch.uint8, device="cuda")
    step = max(1, (1 << 26) // math.prod(rows))
    for b in range(0, blocks, step):
        x = torch.randn((min(step, blocks - b),) + rows, generator=g, device="cuda")
        if kv == "bf16":
            pool[b:b + step] = x
        elif kv == "fp8":
            pool[b:b + step] = (x / (V_SCALE if is_v else K_SCALE)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            pool[b:b + step] = _tiles(x.bfloat16().float().unflatten(2, (-1, 16)), is_v)
    return pool


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    order = rng.permutation(case["seqs"])
    lens, new = (x[order] for x in _lengths(case))
    used = (lens + case["block"] - 1) // case["block"]
    n_pool, width = int(used.sum()), int(used.max())
    ids = rng.permutation(n_pool).astype(np.int32)
    tables = np.full((case["seqs"], width), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(used):
        tables[s, :n] = ids[at:at + n]
        at += n
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    state = {"case": case, "most": int(lens.max()), "tables": torch.from_numpy(tables).cuda(),
             "lens": torch.from_numpy(lens.astype(np.int32)).cuda(), "scale": 1.0 / math.sqrt(dim),
             "k_pool": _pool(case, n_pool, g, False), "v_pool": _pool(case, n_pool, g, True)}
    tokens = int(new.sum())
    if case["op"] == "rope":
        # one row per token: the queries, the keys and the values of all heads, as one projection gives them
        state["qkv"] = normal(tokens, (hq + 2 * hkv) * dim)
        state["norms"] = [(1 + normal(dim) / 8) if case["norm"] else None for _ in range(2)]
        angle = torch.arange(state["most"], dtype=torch.float64)[:, None] * 1e6 ** (
            -torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).float().cuda()
        state["starts"] = None if case["new_hi"] == 1 else torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        state["q_out"] = torch.empty((tokens, hq, dim), dtype=torch.bfloat16, device="cuda")
    else:
        state["q"] = normal(tokens, hq, dim)
        state["out"] = torch.empty_like(state["q"])
    if case["op"] == "fp4":
        state["k_new"], state["v_new"] = normal(tokens, hkv, dim), normal(tokens, hkv, dim)
    if own:
        from paper_2602_11530_amd import binding as pkv
        state["shape"] = pkv.make_shape(case["seqs"], hq, hkv, width, n_pool, head_dim=dim, block_size=case["block"],
                                        max_context_len=state["most"])
        if case["op"] == "rope":
            row = (hq + 2 * hkv) * dim
            state["rope"] = pkv.make_rope(tokens, case["rotary"], state["most"], interleaved=case["interleaved"], norm_eps=EPS,
                                          q_stride=row, k_stride=row, v_stride=row)
        else:
            state["ws"] = torch.empty(pkv.pkv_attn_workspace_bytes(state["shape"]), dtype=torch.uint8, device="cuda")
    return state


# ---------------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"window": _plain_window, "fp4": _plain_fp4, "rope": _plain_rope}[case["op"]](state, case)


def _run_own(state, case):
    from paper_2602_11530_amd import binding as pkv
    tables, lens, shape, kv = state["tables"], state["lens"], state["shape"], case["kv"]
    k_pool, v_pool = state["k_pool"], state["v_pool"]
    if case["op"] == "rope":
        hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
        qkv = state["qkv"]
        args = (qkv, qkv[:, hq * dim:], qkv[:, (hq + hkv) * dim:], *state["norms"], state["cos_sin"], state["q_out"], k_pool, v_pool, tables, lens,
                state["starts"])
        if kv == "fp8":
            pkv.kv_rope_append_fp8(*args, K_SCALE, V_SCALE, state["rope"], shape)
            return [state["q_out"], k_pool.view(torch.float8_e4m3fn), v_pool.view(torch.float8_e4m3fn)]
        pkv.kv_rope_append(*args, state["rope"], shape)
        return [state["q_out"], k_pool, v_pool]
    attn = (state["q"], k_pool, v_pool, tables, lens, state["scale"])
    if case["op"] == "fp4":
        pkv.kv_append_fp4(state["k_new"], state["v_new"], k_pool, v_pool, tables, lens, shape)
        pkv.paged_decode_attn_fp4kv(*attn, state["out"], shape, state["ws"])
        return [state["out"], k_pool, v_pool]
    span = (case["window"], case["sinks"])
    if kv == "fp8":
        pkv.paged_decode_attn_window_fp8kv(*attn, K_SCALE, V_SCALE, *span, state["out"], shape, state["ws"])
    elif kv == "fp4":
        pkv.paged_decode_attn_window_fp4kv(*attn, *span, state["out"], shape, state["ws"])
    else:
        pkv.paged_decode_attn_window(*attn, *span, state["out"], shape, state["ws"])
    return [state["out"]]


def _values(dtype=torch.float32):
    half = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    return torch.tensor(half + [-x for x in half], dtype=dtype, device="cuda")


def _codes(tiles, dim, is_v):
    """Tiles [..., 8.5 D] -> bytes of codes [..., 16 tokens, D / 2] and of scales [..., 16 tokens, D / 32]"""
    packed, scale = tiles[..., :8 * dim], tiles[..., 8 * dim:]
    if is_v:
        w = _dims_together(dim)
        packed = packed.unflatten(-1, (4, dim // w, 4, w // 2)).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    else:
        packed = packed.unflatten(-1, (dim // 32, 16, 16)).transpose(-3, -2).flatten(-2)
    return packed, scale.unflatten(-1, (dim // 32, 16)).transpose(-2, -1)


def _widen(packed, scale):
    code = torch.stack([packed & 15, packed >> 4], dim=-1).flatten(-2)
    x = _values()[code.int()].unflatten(-1, (-1, 32))
    return (x * torch.exp2(scale.float() - 127)[..., None]).flatten(-2)


def _rows(state, case, pool, positions, is_v):
    """Rows at each request's positions [S, N], in fp32: [S, Hkv, N, D]"""
    at = positions.clamp(min=0)
    block, slot = case["block"], at % case["block"]
    ids = state["tables"].gather(1, at // block).clamp(min=0)
    if case["kv"] == "fp4":
        packed, scale = _codes(pool, case["dim"], is_v)                        # views of the pool
        x = _widen(packed[ids, :, slot // 16, slot % 16], scale[ids, :, slot // 16, slot % 16])
    else:
        x = pool[ids, :, slot]
        if case["kv"] == "fp8":
            x = x.view(torch.float8_e4m3fn).float() * (V_SCALE if is_v else K_SCALE)
    return x.float().transpose(1, 2).contiguous()


def _attend(state, case, positions, seen):
    """Softmax attention over the rows at positions [S, N] of which `seen` says which count."""
    group = case["hq"] // case["hkv"]
    k, v = _rows(state, case, state["k_pool"], positions, False), _rows(state, case, state["v_pool"], positions, True)
    q = state["q"].float().unflatten(1, (case["hkv"], group))
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * state["scale"]
    seen = seen[:, None, None, :]
    score = torch.where(seen, score, -torch.inf)
    most = score.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    weight = torch.where(seen, torch.exp(score - most), 0.0)
    total = weight.sum(dim=-1, keepdim=True)
    v = torch.where(seen[:, 0, 0, :, None][:, None], v, 0.0)
    out = torch.matmul(weight, v) / torch.where(total > 0, total, 1.0)
    state["out"].copy_(out.flatten(1, 2))
    return state["out"]


def _plain_window(state, case):
    lens = state["lens"].long()[:, None]
    back = min(case["window"], state["most"])
    first = torch.arange(min(case["sinks"], state["most"]), device="cuda")[None, :].expand(len(lens), -1)
    last = lens - back + torch.arange(back, device="cuda")[None, :]
    seen = torch.cat([first < lens - case["window"], last >= 0], dim=1)        # a first token inside the window counts there
    return [_attend(state, case, torch.cat([first, last], dim=1), seen)]


def _plain_fp4(state, case):
    dim, lens = case["dim"], state["lens"].long()
    at = lens - 1
    slot = at % case["block"]
    ids = state["tables"].gather(1, (at // case["block"])[:, None])[:, 0].long()
    for pool, new, is_v in ((state["k_pool"], state["k_new"], False), (state["v_pool"], state["v_new"], True)):
        code, scale = _quantise(new.float())
        groups = pool[..., 8 * dim:].unflatten(-1, (dim // 32, 16))
        groups[ids, :, slot // 16, :, slot % 16] = scale
        packed = _pair(code)
        if is_v:
            w = _dims_together(dim)
            tiles = pool[..., :8 * dim].unflatten(-1, (4, dim // w, 4, w // 2))
            tiles[ids, :, slot // 16, slot % 16 // 4, :, slot % 4] = packed.unflatten(-1, (-1, w // 2))
        else:
            tiles = pool[..., :8 * dim].unflatten(-1, (dim // 32, 16, 16))
            tiles[ids, :, slot // 16, :, slot % 16] = packed.unflatten(-1, (-1, 16))
    positions = torch.arange(state["most"], device="cuda")[None, :].expand(len(lens), -1)
    out = _attend(state, case, positions, positions < lens[:, None])
    # codes and scales of the new rows are exact (the scale is a power of two), so they are compared as they are
    return [out, state["k_pool"], state["v_pool"]]


def _positions(state, case):
    """Request and position of each new token."""
    lens = state["lens"].long()
    if state["starts"] is None:
        return torch.arange(len(lens), device="cuda"), lens - 1
    starts = state["starts"].long()
    token = torch.arange(len(state["qkv"]), device="cuda")
    request = torch.searchsorted(starts, token, right=True) - 1
    return request, lens[request] - (starts[request + 1] - token)


def _turned(x, norm, cos, sin, interleaved):
    """[T, H, D] in fp32, normalised and with its first dims rotated."""
    if norm is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * norm.float()
    n = cos.shape[-1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], dim=-1).flatten(-2) if interleaved else torch.cat([c, d], dim=-1)
    return torch.cat([turned, x[..., 2 * n:]], dim=-1)


def _plain_rope(state, case):
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    request, position = _positions(state, case)
    cos, sin = state["cos_sin"][position].unsqueeze(1).chunk(2, dim=-1)
    q, k, v = state["qkv"].unflatten(1, (-1, dim)).float().split([hq, hkv, hkv], dim=1)
    state["q_out"].copy_(_turned(q, state["norms"][0], cos, sin, case["interleaved"]))
    ids = state["tables"][request, position // case["block"]].long()
    slot = position % case["block"]
    pools = []
    for pool, x, scale in ((state["k_pool"], _turned(k, state["norms"][1], cos, sin, case["interleaved"]), K_SCALE), (state["v_pool"], v, V_SCALE)):
        if case["kv"] == "fp8":
            pool[ids, :, slot] = (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            pools.append(pool.view(torch.float8_e4m3fn))
        else:
            pool[ids, :, slot] = x.bfloat16()
            pools.append(pool)
    return [state["q_out"], *pools]


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _row_bytes(case):
    return case["hkv"] * case["dim"] * {"bf16": 32, "fp8": 16, "fp4": 8.5}[case["kv"]] / 16


def work(case):
    lens, new = _lengths(case)
    tokens, seqs, dim = int(new.sum()), case["seqs"], case["dim"]
    if case["op"] == "rope":
        rows = tokens * (2 * case["hq"] + 2 * case["hkv"]) * dim * 2 + 2 * tokens * _row_bytes(case)   # in and out
        table = tokens * case["rotary"] * 4 + 4 * int(((new + case["block"] - 1) // case["block"]).sum()) + 8 * seqs
        return {"bytes": rows + table, "flops": tokens * (case["hq"] + case["hkv"]) * (3 * case["rotary"] + (4 * dim if case["norm"] else 0))}
    seen = _visible(case, lens)
    total = int(seen.sum())
    moved = 2 * total * _row_bytes(case) + 2 * tokens * case["hq"] * dim * 2
    moved += 4 * int(((seen + case["block"] - 1) // case["block"]).sum()) + 4 * seqs
    if case["op"] == "fp4":
        moved += 2 * tokens * (case["hkv"] * dim * 2 + _row_bytes(case))
    return {"bytes": moved, "flops": 4 * total * case["hq"] * dim}


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_rope(state, case) if case["op"] == "rope" else _exact_attention(state, case)


def _fp4_value(pool, ids, n, dim, is_v):
    """The first n tokens of the blocks listed, in 64 bits: [n, Hkv, D], from the format's definition, nibble by nibble."""
    tile = pool[ids]                                                         # [blocks, Hkv, units, bytes]
    dims, tokens = torch.arange(dim, device="cuda"), torch.arange(16, device="cuda")[:, None]
    if is_v:
        w = 4 if dim == 64 else 8
        byte = (tokens // 4) * (4 * dim // w) * (w // 2) + (dims // w) * 4 * (w // 2) + (tokens % 4) * (w // 2) + dims % w // 2
    else:
        byte = (dims // 32) * 256 + tokens * 16 + dims % 32 // 2
    code = tile[..., byte] >> (dims % 2 * 4).to(torch.uint8) & 15            # [blocks, Hkv, units, 16, D]
    power = tile[..., 8 * dim + (dims // 32) * 16 + tokens].double() - 127
    low, sign = (code & 7).double(), 1 - 2 * (code >> 3).double()
    size = torch.where(low < 2, low / 2, (1 + low % 2 / 2) * torch.exp2(torch.floor(low / 2) - 1))
    x = (sign * size * torch.exp2(power)).permute(0, 2, 3, 1, 4)
    return x.reshape(-1, x.shape[3], dim)[:n]


def _exact_attention(state, case):
    lens, tables, dim = state["lens"].tolist(), state["tables"].long(), case["dim"]
    group = case["hq"] // case["hkv"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        ids = tables[s, :(n + case["block"] - 1) // case["block"]]
        rows = []
        for pool, pool_scale, is_v in ((state["k_pool"], K_SCALE, False), (state["v_pool"], V_SCALE, True)):
            if case["kv"] == "fp4":
                x = _fp4_value(pool, ids, n, dim, is_v)
            else:
                x = pool[ids]
                if case["kv"] == "fp8":
                    x = x.view(torch.float8_e4m3fn).double() * float(np.float32(pool_scale))
                x = x.double().permute(0, 2, 1, 3).reshape(-1, case["hkv"], dim)[:n]
            rows.append(x)
        if case["op"] == "fp4":                                              # the call's own token
            for x, new in zip(rows, (state["k_new"], state["v_new"])):
                values = new[s].double().reshape(case["hkv"], -1, 32)
                most = values.abs().amax(dim=-1, keepdim=True)
                power = torch.floor(torch.log2(most)) - 2
                power = power + (most >= 7 * torch.exp2(power))
                grid = _values(torch.float64)[:8]
                y = values.abs() / torch.exp2(power)
                # of two values at the same distance the even code's: its neighbours' middles are 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5
                code = (y[..., None] > (grid[1:] + grid[:-1]) / 2).sum(-1)
                tie = (y[..., None] == (grid[1:] + grid[:-1]) / 2).any(-1)
                code = code + (tie & (code % 2 == 1))
                x[n - 1] = (torch.sign(values) * grid[code] * torch.exp2(power)).reshape(case["hkv"], dim)
        t = torch.arange(n, device="cuda")
        seen = (t >= n - case["window"]) | (t < case["sinks"]) if case["op"] == "window" else t >= 0
        k, v = (x[seen].permute(1, 0, 2).contiguous() for x in rows)
        q = state["q"][s].double().view(case["hkv"], group, dim)
        p = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) * float(np.float32(state["scale"])), dim=-1)
        out[s] = torch.bmm(p, v).reshape(case["hq"], dim)
    return [out, None, None] if case["op"] == "fp4" else [out]


def _exact_rope(state, case):
    hq, hkv, dim, block = case["hq"], case["hkv"], case["dim"], case["block"]
    lens = state["lens"].tolist()
    starts = list(range(len(lens) + 1)) if state["starts"] is None else state["starts"].tolist()
    position = torch.cat([torch.arange(n - (b - a), n) for n, a, b in zip(lens, starts, starts[1:])]).cuda()
    request = torch.cat([torch.full((b - a,), s) for s, (a, b) in enumerate(zip(starts, starts[1:]))]).cuda()
    table = state["cos_sin"][position].double()
    half = case["rotary"] // 2
    factor = torch.complex(table[:, :half], table[:, half:])[:, None, :]     # a rotation is a product of complex numbers

    def turn(x, norm):
        x = x.double()
        if norm is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / dim + EPS) * norm.double()
        y = x.clone()
        one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * factor
        y[..., one], y[..., two] = z.real, z.imag
        return y

    x = state["qkv"].view(-1, hq + 2 * hkv, dim)
    q = turn(x[:, :hq], state["norms"][0])
    ids = state["tables"].long()[request, position // block]
    pools = []
    for pool, new, scale in ((state["k_pool"], turn(x[:, hq:hq + hkv], state["norms"][1]), K_SCALE), (state["v_pool"], x[:, hq + hkv:].double(), V_SCALE)):
        values = pool.view(torch.float8_e4m3fn).double() if case["kv"] == "fp8" else pool.double()
        values[ids, :, position % block] = (new / float(np.float32(scale))).clamp(-448, 448) if case["kv"] == "fp8" else new
        pools.append(values)
    return [q, *pools]
