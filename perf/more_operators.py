"""Operators around prompts and around a cache held in 8 bits with scales of its own for each block, with the sizes that a serving program calls
them at.

* ``prompt``  causal attention of new tokens, whole prompts or pieces of them, packed one request behind the other, over the paged cache that
              already holds their keys and values: bf16 pools, e4m3 pools with a scale each (``fp8``) or with one for each block and head (``blk``)
* ``step``    a decode step over ``blk`` pools: the new token's rows are quantised and appended, then every request attends over its cache
* ``append``  new tokens of a fused projection into ``blk`` pools: queries and keys are rotated to their positions, queries go to the
              attention's input, keys and values are quantised and go into the cache

A case is one pass through one of them.  Lengths belong to the case (so its work is known); the values, the order of the requests
and the placement of their blocks come from the seed.

The ``blk`` format: bytes of E4M3 (largest value 448) and for each physical block and KV head a byte b that stands for a scale of 2^(b - 127).
The scales of a pool are an array [blocks][Hkv, rounded up to 16] of their own.  An append gives a block whose first token it writes the smallest
scale, from 2^-117 to 2^119, with which no value that it writes there is beyond 448; a block that held tokens before keeps its scale or takes a
larger one if it has to, and then what it held is rounded to that.
"""
import math

import numpy as np
import torch

own = False

K_SCALE, V_SCALE = 0.0134, 0.0171   # pools with one scale: 448 of them cover 6 and 7.7 sigma
LEAST, MOST = -117, 119             # powers of two of a block's scale


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def _case(name, op, seqs, lo, hi, new_lo=1, new_hi=1, hq=40, hkv=8, dim=128, block=16, kv="bf16", lens_seed=1, **more):
    """`lo` and `hi` bound the tokens that a request has in the cache: before the call's own (prompt, append), or with the one (step)."""
    c = {"op": op, "seqs": seqs, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "hq": hq, "hkv": hkv, "dim": dim, "block": block, "kv": kv,
         "lens_seed": lens_seed, **more}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a handful of short prompts of a small model shard: nothing but latency
        _case("prompt_tiny_b4", "prompt", 4, 0, 0, 17, 120, hq=8, hkv=2),
        # prompts of all lengths in one call
        _case("prompt_b16", "prompt", 16, 0, 0, 100, 2000),
        # one long document (odd length)
        _case("prompt_one_8k", "prompt", 1, 0, 0, 8191, 8191),
        # pieces of prompts behind what is cached, narrow heads, 8-bit pools
        _case("prompt_pieces_d64_fp8", "prompt", 24, 0, 4096, 1, 900, hq=32, hkv=8, dim=64, block=32, kv="fp8"),
        # a piece of one very long prompt behind 32 thousand tokens, 8-bit pools with a scale for each block
        _case("prompt_piece_long_blk", "prompt", 1, 32000, 32000, 512, 512, kv="blk"),
        # a few drafted tokens of every request of an ordinary batch, to be verified at once
        _case("prompt_drafts_b32", "prompt", 32, 1000, 8000, 4, 4),
        # wide heads, 64-token blocks
        _case("prompt_d256_b8", "prompt", 8, 0, 1000, 200, 1500, hq=16, hkv=8, dim=256, block=64),
        # a step of a handful of short requests of a small model shard: nothing but latency
        _case("step_tiny_b4", "step", 4, 17, 300, hq=8, hkv=2, kv="blk"),
        # the ordinary full batch
        _case("step_b64", "step", 64, 1024, 8192, kv="blk"),
        # contexts for which a cache in 8 bits is kept, narrow heads, 32-token blocks
        _case("step_d64_b32_long", "step", 32, 8192, 32768, hq=32, hkv=8, dim=64, block=32, kv="blk"),
        # prompts of all lengths in one call
        _case("append_prompts", "append", 16, 0, 0, 100, 2000, kv="blk", rotary=128, interleaved=False),
        # pieces of prompts behind what is cached, narrow heads of which half is rotated in pairs, 64-token blocks
        _case("append_pieces_d64", "append", 24, 0, 4096, 1, 900, hq=32, hkv=8, dim=64, block=64, kv="blk", rotary=32, interleaved=True),
    ]


_HEADS = [(40, 8), (32, 8), (16, 8), (28, 4), (10, 2), (8, 2), (8, 8), (8, 1)]   # whole models and their shards


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "prompt", "step", "step", "append"])
    dim, block = rng.choice([128, 128, 64, 256]), rng.choice([16, 16, 32, 64])
    hq, hkv = rng.choice(_HEADS)
    kv = rng.choice(["bf16", "fp8", "blk"]) if op == "prompt" else "blk"
    base = dict(hq=hq, hkv=hkv, dim=dim, block=block, kv=kv, lens_seed=rng.randrange(1, 1 << 30))
    if op == "append":
        new_hi = _log_int(rng, 2, 4096)
        return _case(None, op, _log_int(rng, 1, max(1, min(64, (1 << 14) // new_hi))), 0, rng.choice([0, 1000]), max(1, new_hi // 8), new_hi,
                     rotary=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.3, **base)
    if op == "step":
        hi = _log_int(rng, 64, 16384)
        return _case(None, op, _log_int(rng, 1, max(1, min(512, (1 << 29) // (hkv * dim * hi)))), max(1, int(hi * rng.uniform(0.05, 1.0))), hi,
                     **base)
    new_hi = _log_int(rng, 1, 6000)
    new_lo = max(1, int(new_hi * rng.uniform(0.05, 1.0)))
    hi = rng.choice([0, 0, _log_int(rng, 16, 16384)])
    limit = 2 ** 25 * 40 * 128 // (hq * dim)         # pairs of a query and a key in one prompt of 8192 tokens on 40 heads
    hi = max(0, min(hi, limit // new_hi - (new_hi + 1) // 2))
    pairs = new_hi * (hi + (new_hi + 1) // 2)        # the most of a request
    room = min(limit // max(pairs, 1), (1 << 28) // (hkv * dim * (hi + new_hi)))
    return _case(None, op, _log_int(rng, 1, max(1, min(64, room))), hi // 8, hi, new_lo, new_hi, **base)


def _lengths(case):
    """Tokens in the cache once the call's own are there, and the call's own, of each request."""
    rng = np.random.default_rng(case["lens_seed"])
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    lens = rng.integers(lo, hi + 1, size=n)
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=n)
    return (lens, new) if case["op"] == "step" else (lens + new, new)


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _power(most):
    """Of the largest magnitudes: the least e, from LEAST to MOST, with most <= 448 * 2^e."""
    m, e = torch.frexp(most)
    e = e - 9 + (m > 0.875).int()
    return torch.where(most > 0, e, LEAST).clamp(LEAST, MOST)


def _codes(x, e):
    return (x * torch.exp2(-e.float())).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _pool(case, blocks, g, is_v, sizes):
    """One pool of N(0, 1) values times their head's size, and its scales."""
    rows = (case["hkv"], case["block"], case["dim"])
    kv = case["kv"]
    pool = torch.empty((blocks,) + rows, dtype=torch.bfloat16 if kv == "bf16" else torch.uint8, device="cuda")
    scales = torch.zeros((blocks, (case["hkv"] + 15) // 16 * 16), dtype=torch.uint8, device="cuda") if kv == "blk" else None
    step = max(1, (1 << 26) // math.prod(rows))
    for b in range(0, blocks, step):
        x = torch.randn((min(step, blocks - b),) + rows, generator=g, device="cuda")
        if kv == "bf16":
            pool[b:b + step] = x
        elif kv == "fp8":
            pool[b:b + step] = (x / (V_SCALE if is_v else K_SCALE)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        else:
            x = x.mul_(sizes[:, None, None])
            e = _power(x.abs().amax(dim=(2, 3)))
            pool[b:b + step] = _codes(x, e[..., None, None])
            scales[b:b + step, :case["hkv"]] = (e + 127).to(torch.uint8)
    return pool, scales


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
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    op, hq, hkv, dim = case["op"], case["hq"], case["hkv"], case["dim"]
    # heads differ in the size of their keys and values, as trained ones do; of scales for a whole pool they make poor use
    sizes = torch.exp(0.5 * normal(2, hkv)) if case["kv"] == "blk" else torch.ones((2, hkv), device="cuda")
    state = {"case": case, "most": int(lens.max()), "tables": torch.from_numpy(tables).cuda(),
             "lens": torch.from_numpy(lens.astype(np.int32)).cuda(), "scale": 1.0 / math.sqrt(dim),
             "starts": None if op == "step" else torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()}
    state["k_pool"], state["k_scales"] = _pool(case, n_pool, g, False, sizes[0])
    state["v_pool"], state["v_scales"] = _pool(case, n_pool, g, True, sizes[1])
    tokens = int(new.sum())
    if op == "append":
        # one row per token: the queries, the keys and the values of all heads, as one projection gives them
        rows = normal(tokens, hq + 2 * hkv, dim)
        rows[:, hq:] *= sizes.view(2 * hkv, 1)
        state["qkv"] = rows.bfloat16().flatten(1)
        angle = torch.arange(state["most"], dtype=torch.float64)[:, None] * 1e6 ** (
            -torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])
        # a model in bf16 keeps cosines and sines in it; products of two such numbers are exact in 32 bits, so that keys, and the scales of
        # their blocks, are the same however they are computed
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], dim=1).bfloat16().float().cuda()
        state["q_out"] = torch.empty((tokens, hq, dim), dtype=torch.bfloat16, device="cuda")
    else:
        state["q"] = normal(tokens, hq, dim).bfloat16()
        state["out"] = torch.empty_like(state["q"])
    if op == "step":
        state["k_new"], state["v_new"] = ((normal(tokens, hkv, dim) * size[:, None]).bfloat16() for size in sizes)
    if own:
        from paper_2602_11530_amd import binding as pkv
        state["shape"] = pkv.make_shape(case["seqs"], hq, hkv, width, n_pool, head_dim=dim, block_size=case["block"],
                                        max_context_len=state["most"])
        if op == "append":
            row = (hq + 2 * hkv) * dim
            state["rope"] = pkv.make_rope(tokens, case["rotary"], state["most"], interleaved=case["interleaved"], q_stride=row, k_stride=row,
                                          v_stride=row)
        else:
            size = pkv.pkv_attn_workspace_bytes(state["shape"]) if op == "step" else pkv.pkv_prompt_workspace_bytes(state["shape"], tokens)
            state["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return state


# ---------------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    return {"prompt": _plain_prompt, "step": _plain_step, "append": _plain_append}[case["op"]](state, case)


def _blk_outputs(state):
    """Codes as the values they stand for, and the scales' bytes."""
    return [state["k_pool"].view(torch.float8_e4m3fn), state["v_pool"].view(torch.float8_e4m3fn), state["k_scales"], state["v_scales"]]


def _run_own(state, case):
    from paper_2602_11530_amd import binding as pkv
    tables, lens, shape, starts = state["tables"], state["lens"], state["shape"], state["starts"]
    pools, scales = (state["k_pool"], state["v_pool"]), (state["k_scales"], state["v_scales"])
    if case["op"] == "append":
        hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
        qkv = state["qkv"]
        pkv.kv_rope_append_fp8blk(qkv, qkv[:, hq * dim:], qkv[:, (hq + hkv) * dim:], None, None, state["cos_sin"], state["q_out"], *pools, *scales,
                                  tables, lens, starts, state["rope"], shape)
        return [state["q_out"], *_blk_outputs(state)]
    q, out, ws, scale = state["q"], state["out"], state["ws"], state["scale"]
    if case["op"] == "step":
        pkv.kv_append_fp8blk(state["k_new"], state["v_new"], *pools, *scales, tables, lens, shape)
        pkv.paged_decode_attn_fp8blk(q, *pools, *scales, tables, lens, scale, out, shape, ws)
        return [out, *_blk_outputs(state)]
    if case["kv"] == "bf16":
        pkv.paged_prompt_attn(q, *pools, tables, lens, starts, len(q), scale, out, shape, ws)
    elif case["kv"] == "fp8":
        pkv.paged_prompt_attn_fp8kv(q, *pools, tables, lens, starts, len(q), scale, K_SCALE, V_SCALE, out, shape, ws)
    else:
        pkv.paged_prompt_attn_fp8blk(q, *pools, *scales, tables, lens, starts, len(q), scale, out, shape, ws)
    return [out]


def _positions(state):
    """Request and position of each new token."""
    lens = state["lens"].long()
    if state["starts"] is None:
        return torch.arange(len(lens), device="cuda"), lens - 1
    starts = state["starts"].long()
    token = torch.arange(len(state["qkv"] if "qkv" in state else state["q"]), device="cuda")
    request = torch.searchsorted(starts, token, right=True) - 1
    return request, lens[request] - (starts[request + 1] - token)


def _rows(state, case, ids, name):
    """The rows of blocks `ids`, in fp32: [..., Hkv, B, D]"""
    x = state[name + "_pool"][ids]
    if case["kv"] == "bf16":
        return x.float()
    x = x.view(torch.float8_e4m3fn).float()
    if case["kv"] == "fp8":
        return x * (V_SCALE if name == "v" else K_SCALE)
    return x * torch.exp2(state[name + "_scales"][ids][..., :case["hkv"]].float() - 127)[..., None, None]


def _attend(state, case):
    """Each request's new tokens over the tokens up to their own, which the cache holds."""
    group = case["hq"] // case["hkv"]
    lens = state["lens"].tolist()
    starts = range(len(lens) + 1) if state["starts"] is None else state["starts"].tolist()
    for s, n in enumerate(lens):
        ids = state["tables"][s, :(n + case["block"] - 1) // case["block"]].long()
        k, v = (_rows(state, case, ids, name).transpose(0, 1).flatten(1, 2)[:, :n].contiguous() for name in ("k", "v"))   # [Hkv, n, D]
        kt = k.transpose(1, 2).contiguous()
        first, end = starts[s], starts[s + 1]
        step = max(1, (1 << 28) // (case["hq"] * n))
        for a in range(first, end, step):
            b = min(a + step, end)
            q = state["q"][a:b].float().unflatten(1, (case["hkv"], group)).transpose(0, 1).flatten(1, 2)                  # [Hkv, (b - a) G, D]
            score = torch.matmul(q, kt) * state["scale"]
            position = torch.arange(n - (end - a), n - (end - b), device="cuda").repeat_interleave(group)
            score = torch.where(torch.arange(n, device="cuda") <= position[:, None], score, -torch.inf)
            weight = torch.exp(score - score.amax(dim=-1, keepdim=True))
            out = torch.matmul(weight, v) / weight.sum(dim=-1, keepdim=True)
            state["out"][a:b] = out.unflatten(1, (b - a, group)).transpose(0, 1).flatten(1, 2)
    return state["out"]


def _plain_prompt(state, case):
    return [_attend(state, case)]


def _append_blk(state, case, k, v):
    """New tokens' rows [T, Hkv, D] in fp32 into the cache."""
    request, position = _positions(state)
    slot = position % case["block"]
    ids = state["tables"][request, position // case["block"]].long()
    hkv, blocks = case["hkv"], len(state["k_pool"])
    begins = torch.zeros(blocks, dtype=torch.bool, device="cuda")
    begins[ids[slot == 0]] = True
    # where each request's own tokens begin: the one block of it that may hold others
    lens = state["lens"].long()
    count = torch.ones_like(lens) if state["starts"] is None else state["starts"].long().diff()
    first = lens - count
    head = state["tables"].gather(1, (first // case["block"])[:, None])[:, 0].long()
    kept = torch.arange(case["block"], device="cuda") < (first % case["block"])[:, None]
    for x, pool, scales in ((k, state["k_pool"], state["k_scales"]), (v, state["v_pool"], state["v_scales"])):
        most = torch.zeros((blocks, hkv), device="cuda").index_reduce_(0, ids, x.abs().amax(dim=-1), "amax")
        old = scales[:, :hkv].int() - 127
        e = torch.where(begins[:, None], _power(most), torch.maximum(old, _power(most)))
        touched = torch.zeros(blocks, dtype=torch.bool, device="cuda")
        touched[ids] = True
        e = torch.where(touched[:, None], e, old)
        before = pool[head]
        values = before.view(torch.float8_e4m3fn).float() * torch.exp2(old[head].float())[..., None, None]
        again = kept[:, None, :, None] & (e[head] > old[head])[..., None, None]
        pool[head] = torch.where(again, _codes(values, e[head][..., None, None]), before)
        pool[ids, :, slot] = _codes(x, e[ids][..., None])
        scales[:, :hkv] = (e + 127).to(torch.uint8)


def _plain_step(state, case):
    _append_blk(state, case, state["k_new"].float(), state["v_new"].float())
    return [_attend(state, case), *_blk_outputs(state)]


def _turned(x, cos, sin, interleaved):
    """[T, H, D] in fp32 with its first dims rotated."""
    n = cos.shape[-1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], dim=-1).flatten(-2) if interleaved else torch.cat([c, d], dim=-1)
    return torch.cat([turned, x[..., 2 * n:]], dim=-1)


def _plain_append(state, case):
    hq, hkv, dim = case["hq"], case["hkv"], case["dim"]
    _, position = _positions(state)
    cos, sin = state["cos_sin"][position].unsqueeze(1).chunk(2, dim=-1)
    q, k, v = state["qkv"].unflatten(1, (-1, dim)).float().split([hq, hkv, hkv], dim=1)
    state["q_out"].copy_(_turned(q, cos, sin, case["interleaved"]))
    _append_blk(state, case, _turned(k, cos, sin, case["interleaved"]), v)
    return [state["q_out"], *_blk_outputs(state)]


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    lens, new = _lengths(case)
    lens, new = lens.astype(object), new.astype(object)
    tokens, seqs, hq, hkv, dim, block = int(new.sum()), case["seqs"], case["hq"], case["hkv"], case["dim"], case["block"]
    blocks = int(((lens + block - 1) // block).sum())
    if case["op"] == "append":
        rows = tokens * (2 * hq + 2 * hkv) * dim * 2 + 2 * tokens * hkv * dim          # in and out
        written = sum(int((n - 1) // block - (n - m) // block + 1) for n, m in zip(lens, new))
        return {"bytes": rows + tokens * case["rotary"] * 4 + written * (4 + 2 * hkv) + 8 * seqs,
                "flops": tokens * (hq + hkv) * 3 * case["rotary"]}
    held = int(lens.sum()) * hkv * dim * (2 if case["kv"] == "bf16" else 1) + (blocks * hkv if case["kv"] == "blk" else 0)   # K, or V
    moved = 2 * held + 2 * tokens * hq * dim * 2 + 4 * blocks + 8 * seqs
    if case["op"] == "step":
        moved += 2 * tokens * hkv * (3 * dim + 1)
        pairs = int(lens.sum())
    else:
        pairs = sum(int(m * (n - m) + m * (m + 1) // 2) for n, m in zip(lens, new))
    return {"bytes": moved, "flops": 4 * pairs * hq * dim}


def exact(case, seed):
    state = prepare(case, seed)
    hq, hkv, dim, block = case["hq"], case["hkv"], case["dim"], case["block"]
    lens, tables = state["lens"].tolist(), state["tables"].tolist()
    starts = list(range(len(lens) + 1)) if case["op"] == "step" else state["starts"].tolist()
    names = ("k", "v")
    fresh = None
    if case["op"] == "step":
        fresh = {"k": state["k_new"].double(), "v": state["v_new"].double()}
    elif case["op"] == "append":
        x = state["qkv"].view(-1, hq + 2 * hkv, dim).double()
        half = case["rotary"] // 2
        position = torch.cat([torch.arange(n - (b - a), n) for n, a, b in zip(lens, starts, starts[1:])]).cuda()
        table = state["cos_sin"][position].double()
        factor = torch.complex(table[:, :half].contiguous(), table[:, half:].contiguous())[:, None, :]   # a rotation is a product of complex numbers
        one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(x[:, :hq + hkv, one].contiguous(), x[:, :hq + hkv, two].contiguous()) * factor
        x[:, :hq + hkv, one], x[:, :hq + hkv, two] = z.real, z.imag
        fresh = {"k": x[:, hq:hq + hkv], "v": x[:, hq + hkv:]}
    held, power = {}, {}
    for name in names:
        pool = state[name + "_pool"]
        if case["kv"] == "bf16":
            held[name], power[name] = pool, None
        elif case["kv"] == "fp8":
            held[name], power[name] = pool.view(torch.float8_e4m3fn), None
        else:
            held[name], power[name] = pool.view(torch.float8_e4m3fn).double(), state[name + "_scales"][:, :hkv].double() - 127
    if fresh is not None:
        for s, n in enumerate(lens):
            m = starts[s + 1] - starts[s]
            for b in range((n - m) // block, (n - 1) // block + 1):
                id_, lo, hi = tables[s][b], max(n - m, b * block), min(n, (b + 1) * block)
                for name in names:
                    rows = fresh[name][starts[s + 1] - (n - lo):starts[s + 1] - (n - hi)].transpose(0, 1)   # [Hkv, tokens, D]
                    most = rows.abs().amax(dim=(1, 2))
                    e = torch.ceil(torch.log2(most / 448))
                    e = torch.where(most > 448 * torch.exp2(e), e + 1, torch.where(most <= 448 * torch.exp2(e - 1), e - 1, e)).clamp(LEAST, MOST)
                    if lo > b * block:                                       # what the block held before keeps its value
                        was = power[name][id_]
                        e = torch.maximum(e, was)
                        held[name][id_, :, :lo - b * block] *= torch.exp2(was - e)[:, None, None]
                    held[name][id_, :, lo - b * block:hi - b * block] = rows * torch.exp2(-e)[:, None, None]
                    power[name][id_] = e
    if case["op"] == "append":
        scales = []
        for name in names:
            full = state[name + "_scales"].clone()
            full[:, :hkv] = (power[name] + 127).to(torch.uint8)
            scales.append(full)
        return [x[:, :hq].contiguous(), held["k"], held["v"], *scales]
    group = hq // hkv
    out = torch.empty(state["q"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(lens):
        ids = torch.tensor(tables[s][:(n + block - 1) // block], device="cuda")
        rows = {}
        for name in names:
            x = held[name][ids].double()
            if case["kv"] == "fp8":
                x = x * float(np.float32(V_SCALE if name == "v" else K_SCALE))
            elif case["kv"] == "blk":
                last = n - 1 - (len(ids) - 1) * block
                if case["op"] == "step":                                     # codes of the block that was written are those that are held
                    x[-1, :, :last + 1] = x[-1, :, :last + 1].float().to(torch.float8_e4m3fn).double()
                x = x * torch.exp2(power[name][ids])[..., None, None]
            rows[name] = x.permute(1, 0, 2, 3).reshape(hkv, -1, dim)[:, :n].contiguous()
        m = starts[s + 1] - starts[s]
        at = torch.arange(n, device="cuda")
        for h in range(hq):
            k, v = rows["k"][h // group], rows["v"][h // group]
            for a in range(0, m, 4096):
                q = state["q"][starts[s] + a:min(starts[s] + a + 4096, starts[s + 1]), h].double()
                score = torch.mm(q, k.t().contiguous()) * float(np.float32(state["scale"]))
                own_at = torch.arange(n - m + a, n - m + a + len(q), device="cuda")
                score = score.masked_fill(at[None, :] > own_at[:, None], -torch.inf)
                out[starts[s] + a:starts[s] + a + len(q), h] = torch.mm(torch.softmax(score, dim=-1), v)
    return [out] if case["op"] == "prompt" else [out, None, None, None, None]
