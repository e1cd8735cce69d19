"""Pools with a scale for each block and KV head: appends byte for byte, attention of steps, the copies."""
import numpy as np
import pytest
import torch

import plain
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from prompt_util import make_batch, plain_append, pools_of, refresh, scale_row, shape_of, upload

pytestmark = pytest.mark.gpu


def step_attention(b, p, max_context_len=0, stream=None):
    shape = shape_of(b, max_context_len)
    ws = torch.full((max(pkv.pkv_attn_workspace_bytes(shape), 16),), 0xa5, dtype=torch.uint8, device="cuda")
    q = to_dev(b.q_bits)
    out = torch.full(b.q_bits.shape, 0x7FC1, dtype=torch.int16, device="cuda")
    tables, lens = to_dev(b.tables), to_dev(b.lens)
    if stream is not None:
        torch.cuda.synchronize()
    pkv.paged_decode_attn_fp8blk(q, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, b.scale, out, shape, ws, stream)
    torch.cuda.synchronize()
    return to_bits(out)


def values_of(b):
    return wl.bf16_bits_to_f64(b.q_bits).reshape(b.q_bits.shape)


@pytest.mark.parametrize("dim,block", [(128, 16), (64, 32), (256, 64), (128, 64), (64, 16), (256, 16)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (8, 8), (5, 1), (16, 2)])
def test_attention_of_steps(dim, block, hq, hkv):
    lens = [1, 15, 16, 17, 33, 64, 100, 500, 1500]
    b = make_batch(np.array(lens) - 1, [1] * len(lens), hq, hkv, dim, block, dim + hq)
    p = pools_of(b, "blk")
    plain.within(step_attention(b, p), *plain.attention(values_of(b), p.k, p.v, b.tables, b.lens, b.scale))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("seqs,lo,hi", [(3, 1, 90), (70, 1, 200), (40, 100, 2500), (300, 1, 64)])
def test_batches(dim, seqs, lo, hi):
    """Cut along segments or not, long shares and short ones; lengths of zero among them."""
    rng = np.random.default_rng(seqs + dim)
    lens = rng.integers(lo, hi + 1, seqs)
    b = make_batch(lens - 1, [1] * seqs, 4, 2, dim, 16, seqs)
    b.lens[rng.random(seqs) < 0.1] = 0
    p = pools_of(b, "blk")
    want = plain.attention(values_of(b), p.k, p.v, b.tables, b.lens, b.scale)
    plain.within(step_attention(b, p), *want)
    plain.within(step_attention(b, p, max_context_len=int(b.lens.max())), *want)


def test_long_shares_of_wide_heads():
    b = make_batch([6000] * 20, [1] * 20, 8, 8, 256, 64, 1)
    p = pools_of(b, "blk")
    got = step_attention(b, p, max_context_len=6001)
    pick = [0, 7, 19]
    q = values_of(b)
    want, off = plain.attention(q[pick], p.k, p.v, b.tables[pick], b.lens[pick], b.scale)
    plain.within(got[pick], want, off)


@pytest.mark.expects_id_faults
def test_blocks_outside_the_pool_and_unused_bytes(id_faults):
    b = make_batch([99, 40, 15], [1, 1, 1], 8, 2, 128, 16, 2, spare=2)
    p = pools_of(b, "blk")
    b.tables[0][2], b.tables[2][0] = -7, b.num_blocks + 5
    used = np.zeros((b.num_blocks, b.block), bool)
    for s, n in enumerate(b.lens):
        t = np.arange(n)
        ids = b.tables[s][t // b.block]
        ok = (ids >= 0) & (ids < b.num_blocks)
        used[ids[ok], t[ok] % b.block] = True
    for name in "kv":
        getattr(p, name + "_bits")[np.broadcast_to(~used[:, None, :, None], p.k_bits.shape)] = wl.E4M3_NAN
        getattr(p, name + "_scales")[~used.any(1)] = 255
    refresh(p, b)
    upload(p)
    got = step_attention(b, p)
    plain.within(got, *plain.attention(values_of(b), p.k, p.v, b.tables, b.lens, b.scale))
    assert (got[2] == 0).all() and int(id_faults.item()) == 4


def test_nan_and_infinite_scales_stay_where_they_are():
    b = make_batch([63], [1], 4, 2, 128, 16, 3)
    p = pools_of(b, "blk")
    p.v_scales[b.tables[0][1], 1] = 255
    upload(p)
    got = wl.bf16_bits_to_f64(step_attention(b, p)).reshape(b.q_bits.shape)
    assert np.isfinite(got[0, :2]).all() and not np.isfinite(got[0, 2:]).any()


def compare_pools(p, b):
    for name in "kv":
        got = getattr(p, name + "_dev").cpu().numpy()
        bad = np.argwhere(got != getattr(p, name + "_bits"))
        assert not len(bad), (name, len(bad), bad[:5].tolist(), got[tuple(bad[0])], getattr(p, name + "_bits")[tuple(bad[0])])
        scales = getattr(p, name[0] + "s_dev").cpu().numpy()
        assert np.array_equal(scales, getattr(p, name + "_scales")), (name, np.argwhere(scales != getattr(p, name + "_scales"))[:5].tolist())


def new_rows(b, tokens, spread=3.0):
    """Keys and values of very different sizes, bf16 bits and values."""
    size = np.exp(spread * b.rng.standard_normal((2, tokens, b.hkv, 1)))
    bits = [wl.f32_to_bf16_bits(b.rng.standard_normal((tokens, b.hkv, b.dim)).astype(np.float32) * s.astype(np.float32)) for s in size]
    return bits, [wl.bf16_bits_to_f64(x).reshape(x.shape) for x in bits]


@pytest.mark.parametrize("dim,block,hkv", [(128, 16, 8), (64, 32, 2), (256, 64, 3), (128, 64, 1), (64, 16, 17), (256, 32, 1)])
def test_append_of_steps(dim, block, hkv):
    """Blocks that begin, that keep their scales and whose scales grow."""
    lens = list(range(1, 70)) + [500]
    b = make_batch(np.array(lens) - 1, [1] * len(lens), hkv, hkv, dim, block, dim + hkv)
    p = pools_of(b, "blk")
    for turn in range(3):
        bits, values = new_rows(b, len(lens))
        pkv.kv_append_fp8blk(to_dev(bits[0]), to_dev(bits[1]), p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables), to_dev(b.lens), shape_of(b))
        torch.cuda.synchronize()
        plain_append(p, b, values, [(s, int(n) - 1) for s, n in enumerate(b.lens)])
        compare_pools(p, b)


@pytest.mark.parametrize("dim,block", [(128, 16), (64, 64), (256, 32)])
def test_append_of_every_kind_of_value(dim, block):
    """Zeros of both signs, subnormals, borders of a scale, the largest ones, infinities, NaN."""
    rows = np.array([0x0000, 0x8000, 0x0001, 0x8001, 0x0080, 0x7F7F, 0xFF7F, 0x7F80, 0xFF80, 0x7FC0, 0x3F80, 0x43E0, 0x43E1, 0xC3E0, 0xC3E1, 0x3FE0,
                     0x3FE1, 0x0480, 0x0460, 0x7B60, 0x7F60, 0x7F61], np.uint16)
    tokens = len(rows)
    b = make_batch(np.arange(tokens) % 3, [1] * tokens, 2, 2, dim, block, 4)
    p = pools_of(b, "blk")
    bits = []
    for _ in range(2):
        x = np.zeros((tokens, 2, dim), np.uint16)
        x[:, 0, 5] = rows
        x[:, 1] = wl.normal_bf16(b.rng, (tokens, dim)) & 0xBFFF     # small values next to one of them
        x[:, 1, dim - 1] = rows
        bits.append(x)
    values = [wl.bf16_bits_to_f64(x).reshape(x.shape) for x in bits]
    pkv.kv_append_fp8blk(to_dev(bits[0]), to_dev(bits[1]), p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables), to_dev(b.lens), shape_of(b))
    torch.cuda.synchronize()
    plain_append(p, b, values, [(s, int(n) - 1) for s, n in enumerate(b.lens)])
    for name in "kv":    # a NaN may be either one
        dev = getattr(p, name + "_dev")
        got, want = dev.cpu().numpy(), getattr(p, name + "_bits")
        same = (got == want) | ((got & 0x7F) == 0x7F) & ((want & 0x7F) == 0x7F)
        assert same.all(), (name, np.argwhere(~same)[:5].tolist())
        assert np.array_equal(getattr(p, name + "s_dev").cpu().numpy(), getattr(p, name + "_scales"))


@pytest.mark.parametrize("dim,block,hkv,hq", [(128, 16, 8, 40), (64, 32, 2, 6), (256, 64, 3, 6), (128, 64, 1, 8), (64, 16, 2, 2)])
@pytest.mark.parametrize("queries", [True, False])
def test_prompts_and_pieces(dim, block, hkv, hq, queries):
    """Not rotated, so that scales and bytes are the definition's to the bit; rows of one projection."""
    b = make_batch([0, 5, 16, 100, 31, 0, 3], [200, 7, 64, 1, 33, 0, 40], hq, hkv, dim, block, dim, lead=2, tail=3)
    p = pools_of(b, "blk")
    (k, v), values = new_rows(b, b.tokens)
    row = np.concatenate([b.q_bits, k, v], axis=1)
    qkv = to_dev(row).flatten(1)
    rope = pkv.make_rope(b.tokens, 0, 0, q_stride=qkv.shape[1], k_stride=qkv.shape[1], v_stride=qkv.shape[1])
    q_out = torch.full(b.q_bits.shape, 0x7FC1, dtype=torch.int16, device="cuda") if queries else None
    pkv.kv_rope_append_fp8blk(qkv if queries else None, qkv[:, hq * dim:], qkv[:, (hq + hkv) * dim:], None, None, None, q_out, p.k_dev, p.v_dev, p.ks_dev,
                              p.vs_dev, to_dev(b.tables), to_dev(b.lens), to_dev(b.starts), rope, shape_of(b))
    torch.cuda.synchronize()
    at = plain.positions(b.lens, b.starts, 1 << 30, b.tokens)
    plain_append(p, b, values, at)
    compare_pools(p, b)
    if queries:
        has = np.array([s >= 0 for s, _ in at])
        got = to_bits(q_out)
        assert np.array_equal(got[has], b.q_bits[has]) and (got[~has] == 0x7FC1).all()


@pytest.mark.parametrize("dim,rotary,interleaved,norm", [(128, 128, False, True), (64, 32, True, False), (256, 128, False, True), (128, 64, True, True),
                                                         (64, 64, False, False)])
@pytest.mark.parametrize("tokens", ["few", "many"])
def test_normalised_and_rotated(dim, rotary, interleaved, norm, tokens):
    """The rows are those of kv_rope_append to the bit of a fp32 number; with its bf16 pools as what was there, each value is off by its rounding."""
    new = [30, 1, 70] if tokens == "few" else [700, 1, 500]
    b = make_batch([0, 20, 5], new, 8, 2, dim, 16, dim + rotary)
    p = pools_of(b, "blk")
    qkv = to_dev(wl.normal_bf16(b.rng, (b.tokens, (b.hq + 2 * b.hkv) * dim)))
    norms = [to_dev(wl.normal_bf16(b.rng, (dim,))) if norm else None for _ in range(2)]
    most = int(b.lens.max())
    angle = np.arange(most)[:, None] / 100.0 ** (np.arange(rotary // 2) / (rotary // 2))
    cos_sin = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
    rope = pkv.make_rope(b.tokens, rotary, most, interleaved=interleaved, q_stride=qkv.shape[1], k_stride=qkv.shape[1], v_stride=qkv.shape[1])
    shape = shape_of(b, most)
    q_outs = [torch.full((b.tokens, b.hq, dim), 0x7FC1, dtype=torch.int16, device="cuda") for _ in range(2)]
    tables, lens, starts = to_dev(b.tables), to_dev(b.lens), to_dev(b.starts)
    rows = (qkv, qkv[:, b.hq * dim:], qkv[:, (b.hq + b.hkv) * dim:], *norms, cos_sin)
    wide = [torch.zeros((b.num_blocks, b.hkv, b.block, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pkv.kv_rope_append(*rows, q_outs[0], *wide, tables, lens, starts, rope, shape)
    before = [x.copy() for x in (p.k, p.v)]
    pkv.kv_rope_append_fp8blk(*rows, q_outs[1], p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, starts, rope, shape)
    torch.cuda.synchronize()
    assert torch.equal(*q_outs)
    mine, cached = np.zeros((2, b.num_blocks, b.block), bool)
    for s, n in enumerate(b.lens):
        t = np.arange(int(n))
        own = t >= int(n) - int(b.new[s])
        mine[b.tables[s][t[own] // b.block], t[own] % b.block] = True
        cached[b.tables[s][t[~own] // b.block], t[~own] % b.block] = True
    for name, x, old, was in zip("kv", wide, before, (p.k_scales.copy(), p.v_scales.copy())):
        setattr(p, name + "_bits", getattr(p, name + "_dev").cpu().numpy())
        setattr(p, name + "_scales", getattr(p, name + "s_dev").cpu().numpy())
        refresh(p, b)
        got, want = getattr(p, name), x.double().cpu().numpy()
        scale = 2.0 ** (getattr(p, name + "_scales")[:, :b.hkv].astype(float) - 127)[..., None, None]
        # bf16 is 2^-8 of the value off, e4m3 2^-4 of it or 2^-10 of the scale
        off = 2.0 ** -8 * np.abs(want) + np.maximum(2.0 ** -4 * np.abs(want) * (1 + 2.0 ** -8), 2.0 ** -10 * scale)
        where = np.broadcast_to(mine[:, None, :, None], want.shape)
        assert (np.abs(got - want) <= off)[where].all()
        # the largest value of a block is in its scale's upper half, unless the block had its scale before
        fresh = mine[:, 0]
        top = np.abs(want).max(axis=(2, 3)) / scale[..., 0, 0]
        assert (top[fresh] > 224 * (1 - 2.0 ** -7)).all() and (top <= 448 * (1 + 2.0 ** -7)).all()
        # what was cached is what it was, to the rounding of a scale that has grown
        kept = np.broadcast_to(cached[:, None, :, None], want.shape)
        rounded = np.where(scale > 2.0 ** (was[:, :b.hkv].astype(float) - 127)[..., None, None], np.maximum(2.0 ** -4 * np.abs(old), 2.0 ** -10 * scale), 0)
        assert (np.abs(got - old) <= rounded)[kept].all()


@pytest.mark.expects_id_faults
def test_append_refuses_what_it_must(id_faults):
    b = make_batch([20, 40, 0, 5], [30, 1, 20, 4], 4, 2, 128, 16, 6)
    p = pools_of(b, "blk")
    b.tables[0][2], b.tables[1][2] = b.num_blocks, -1
    b.lens[2], b.lens[3] = 8, 0             # 20 new tokens of a context of 8, 4 of one of 0
    (k, v), values = new_rows(b, b.tokens)
    pkv.kv_rope_append_fp8blk(None, to_dev(k), to_dev(v), None, None, None, None, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables), to_dev(b.lens),
                              to_dev(b.starts), pkv.make_rope(b.tokens, 0, 0), shape_of(b))
    torch.cuda.synchronize()
    plain_append(p, b, values, plain.positions(b.lens, b.starts, 1 << 30, b.tokens))
    compare_pools(p, b)
    assert int(id_faults.item()) == 2


def test_a_token_at_a_time_is_the_attention_of_what_was_appended():
    """Appends of single tokens and of a piece, attention of steps and of the piece, copies of blocks with their scales, all together."""
    b = make_batch([0, 0], [40, 23], 8, 2, 128, 16, 7, spare=20)
    p = pools_of(b, "blk")
    room = np.full((2, 8), -1, np.int32)
    ids = b.rng.permutation(b.num_blocks)[:8].astype(np.int32)
    room[0, :4], room[1, :4] = ids[:4], ids[4:]
    b.tables = room
    (k, v), values = new_rows(b, b.tokens, 1.0)
    tables, starts = to_dev(b.tables), to_dev(b.starts)
    shape = shape_of(b)
    pkv.kv_rope_append_fp8blk(None, to_dev(k), to_dev(v), None, None, None, None, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, to_dev(b.lens), starts,
                              pkv.make_rope(b.tokens, 0, 0), shape)
    plain_append(p, b, values, plain.positions(b.lens, b.starts, 1 << 30, b.tokens))
    from prompt_util import check, plain_prompt, run_prompt
    check(b, run_prompt(b, p), *plain_prompt(b, p))
    b.q_bits = wl.normal_bf16(b.rng, (2, 8, 128))
    for turn in range(20):
        b.lens = b.lens + 1
        bits, values = new_rows(b, 2, 1.0)
        pkv.kv_append_fp8blk(to_dev(bits[0]), to_dev(bits[1]), p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, to_dev(b.lens), shape)
        plain_append(p, b, values, [(s, int(n) - 1) for s, n in enumerate(b.lens)])
        plain.within(step_attention(b, p), *plain.attention(values_of(b), p.k, p.v, b.tables, b.lens, b.scale))
    compare_pools(p, b)
    # to other blocks, scales and all
    first = step_attention(b, p)
    free = np.setdiff1d(np.arange(b.num_blocks), ids)[:8].astype(np.int32)
    nbytes, row = 2 * 16 * 128, pkv.pkv_fp8blk_scale_bytes(shape)
    assert row == scale_row(2)
    for x, size in ((p.k_dev, nbytes), (p.v_dev, nbytes), (p.ks_dev, row), (p.vs_dev, row)):
        pkv.kv_blocks_move(x, to_dev(ids), x, to_dev(free), 8, size, b.num_blocks, b.num_blocks)
    lookup = dict(zip(ids.tolist(), free.tolist()))
    b.tables = np.vectorize(lambda i: lookup.get(i, -1))(b.tables).astype(np.int32)
    assert np.array_equal(first, step_attention(b, p))


def test_captured_and_on_another_stream():
    b = make_batch([99, 700, 15], [1, 1, 1], 8, 2, 128, 16, 8)
    p = pools_of(b, "blk")
    want = step_attention(b, p)
    assert np.array_equal(want, step_attention(b, p, stream=torch.cuda.Stream()))
    (k, v), values = new_rows(b, 3)
    k, v, tables, lens, q, shape = to_dev(k), to_dev(v), to_dev(b.tables), to_dev(b.lens), to_dev(b.q_bits), shape_of(b)
    out = torch.empty(b.q_bits.shape, dtype=torch.int16, device="cuda")
    ws = torch.empty(pkv.pkv_attn_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkv.kv_append_fp8blk(k, v, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, shape)
        pkv.paged_decode_attn_fp8blk(q, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, b.scale, out, shape, ws)
    plain_append(p, b, values, [(s, int(n) - 1) for s, n in enumerate(b.lens)])
    want = plain.attention(values_of(b), p.k, p.v, b.tables, b.lens, b.scale)
    for _ in range(3):
        out.fill_(0x7FC1)
        graph.replay()
        torch.cuda.synchronize()
        plain.within(to_bits(out), *want)
    compare_pools(p, b)


@pytest.mark.parametrize("dim,block", [(128, 16), (64, 64)])
def test_appends_behind_scales_of_any_byte(dim, block):
    """Blocks that were not filled by appends may hold scales that those would not choose: they are kept, or grow, as any other."""
    bytes_ = [0, 1, 9, 10, 11, 120, 127, 245, 246, 247, 253, 254, 255]
    b = make_batch([5] * len(bytes_), [3] * len(bytes_), 2, 1, dim, block, 9)
    p = pools_of(b, "blk")
    for s, byte in enumerate(bytes_):
        p.k_scales[b.tables[s][0], 0] = byte
        p.v_scales[b.tables[s][0], 0] = bytes_[-1 - s]
    refresh(p, b)
    upload(p)
    (k, v), values = new_rows(b, b.tokens)
    pkv.kv_rope_append_fp8blk(None, to_dev(k), to_dev(v), None, None, None, None, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables), to_dev(b.lens),
                              to_dev(b.starts), pkv.make_rope(b.tokens, 0, 0), shape_of(b))
    torch.cuda.synchronize()
    plain_append(p, b, values, plain.positions(b.lens, b.starts, 1 << 30, b.tokens))
    for name in "kv":   # what a block of NaN holds is nothing
        nan = getattr(p, name + "_scales")[:, 0] == 255
        getattr(p, name + "_bits")[nan] = getattr(p, name + "_dev").cpu().numpy()[nan]
    compare_pools(p, b)


def test_beyond_4_gib():
    """150 000 blocks of 32 KiB, the requests' own on both sides of 4 GiB and at the end: appends, attention of prompts and of steps."""
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GiB of free device memory")
    from prompt_util import check, plain_prompt, run_prompt
    large, hkv, dim = 150_000, 8, 256
    b = make_batch([0, 170, 1000], [37, 30, 1], 16, hkv, dim, 16, 10)
    nbytes = hkv * 16 * dim
    assert large * nbytes > 1 << 32
    small = pools_of(b, "blk")
    place = np.concatenate([[large - 1, (1 << 32) // nbytes, (1 << 32) // nbytes + 1],
                            b.rng.choice(np.arange((1 << 32) // nbytes + 2, large - 1), b.num_blocks - 3, replace=False)])
    p = pools_of(b, "blk")
    p.k_dev, p.v_dev = (torch.zeros((large, hkv, 16, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    p.ks_dev, p.vs_dev = (torch.zeros((large, scale_row(hkv)), dtype=torch.uint8, device="cuda") for _ in range(2))
    at = to_dev(place.astype(np.int64))
    tables, count = b.tables, b.num_blocks
    far = np.where(tables >= 0, place[tables], -1).astype(np.int32)
    (k, v), values = new_rows(b, b.tokens, 1.0)
    for name in "kv":
        getattr(p, name + "_dev")[at] = to_dev(getattr(small, name + "_bits"))
        getattr(p, name[0] + "s_dev")[at] = to_dev(getattr(small, name + "_scales"))
    b.tables, b.num_blocks = far, large
    pkv.kv_rope_append_fp8blk(None, to_dev(k), to_dev(v), None, None, None, None, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(far), to_dev(b.lens),
                              to_dev(b.starts), pkv.make_rope(b.tokens, 0, 0), shape_of(b))
    got = run_prompt(b, p)
    q = b.q_bits
    b.q_bits = q[:3].copy()
    step = step_attention(b, p)
    b.q_bits, b.tables, b.num_blocks = q, tables, count
    plain_append(small, b, values, plain.positions(b.lens, b.starts, 1 << 30, b.tokens))
    for name in "kv":
        assert np.array_equal(getattr(p, name + "_dev")[at].cpu().numpy(), getattr(small, name + "_bits"))
        assert np.array_equal(getattr(p, name[0] + "s_dev")[at].cpu().numpy(), getattr(small, name + "_scales"))
    check(b, got, *plain_prompt(b, small))
    b.q_bits = q[:3].copy()
    plain.within(step, *plain.attention(values_of(b), small.k, small.v, tables, b.lens, b.scale))


@pytest.mark.parametrize("hkv", [17, 40])
def test_more_kv_heads_than_one_row_of_scales(hkv):
    b = make_batch([30, 0, 1], [20, 50, 1], hkv, hkv, 64, 32, hkv)
    p = pools_of(b, "blk")
    (k, v), values = new_rows(b, b.tokens, 1.0)
    pkv.kv_rope_append_fp8blk(None, to_dev(k), to_dev(v), None, None, None, None, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables), to_dev(b.lens),
                              to_dev(b.starts), pkv.make_rope(b.tokens, 0, 0), shape_of(b))
    from prompt_util import check, plain_prompt, run_prompt
    got = run_prompt(b, p)
    plain_append(p, b, values, plain.positions(b.lens, b.starts, 1 << 30, b.tokens))
    compare_pools(p, b)
    check(b, got, *plain_prompt(b, p))
    b.q_bits = b.q_bits[:3]
    plain.within(step_attention(b, p), *plain.attention(values_of(b), p.k, p.v, b.tables, b.lens, b.scale))
