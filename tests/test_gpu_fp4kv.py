"""The cache held in 4 bits: the append against the format's definition byte by byte, the attention over it against a plain implementation in 64
bits, and the copies of its blocks."""
import numpy as np
import pytest
import torch

import plain
from formats_util import attend, make_batch, pools_of, poison, shape_of
from gpu_util import to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl

pytestmark = pytest.mark.gpu


def append(b, pools, k_new, v_new, lens=None, **kw):
    pkv.kv_append_fp4(to_dev(k_new), to_dev(v_new), pools.k_dev, pools.v_dev, to_dev(b.tables), to_dev(b.lens if lens is None else lens),
                      shape_of(b, **kw))
    torch.cuda.synchronize()
    return pools.k_dev.cpu().numpy(), pools.v_dev.cpu().numpy()


def expected(b, pools, k_new, v_new, lens, requests):
    found = []
    for bits, new, is_v in ((pools.k_bits, k_new, False), (pools.v_bits, v_new, True)):
        pool = bits.copy()
        t = np.array([lens[s] - 1 for s in requests])
        rows = wl.bf16_bits_to_f64(new).reshape(new.shape)[requests]
        plain.put(pool, b.dim, b.tables[requests, t // b.block], t % b.block, rows, is_v)
        found.append(pool)
    return found


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 32, 64])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (10, 5), (40, 40)])
def test_append_writes_its_rows_and_nothing_else(device, dim, block, hq, hkv):
    b = make_batch([1, 0, block, block + 1, 5 * block - 1, 16, 17, 200], hq, hkv, dim, block, seed=21, spare=3)
    pools = pools_of(b, "fp4")
    new = [wl.normal_bf16(b.rng, (len(b.lens), hkv, dim)) for _ in range(2)]
    got = append(b, pools, *new)
    want = expected(b, pools, *new, b.lens, [s for s, n in enumerate(b.lens) if n])
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("dim,hkv", [(64, 3), (128, 8), (256, 7)])
def test_append_for_many_requests(device, dim, hkv):
    b = make_batch(np.random.default_rng(1).integers(0, 40, 1200), hkv, hkv, dim, 16, seed=24)
    pools = pools_of(b, "fp4")
    new = [wl.normal_bf16(b.rng, (len(b.lens), hkv, dim)) for _ in range(2)]
    got = append(b, pools, *new)
    want = expected(b, pools, *new, b.lens, [s for s, n in enumerate(b.lens) if n])
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_append_of_every_kind_of_value(device):
    """Every finite bf16 value as the largest of a group, all ties between codes, values below a group's smallest, infinities and NaN."""
    rng = np.random.default_rng(5)
    bits = np.arange(65536, dtype=np.uint16)
    rows = [bits.reshape(-1, 32)]                                        # neighbours: one binade, all signs; NaN and infinities at the ends
    power = rng.integers(1, 250, 4096).astype(np.uint16)
    codes = np.array([0, .24, .25, .26, .5, .74, .75, .76, 1, 1.24, 1.25, 1.26, 1.5, 1.74, 1.75, 1.76, 2, 2.49, 2.5, 2.51, 3, 3.49, 3.5, 3.51, 4, 4.9, 5,
                      5.1, 6, 6.5, 6.95, -5])
    with np.errstate(over="ignore"):
        x = (codes[None] * 2.0 ** (power[:, None].astype(np.float64) - 125)).astype(np.float32)
    rows.append(wl.f32_to_bf16_bits(x))
    mixed = rng.integers(0, 65536, (4096, 32)).astype(np.uint16)         # any bits together
    rows.append(mixed)
    spread = wl.normal_bf16(rng, (2048, 32))
    spread[::3, 0], spread[1::3, 31], spread[2::9, 7] = wl.BF16_INF, 0xff80, wl.BF16_NAN
    rows.append(spread)
    groups = np.concatenate(rows)
    S, hkv, dim = 192, 16, 128
    groups = np.concatenate([groups, np.zeros((S * hkv * 4 - len(groups), 32), np.uint16)]).reshape(S, hkv, dim)
    b = make_batch(np.full(S, 7), hkv, hkv, dim, 16, seed=22)
    pools = pools_of(b, "fp4")
    got = append(b, pools, groups, groups[::-1].copy())
    want = expected(b, pools, groups, groups[::-1].copy(), b.lens, list(range(S)))
    for g, w, is_v in zip(got, want, (False, True)):
        scale = np.s_[..., 8 * dim:]
        assert np.array_equal(g[scale], w[scale])
        assert np.array_equal(plain.decode(g, dim, is_v), plain.decode(w, dim, is_v), equal_nan=True)
        code_at, scale_at, _ = plain._places(dim, is_v)
        number = w[..., scale_at] != 255                                 # the codes of a NaN group say nothing
        assert np.array_equal(g[..., code_at][number], w[..., code_at][number])


@pytest.mark.expects_id_faults
def test_append_skips(device, id_faults):
    b = make_batch([40, 20, 300, 5, 64], 4, 2, 128, 16, seed=23, spare=2)
    pools = pools_of(b, "fp4")
    new = [wl.normal_bf16(b.rng, (5, 2, 128)) for _ in range(2)]
    right = b.tables.copy()
    b.tables[0, 2], b.tables[3, 0] = -1, b.num_blocks
    lens = np.array([40, -3, 300, 5, 64], np.int32)
    got = append(b, pools, *new, lens=lens, max_context_len=128)
    b.tables = right
    want = expected(b, pools, *new, np.minimum(lens, 128), [2, 4])       # the bound's last position, as attention sees it
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    assert int(id_faults.item()) == 2


@pytest.mark.parametrize("dim,block", [(64, 32), (128, 16), (256, 64)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (5, 1), (8, 8)])
def test_attention(device, dim, block, hq, hkv):
    b = make_batch([0, 1, 15, 16, 17, 33, 100, 5, 257, 1600, 64, 48], hq, hkv, dim, block, seed=31)
    pools = pools_of(b, "fp4")
    want, off = plain.attention(b.q, pools.k, pools.v, b.tables, b.lens, b.scale)
    plain.within(attend(b, pools), want, off)
    plain.within(attend(b, pools, partition_size=128, max_context_len=1600), want, off)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("seqs,hkv,longest", [(70, 2, 300), (300, 1, 120), (90, 2, 1500), (230, 2, 900), (1, 8, 8191), (2048, 1, 20)])
def test_attention_of_many_requests_and_long_ones(device, dim, seqs, hkv, longest):
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, longest + 1, seqs)
    lens[0] = longest
    b = make_batch(lens, 2 * hkv, hkv, dim, 16, seed=seqs)
    pools = pools_of(b, "fp4")
    want, off = plain.attention(b.q, pools.k, pools.v, b.tables, b.lens, b.scale)
    plain.within(attend(b, pools), want, off)
    plain.within(attend(b, pools, max_context_len=longest), want, off)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_every_code_and_scale_of_v(device, dim):
    """One-token requests: the row is the token's V, widened exactly."""
    S, hkv = 246, 2
    b = make_batch(np.full(S, 1), hkv, hkv, dim, 16, seed=33)
    pools = pools_of(b, "fp4")
    code_at, scale_at, _ = plain._places(dim, True)
    pool = pools.v_bits
    for s in range(S):
        tile = pool[b.tables[s, 0], :, 0]
        tile[:, code_at[0, ::2]] = b.rng.integers(0, 256, (hkv, dim // 2))
        tile[:, scale_at[0, ::32]] = 7 + (s + np.arange(dim // 32)) % 246        # every scale that the append writes
    pools.v_dev = to_dev(pool)
    v = plain.decode(pool, dim, True)[b.tables[:, 0], :, 0]
    got = wl.bf16_bits_to_f64(attend(b, pools)).reshape(S, hkv, dim)
    assert np.array_equal(got, v)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_unused_slots_may_hold_anything(device, dim):
    b = make_batch([1, 5, 16, 17, 40, 100], 4, 2, dim, 32, seed=34, spare=3)
    pools = pools_of(b, "fp4")
    want, off = plain.attention(b.q, pools.k, pools.v, b.tables, b.lens, b.scale)
    used = np.zeros((b.num_blocks, 32), bool)
    for s, n in enumerate(b.lens):
        for t in range(n):
            used[b.tables[s, t // 32], t % 32] = True
    poison(pools, "fp4", ~used)
    plain.within(attend(b, pools), want, off)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_nan_stays_where_it_belongs(device, dim):
    b = make_batch([50, 50, 700], 4, 2, dim, 16, seed=35)
    pools = pools_of(b, "fp4")
    _, scale_at, _ = plain._places(dim, False)
    pools.k_bits[b.tables[0, 1], 0, 0, scale_at[3, 32]] = 255        # token 19 of request 0, KV head 0, dims 32..63
    pools.v_bits[b.tables[1, 2], 1, 0, scale_at[5, 0]] = 255         # token 37 of request 1, KV head 1, dims 0..31
    pools.k_dev, pools.v_dev = to_dev(pools.k_bits), to_dev(pools.v_bits)
    out = np.isnan(wl.bf16_bits_to_f64(attend(b, pools)).reshape(3, 4, dim))
    want = np.zeros_like(out)
    want[0, :2] = True
    want[1, 2:, :32] = True
    assert np.array_equal(out, want)


@pytest.mark.parametrize("dim,block,hkv", [(64, 16, 1), (128, 16, 8), (256, 64, 3)])
def test_blocks_are_copied_as_they_are(device, dim, block, hkv):
    """A request leaves through a staging image and pinned host memory, and another pool: its rows are the same to the bit."""
    b = make_batch([300, 75], 2 * hkv, hkv, dim, block, seed=36, spare=20)
    pools = pools_of(b, "fp4")
    shape = shape_of(b)
    size, NB = pkv.pkv_fp4_block_bytes(shape), b.num_blocks
    before = attend(b, pools)
    used = [(int(n) + block - 1) // block for n in b.lens]
    old = np.concatenate([b.tables[s, :n] for s, n in enumerate(used)]).astype(np.int32)
    free = np.setdiff1d(np.arange(NB), old).astype(np.int32)
    n = used[1]
    ids, new = to_dev(b.tables[1, :n]), to_dev(free[:n])
    staging = torch.empty(n * size, dtype=torch.uint8, device="cuda")
    host = torch.empty(n * size, dtype=torch.uint8, pin_memory=True)
    pkv.kv_blocks_offload(pools.k_dev, ids, staging, host, n, size, NB)
    pkv.kv_blocks_reload(host, staging, pools.k_dev, new, n, size, NB)
    pkv.kv_blocks_gather(pools.v_dev, ids, staging, n, size, NB)
    pkv.kv_blocks_scatter(staging, pools.v_dev, new, n, size, NB)
    b.tables[1, :n] = free[:n]
    assert np.array_equal(attend(b, pools), before)
    other = [torch.zeros_like(pools.k_dev) for _ in range(2)]
    everything = to_dev(np.arange(NB, dtype=np.int32))
    for src, dst in ((pools.k_dev, other[0]), (pools.v_dev, other[1])):
        pkv.kv_blocks_move(src, everything, dst, everything, NB, size, NB, NB)
    pools.k_dev, pools.v_dev = other
    assert np.array_equal(attend(b, pools), before)
