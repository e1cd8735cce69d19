"""Attention of prompts and pieces of them against plain rows in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from prompt_util import KINDS, check, make_batch, plain_prompt, pools_of, run_prompt, shape_of, upload

pytestmark = pytest.mark.gpu


def both(b, p, **kw):
    got = run_prompt(b, p, **kw)
    check(b, got, *plain_prompt(b, p, kw.get("max_context_len") or None, kw.get("scale")))
    return got


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,block", [(128, 16), (64, 32), (256, 64), (128, 64), (64, 16), (256, 16)])
def test_prompts_of_all_lengths(kind, dim, block):
    new = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129, 200]
    b = make_batch(np.zeros(len(new), int), new, 8, 2, dim, block, dim + block)
    both(b, pools_of(b, kind))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,dim", [(1, 1, 128), (40, 8, 128), (15, 3, 64), (16, 1, 128), (13, 1, 64), (8, 8, 128), (7, 1, 256), (8, 1, 256),
                                        (33, 3, 128), (6, 2, 64), (12, 1, 128), (28, 4, 128)])
def test_heads(kind, hq, hkv, dim):
    b = make_batch([0, 100, 37], [70, 19, 1], hq, hkv, dim, 16, hq)
    both(b, pools_of(b, kind))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 4, 40])
def test_pieces_behind_long_contexts(kind, dim, new):
    """Few rows: contexts are cut and joined."""
    b = make_batch([3000, 0, 511, 512, 1700], [new] * 5, 8, 2, dim, 16, new)
    assert pkv.pkv_prompt_workspace_bytes(shape_of(b), b.tokens) > 0
    both(b, pools_of(b, kind))


def test_mixed_with_steps_and_without_tokens():
    b = make_batch([0, 500, 3, 64, 0, 900, 0], [300, 1, 0, 1, 0, 64, 1], 10, 2, 128, 16, 3)
    both(b, pools_of(b, "bf16"))


@pytest.mark.parametrize("seqs", [62, 63, 64, 65, 127, 128, 300, 2048])
def test_many_requests(seqs):
    rng = np.random.default_rng(seqs)
    b = make_batch(rng.integers(0, 30, seqs), rng.integers(0, 12, seqs), 4, 2, 64, 16, seqs)
    both(b, pools_of(b, "bf16"))


@pytest.mark.parametrize("kind", KINDS)
def test_one_token_each_without_starts(kind):
    b = make_batch([0, 5, 130, 700], [1, 1, 1, 1], 8, 2, 128, 16, 5)
    p = pools_of(b, kind)
    assert np.array_equal(both(b, p), both(b, p, starts=False))


@pytest.mark.parametrize("lead,tail", [(0, 5), (3, 0), (300, 70)])
def test_padding_is_left_as_it_was(lead, tail):
    b = make_batch([0, 20], [40, 30], 8, 2, 128, 16, lead, lead=lead, tail=tail)
    both(b, pools_of(b, "bf16"))


def test_tokens_without_a_position():
    b = make_batch([0, 0, 10], [60, 300, 20], 8, 2, 128, 16, 6)
    b.lens = np.array([20, 0, 30], np.int32)      # 60 and 300 new tokens of contexts of 20 and 0
    both(b, pools_of(b, "bf16"))


@pytest.mark.parametrize("bound", [1, 60, 200])
def test_bound_on_the_lengths(bound):
    b = make_batch([0, 100, 0], [30, 100, 150], 8, 2, 128, 16, 7)
    both(b, pools_of(b, "bf16"), max_context_len=bound)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales(scale):
    b = make_batch([0, 100], [70, 20], 8, 2, 128, 16, 8)
    both(b, pools_of(b, "bf16"), scale=scale)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cached,new", [(0, 100), (50, 90), (1000, 4)])
def test_nothing_behind_a_token_reaches_its_row(kind, cached, new):
    """NaN and infinities in K and V of some tokens, and in all slots and blocks that no token has."""
    b = make_batch([cached, cached // 2], [new, new], 8, 2, 128, 16, cached + new, spare=3)
    p = pools_of(b, kind)
    free = np.ones((b.num_blocks, b.block), bool)
    for s, n in enumerate(b.lens):
        t = np.arange(n)
        free[b.tables[s][t // b.block], t % b.block] = False
    nan = wl.BF16_NAN if kind == "bf16" else wl.E4M3_NAN
    for name in "kv":
        bits = getattr(p, name + "_bits")
        bits[np.broadcast_to(free[:, None, :, None], bits.shape)] = nan
    bad = []
    for s in range(2):
        n = int(b.lens[s])
        for at, name, kvh, dim in ((n - new // 2, "v", 0, 3), (n - 2, "v", 1, 70), (n - 1, "k", 0, 9), (n - new // 3 - 1, "v", 0, 127)):
            id_ = b.tables[s][at // b.block]
            getattr(p, name + "_bits")[id_, kvh, at % b.block, dim] = nan if name == "k" or kind != "bf16" or dim != 70 else 0x7F80
            getattr(p, name)[id_, kvh, at % b.block, dim] = np.nan if name == "k" or kind != "bf16" or dim != 70 else np.inf
            bad.append((s, at, name, kvh, dim))
    upload(p)
    got = run_prompt(b, p)
    want, off, has = plain_prompt(b, p)
    # which elements see something that is not finite
    hit = np.zeros(want.shape, bool)
    for s, at, name, kvh, dim in bad:
        i = int(b.starts[s + 1]) - (int(b.lens[s]) - at)
        rows = slice(max(i, int(b.starts[s])), int(b.starts[s + 1]))
        heads = slice(kvh * 4, kvh * 4 + 4)
        hit[rows, heads, slice(None) if name == "k" else dim] = True
    value = wl.bf16_bits_to_f64(got).reshape(want.shape)
    assert not np.isfinite(value[hit]).any()
    assert np.isfinite(value[~hit & has[:, None, None]]).all()
    check(b, got, want, np.where(hit, np.inf, off), has)


@pytest.mark.expects_id_faults
@pytest.mark.parametrize("kind", KINDS)
def test_blocks_outside_the_pool(id_faults, kind):
    b = make_batch([100, 16, 0], [60, 3, 20], 8, 2, 128, 16, 9)
    p = pools_of(b, kind)
    b.tables[0][1], b.tables[0][4], b.tables[2][0], b.tables[2][1] = -1, b.num_blocks, 2 ** 31 - 1, -2 ** 31
    got = run_prompt(b, p)
    check(b, got, *plain_prompt(b, p))
    assert (got[b.starts[2]:] == 0).all()         # nothing left to see
    # one for each unit, KV head and group of tokens (32 of them with four heads to a KV head) that meet
    assert int(id_faults.item()) == 2 * 2 * 2 + 2 * 2


@pytest.mark.parametrize("kind", KINDS)
def test_blocks_anywhere_give_the_same_bits(kind):
    b = make_batch([700, 30], [50, 90], 8, 2, 128, 16, 10, spare=9)
    p = pools_of(b, kind)
    first = run_prompt(b, p)
    order = b.rng.permutation(b.num_blocks)
    for name in ("k_bits", "v_bits", "k", "v") + (("k_scales", "v_scales") if kind == "blk" else ()):
        x = np.empty_like(getattr(p, name))
        x[order] = getattr(p, name)
        setattr(p, name, x)
    b.tables = np.where(b.tables >= 0, order[b.tables], b.tables).astype(np.int32)
    upload(p)
    assert np.array_equal(first, run_prompt(b, p))


def test_a_request_does_not_depend_on_the_others_contents():
    b = make_batch([10, 400, 0], [40, 70, 64], 8, 2, 128, 16, 11)
    p = pools_of(b, "bf16")
    first = run_prompt(b, p)
    ids = b.tables[1][:int((b.lens[1] + 15) // 16)]
    p.k_bits[ids] = p.v_bits[ids] = wl.BF16_NAN
    upload(p)
    again = run_prompt(b, p)
    rows = np.r_[0:40, 110:174]
    assert np.array_equal(first[rows], again[rows])


def test_written_in_place():
    b = make_batch([0, 900], [100, 5], 8, 2, 128, 16, 12)
    p = pools_of(b, "bf16")
    for batch in (b, make_batch([900], [4], 8, 2, 128, 16, 13)):
        p = pools_of(batch, "bf16")
        first = run_prompt(batch, p)
        q = torch.from_numpy(batch.q_bits.view(np.int16)).cuda()
        assert np.array_equal(first, run_prompt(batch, p, q=q, out=q))


def test_equal_keys_and_values():
    """V of ones gives ones; keys that are all the same give the mean."""
    b = make_batch([0], [200], 4, 2, 128, 16, 14)
    p = pools_of(b, "bf16")
    p.v_bits[:] = 0x3F80
    upload(p)
    got = wl.bf16_bits_to_f64(run_prompt(b, p)).reshape(b.q_bits.shape)
    assert np.abs(got - 1).max() <= 2.0 ** -7      # weights are rounded, their sum is not
    first = run_prompt(b, p)[0]
    assert (first == 0x3F80).all()                  # a token alone


def test_on_another_stream_and_captured():
    b = make_batch([0, 1500, 3], [130, 6, 40], 8, 2, 128, 16, 15)
    p = pools_of(b, "blk")
    want = run_prompt(b, p)
    side = torch.cuda.Stream()
    assert np.array_equal(want, run_prompt(b, p, stream=side))
    outs = [torch.empty(b.q_bits.shape, dtype=torch.int16, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    tables, lens, starts, q = (torch.from_numpy(x).cuda() for x in (b.tables, b.lens, b.starts, b.q_bits.view(np.int16)))
    shape = shape_of(b)
    ws = [torch.empty(pkv.pkv_prompt_workspace_bytes(shape, b.tokens), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for o, w in zip(outs, ws):
            pkv.paged_prompt_attn_fp8blk(q, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, starts, b.tokens, b.scale, o, shape, w)
    for _ in range(3):
        for o in outs:
            o.fill_(0x7FC1)
        graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert np.array_equal(o.cpu().numpy().view(np.uint16), want)
