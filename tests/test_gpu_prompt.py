"""Attention of prompts and pieces of them against plain rows in 64 bits."""
import numpy as np
import pytest
import torch

import plain
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from prompt_util import KINDS, check, make_batch, plain_append, plain_prompt, pools_of, refresh, run_prompt, shape_of, upload

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


def test_scales_that_are_not_finite():
    """Of V's blocks with a scale of NaN, or one whose products are infinite, only the rows that see a token of them have anything."""
    b = make_batch([20, 0], [70, 90], 4, 2, 128, 16, 16)
    p = pools_of(b, "blk")
    p.v_scales[b.tables[0][4], 1], p.v_scales[b.tables[1][1], 0] = 255, 254       # tokens 64 to 79 and 16 to 31
    p.v_bits[b.tables[1][1], 0] = 0x7E                                            # 448
    upload(p)
    got = wl.bf16_bits_to_f64(run_prompt(b, p)).reshape(b.q_bits.shape)
    at = b.lens.repeat(b.new) - np.repeat(b.starts[1:], b.new) + np.arange(b.tokens)
    bad = np.zeros(got.shape, bool)
    bad[(np.arange(b.tokens) < 70) & (at >= 64), 2:] = True
    bad[(np.arange(b.tokens) >= 70) & (at >= 16), :2] = True
    assert np.isfinite(got[~bad]).all() and not np.isfinite(got[bad]).any()
    refresh(p, b)
    with np.errstate(all="ignore"):
        want, off, has = plain_prompt(b, p)
    check(b, run_prompt(b, p), np.where(bad, np.nan, want), np.where(bad, np.inf, off), has)


@pytest.mark.parametrize("kind", KINDS)
def test_long_tables(kind):
    """Contexts of many windows of the table, most entries behind them empty, a bound far above the lengths."""
    b = make_batch([5000, 9000, 0, 2047], [3, 33, 2, 1], 4, 1, 64, 16, 17)
    b.tables = np.concatenate([b.tables, np.full((4, 3000), -1, np.int32)], axis=1)
    b.tables[:, -1] = 2 ** 31 - 1
    p = pools_of(b, kind)
    check(b, run_prompt(b, p), *plain_prompt(b, p))


def test_two_calls_at_once():
    """On two streams, with a workspace each, over the same pools."""
    a = make_batch([3000, 5], [4, 60], 8, 2, 128, 16, 18)
    p = pools_of(a, "fp8")
    assert pkv.pkv_prompt_workspace_bytes(shape_of(a), a.tokens) > 0
    want = run_prompt(a, p)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [run_prompt(a, p, stream=s, wait=False) for s in streams]
        torch.cuda.synchronize()
        assert all(np.array_equal(want, to_bits(x)) for x in got)


def test_rows_beyond_4_gib():
    """A call whose queries are 4.6 GiB: the last requests' rows are right, and the first one's."""
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB of free device memory")
    heads, dim, seqs, new = 64, 256, 1100, 135
    b = make_batch([0] * 3, [new] * 3, heads, 8, dim, 64, 19)
    p = pools_of(b, "bf16")
    # the three requests again and again, over the same blocks
    tables, starts = np.tile(b.tables, (seqs // 3 + 1, 1))[:seqs], (np.arange(seqs + 1) * new).astype(np.int32)
    lens, tokens = np.full(seqs, new, np.int32), seqs * new
    assert tokens * heads * dim * 2 > 1 << 32
    few = to_dev(b.q_bits)
    q = few.repeat(seqs // 3 + 1, 1, 1)[:tokens].contiguous()
    out = torch.full_like(q, 0x7FC1)
    shape = pkv.make_shape(seqs, heads, 8, tables.shape[1], b.num_blocks, dim, 64, 0, 0)
    ws = torch.empty(max(pkv.pkv_prompt_workspace_bytes(shape, tokens), 16), dtype=torch.uint8, device="cuda")
    pkv.paged_prompt_attn(q, p.k_dev, p.v_dev, to_dev(tables), to_dev(lens), to_dev(starts), tokens, b.scale, out, shape, ws)
    torch.cuda.synchronize()
    first = out[:3 * new]
    check(b, to_bits(first), *plain_prompt(b, p))
    whole = seqs // 3 * 3 * new
    assert torch.equal(out[:whole].view(seqs // 3, -1), first.reshape(1, -1).expand(seqs // 3, -1))
    assert torch.equal(out[whole:], first[:tokens - whole])


def test_one_token_after_another_as_a_program_goes():
    """Prompts, then steps, each captured in a graph of its own; the graphs share one workspace and run in turn on one stream."""
    b = make_batch([0, 0], [70, 33], 8, 2, 128, 16, 20, spare=20)
    p = pools_of(b, "blk")
    b.tables = b.rng.permutation(b.num_blocks)[:2 * 8].reshape(2, 8).astype(np.int32)
    total = 6
    rows = [wl.normal_bf16(b.rng, (b.tokens + 2 * total, h, 128)) for h in (8, 2, 2)]
    q, k, v = (to_dev(x) for x in rows)
    tables, starts, step_starts = to_dev(b.tables), to_dev(b.starts), None
    lens = to_dev(b.lens)
    shape = shape_of(b)
    need = max(pkv.pkv_prompt_workspace_bytes(shape, b.tokens), pkv.pkv_attn_workspace_bytes(shape), 16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    q_in, k_in, v_in = (torch.empty((2, h, 128), dtype=torch.int16, device="cuda") for h in (8, 2, 2))
    turned, turned_step = torch.empty_like(q[:b.tokens]), torch.empty_like(q_in)
    out, out_step = torch.empty_like(turned), torch.empty_like(turned_step)

    def prompt():
        pkv.kv_rope_append_fp8blk(q[:b.tokens], k[:b.tokens], v[:b.tokens], None, None, None, turned, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens,
                                  starts, pkv.make_rope(b.tokens, 0, 0), shape)
        pkv.paged_prompt_attn_fp8blk(turned, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, starts, b.tokens, b.scale, out, shape, ws)

    def step():
        pkv.kv_rope_append_fp8blk(q_in, k_in, v_in, None, None, None, turned_step, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, step_starts,
                                  pkv.make_rope(2, 0, 0), shape)
        pkv.paged_decode_attn_fp8blk(turned_step, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, tables, lens, b.scale, out_step, shape, ws)

    torch.cuda.synchronize()
    graphs = []
    for run in (prompt, step):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
    values = [wl.bf16_bits_to_f64(x).reshape(x.shape) for x in rows[1:]]
    first_lens, all_q = b.lens.copy(), rows[0]
    fresh = {name: getattr(p, name).copy() for name in ("k_bits", "v_bits", "k_scales", "v_scales")}
    for turn in range(2):      # the same program twice, over what the first left in the pools
        b.lens = first_lens.copy()
        lens.copy_(to_dev(b.lens))
        graphs[0].replay()
        torch.cuda.synchronize()
        plain_append(p, b, [x[:b.tokens] for x in values], plain.positions(b.lens, b.starts, 1 << 30, b.tokens))
        b.q_bits = all_q[:b.tokens]
        check(b, to_bits(out), *plain_prompt(b, p))
        for i in range(total):
            at = b.tokens + 2 * i
            b.lens = b.lens + 1
            for x, y in ((q_in, q), (k_in, k), (v_in, v)):
                x.copy_(y[at:at + 2])
            lens.add_(1)
            graphs[1].replay()
            torch.cuda.synchronize()
            plain_append(p, b, [x[at:at + 2] for x in values], [(s, int(n) - 1) for s, n in enumerate(b.lens)])
            b.q_bits = all_q[at:at + 2]
            got = to_bits(out_step)
            query = wl.bf16_bits_to_f64(b.q_bits).reshape(b.q_bits.shape)
            plain.within(got, *plain.attention(query, p.k, p.v, b.tables, b.lens, b.scale))
            # the same step as a prompt of one token each
            b.starts, kept = np.arange(3, dtype=np.int32), (b.starts, b.tokens)
            b.tokens = 2
            check(b, run_prompt(b, p), *plain_prompt(b, p))
            b.starts, b.tokens = kept
        for name in ("k", "v"):
            assert np.array_equal(getattr(p, name + "_dev").cpu().numpy(), getattr(p, name + "_bits"))
            assert np.array_equal(getattr(p, name + "s_dev").cpu().numpy(), getattr(p, name + "_scales"))
    assert any(not np.array_equal(fresh[n], getattr(p, n)) for n in fresh)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,dim,block", [(8, 2, 128, 16), (16, 2, 64, 64), (6, 2, 256, 32), (13, 1, 128, 32)])
@pytest.mark.parametrize("longest", [40, 3000])
def test_few_rows(kind, hq, hkv, dim, block, longest):
    """A few tokens of each request, of one more than a wavefront has rows for, of one none; contexts from nothing to long."""
    rng = np.random.default_rng(hq + longest)
    new = rng.integers(1, 3, 24)
    new[3], new[7] = 45 * 2 * hkv // hq + 1, 0
    cached = rng.integers(0, longest, 24)
    cached[[0, 5, 9]] = 0, 31, 127
    b = make_batch(cached, new, hq, hkv, dim, block, hq + dim, lead=1, tail=2)
    assert b.tokens <= 24 * (32 * hkv // hq)
    both(b, pools_of(b, kind))


@pytest.mark.expects_id_faults
@pytest.mark.parametrize("kind", KINDS)
def test_few_rows_with_blocks_outside_the_pool(id_faults, kind):
    b = make_batch([500, 16, 0, 300], [4, 3, 2, 1], 8, 2, 128, 16, 21)
    p = pools_of(b, kind)
    b.tables[0][1], b.tables[0][30], b.tables[2][0], b.tables[3][9] = -1, b.num_blocks, 2 ** 31 - 1, -2 ** 31
    got = run_prompt(b, p)
    check(b, got, *plain_prompt(b, p))
    assert (got[b.starts[2]:b.starts[3]] == 0).all()
    assert int(id_faults.item()) == 4 * 2         # a unit each, for each KV head


def test_few_rows_without_finite_scales():
    b = make_batch([70, 200, 30], [3, 4, 2], 4, 2, 128, 16, 22)
    p = pools_of(b, "blk")
    p.v_scales[b.tables[0][4], 1], p.v_scales[b.tables[1][12], 0] = 255, 254      # tokens 64 to 79 of 73, 192 to 207 of 204
    p.v_bits[b.tables[1][12], 0] = 0x7E
    upload(p)
    got = wl.bf16_bits_to_f64(run_prompt(b, p)).reshape(b.q_bits.shape)
    bad = np.zeros(got.shape, bool)
    bad[:3, 2:], bad[3:7, :2] = True, True
    assert np.isfinite(got[~bad]).all() and not np.isfinite(got[bad]).any()


@pytest.mark.parametrize("kind", KINDS)
def test_few_rows_are_those_of_many(kind):
    """The same tokens beside a request that has many: other workgroups, rows within twice the tolerance of each other."""
    b = make_batch([900, 40], [3, 2], 8, 2, 128, 16, 23)
    p = pools_of(b, kind)
    few = wl.bf16_bits_to_f64(run_prompt(b, p)).reshape(b.q_bits.shape)
    want, off, has = plain_prompt(b, p)
    b.tables = np.concatenate([b.tables, b.tables[:1]])
    b.new, b.lens = np.r_[b.new, 500].astype(np.int32), np.r_[b.lens, 500].astype(np.int32)
    b.starts = np.r_[b.starts, b.starts[-1] + 500].astype(np.int32)
    b.tokens += 500
    b.q_bits = np.concatenate([b.q_bits, wl.normal_bf16(b.rng, (500, 8, 128))])
    many = wl.bf16_bits_to_f64(run_prompt(b, p)).reshape(b.q_bits.shape)[:5]
    assert (np.abs(few - want) <= off).all() and (np.abs(many - want) <= off).all() and has.all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,dim,new", [(40, 20, 128, 200), (16, 8, 256, 500), (24, 24, 64, 330)])
def test_longest_work_first(kind, hq, hkv, dim, new):
    """More workgroups than run at once: requests of all lengths, some without tokens, one with more tokens than positions; rows of picked requests."""
    rng = np.random.default_rng(hq)
    many = rng.integers(1, new + 1, 30)
    many[[4, 29]], many[11] = 0, 1
    b = make_batch(rng.integers(0, 600, 30), many, hq, hkv, dim, 16, hq, lead=3, tail=70)
    b.lens[7] = many[7] // 3
    p = pools_of(b, kind)
    got = run_prompt(b, p)
    # the same bits in the order of the requests, as 65 of them are taken
    few = b.lens, b.starts, b.tables
    b.lens = np.r_[b.lens, np.zeros(35, np.int32)].astype(np.int32)
    b.starts = np.r_[b.starts, np.full(35, b.starts[-1])].astype(np.int32)
    b.tables = np.concatenate([b.tables, np.full((35, b.tables.shape[1]), -1, np.int32)])
    assert np.array_equal(got, run_prompt(b, p))
    b.lens, b.starts, b.tables = few
    pick = [0, 7, 11, 23]
    for s in pick:
        one = make_batch([0], [int(many[s])], hq, hkv, dim, 16, 1)
        one.lens, one.tables, one.num_blocks, one.scale = b.lens[s:s + 1], b.tables[s:s + 1], b.num_blocks, b.scale
        rows = slice(int(b.starts[s]), int(b.starts[s + 1]))
        one.q_bits = b.q_bits[rows]
        check(one, got[rows], *plain_prompt(one, p))
    assert (got[:3] == 0x7FC1).all() and (got[b.starts[-1]:] == 0x7FC1).all()
