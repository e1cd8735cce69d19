"""NaN in a part of a context that is attended over by itself and joined with the others: pieces of prompts, shares of decode steps.  It reaches every row
that sees it, also where it is all that a piece has, or where the other pieces' scores are far larger; all else keeps its bits."""
import numpy as np
import pytest
import torch

import formats_util
import plain
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from prompt_util import KINDS, make_batch, plain_prompt, pools_of, run_prompt, shape_of, upload

pytestmark = pytest.mark.gpu


def nan_of(kind):
    return wl.BF16_NAN if kind == "bf16" else wl.E4M3_NAN


def values(bits, like):
    return wl.bf16_bits_to_f64(np.asarray(bits)).reshape(like.shape)


def only_there(b, got, clean, nan):
    """NaN where it has to be, the bits of the clean call elsewhere."""
    found = np.isnan(values(got, b.q_bits))
    assert np.array_equal(found, nan), (np.argwhere(found != nan)[:5].tolist(), int(found.sum()), int(nan.sum()))
    got, clean = np.asarray(got).reshape(nan.shape), np.asarray(clean).reshape(nan.shape)
    assert np.array_equal(got[~nan], clean[~nan])


def nan_queries(b, nan, got, clean, want, off, has):
    """A row of NaN raises no reference maximum, so that the rows beside it, of its request and KV head, may have theirs raised at other tiles: those are
    right to their tolerance, the others' bits are kept."""
    got, clean = (np.asarray(x).reshape(nan.shape) for x in (got, clean))
    rows = nan[:, :, 0].reshape(len(nan), b.hkv, -1).any(-1)                     # of tokens and KV heads
    request = np.repeat(np.arange(len(b.lens)), b.new)
    beside = np.stack([rows[request == s].any(0) for s in range(len(b.lens))])[request].repeat(b.hq // b.hkv, 1)
    assert np.array_equal(np.isnan(values(got, got)), nan)
    assert np.array_equal(got[~beside], clean[~beside])
    bad = ~(np.abs(values(got, got) - want) <= off) & ~nan & has[:, None, None]
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())


def slot_of(b, s, t):
    return b.tables[s][t // b.block], t % b.block


# what the plan cuts: one token of each of many requests, which are four wavefronts' rows, and pieces of prompts, which are a workgroup's
CUT = {"few": ([32 * i for i in range(41)], 1), "many": ([64 * i + 25 for i in range(20)], 40)}


def cut_batch(how, dim, seed):
    cached, new = CUT[how]
    b = make_batch(cached, [new] * len(cached), 8, 2, dim, 16, seed)
    assert pkv.pkv_prompt_workspace_bytes(shape_of(b), b.tokens) > 0
    assert ((b.lens % 32 == 1).all() if how == "few" else (b.lens % 64 == 1).all())      # the last key begins a tile, and a piece somewhere
    return b


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("how", CUT)
def test_prompts_newest_key(how, dim, kind):
    b = cut_batch(how, dim, dim)
    p = pools_of(b, kind)
    clean = run_prompt(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    for s, n in enumerate(b.lens):
        id_, slot = slot_of(b, s, int(n) - 1)
        p.k_bits[id_, s % 2, slot, 11] = nan_of(kind)
        nan[b.starts[s + 1] - 1, 4 * (s % 2):4 * (s % 2) + 4] = True
    upload(p)
    only_there(b, run_prompt(b, p), clean, nan)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("how", CUT)
def test_prompts_queries(how, kind):
    b = cut_batch(how, 128, 1)
    p = pools_of(b, kind)
    clean = run_prompt(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    nan[np.arange(0, b.tokens, 3), np.arange(0, b.tokens, 3) % 8] = True
    plain_rows = plain_prompt(b, p)
    b.q_bits = np.where(nan & (np.arange(128) == 77), wl.BF16_NAN, b.q_bits).astype(np.uint16)
    nan_queries(b, nan, run_prompt(b, p), clean, *plain_rows)


def aligned_first_key(b, p):
    """The first key of each request and KV head is far along that head's first query, so that those rows weigh nothing else."""
    for s in range(len(b.lens)):
        id_, slot = slot_of(b, s, 0)
        for h in range(b.hkv):
            first = values(b.q_bits[b.starts[s], h * (b.hq // b.hkv)], np.zeros(b.dim))
            p.k_bits[id_, h, slot] = wl.f32_to_bf16_bits((first * 32).astype(np.float32))


@pytest.mark.parametrize("how", CUT)
def test_prompts_far_below_the_largest_score(how):
    """V of a key whose weight is below the least number: 32 |q|^2 / sqrt(128) is some 360, 520 in powers of two."""
    b = cut_batch(how, 128, 2)
    p = pools_of(b, "bf16")
    aligned_first_key(b, p)
    upload(p)
    clean = run_prompt(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    for s, n in enumerate(b.lens):
        if n < 100:
            continue
        at = int(n) - int(b.new[s]) - 20 - s      # a key that all new tokens see
        id_, slot = slot_of(b, s, at)
        p.v_bits[id_, 1, slot, 5 + s] = wl.BF16_NAN
        nan[b.starts[s]:b.starts[s + 1], 4:, 5 + s] = True
    upload(p)
    only_there(b, run_prompt(b, p), clean, nan)


@pytest.mark.parametrize("name", ["k", "v"])
def test_prompts_scales(name):
    """A scale of NaN for a block that is all that a piece has."""
    b = make_batch([32 * i + 15 for i in range(41)], [1] * 41, 8, 2, 128, 16, 3)
    assert pkv.pkv_prompt_workspace_bytes(shape_of(b), b.tokens) > 0
    p = pools_of(b, "blk")
    clean = run_prompt(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    for s, n in enumerate(b.lens):
        getattr(p, name + "_scales")[slot_of(b, s, int(n) - 1)[0], s % 2] = 255
        nan[s, 4 * (s % 2):4 * (s % 2) + 4] = True
    upload(p)
    only_there(b, run_prompt(b, p), clean, nan)


def step(b, p, max_context_len=0):
    """Decode attention over any kind of pools."""
    if p.kind != "blk":
        return formats_util.attend(b, p, max_context_len=max_context_len)
    shape = shape_of(b, max_context_len)
    ws = torch.full((max(pkv.pkv_attn_workspace_bytes(shape), 16),), 0xa5, dtype=torch.uint8, device="cuda")
    out = torch.full(b.q_bits.shape, 0x7FC1, dtype=torch.int16, device="cuda")
    pkv.paged_decode_attn_fp8blk(to_dev(b.q_bits), p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables), to_dev(b.lens), b.scale, out, shape, ws)
    torch.cuda.synchronize()
    return to_bits(out)


# lengths of which the last token has a block of its own: a wavefront's only one where a segment has a workgroup, a share's where there are as many blocks
# as wavefronts, and somewhere among long shares
STEPS = {"workgroup": [17, 33, 81, 1, 177], "shares": [16 * i + 1 for i in range(40)], "records": [16 * i + 1 for i in range(40, 150, 8)]}


def step_batch(how, dim, seed):
    lens = STEPS[how]
    b = make_batch(np.array(lens) - 1, [1] * len(lens), 8, 2, dim, 16, seed)
    b.q = values(b.q_bits, b.q_bits)
    return b


def only_newest_key(b, p, kind, bound):
    clean = step(b, p, bound)
    nan = np.zeros(b.q_bits.shape, bool)
    for s, n in enumerate(b.lens):
        id_, slot = slot_of(b, s, int(n) - 1)
        p.k_bits[id_, s % 2, slot, 11] = nan_of(kind)
        nan[s, 4 * (s % 2):4 * (s % 2) + 4] = True
    upload(p)
    only_there(b, step(b, p, bound), clean, nan)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("how", STEPS)
def test_steps_newest_key(how, dim, kind):
    b = step_batch(how, dim, dim)
    only_newest_key(b, pools_of(b, kind), kind, int(b.lens.max()))


@pytest.mark.parametrize("kind", [*KINDS, "fp4"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("how", STEPS)
def test_steps_queries(how, dim, kind):
    """No score of the row is a number: no wavefront has a maximum."""
    b = step_batch(how, dim, 4)
    p = formats_util.pools_of(b, "fp4") if kind == "fp4" else pools_of(b, kind)
    clean = step(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    nan[np.arange(len(b.lens)), np.arange(len(b.lens)) % 8] = True
    plain_rows = plain.attention(b.q, p.k, p.v, b.tables, b.lens, b.scale)
    b.q_bits = np.where(nan & (np.arange(dim) == 7), wl.BF16_NAN, b.q_bits).astype(np.uint16)
    nan_queries(b, nan, step(b, p), clean, *plain_rows, np.ones(len(b.lens), bool))


@pytest.mark.parametrize("how", STEPS)
def test_steps_far_below_the_largest_score(how):
    b = step_batch(how, 128, 5)
    p = pools_of(b, "bf16")
    aligned_first_key(b, p)
    upload(p)
    clean = step(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    for s, n in enumerate(b.lens):
        if n < 30:
            continue
        id_, slot = slot_of(b, s, int(n) - 1 - 2 * s)
        p.v_bits[id_, 1, slot, 5 + s] = wl.BF16_NAN
        nan[s, 4:, 5 + s] = True
    upload(p)
    only_there(b, step(b, p), clean, nan)


@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("how", STEPS)
def test_steps_scales(how, name):
    b = step_batch(how, 128, 6)
    p = pools_of(b, "blk")
    clean = step(b, p)
    nan = np.zeros(b.q_bits.shape, bool)
    for s, n in enumerate(b.lens):
        getattr(p, name + "_scales")[slot_of(b, s, int(n) - 1)[0], s % 2] = 255
        nan[s, 4 * (s % 2):4 * (s % 2) + 4] = True
    upload(p)
    only_there(b, step(b, p), clean, nan)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
def test_steps_with_a_window(kind):
    b = step_batch("records", 128, 7)
    p = formats_util.pools_of(b, kind)
    clean = formats_util.attend(b, p, window=3000, sinks=5)
    nan = np.zeros(b.q_bits.shape, bool)
    nan[np.arange(len(b.lens)), np.arange(len(b.lens)) % 8] = True
    plain_rows = plain.attention(b.q, p.k, p.v, b.tables, b.lens, b.scale, 3000, 5)
    b.q_bits = np.where(nan & (np.arange(128) == 7), wl.BF16_NAN, b.q_bits).astype(np.uint16)
    nan_queries(b, nan, formats_util.attend(b, p, window=3000, sinks=5), clean, *plain_rows, np.ones(len(b.lens), bool))
