"""Infinite values in K: a score of minus infinity weighs nothing wherever its key lies in the cut of a context, a row that has no other score is NaN, and so
is one with a score of plus infinity, as the formula has it."""
import numpy as np
import pytest
import torch

import formats_util
from gpu_util import to_dev
from paper_2602_11530_amd import workloads as wl
from prompt_util import make_batch, pools_of, run_prompt
from test_gpu_nan_pieces import CUT, STEPS, slot_of, step_batch, values

pytestmark = pytest.mark.gpu


def rows_of(b, p, tokens, weight_bits):
    """Rows in 64 bits and how far a result may be from them, (request, keys seen) of each token given.  Keys with a score of minus infinity are
    left out.  The errors are those of prompt_util.plain_prompt, with weights held to 2^-weight_bits."""
    out, off = np.zeros((2, len(tokens), b.hq, b.dim))
    group = b.hq // b.hkv
    q = values(b.q_bits, b.q_bits)
    for i, (s, m) in enumerate(tokens):
        t = np.arange(m)
        ids = b.tables[s][t // b.block]
        for h in range(b.hq):
            k, v = p.k[ids, h // group, t % b.block], p.v[ids, h // group, t % b.block]
            with np.errstate(invalid="ignore"):
                score = k @ q[i, h] * float(np.float32(b.scale))
            if np.isnan(score).any() or (score == np.inf).any() or (score == -np.inf).all():
                out[i, h] = np.nan
                continue
            k, v, score = k[score > -np.inf], v[score > -np.inf], score[score > -np.inf]
            w = np.exp(score - score.max())
            w /= w.sum()
            out[i, h] = w @ v
            d = b.dim * 2.0 ** -24 * (np.abs(k) @ np.abs(q[i, h])).max() * b.scale + 2.0 ** -21 * (1 + np.abs(score).max())
            off[i, h] = (2 * d + 2.0 ** -weight_bits + m * 2.0 ** -23) * (w @ np.abs(v))
    return out, off + 2.0 ** -8 * np.abs(out) + 2.0 ** -130


def compare(got, want, off):
    got = values(got, want)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), (np.argwhere(np.isnan(got) != nan)[:5].tolist(), int(np.isnan(got).sum()), int(nan.sum()))
    bad = ~(np.abs(got - want) <= off) & ~nan
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], off[bad][:3])


def infinite(b, p, s, tokens, dim=11):
    """K of those tokens of a request: infinite, of both signs by the KV head, so that of each group's heads some have one score and some the other."""
    for t in tokens:
        id_, slot = slot_of(b, s, int(t))
        for h in range(b.hkv):
            p.k_bits[id_, h, slot, dim] = (0x7F80, 0xFF80)[(h + s) % 2]
    p.k = wl.bf16_bits_to_f64(p.k_bits).reshape(p.k_bits.shape)
    p.k_dev = to_dev(p.k_bits)


def alike(b):
    """Queries of a group that all have one sign where K is infinite, in some requests: no wavefront has another score then."""
    first = b.starts[:-1:2] if hasattr(b, "starts") else np.arange(0, len(b.q_bits), 2)
    for i in first:
        b.q_bits[i, :, 11] = (b.q_bits[i, :, 11] & 0x7FFF) | np.repeat([0x8000, 0] * (b.hkv // 2), b.hq // b.hkv)
    b.q = values(b.q_bits, b.q_bits)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("how", STEPS)
@pytest.mark.parametrize("where", ["newest", "first block", "all"])
def test_steps(how, dim, where):
    b = step_batch(how, dim, dim + 1)
    alike(b)
    p = pools_of(b, "bf16")
    for s, n in enumerate(b.lens):
        infinite(b, p, s, [n - 1] if where == "newest" else range(min(int(n), 16)) if where == "first block" else range(int(n)) if s < 6 else [])
    got = formats_util.attend(b, p)
    compare(got, *rows_of(b, p, [(s, int(n)) for s, n in enumerate(b.lens)], 15))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("how", CUT)
@pytest.mark.parametrize("where", ["newest", "first block", "all"])
def test_prompts(how, dim, where):
    cached, new = CUT[how]
    b = make_batch(cached, [new] * len(cached), 8, 2, dim, 16, dim + 2)
    alike(b)
    p = pools_of(b, "bf16")
    for s, n in enumerate(b.lens):
        infinite(b, p, s, [n - 1] if where == "newest" else range(min(int(n), 16)) if where == "first block" else range(int(n)) if s < 6 else [])
    tokens = [(s, int(b.lens[s]) - int(b.new[s]) + i + 1) for s in range(len(b.lens)) for i in range(int(b.new[s]))]
    compare(run_prompt(b, p), *rows_of(b, p, tokens, 8))


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompts_whole(dim):
    """Contexts that are not cut; the first token sees nothing but itself."""
    b = make_batch([0] * 30, [40] * 30, 32, 8, dim, 16, dim + 3)
    alike(b)
    p = pools_of(b, "bf16")
    for s in range(30):
        infinite(b, p, s, range(1 + s % 3))
    tokens = [(s, i + 1) for s in range(30) for i in range(40)]
    compare(run_prompt(b, p), *rows_of(b, p, tokens, 8))


@pytest.mark.expects_id_faults
@pytest.mark.parametrize("how", ["steps", "few", "many"])
def test_rows_without_blocks_are_zeros(id_faults, how):
    """Nothing seen is not the same as nothing that weighs anything."""
    new = 40 if how == "many" else 1
    b = make_batch([500, 100, 700, 0], [new] * 4, 8, 2, 128, 16, 9)
    b.q = values(b.q_bits, b.q_bits)
    p = pools_of(b, "bf16")
    for s in (0, 1, 2):
        infinite(b, p, s, range(int(b.lens[s])))
    b.tables[1] = np.where(b.tables[1] >= 0, b.num_blocks, -1)
    b.tables[3] = -1
    run = formats_util.attend if how == "steps" else run_prompt
    got = values(run(b, p), b.q_bits).reshape(4, new, 8, 128)
    assert (got[[1, 3]] == 0).all() and np.isnan(got[[0, 2]]).all() and int(id_faults.item()) > 0
