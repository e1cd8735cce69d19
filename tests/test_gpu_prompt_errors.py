"""How far rows of prompts are from those in 64 bits, all together: a key that is lost or taken twice is some 1/sqrt(keys) of a row, ten times what roundings are."""
import numpy as np
import pytest

from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from prompt_util import KINDS, encode, make_batch, pools_of, power_of, refresh, run_prompt, shape_of, upload

pytestmark = pytest.mark.gpu

# A rounding to bf16 is off by up to half a step, evenly over that, and steps are 2^-7 of the power of two below a value: its mean square is
# (step)^2 / 12.  That of a weight is at most (2^-7 w)^2 / 12, where its mantissa is 1.
STEP = 2.0 ** -7
# Roundings are independent.  A row's part is taken relative to its own size, so that long contexts, whose rows are small, count as much as short ones.  The sum of N
# even squares is within 1 / sqrt(N) of its mean in some two of three cases; N is 4000 at the least here, but a row's weights are shared by its dims, so that of
# weights there are fewer: 20 % of a mean square is more than four times that where there are 500 of them.
MARGIN = 1.1


def pools(b, kind):
    """Values of about one, so that a row has weights of many keys: those of prompt_util differ so much by the block that one key has nearly all."""
    p = pools_of(b, kind)
    if kind == "blk":
        for name in "kv":
            x = b.rng.standard_normal(p.k.shape) * np.exp(0.2 * b.rng.standard_normal((b.num_blocks, b.hkv, 1, 1)))
            e = power_of(np.abs(x).max(axis=(2, 3)))
            getattr(p, name + "_bits")[:] = encode(x / 2.0 ** e[..., None, None])
            getattr(p, name + "_scales")[:, :b.hkv] = e + 127
        refresh(p, b)
        upload(p)
    return p


def squares(b, p):
    """Of the rows of those tokens: the reference, the mean squares of its rounding and of the weights'."""
    q = wl.bf16_bits_to_f64(b.q_bits).reshape(b.q_bits.shape)
    group = b.hq // b.hkv
    out, weights = np.zeros(q.shape), np.zeros(q.shape)
    for s, n in enumerate(b.lens):
        t = np.arange(int(n))
        ids = b.tables[s][t // b.block]
        k, v = p.k[ids, :, t % b.block], p.v[ids, :, t % b.block]
        for i in range(int(b.starts[s]), int(b.starts[s + 1])):
            m = int(n) - int(b.starts[s + 1]) + i + 1
            for h in range(b.hkv):
                heads = slice(h * group, (h + 1) * group)
                score = q[i, heads] @ k[:m, h].T * b.scale
                w = np.exp(score - score.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[i, heads] = w @ v[:m, h]
                weights[i, heads] = (w * w) @ (v[:m, h] ** 2)
    step = STEP * 2.0 ** np.floor(np.log2(np.abs(out)))
    return out, (step ** 2).sum(-1) / 12, STEP ** 2 * weights.sum(-1) / 12


def error(b, p, one_number):
    """Rows, and of each head's row the squares of its error and of the bound without a margin, relative to its size."""
    out, rounding, weights = squares(b, p)
    got = wl.bf16_bits_to_f64(run_prompt(b, p)).reshape(out.shape)
    size = (out ** 2).sum(-1)
    found, bound = ((got - out) ** 2).sum(-1) / size, (rounding + (weights if one_number else 0)) / size
    print(f"relative L2 {np.sqrt(found.mean()):.6f}, bound {MARGIN * np.sqrt(bound.mean()):.6f}")
    assert found.mean() <= MARGIN ** 2 * bound.mean()
    return got, bound


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,hq,hkv", [(64, 8, 2), (128, 8, 2), (256, 8, 2), (128, 5, 1), (64, 16, 1)])
@pytest.mark.parametrize("new", [1, 2])
def test_few_rows(kind, dim, hq, hkv, new):
    """Over bf16 pools weights are two bf16 numbers, as in the decode kernels: there is the rounding of the rows and nothing else."""
    b = make_batch([4000, 30, 1999, 700, 0, 512, 1200, 3100], [new] * 8, hq, hkv, dim, 16, dim + new)
    assert b.tokens <= 8 * (32 * hkv // hq)
    error(b, pools(b, kind), kind != "bf16")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,block", [(64, 32), (128, 16), (256, 64)])
@pytest.mark.parametrize("cut", [True, False])
def test_many_rows(kind, dim, block, cut):
    b = make_batch([3000, 700], [40, 33], 8, 2, dim, block, dim) if cut else make_batch([0] * 40, [40] * 40, 32, 8, dim, block, dim)
    assert (pkv.pkv_prompt_workspace_bytes(shape_of(b), b.tokens) > 0) == cut
    error(b, pools(b, kind), True)


@pytest.mark.parametrize("kind", KINDS)
def test_one_key_of_thousands(kind):
    """The bound finds a key of 3000 that the reference weighs otherwise than the kernel."""
    b = make_batch([3000, 3000], [2, 40], 8, 2, 128, 16, 5)
    p = pools(b, kind)
    got, bound = error(b, p, True)
    for s in range(2):
        p.k[b.tables[s][70], :, 3] = 0
    other, _, _ = squares(b, p)
    assert (((got - other) ** 2).sum(-1) / (other ** 2).sum(-1)).mean() > 2 * MARGIN ** 2 * bound.mean()
