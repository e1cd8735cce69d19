"""Appends into pools with a scale for each block and KV head: signalling NaN among the values, padding far behind the last request."""
import numpy as np
import pytest
import torch

import plain
from gpu_util import to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from prompt_util import make_batch, plain_append, pools_of, shape_of

pytestmark = pytest.mark.gpu

SIGNALLING = [0x7F81, 0x7FBF, 0xFF81, 0xFFBF]
NANS = SIGNALLING + [0x7FC0, 0xFFFF]


def compare(p):
    """Bytes and scales as they have to be; a NaN may be either one."""
    for name in "kv":
        got, want = getattr(p, name + "_dev").cpu().numpy(), getattr(p, name + "_bits")
        same = (got == want) | ((got & 0x7F) == 0x7F) & ((want & 0x7F) == 0x7F)
        scales = getattr(p, name + "s_dev").cpu().numpy()
        wrong = np.argwhere(scales != getattr(p, name + "_scales"))
        assert not len(wrong), (name, len(wrong), wrong[:5].tolist())
        assert same.all(), (name, int((~same).sum()), np.argwhere(~same)[:5].tolist())


def append(b, p, bits, starts=True, norm=None):
    rope = pkv.make_rope(b.tokens, 0, 0)
    pkv.kv_rope_append_fp8blk(None, to_dev(bits[0]), to_dev(bits[1]), None, norm, None, None, p.k_dev, p.v_dev, p.ks_dev, p.vs_dev, to_dev(b.tables),
                              to_dev(b.lens), to_dev(b.starts) if starts else None, rope, shape_of(b))
    torch.cuda.synchronize()
    at = plain.positions(b.lens, b.starts if starts else None, 1 << 30, b.tokens)
    plain_append(p, b, [wl.bf16_bits_to_f64(x).reshape(x.shape) for x in bits], at)
    compare(p)


def rows(b):
    """Small values, so that a scale taken from a NaN leaves nothing of them, and one of them larger than what blocks hold."""
    out = []
    for _ in range(2):
        x = wl.normal_bf16(b.rng, (b.tokens, b.hkv, b.dim))
        x[::2, :, b.dim // 2 + 1] = 0x4280      # 64
        out.append(x)
    return out


@pytest.mark.parametrize("dim,block", [(128, 16), (64, 64), (256, 32)])
@pytest.mark.parametrize("cached", [0, 5])
def test_signalling_nan_in_a_step(dim, block, cached):
    """In every place of a row, of a block that begins or that holds tokens."""
    b = make_batch([cached] * dim, [1] * dim, 2, 2, dim, block, dim + cached)
    p = pools_of(b, "blk")
    bits = rows(b)
    for s in range(dim):
        for i, x in enumerate(bits):
            x[s, s % 2, s] = NANS[(s // 2 + i) % len(NANS)]
    append(b, p, bits, starts=False)


@pytest.mark.parametrize("dim,block", [(128, 16), (64, 64), (256, 32), (128, 64)])
@pytest.mark.parametrize("cached", [0, 5])
def test_signalling_nan_in_a_piece(dim, block, cached):
    """In every place of a row and every row that a lane has."""
    b = make_batch([cached] * dim, [3 + s % (block + 9) for s in range(dim)], 2, 2, dim, block, dim + block + cached)
    p = pools_of(b, "blk")
    bits = rows(b)
    for s in range(dim):
        for i, x in enumerate(bits):
            x[b.starts[s] + s * 7 % int(b.new[s]), (s + i) % 2, s] = NANS[(s + i) % len(NANS)]
    append(b, p, bits)


def test_nothing_but_nan_and_infinities():
    b = make_batch([0, 3, 0, 3, 20], [1, 1, 6, 6, 30], 2, 2, 128, 16, 1)
    p = pools_of(b, "blk")
    bits = [np.full((b.tokens, 2, 128), x, np.uint16) for x in (0x7F81, 0xFFBF)]
    bits[0][:, 0, ::3] = 0x7F80
    bits[1][:, 1, 1::3] = 0xFF80
    append(b, p, bits)


@pytest.mark.parametrize("dim,block", [(128, 16), (64, 64), (256, 32)])
def test_padding_of_thousands_of_tokens(dim, block):
    """All slots of the tokens behind the last request fall to it."""
    b = make_batch([0, 40, 7], [30, 1, 50], 2, 2, dim, block, dim, tail=9000)
    append(b, pools_of(b, "blk"), rows(b))
