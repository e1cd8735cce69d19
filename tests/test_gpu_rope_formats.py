"""Rotated appends: partial and interleaved rotations into every kind of pool, by both launches,
queries in place and rows without gaps."""
import numpy as np
import pytest
import torch

from formats_util import KINDS, make_batch, pools_of, shape_of
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv
from paper_2602_11530_amd import workloads as wl
from test_gpu_rope import check, run, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("dim,block", [(64, 32), (128, 16), (256, 64)])
@pytest.mark.parametrize("rotary", [0, 16, 32, 48, 64, 80, 112, 128, 240, 256])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(device, kind, dim, block, rotary, interleaved):
    if rotary > dim:
        pytest.skip("more than a row")
    b = make_batch([30, 200], 4, 2, dim, block, seed=rotary)
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools, starts_of([30, 5]), rotary=rotary, interleaved=interleaved))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,hq,hkv", [(64, 8, 1), (64, 20, 5), (128, 3, 1), (128, 12, 4), (256, 2, 1), (256, 10, 5)])
@pytest.mark.parametrize("rotary,interleaved", [(0, False), (16, False), (48, True), (48, False), (64, True)])
def test_rotations_of_many_tokens(device, kind, dim, hq, hkv, rotary, interleaved):
    """From 1024 tokens on, by both of the launches for them."""
    new = np.array([0, 700, 1, 0, 333, 40, 2])
    b = make_batch(new + np.array([3, 0, 17, 0, 5, 1, 100]), hq, hkv, dim, 16, seed=rotary + dim, spare=2)
    pools = pools_of(b, kind)
    check(b, pools, run(b, pools, starts_of(new), rotary=rotary, interleaved=interleaved))


@pytest.mark.parametrize("dim,hq,hkv", [(64, 8, 1), (128, 12, 4), (128, 40, 8), (256, 10, 5)])
@pytest.mark.parametrize("rotary,interleaved", [(64, False), (48, True)])
def test_many_tokens_in_place(device, dim, hq, hkv, rotary, interleaved):
    new = np.array([900, 1, 300, 17])
    b = make_batch(new + np.array([0, 40, 3, 100]), hq, hkv, dim, 16, seed=dim + hkv)
    pools = pools_of(b, "bf16")
    check(b, pools, run(b, pools, starts_of(new), rotary=rotary, interleaved=interleaved, in_place=True, gap=8))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens", [5, 1200])
def test_rows_without_gaps(device, kind, tokens):
    """Queries, keys and values each for themselves, strides 0: as from one projection."""
    hq, hkv, dim = 4, 2, 128
    b = make_batch(np.full(tokens, 3), hq, hkv, dim, 16, seed=71)
    fused, apart = pools_of(b, kind), pools_of(b, kind)
    apart.k_dev, apart.v_dev = fused.k_dev.clone(), fused.v_dev.clone()
    rows = to_dev(wl.normal_bf16(b.rng, (tokens, hq + 2 * hkv, dim)))
    table, tables, lens = to_dev(b.rng.standard_normal((16, dim)).astype(np.float32)), to_dev(b.tables), to_dev(b.lens)
    weight = to_dev(wl.normal_bf16(b.rng, (dim,)))
    name = "kv_rope_append" + {"bf16": "", "fp8": "_fp8", "fp4": "_fp4"}[kind]
    scales = (0.0134, 0.0171) if kind == "fp8" else ()
    parts = [x.contiguous() for x in rows.split([hq, hkv, hkv], dim=1)]
    row, outs = (hq + 2 * hkv) * dim, []
    for pools, (q, k, v), stride in ((fused, (rows, rows[:, hq:], rows[:, hq + hkv:]), row), (apart, parts, 0)):
        q_out = torch.zeros((tokens, hq, dim), dtype=torch.int16, device="cuda")
        rope = pkv.make_rope(tokens, dim, 16, q_stride=stride, k_stride=stride, v_stride=stride)
        getattr(pkv, name)(q, k, v, weight, weight, table, q_out, pools.k_dev, pools.v_dev, tables, lens, None, *scales, rope, shape_of(b))
        outs.append(q_out)
    torch.cuda.synchronize()
    assert to_bits(outs[0]).any() and torch.equal(*outs)
    assert torch.equal(fused.k_dev, apart.k_dev) and torch.equal(fused.v_dev, apart.v_dev)
