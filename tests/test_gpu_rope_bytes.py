"""Rows that are neither normalised nor rotated go into the pools as the plain appends put them, byte for byte."""
import numpy as np
import pytest
import torch

from formats_util import KINDS, make_batch, pools_of, shape_of
from gpu_util import to_bits, to_dev
from paper_2602_11530_amd import binding as pkv

pytestmark = pytest.mark.gpu

SCALES = {"bf16": [()], "fp4": [()],     # beyond 2^60 the quotient is divided out
          "fp8": [(0.0134, 0.0171), (1.0, 0.75), (2.0 ** -70, 2.0 ** 70), (3e-38, 1e38), (1e-45, 0.1), (2.0 ** 60, 2.0 ** -60)]}


@pytest.mark.parametrize("kind,scales", [(k, s) for k in KINDS for s in SCALES[k]])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_as_they_are_are_the_append(device, kind, scales, dim):
    """Every bf16 value, zeros of both signs, infinities and NaN among them: without norm and rotation the bytes are the append's."""
    S, hkv = 65536 // (2 * dim), 2
    bits = np.arange(65536, dtype=np.uint16).reshape(S, hkv, dim)
    b = make_batch(np.full(S, 5), 1, 1, dim, 16, seed=70)
    b.hq = b.hkv = hkv
    pools = [pools_of(b, kind) for _ in range(2)]
    for x, y in (("k_dev", "k_bits"), ("v_dev", "v_bits")):
        setattr(pools[1], x, getattr(pools[0], x).clone())
    shape = shape_of(b)
    suffix = {"bf16": "", "fp8": "_fp8", "fp4": "_fp4"}[kind]
    tables, lens = to_dev(b.tables), to_dev(b.lens)
    getattr(pkv, "kv_append" + suffix)(to_dev(bits), to_dev(bits[::-1].copy()), pools[0].k_dev, pools[0].v_dev, tables, lens, *scales, shape)
    q = np.concatenate([bits, bits, bits[::-1]], axis=1)
    d = to_dev(q)
    q_out = torch.zeros((S, hkv, dim), dtype=torch.int16, device="cuda")
    row = 3 * hkv * dim
    rope = pkv.make_rope(S, 0, 0, q_stride=row, k_stride=row, v_stride=row)
    getattr(pkv, "kv_rope_append" + suffix)(d, d[:, hkv:], d[:, 2 * hkv:], None, None, None, q_out, pools[1].k_dev, pools[1].v_dev, tables, lens, None,
                                            *scales, rope, shape)
    torch.cuda.synchronize()
    number = (bits & 0x7fff) <= 0x7f80                          # of a NaN it is said only that it is one
    assert np.array_equal(to_bits(q_out)[number], bits[number])
    for x in ("k_dev", "v_dev"):
        want, got = (getattr(p, x).cpu().numpy() for p in pools)
        if kind == "bf16":
            want, got = (np.where((a.view(np.uint16) & 0x7fff) > 0x7f80, 0x7fff, a.view(np.uint16)) for a in (want, got))
        elif kind == "fp8":
            want, got = (np.where((a & 0x7f) == 0x7f, 0x7f, a) for a in (want, got))
        assert not (want != got).any(), (x, np.argwhere(want != got)[:4].tolist(), want[want != got][:4], got[want != got][:4])
