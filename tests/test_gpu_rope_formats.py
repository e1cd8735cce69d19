"""Rotated appends: partial and interleaved rotations into every kind of pool, by both launches."""
import numpy as np
import pytest

from formats_util import KINDS, make_batch, pools_of
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
