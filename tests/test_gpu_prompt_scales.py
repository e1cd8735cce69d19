"""Softmax scales that are not numbers: rows of NaN, as decode attention gives them."""
import numpy as np
import pytest

from prompt_util import KINDS, make_batch, pools_of, run_prompt
from test_gpu_nan_pieces import CUT, values
from test_gpu_prompt import both

pytestmark = pytest.mark.gpu

BATCHES = {**{how: (cached, [new] * len(cached)) for how, (cached, new) in CUT.items()}, "whole": ([0] * 30, [40] * 30)}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("how", BATCHES)
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
def test_scales_that_are_no_numbers(how, kind, scale):
    b = make_batch(*BATCHES[how], 8, 2, 128, 16, 1, lead=2, tail=3)
    got = run_prompt(b, pools_of(b, kind), scale=scale)
    assert np.isnan(values(got, b.q_bits)).all()                              # padding holds a NaN of its own
    assert (got[:2] == 0x7FC1).all() and (got[-3:] == 0x7FC1).all() and (got[2:-3] != 0x7FC1).any()


@pytest.mark.parametrize("how", BATCHES)
@pytest.mark.parametrize("scale", [1e-30, -1e-38, 1e-45])
def test_smallest_scales(how, scale):
    """Below the normal numbers, too: the mean of V."""
    b = make_batch(*BATCHES[how], 8, 2, 128, 16, 2)
    both(b, pools_of(b, "bf16"), scale=scale)
