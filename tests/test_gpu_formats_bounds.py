"""Windows and 4-bit pools: no bit of a row depends on the bound on the lengths, whatever launch it leads to."""
import numpy as np
import pytest

import plain
from formats_util import KINDS, attend, make_batch, pools_of

pytestmark = pytest.mark.gpu


# segments: as many as a launch has workgroups, and up to twice that; windows that keep a segment short, and that do not
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind,window,sinks", [(k, w, s) for k in KINDS for w, s in ((60, 4), (150, 20), (2000, 4))]
                         + [("fp4", None, None)])
@pytest.mark.parametrize("seqs,hkv", [(32, 8), (60, 5), (96, 4), (128, 4)])
def test_rows_are_the_same_under_every_bound(device, dim, kind, window, sinks, seqs, hkv):
    rng = np.random.default_rng(seqs + dim)
    b = make_batch(rng.integers(0, 200, seqs), 2 * hkv, hkv, dim, 16, seed=seqs)
    wide = np.full((seqs, 1600 // 16), -1, np.int32)
    wide[:, :b.tables.shape[1]] = b.tables
    b.tables = wide
    pools = pools_of(b, kind)
    loose = attend(b, pools, window, sinks)
    some = slice(0, seqs, 7)
    want, off = plain.attention(b.q[some], pools.k, pools.v, b.tables[some], b.lens[some], b.scale, window, sinks or 0)
    plain.within(loose[some], want, off)
    for bound in (int(b.lens.max()), 700, 1000):
        assert np.array_equal(attend(b, pools, window, sinks, max_context_len=bound), loose), bound


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(None, None), (500, 70), (5000, 0)])
@pytest.mark.parametrize("seqs,hkv", [(1, 1), (9, 8)])
def test_few_segments_of_tiles_up_to_the_longest_that_are_cut(device, dim, window, sinks, seqs, hkv):
    """Segments of up to 12 units a wavefront, a token less and a unit more."""
    longest = 16 * 12 * (4 if dim == 256 else 8)
    for most in (longest, longest - 17, longest + 1):
        b = make_batch([most, *np.random.default_rng(3).integers(1, most, seqs - 1)], 2 * hkv, hkv, dim, 16, seed=seqs + most)
        wide = np.full((seqs, 5 * longest // 32), -1, np.int32)
        wide[:, :b.tables.shape[1]] = b.tables
        b.tables = wide
        pools = pools_of(b, "fp4")
        loose = attend(b, pools, window, sinks)
        want, off = plain.attention(b.q, pools.k, pools.v, b.tables, b.lens, b.scale, window, sinks or 0)
        plain.within(loose, want, off)
        assert np.array_equal(attend(b, pools, window, sinks, max_context_len=most), loose)
