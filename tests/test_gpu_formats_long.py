"""Shares of more units than a wavefront describes at a time (64), over 4-bit pools and with windows: descriptors are taken over from window to window, pairs
of tiles end at a window's end, segments straddle both and the shares.  Many table entries share a few hundred blocks, so the pools stay small."""
import numpy as np
import pytest

import plain
import routes
from formats_util import KINDS, attend, make_batch, pools_of

pytestmark = pytest.mark.gpu

BLOCKS = 300


def units_seen(n, window, sinks):
    t = np.arange(n)
    return len(np.unique(t[(t >= n - window) | (t < sinks)] // 16))


def long_batch(dim, share, window, sinks, seed, hkv=8):
    """Requests of 50 to 4000 tokens, as many as give every wavefront `share` units; some of up to 30000, empty and tiny ones among them."""
    rng = np.random.default_rng(seed)
    lens, units = [], 0
    want = share * routes.full_waves(dim) // hkv
    while units < want:
        kind = len(lens) % 40
        n = 0 if kind == 7 else int(rng.integers(1, 40) if kind in (11, 12) else rng.integers(4000, 30000) if kind == 20 else 50 * 80 ** rng.random())
        units += units_seen(n, window, sinks)
        lens.append(n)
    b = make_batch(np.zeros(len(lens), np.int32), hkv, hkv, dim, 16, seed)
    b.lens, b.num_blocks = np.asarray(lens, np.int32), BLOCKS
    b.tables = rng.integers(0, BLOCKS, (len(lens), (max(lens) + 15) // 16)).astype(np.int32)
    b.tables[np.arange(b.tables.shape[1])[None, :] >= (b.lens[:, None] + 15) // 16] = -1
    assert share * 0.99 < hkv * units / routes.full_waves(dim) < share * 1.2
    return b


def some(b):
    """The first and the last request, a long one, and others of all lengths: some hundred segments, of which every second or third has a window's end."""
    return np.unique([0, len(b.lens) - 1, 20, *np.random.default_rng(1).integers(0, len(b.lens), 24)])


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("share,partition", [(65, 0), (66, 48), (128, 16), (200, 80)])
@pytest.mark.parametrize("kind,window,sinks", [("fp4", None, 0)] + [(k, 1501, 70) for k in KINDS])
def test_long_shares(device, dim, share, partition, kind, window, sinks):
    b = long_batch(dim, share, 1 << 30 if window is None else window, sinks, seed=share + dim)
    pools = pools_of(b, kind)
    got, at = attend(b, pools, window, sinks, partition_size=partition), some(b)
    want, off = plain.attention(b.q[at], pools.k, pools.v, b.tables[at], b.lens[at], b.scale, window, sinks)
    plain.within(got[at], want, off)
