"""The plain implementations that the tests of the 4-bit format compare with, pinned to values worked out by hand (no GPU)."""
import numpy as np
import pytest

import plain


def test_codes_and_scales():
    x = np.zeros((1, 64))
    x[0, :9] = [6, -5, 5.1, 2.5, 1.75, -0.25, 0.26, -0.0, 0.75]
    x[0, 32:35] = [7, 1, 0.5]                # 7 would be rounded to 8: the scale is 2
    code, scale = plain.quantise(x)
    assert code[0, :9].tolist() == [7, 8 + 6, 7, 4, 4, 8, 1, 8, 2]
    assert scale.tolist() == [[127, 128]]
    assert code[0, 32:35].tolist() == [6, 1, 0]     # 3.5 -> 4, 0.5, 0.25 -> 0


@pytest.mark.parametrize("most,scale", [(6.99, 127), (4.0, 127), (3.49, 126), (3.5, 127), (0.0, 7), (2.0 ** -130, 7), (3.0e38, 252),
                                        (np.inf, 252), (np.nan, 255)])
def test_scales(most, scale):
    x = np.zeros((1, 32))
    x[0, 5] = most
    assert plain.quantise(x)[1].tolist() == [[scale]]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("is_v", [False, True])
def test_tiles_hold_every_value_once(dim, is_v):
    code_at, scale_at, _ = plain._places(dim, is_v)
    assert sorted(code_at.ravel().tolist()) == sorted(2 * list(range(8 * dim)))
    assert sorted(scale_at.ravel().tolist()) == sorted(32 * list(range(8 * dim, plain.tile_bytes(dim))))
    rng = np.random.default_rng(3)
    code, power = rng.integers(0, 16, (2, 3, 32, dim)), rng.integers(-4, 5, (2, 3, 32, dim // 32))
    x = np.where(code >= 8, -1, 1) * plain.E2M1[code & 7] * 2.0 ** np.repeat(power, 32, -1)
    assert np.array_equal(plain.decode(plain.encode(x, is_v), dim, is_v), x)


def test_attention_sees_the_window_and_the_sinks():
    k = np.zeros((4, 1, 16, 64))
    v = np.arange(64.0).reshape(4, 1, 16, 1).repeat(64, 3)
    tables, q = np.arange(4)[None], np.ones((1, 1, 64))
    mean = lambda **kw: plain.attention(q, k, v, tables, [50], 1.0, **kw)[0][0, 0, 0]  # noqa: E731
    assert np.isclose(mean(), np.arange(50).mean())
    assert np.isclose(mean(window=3, sinks=2), np.mean([0, 1, 47, 48, 49]))
    assert np.isclose(mean(window=0, sinks=2), 0.5) and mean(window=0, sinks=0) == 0
    assert np.isclose(mean(window=45, sinks=20), np.arange(50).mean())
