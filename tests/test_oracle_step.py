"""Pins of the step oracle: masks and attention against plain loops, the
4-bit grid against every code and midpoint."""
import math

import numpy as np
import pytest

from oracle.attention import causal_gqa_attention
from oracle.step import (E2M1, e2m1_decode, e2m1_encode, rms_norm, step_attention,
                         visible_keys)


@pytest.mark.parametrize("pos,lo,window,sinks,expect", [
    (5, 0, 0, 0, [0, 1, 2, 3, 4, 5]),
    (5, 2, 0, 3, [2, 3, 4, 5]),          # sinks add nothing without a window
    (5, 0, 1, 0, [5]),
    (5, 0, 2, 1, [0, 4, 5]),
    (5, 2, 2, 1, [2, 4, 5]),             # sinks count from the first key
    (5, 0, 100, 7, [0, 1, 2, 3, 4, 5]),
    (1, 0, 1, 7, [0, 1]),                # sinks past the row are not visible
    (5, 6, 3, 2, []),
    (-1, 0, 0, 0, []),
])
def test_visible_keys(pos, lo, window, sinks, expect):
    assert np.nonzero(visible_keys(pos, lo, window, sinks, 8))[0].tolist() == expect


def test_attention_without_window_is_the_causal_oracle():
    rng = np.random.default_rng(0)
    q, K, V = rng.normal(size=(3, 4, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    out, lse, mag, top = step_attention(q, [2, 5, 8], [0, 1, 0], K, V)
    ref, rlse = causal_gqa_attention(q, [2, 5, 8], K, V, kv_lo=[0, 1, 0])
    np.testing.assert_allclose(out, ref, rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(lse, rlse, rtol=1e-12)
    assert (mag >= np.abs(out) - 1e-15).all() and (top > 0).all()


def test_attention_with_window_by_loops():
    rng = np.random.default_rng(1)
    q, K, V = rng.normal(size=(1, 2, 4)), rng.normal(size=(7, 1, 4)), rng.normal(size=(7, 1, 4))
    out, lse, _, _ = step_attention(q, [6], [1], K, V, window=2, n_sinks=1)
    for h in range(2):
        keys = [1, 5, 6]
        s = [sum(q[0, h, i] * K[j, 0, i] for i in range(4)) / 2.0 for j in keys]
        z = sum(math.exp(x) for x in s)
        for i in range(4):
            want = sum(math.exp(x) * V[j, 0, i] for x, j in zip(s, keys)) / z
            assert out[0, h, i] == pytest.approx(want, rel=1e-12)
        assert lse[0, h] == pytest.approx(math.log(z), rel=1e-12)


def test_rows_that_see_nothing():
    z = np.ones((4, 1, 4))
    out, lse, _, _ = step_attention(np.ones((2, 1, 4)), [-1, 2], [0, 3], z, z, window=1)
    assert not out.any() and np.isneginf(lse).all()


def test_norm():
    x = np.array([[3.0, -4.0]])
    np.testing.assert_allclose(rms_norm(x, [2.0, 1.0], 0.5), [[6 / math.sqrt(13), -4 / math.sqrt(13)]])


def test_e2m1_grid_and_ties():
    # scale 1: a block with its largest magnitude in (3, 6]
    vals = [6, -6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, .2501, .7499, 5.001, 0, -0.0]
    want = [6, -6, 0, 1, 1, 2, 2, 4, 4, -0.0, -1, .5, .5, 6, 0, -0.0]
    x = np.array(vals + list(E2M1) + list(-E2M1), dtype=np.float64)
    codes, scale = e2m1_encode(x)
    assert scale.tolist() == [127]
    back = e2m1_decode(codes, scale)
    np.testing.assert_array_equal(back, want + list(E2M1) + list(-E2M1))
    assert np.signbit(back[9]) and np.signbit(back[15]) and not np.signbit(back[14])
    assert codes[0] == 0xf7 and codes[1] == 0x20


@pytest.mark.parametrize("amax,k", [(6.0, 0), (6.001, 1), (3.001, 0), (3.0, -1), (1.0, -2),
                                    (2.0 ** -130, -126), (0.0, 0), (3e38, 126)])
def test_e2m1_scale(amax, k):
    x = np.zeros(32)
    x[7] = -amax
    assert e2m1_encode(x)[1].tolist() == [k + 127]


def test_e2m1_non_finite_block():
    x = np.ones(64)
    x[40] = np.inf
    codes, scale = e2m1_encode(x)
    assert scale[1] == 255 and scale[0] == 125
    back = e2m1_decode(codes, scale)
    assert np.isnan(back[32:]).all() and (back[:32] == 1).all()
