"""Pins of the cache oracle to things other than itself: the decoder oracle's
rotation and causal attention, the norm's definition, the 4-bit format's levels,
its smallest scale and its error bound, and what an evicted page, a window and
first tokens leave visible."""
import numpy as np
import pytest

from oracle.cache import LEVELS, PagedCache, mxfp4_block, mxfp4_rows, mxfp4_values, qk_norm_rope, rope_axes
from oracle.decoder import causal_attention, rms_norm
from oracle.predictor import rope


def test_axes_in_runs_and_in_turn():
    assert rope_axes([2, 1, 1], False) == [0, 0, 1, 2]
    assert rope_axes([3, 1, 2], True) == [0, 1, 2, 0, 2, 0]
    assert rope_axes([0, 2], True) == [1, 1]


def test_rotation_is_the_decoders_for_one_axis_and_norm_is_rms():
    rng = np.random.default_rng(0)
    x, pos, g = rng.standard_normal((5, 3, 64)), np.array([0, 1, 7, 200, 4000]), rng.standard_normal(64)
    got = qk_norm_rope(x, pos[None], g, 64, [32], eps=1e-5)
    for h in range(3):
        np.testing.assert_allclose(got[:, h], rope(rms_norm(x[:, h], g, 1e-5), pos, 10000.0), atol=1e-12)
    # equal positions on all axes are one axis; values past rot stay
    three = qk_norm_rope(x, np.stack([pos] * 3), None, 32, [4, 6, 6], interleaved=True)
    np.testing.assert_allclose(three[..., :32], qk_norm_rope(x, pos[None], None, 32, [16])[..., :32])
    np.testing.assert_array_equal(three[..., 32:], x[..., 32:])


def test_four_bit_levels_are_fixed_points_and_the_scale_is_the_smallest():
    for e in (-126, -3, 0, 100):
        block = np.array([s * v * 2.0 ** e for s in (1, -1) for v in LEVELS] * 2)
        codes, byte = mxfp4_block(block)
        assert byte == max(e, -126) + 127
        np.testing.assert_array_equal(mxfp4_values(codes, byte), block)
    assert mxfp4_block([7.0] + [0.0] * 31)[1] == 127 and mxfp4_block([7.0001] + [0.0] * 31)[1] == 128
    assert mxfp4_block([0.0] * 32) == ([0] * 32, 1)
    assert mxfp4_block([float("inf")] + [1.0] * 31)[1] == 255 and np.isnan(mxfp4_values([0], 255)).all()


def test_four_bit_error_is_half_a_step_and_storing_again_changes_nothing():
    x = np.random.default_rng(1).standard_normal((50, 64)) * np.exp(np.random.default_rng(2).standard_normal((50, 1)))
    y = mxfp4_rows(x)
    top = 2.0 ** np.ceil(np.log2(np.abs(x.reshape(-1, 32)).max(1) / 7.0))
    step = np.where(np.abs(y.reshape(-1, 32)) / top[:, None] < 2, 0.5, np.where(np.abs(y.reshape(-1, 32)) / top[:, None] < 4, 1, 2))
    assert (np.abs(x - y).reshape(-1, 32) <= 0.5 * step * top[:, None] + 1e-15).all()
    np.testing.assert_array_equal(mxfp4_rows(y), y)


def _filled(rng, n, table, page=16, n_pages=40, heads=2, d=64):
    c = PagedCache(n_pages, page, table)
    k, v = rng.standard_normal((2, n, heads, d))
    c.append([n], [0, n], k, v)
    return c, k, v


def test_attention_is_the_decoders_and_in_two_parts_the_same():
    rng = np.random.default_rng(3)
    n, table = 37, [[5, 0, 7]]
    c, k, v = _filled(rng, n, table)
    q = rng.standard_normal((n, 4, 64))
    out, _ = c.attention([n], [0, n], q, 64 ** -0.5)
    for h in range(4):
        np.testing.assert_allclose(out[:, h], causal_attention(q[:, h], k[:, h // 2], v[:, h // 2]), atol=1e-12)
    d = PagedCache(40, 16, table)
    d.append([20], [0, 20], k[:20], v[:20])
    first, _ = d.attention([20], [0, 20], q[:20], 64 ** -0.5)
    d.append([37], [0, 17], k[20:], v[20:])
    rest, _ = d.attention([37], [0, 17], q[20:], 64 ** -0.5)
    np.testing.assert_allclose(np.concatenate([first, rest]), out, atol=1e-12)


def test_window_and_first_tokens_and_evicted_pages():
    rng = np.random.default_rng(4)
    n = 50
    c, k, v = _filled(rng, n, [[3, 1, 4, 9]])
    q = rng.standard_normal((1, 2, 64))
    out, _ = c.attention([n], [0, 1], q, 1.0, window=10, sinks=3)
    see = [0, 1, 2] + list(range(40, 50))
    for h in range(2):
        p = np.exp(k[see, h] @ q[0, h])
        np.testing.assert_allclose(out[0, h], (p / p.sum()) @ v[see, h], atol=1e-10)
    c.table = [[3, -1, 4, 9]]      # page 1 (tokens 16..31) was outside the window anyway
    again, _ = c.attention([n], [0, 1], q, 1.0, window=10, sinks=3)
    np.testing.assert_array_equal(out, again)
    c.table = [[-1, 40, -7, 99]]
    none, spread = c.attention([n], [0, 1], q, 1.0)
    assert not none.any() and not spread.any()


@pytest.mark.parametrize("n,length", [(4, 2), (3, 0), (2, -5)])
def test_rows_before_the_first_token_see_nothing(n, length):
    c = PagedCache(4, 16, [[0, 1]])
    k = np.ones((n, 1, 64))
    c.append([length], [0, n], k, k)
    out, _ = c.attention([length], [0, n], k, 1.0)
    keep = max(0, length)
    assert not out[:n - keep].any() and (out[n - keep:] == 1).all()
