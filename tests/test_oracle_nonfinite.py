"""Pins of the long-context oracles where keys or queries are no numbers or infinite, by hand."""
import numpy as np
import pytest

import oracle
from paper_2504_00030_b200 import synth


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_queries_that_are_not_finite_score_nothing(value):
    """All whole numbers of the row and kv head are 0, whichever head holds it and wherever it stands among the larger ones."""
    rng = np.random.default_rng(1)
    bounds = np.sort(rng.integers(-127, 128, (12, 1, 2, 64)), 2)[:, :, ::-1].astype(np.int8)
    scales, table = rng.uniform(0.01, 0.02, (12, 1)).astype(np.float32), np.arange(12, dtype=np.int32)
    for g, d in ((0, 0), (1, 63), (3, 20)):
        q = rng.standard_normal((4, 64)).astype(np.float32)
        q[g, d], q[2, 5] = value, 3e38
        score, chosen = oracle.page_choice(synth.bf16_bits(q), bounds, scales, 0, table, 12, 5, 1, 1)
        assert (score == 0).all() and np.nonzero(chosen)[0].tolist() == [0, 1, 2, 3, 11]


@pytest.mark.parametrize("value,scale", [(np.nan, np.nan), (np.inf, np.inf), (-np.inf, np.inf)])
def test_keys_that_are_not_finite_leave_their_mark_in_the_scale(value, scale):
    k = np.ones((3, 2, 16, 64), np.float32)
    k[1, 0, 4, 9] = value
    k[1, 0, 5, 9], k[1, 0, 6, 8] = -7.0, 9.0                    # other keys of the channel, a larger one of another
    k[2, :, 3:] = value                                         # behind the length
    bounds, scales = oracle.page_bounds_update(synth.bf16_bits(k), [2 * 16 * 64, 16 * 64, 64, 1], [[1, 2]], [19], [0], np.full((3, 2, 2, 64), 9, np.int8),
                                               np.full((3, 2), 7.0, np.float32))
    np.testing.assert_array_equal(scales[1:], np.array([[scale, 1 / 127], [1 / 127, 1 / 127]], np.float32))
    assert (bounds[1, 0] == 0).all() and (bounds[1, 1] == 127).all() and (bounds[2] == 127).all()


def test_a_channel_that_is_no_number_throughout():
    k = np.ones((1, 1, 16, 64), np.float32)
    k[0, 0, :, 3] = np.nan
    bounds, scales = oracle.page_bounds_update(synth.bf16_bits(k), [16 * 64, 16 * 64, 64, 1], [[0]], [16], [0], np.full((1, 1, 2, 64), 9, np.int8),
                                               np.zeros((1, 1), np.float32))
    assert np.isnan(scales[0, 0]) and (bounds == 0).all()
