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
