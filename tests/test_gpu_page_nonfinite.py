"""Queries that are no numbers or infinite in the choice of pages, against the oracle."""
import numpy as np
import pytest

import oracle
from tests.longctx import config, lists_to_arrays
from tests.test_gpu_page_select import select_gpu, setup

pytestmark = pytest.mark.gpu

NAN, NNAN, INF, NINF = 0x7fc0, 0xffc1, 0x7f80, 0xff80


@pytest.mark.parametrize("hq,hkv,head_dim", [(8, 2, 128), (7, 1, 64)])
def test_queries(hq, hkv, head_dim):
    """A row whose queries of a kv head are not all finite scores 0 on every page there: the lowest pages; other rows and heads
    choose as ever."""
    cfg = config("pn", 2, hq, hkv, head_dim, 98)
    sl, g = [1800, 900], [5, 2]
    table, cu, q, bounds, scales = setup(cfg, sl, g, 5, 3)
    for r, h, bits in ((0, 0, NAN), (2, hq - 1, NNAN), (3, 1, INF), (4, 2, NINF), (7, 0, NAN)):
        q[r, h, (r * 11) % head_dim] = bits
    pl, rm, n, status = select_gpu(cfg, q, bounds, scales, table, sl, g, cu, 5, 12, 1, 2)
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, sl, g, cu, 12, 1, 2), pl.shape[2])
    used = np.arange(pl.shape[2]) < n[..., None]
    assert status == 0 and (n == ref[2]).all()
    np.testing.assert_array_equal(np.where(used, pl, -1), ref[0])
    np.testing.assert_array_equal(np.where(used, rm, 0), ref[1])
    mine = [int(p) for p, mask in zip(pl[0, 0, :n[0, 0]], rm[0, 0, :n[0, 0]]) if int(mask) & 1]
    assert mine == list(range(10)) + [111, 112]           # row 0 is at position 1794, on page 112
