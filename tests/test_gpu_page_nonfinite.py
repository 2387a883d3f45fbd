"""Keys and queries that are no numbers or infinite, in the bounds of pages and in the choice by them, against the oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16
from tests.longctx import config, lists_to_arrays
from tests.test_gpu_page_bounds import check as check_bounds
from tests.test_gpu_page_select import select_gpu, setup

pytestmark = pytest.mark.gpu

NAN, NNAN, INF, NINF = 0x7fc0, 0xffc1, 0x7f80, 0xff80


def spoiled(cfg, length):
    """Cache of one sequence whose pages 1 to 7 hold such keys, each in another way."""
    kv = synth.make_kv(cfg, np.array([length], np.int32))
    k, at = kv.k_pool, kv.block_table[0]
    k[at[1], 0, 5, 3] = NAN
    k[at[2], 0, :, 7] = NNAN                              # a channel throughout
    k[at[3]] = NAN                                        # everything
    k[at[4], 0, 2, 1], k[at[4], 1, 2, 1] = INF, NINF
    k[at[5], 1, 0, cfg.head_dim - 1], k[at[5], 1, 1, 0] = NAN, INF
    k[at[6], 0, 15, 2], k[at[6], 0, 14, 2] = NINF, INF
    k[at[7], 0, :, 0], k[at[7], 0, 3, 9] = 0, NAN
    return kv


@pytest.mark.parametrize("slot_major", [False, True])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_bounds(head_dim, slot_major):
    """The scale is what the keys have of it: NaN, or infinite; the whole numbers are 0."""
    cfg = config("pn", 1, 4, 2, head_dim, 96)
    kv = spoiled(cfg, 150)
    kv.k_pool[kv.block_table[0, 9], :, 6:] = NAN          # behind the length: not looked at
    bounds, scales = check_bounds(cfg, [150], first=[0], kv=kv, slot_major=slot_major)
    at = kv.block_table[0]
    assert np.isnan(scales[at[[1, 2, 3, 3, 5, 7]], [0, 0, 0, 1, 1, 0]]).all() and np.isinf(scales[at[[4, 4, 6]], [0, 1, 0]]).all()
    assert np.isfinite(scales[at[[0, 1, 2, 5, 6, 7, 8, 9, 9]], [0, 1, 1, 0, 1, 1, 0, 0, 1]]).all()
    assert (bounds[at[3]] == 0).all() and (bounds[at[2], 0] == 0).all() and (bounds[at[4]] == 0).all()


def test_such_pages_are_read():
    """Bounds as the library makes them of such keys, and the choice by them: every row of their head reads those pages."""
    cfg = config("pn", 1, 8, 2, 128, 97)
    length, gamma, cu = 2000, 4, np.array([0, 5], np.int32)
    kv = spoiled(cfg, length)
    n = kv.k_pool.shape[0]
    pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    bounds, scales = torch.zeros((n, 2, 2, 128), dtype=torch.int8, device=DEV), torch.zeros((n, 2), device=DEV)
    sl = np.array([length], np.int32)
    sv.spec_page_bounds_update(pool, bounds, scales, dev(kv.block_table), dev(sl), first=dev(np.zeros(1, np.int32)), max_new=length)
    bounds, scales = bounds.cpu().numpy(), scales.cpu().numpy()
    q = synth.make_q(cfg, 5)
    pl, rm, m, status = select_gpu(cfg, q, bounds, scales, kv.block_table, sl, [gamma], cu, gamma, 16, 1, 2)
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, kv.block_table, sl, [gamma], cu, 16, 1, 2), pl.shape[2])
    used = np.arange(pl.shape[2]) < m[..., None]
    assert status == 0 and (m == ref[2]).all()
    np.testing.assert_array_equal(np.where(used, pl, -1), ref[0])
    np.testing.assert_array_equal(np.where(used, rm, 0), ref[1])
    for h, pages in ((0, {1, 2, 3, 4, 6, 7}), (1, {3, 4, 5})):
        assert pages <= {int(p) for p, mask in zip(pl[0, h, :m[0, h]], rm[0, h, :m[0, h]]) if mask == 31}


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
