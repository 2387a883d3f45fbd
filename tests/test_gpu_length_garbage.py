"""Lengths that are not a sequence's, up to the largest 32-bit numbers, on the device: reported and skipped, the batch's other
sequences computed as ever."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests import test_gpu_attn_pages as pages
from tests import test_gpu_attn_prefix as prefixes
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import attn_close, config, f64, lists_to_arrays, status_word
from tests.test_gpu_page_select import select_gpu, setup

pytestmark = pytest.mark.gpu

LAST = 2 ** 31 - 1
GARBAGE = [LAST, LAST - 14, LAST - 15, LAST - 16, 2 ** 30, -1, -LAST - 1, 0]


def batch(cfg):
    """A sequence that makes sense in front of and behind each that does not."""
    sl = np.full(17, 100, np.int32)
    sl[1::2] = GARBAGE
    kv, q = synth.make_kv(cfg, np.full(17, 100, np.int32)), synth.make_q(cfg, 17 * 2)
    return sl, np.ones(17, np.int32), np.arange(0, 35, 2, dtype=np.int32), kv, q


def check(cfg, o, lse, status, kv, q, gamma, cu):
    assert status == sv.SV_DEV_BAD_LEN
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, np.full(17, 100), gamma, cu, cfg.hkv, cfg.head_dim ** -0.5)
    good = np.arange(34)[np.arange(34) // 2 % 2 == 0]
    attn_close(o, lse, *ref, good)
    rest = np.setdiff1d(np.arange(34), good)
    assert (o[rest] == 7.0).all() and (lse[rest] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,head_dim,gmax", [(8, 2, 128, 1), (8, 2, 64, 1), (16, 1, 64, 40), (16, 1, 128, 12), (16, 1, 128, 40)])
def test_verify_attention(hq, hkv, head_dim, gmax):
    cfg = config("lg", 17, hq, hkv, head_dim, 120)
    sl, gamma, cu, kv, q = batch(cfg)
    pool, qd, status = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q), status_word()
    o, lse = torch.full_like(qd, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    ws = workspace(sv.spec_verify_attn_workspace_bytes(17, gmax, hq, hkv, head_dim, 112))
    sv.spec_verify_attn(qd, o, pool, dev(kv.block_table), dev(sl), dev(gamma), dev(cu), gmax, 112, workspace=ws, lse=lse, device_status=status)
    torch.cuda.synchronize()
    check(cfg, f64(o), lse.cpu().numpy().astype(np.float64), int(status.item()), kv, q, gamma, cu)


@pytest.mark.parametrize("hq,gmax", [(8, 1), (32, 9)])
def test_listed_pages_and_prefixes(hq, gmax):
    cfg = config("lg", 17, hq, 2, 128, 121)
    sl, gamma, cu, kv, q = batch(cfg)
    every = lists_to_arrays([[(list(range(7)), [3] * 7)] * 2] * 17, 7)
    o, lse, status = pages.attend(cfg, kv, q, sl, gamma, cu, gmax, every, most=112)
    check(cfg, o, lse, status, kv, q, gamma, cu)
    kv = prefixes.build(cfg, np.full(17, 100), np.zeros(17, int), [64])
    o, lse, status = prefixes.attend(cfg, kv, q, sl, gamma, cu, gmax, [0] * 17, [64], most=112)
    check(cfg, o, lse, status, kv, q, gamma, cu)


def test_page_choice_and_bounds():
    cfg = config("lg", 17, 8, 2, 128, 122)
    sl, gamma, cu, kv, q = batch(cfg)
    table, _, _, bounds, scales = setup(cfg, [100] * 17, [1] * 17, 1, 1)
    pl, rm, n, status = select_gpu(cfg, q, bounds, scales, table, sl, gamma, cu, 1, 4, 1, 1, most=112)
    assert status == sv.SV_DEV_BAD_LEN and (n[1::2] == 0).all()
    ref = oracle.page_select(q, bounds, scales, table, np.full(17, 100), gamma, cu, 4, 1, 1)
    for b in range(0, 17, 2):
        for h in range(2):
            assert (pl[b, h, :n[b, h]].tolist(), rm[b, h, :n[b, h]].tolist()) == (ref[b][h][0], ref[b][h][1])
    pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    shape = (kv.k_pool.shape[0], 2)
    db, ds, status = torch.zeros((*shape, 2, 128), dtype=torch.int8, device=DEV), torch.zeros(shape, device=DEV), status_word()
    sv.spec_page_bounds_update(pool, db, ds, dev(kv.block_table), dev(sl), gamma=dev(gamma), max_new=2, device_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == sv.SV_DEV_BAD_LEN
    fine = np.where(np.arange(17) % 2 == 0, 100, 0)
    ref = oracle.page_bounds_update(kv.k_pool, kv.strides, kv.block_table, fine, np.where(fine > 0, 98, 0), np.zeros((*shape, 2, 128), np.int8), np.zeros(shape, np.float32))
    np.testing.assert_array_equal(db.cpu().numpy(), ref[0])
    np.testing.assert_array_equal(ds.cpu().numpy(), ref[1])
