"""Calls at the edges of what the long-context calls allow: nothing to do at all, group sizes that leave most of a row tile empty,
outputs left out."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests import test_gpu_attn_pages as pages
from tests import test_gpu_attn_prefix as prefixes
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import attn_close, config, f64, lists_to_arrays
from tests.test_gpu_page_select import check as check_choice
from tests.test_gpu_page_select import select_gpu, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [1, 5, 600])
@pytest.mark.parametrize("hq,gmax", [(8, 2), (32, 16)])
def test_every_sequence_skipped(batch, hq, gmax):
    cfg = config("le", batch, hq, 2, 128, 140)
    sl, gamma, cu = np.zeros(batch, np.int32), np.zeros(batch, np.int32), np.arange(batch + 1, dtype=np.int32)
    kv, q = synth.make_kv(cfg, np.full(batch, 20)), synth.make_q(cfg, batch)
    arrays = lists_to_arrays([[([0], [1])] * 2] * batch, 2)
    for o, lse, status in (pages.attend(cfg, kv, q, sl, gamma, cu, gmax, arrays, most=32),
                           prefixes.attend(cfg, kv, q, sl, gamma, cu, gmax, [0] * batch, [16], most=32)):
        assert status == sv.SV_DEV_BAD_LEN and (o == 7.0).all() and (lse == 7.0).all()
    table, _, _, bounds, scales = setup(cfg, [700] * batch, [0] * batch, 0, 1)
    pl, _, n, status = select_gpu(cfg, q, bounds, scales, table, sl, gamma, cu, gmax, 5, 1, 1, most=700)
    assert status == sv.SV_DEV_BAD_LEN and (n == 0).all() and (pl == -7).all()


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("group", [65, 100, 127])
def test_groups_of_which_a_row_tile_holds_one_position(group, head_dim):
    cfg = config("le", 3, group * 2, 2, head_dim, 141)
    pages.check(cfg, [400, 17, 1500], [0, 0, 0], every=True)
    pages.check(cfg, [400, 17, 1500], [6, 1, 3], every=True)
    prefixes.check(cfg, [400, 330, 1500], [4, 0, 1], [0, 0, 0], [320])
    check_choice(cfg, [400, 17, 1500], [6, 1, 3], 6, 9, 1, 2)


@pytest.mark.parametrize("gmax", [0, 8])
def test_without_the_log_sum_exp(gmax):
    cfg = config("le", 3, 16, 2, 128, 142)
    sl, gamma, cu = np.array([900, 850, 870], np.int32), np.full(3, gmax, np.int32), np.arange(0, 3 * gmax + 4, gmax + 1, dtype=np.int32)
    kv, q = prefixes.build(cfg, sl, [0, 0, 0], [800]), synth.make_q(cfg, 3 * (gmax + 1))
    pool, qd = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q)
    common = (pool, dev(kv.block_table), dev(sl), dev(gamma), dev(cu), gmax, 900)
    arrays = lists_to_arrays([[(list(range((n + 15) // 16)), [2 ** (gmax + 1) - 1] * ((n + 15) // 16))] * 2 for n in sl], 57)
    outs = torch.zeros_like(qd), torch.zeros_like(qd)
    sv.spec_verify_attn_pages(qd, outs[0], *common, dev(arrays[0]), dev(arrays[1].view(np.int64)), dev(arrays[2]),
                              workspace(sv.spec_verify_attn_pages_workspace_bytes(3, gmax, 16, 2, 128)))
    sv.spec_verify_attn_prefix(qd, outs[1], *common, dev(np.zeros(3, np.int32)), dev(np.array([800], np.int32)),
                               workspace(sv.spec_verify_attn_prefix_workspace_bytes(3, gmax, 16, 2, 128, 1)))
    torch.cuda.synchronize()
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, 2, 128 ** -0.5)
    for o in outs:
        attn_close(f64(o), None, *ref, np.arange(3 * (gmax + 1)))
