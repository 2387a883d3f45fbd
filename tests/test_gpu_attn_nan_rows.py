"""spec_verify_attn with queries that are no numbers or infinite: NaN in the output and in the log-sum-exp of those rows and heads
alone, for keys in one block's share and for keys split over many."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests import test_gpu_attn_pages as pages
from tests import test_gpu_attn_prefix as prefixes
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import config, f64, lists_to_arrays
from tests.test_gpu_attn_nonfinite import same, spoil

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,head_dim,gmax", [(8, 2, 128, 3), (64, 8, 128, 16), (32, 2, 128, 12), (12, 12, 64, 4), (8, 1, 64, 40)])
@pytest.mark.parametrize("batch,longest", [(1, 6000), (3, 1500), (150, 200)])
def test_verify_attention(hq, hkv, head_dim, gmax, batch, longest):
    cfg = config("nr", batch, hq, hkv, head_dim, 150)
    rng = np.random.default_rng(150)
    gamma = rng.integers(0, gmax + 1, batch).astype(np.int32)
    sl = rng.integers(max(gmax + 1, longest // 2), longest + 1, batch).astype(np.int32)
    sl[0] = longest
    cu, _ = synth.prefix(gamma)
    kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, int(cu[-1]))
    spoil(rng, q, kv)
    verify(cfg, kv, q, sl, gamma, cu, gmax, longest)


def verify(cfg, kv, q, sl, gamma, cu, gmax, longest):
    batch, (_, hq, head_dim), hkv = len(sl), q.shape, cfg.hkv
    pool, qd = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q)
    o, lse = torch.zeros_like(qd), torch.zeros(q.shape[:2], device=DEV)
    ws = workspace(sv.spec_verify_attn_workspace_bytes(batch, gmax, hq, hkv, head_dim, longest))
    sv.spec_verify_attn(qd, o, pool, dev(kv.block_table), dev(sl), dev(gamma), dev(cu), gmax, longest, ws, lse=lse)
    torch.cuda.synchronize()
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, hkv, head_dim ** -0.5)
    same(f64(o), lse.cpu().numpy().astype(np.float64), ref, np.arange(int(cu[-1])))


@pytest.mark.parametrize("hq,hkv,head_dim,gmax", [(8, 2, 128, 3), (64, 8, 128, 16), (32, 2, 128, 12), (12, 12, 64, 4), (8, 1, 64, 40)])
@pytest.mark.parametrize("batch,longest", [(1, 6000), (150, 200)])
def test_nothing_but_scores_of_minus_infinity(hq, hkv, head_dim, gmax, batch, longest):
    """0 / 0 in every attention but that over lists, where such a row counts as one without keys."""
    cfg = config("nr", batch, hq, hkv, head_dim, 151)
    rng = np.random.default_rng(151)
    gamma = rng.integers(0, gmax + 1, batch).astype(np.int32)
    sl = rng.integers(max(gmax + 1, longest // 2), longest + 1, batch).astype(np.int32)
    sl[0] = longest
    cu, _ = synth.prefix(gamma)
    group, prefix = [0] * batch, [32]
    kv, q = prefixes.build(cfg, sl, group, prefix), synth.make_q(cfg, int(cu[-1]))
    kv.k_pool[..., 3] = synth.bf16_bits(np.ones(1, np.float32))[0]
    pick = rng.random(q.shape[:2]) < 1 / 6
    pick.reshape(-1)[0] = True
    q[pick, 3] = 0xff80
    verify(cfg, kv, q, sl, gamma, cu, gmax, longest)
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, hkv, head_dim ** -0.5)
    rows = np.arange(int(cu[-1]))
    o, lse, status = prefixes.attend(cfg, kv, q, sl, gamma, cu, gmax, group, prefix)
    assert status == 0
    same(o, lse, ref, rows)
    lists = lists_to_arrays([[(list(range((n + 15) // 16)), [2 ** (int(g) + 1) - 1] * ((n + 15) // 16))] * hkv for n, g in zip(sl, gamma)], (longest + 15) // 16)
    o, lse, status = pages.attend(cfg, kv, q, sl, gamma, cu, gmax, lists)
    assert status == 0 and (o[pick] == 0).all() and (lse[pick] == -np.inf).all() and np.isfinite(o[~pick]).all() and np.isfinite(lse[~pick]).all()
