"""spec_verify_attn with queries that are no numbers or infinite: NaN in the output and in the log-sum-exp of those rows and heads
alone, for keys in one block's share and for keys split over many."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import config, f64
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
    pool, qd = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q)
    o, lse = torch.zeros_like(qd), torch.zeros(q.shape[:2], device=DEV)
    ws = workspace(sv.spec_verify_attn_workspace_bytes(batch, gmax, hq, hkv, head_dim, longest))
    sv.spec_verify_attn(qd, o, pool, dev(kv.block_table), dev(sl), dev(gamma), dev(cu), gmax, longest, ws, lse=lse)
    torch.cuda.synchronize()
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, hkv, head_dim ** -0.5)
    same(f64(o), lse.cpu().numpy().astype(np.float64), ref, np.arange(int(cu[-1])))
