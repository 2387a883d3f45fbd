"""The long-context calls from several host threads of one process, on streams and workspaces of their own."""
import ctypes as C
import threading

import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import attn_close, config, f64, lists_to_arrays
from tests.test_gpu_attn_pages import random_lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head_dim", [64, 128])
def test_blocks_of_different_sizes_over_lists(head_dim):
    """Two sizes of block that are one kernel's with different amounts of shared memory, and one of another kernel."""
    lib, steps, runs = sv.load(), 1500, []
    for k, (hq, gmax) in enumerate(((4, 2), (16, 7), (32, 16))):
        cfg = config("lt", 3, hq, 2, head_dim, 110 + k)
        sl, gamma = np.array([300, 90, 200], np.int32), np.array([gmax, 0, gmax], np.int32)
        cu, _ = synth.prefix(gamma)
        kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, int(cu[-1]))
        arrays = lists_to_arrays(random_lists(np.random.default_rng(k), sl, gamma, 2, 0.6), 20)
        pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
        qd = dev_bf16(q)
        o, lse = torch.zeros_like(qd), torch.zeros(q.shape[:2], device=DEV)
        d = [dev(kv.block_table), dev(sl), dev(gamma), dev(cu), dev(arrays[0]), dev(arrays[1].view(np.int64)), dev(arrays[2])]
        p = sv.AttnPagesParams(sv.attn_params(qd, o, pool, *d[:4], gmax, 300, lse=lse), d[4].data_ptr(), d[5].data_ptr(), d[6].data_ptr(), 20)
        ws = workspace(sv.spec_verify_attn_pages_workspace_bytes(3, gmax, hq, 2, head_dim))
        ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, 2, head_dim ** -0.5, *arrays)
        runs.append((p, ws, torch.cuda.Stream(), (qd, d, pool), o, lse, ref, int(cu[-1])))
    torch.cuda.synchronize()
    start, statuses = threading.Barrier(len(runs)), [set() for _ in runs]

    def worker(k):
        torch.cuda.set_device(DEV)
        p, ws, stream = runs[k][:3]
        start.wait()
        for _ in range(steps):
            statuses[k].add(lib.spec_verify_attn_pages(C.byref(p), ws.data_ptr(), ws.numel(), stream.cuda_stream))

    threads = [threading.Thread(target=worker, args=(k,)) for k in range(len(runs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert statuses == [{sv.SV_OK}] * len(runs)
    for _, _, _, _, o, lse, ref, rows in runs:
        attn_close(f64(o), lse.cpu().numpy().astype(np.float64), *ref, np.arange(rows))
