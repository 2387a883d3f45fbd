"""Attention over parts of the cache where pairs of different shapes follow one another in a block: row tiles and warps
without rows, rows that begin with a partial, workspaces on any 16 bytes.  Float64 oracle, and bits that stay from run to run."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16
from tests.longctx import attn_close, config, f64, lists_to_arrays, status_word
from tests.test_gpu_attn_pages import random_lists
from tests.test_gpu_attn_prefix import build

pytestmark = pytest.mark.gpu


def check(cfg, sl, gamma, gmax, group=None, prefix=None, louder=None, lists=None, runs=4, ws_offset=0):
    """Prefix attention (group, prefix) or attention over lists; louder: keys from that page on are scaled by it."""
    sl, gamma = np.asarray(sl, np.int32), np.asarray(gamma, np.int32)
    B = len(sl)
    cu, _ = synth.prefix(gamma)
    kv = build(cfg, sl, group, prefix) if lists is None else synth.make_kv(cfg, sl)
    if louder is not None:
        own = np.unique(np.concatenate([kv.block_table[b, louder[0]:(sl[b] + 15) // 16] for b in range(B)]))
        k = synth.bf16_to_f32(kv.k_pool)
        k[own] *= louder[1]
        kv = synth.KVState(synth.bf16_bits(k), kv.v_pool, kv.block_table, kv.strides)
    q = synth.make_q(cfg, int(cu[-1]))
    pool, qd = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q)
    i32 = lambda a: dev(np.ascontiguousarray(a, np.int32))  # noqa: E731
    if lists is None:
        n = sv.spec_verify_attn_prefix_workspace_bytes(B, gmax, cfg.hq, cfg.hkv, cfg.head_dim, len(prefix))
    else:
        n = sv.spec_verify_attn_pages_workspace_bytes(B, gmax, cfg.hq, cfg.hkv, cfg.head_dim)
    ws = torch.zeros(n + 64, dtype=torch.uint8, device=DEV)
    assert ws.data_ptr() % 64 == 0
    ws = ws[ws_offset:ws_offset + n]
    table, sld, gd, cud = i32(kv.block_table), i32(sl), i32(gamma), i32(cu)
    first = None
    for _ in range(runs):
        o, lse, status = torch.full_like(qd, 7.0), torch.full(q.shape[:2], 7.0, device=DEV), status_word()
        if lists is None:
            sv.spec_verify_attn_prefix(qd, o, pool, table, sld, gd, cud, gmax, int(sl.max()), i32(group), i32(prefix), ws, lse=lse, device_status=status)
        else:
            sv.spec_verify_attn_pages(qd, o, pool, table, sld, gd, cud, gmax, int(sl.max()), dev(lists[0]), dev(lists[1].view(np.int64)), dev(lists[2]),
                                      ws, lse=lse, device_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        if first is None:
            first = (o, lse)
            ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, cfg.hkv, cfg.head_dim ** -0.5, *(lists or ()))
            attn_close(f64(o), lse.cpu().numpy().astype(np.float64), *ref, np.arange(int(cu[-1])))
        else:
            assert torch.equal(o, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("head_dim", [64, 128])
def test_row_tiles_without_rows(head_dim):
    """Two row tiles of 16 positions to a pair, and more pairs than blocks, many of them with rows in the first tile alone."""
    rng = np.random.default_rng(71)
    cfg = config("ar", 60, 32, 4, head_dim, 71)
    group = np.arange(60) // 2                                       # groups of two sequences: from 2 to 36 positions
    prefix = [int(rng.integers(5, 20)) * 16 for _ in range(30)]
    gamma = rng.integers(0, 18, 60)
    sl = [prefix[g] + int(gamma[b]) + 1 + int(rng.integers(0, 60)) for b, g in enumerate(group)]
    check(cfg, sl, gamma, 17, group, prefix)
    gamma = rng.integers(0, 41, 60)                                  # the sequences' own pairs: up to 41 positions
    sl = [int(gamma[b]) + 1 + int(rng.integers(0, 300)) for b in range(60)]
    check(cfg, sl, gamma, 40, [-1] * 60, [16])
    lists = lists_to_arrays(random_lists(rng, sl, gamma, 4, 0.5), 22)
    check(cfg, sl, gamma, 40, lists=lists)


@pytest.mark.parametrize("gmax", [0, 3, 15, 20])
def test_own_keys_that_outweigh_the_prefix(gmax):
    """The first tile behind the prefix raises the maximum, so that the partial is scaled as soon as it is there."""
    rng = np.random.default_rng(72)
    cfg = config("ar", 40, 16, 2, 128, 72, q_scale=1.5)
    gamma = rng.integers(0, gmax + 1, 40)
    gamma[0] = gmax
    check(cfg, 128 + gamma + 1 + rng.integers(20, 200, 40), gamma, gmax, [0] * 40, [128], louder=(8, 4.0))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("gmax", [7, 15, 33])
def test_warps_without_rows_before_warps_with(gmax, head_dim):
    """Pairs of one and of many rows take turns in a block, all behind prefixes."""
    rng = np.random.default_rng(73)
    cfg = config("ar", 100, 64, 8, head_dim, 73)
    group = np.arange(100) % 3
    gamma = np.where(rng.random(100) < 0.5, 0, gmax)
    check(cfg, 160 + gamma + 1 + rng.integers(0, 90, 100), gamma, gmax, group, [160, 96, 128])


@pytest.mark.parametrize("offset", [16, 32, 48])
def test_workspace_on_any_16_bytes(offset):
    rng = np.random.default_rng(74)
    cfg = config("ar", 4, 16, 2, 128, 74)
    sl, gamma = np.array([900, 850, 1200, 870], np.int32), np.array([2, 0, 3, 1])
    check(cfg, sl, gamma, 3, [0] * 4, [800], ws_offset=offset)
    check(cfg, sl, gamma, 3, lists=lists_to_arrays(random_lists(rng, sl, gamma, 2, 0.5, every=True), 80), ws_offset=offset)


@pytest.mark.parametrize("hq", [2, 16])
def test_more_sequences_than_threads(hq):
    """The shares of work are found in several rounds: one and two row tiles (1 and 8 heads of 17 rows)."""
    rng = np.random.default_rng(75)
    B, gmax = 420, 16
    cfg = config("ar", B, hq, 2, 64, 75)
    gamma = rng.integers(0, gmax + 1, B)
    sl = gamma + 1 + rng.integers(0, 120, B)
    check(cfg, sl, gamma, gmax, lists=lists_to_arrays(random_lists(rng, sl, gamma, 2, 0.5), 9), runs=2)
    check(cfg, sl + 48, gamma, gmax, rng.integers(-1, 5, B), [48, 16, 32, 48, 48], runs=2)


def test_blocks_of_hundreds_of_rows():
    """Rows of one sequence over several pairs: a prompt's part behind a shared prefix."""
    check(config("ar", 3, 8, 2, 128, 76), [1500, 1300, 900], [700, 3, 0], 700, [0, 0, 0], [592], runs=2)
    check(config("ar", 2, 4, 4, 64, 76), [2100, 300], [1999, 100], 2047, [-1, -1], [16], runs=2)


def test_largest_batch():
    """8192 sequences, as many as may share prefixes; lists for three times 8192 owners."""
    rng = np.random.default_rng(77)
    sl = rng.integers(17, 60, 8192)
    check(config("ar", 8192, 3, 3, 64, 77), sl, np.zeros(8192, int), 0, rng.integers(-1, 8, 8192), [16] * 8, runs=2)
    check(config("ar", 8192, 3, 3, 64, 77), sl, np.zeros(8192, int), 0, lists=lists_to_arrays(random_lists(rng, sl, np.zeros(8192, int), 3, 0.6), 4), runs=2)
