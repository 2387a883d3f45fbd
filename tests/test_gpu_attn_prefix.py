"""spec_verify_attn_prefix on the GPU against the float64 oracle of the verify attention over the same block tables."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import attn_close, config, f64, status_word

pytestmark = pytest.mark.gpu


def build(cfg, sl, group, prefix_len):
    """Cache of sequences whose members share their group's prefix pages."""
    sl, group = np.asarray(sl, np.int32), np.asarray(group)
    kv = synth.make_kv(cfg, sl)
    table = kv.block_table.copy()
    for g, n in enumerate(prefix_len):
        members = [b for b in range(len(sl)) if group[b] == g]
        whole = max(members, key=lambda b: sl[b], default=0)               # a member that has all of the prefix, if one has
        for b in members:
            m = min(n // 16, (int(sl[b]) + 15) // 16, (int(sl[whole]) + 15) // 16)
            table[b, :m] = kv.block_table[whole, :m]
    return synth.KVState(kv.k_pool, kv.v_pool, table, kv.strides)


def attend(cfg, kv, q, sl, gamma, cu, gmax, group, prefix_len, most=None, table=None):
    B = len(sl)
    pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    qd = dev_bf16(q)
    o, lse, status = torch.full_like(qd, 7.0), torch.full(q.shape[:2], 7.0, device=DEV), status_word()
    most = most or int(max(sl))
    ws = workspace(sv.spec_verify_attn_prefix_workspace_bytes(B, gmax, cfg.hq, cfg.hkv, cfg.head_dim, len(prefix_len)))
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    sv.spec_verify_attn_prefix(qd, o, pool, i32(kv.block_table if table is None else table), i32(sl), i32(gamma), i32(cu), gmax, most, i32(group),
                               i32(prefix_len), ws, lse=lse, device_status=status)
    torch.cuda.synchronize()
    return f64(o), lse.cpu().numpy().astype(np.float64), int(status.item())


def check(cfg, sl, gamma, group, prefix_len, gmax=None, padded=False, status=0):
    sl, gamma = np.asarray(sl, np.int32), np.asarray(gamma, np.int32)
    gmax = int(gamma.max()) if gmax is None else gmax
    cu, _ = synth.padded_offsets(len(sl), gmax) if padded else synth.prefix(gamma)
    kv, q = build(cfg, sl, group, prefix_len), synth.make_q(cfg, int(cu[-1]))
    o, lse, st = attend(cfg, kv, q, sl, gamma, cu, gmax, group, prefix_len)
    assert st == status
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, cfg.hkv, cfg.head_dim ** -0.5)
    rows = np.concatenate([np.arange(cu[b], cu[b] + gamma[b] + 1) for b in range(len(sl))])
    attn_close(o, lse, *ref, rows)
    rest = np.setdiff1d(np.arange(q.shape[0]), rows)
    assert (o[rest] == 7.0).all() and (lse[rest] == 7.0).all()


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (14, 2), (24, 1), (128, 1)])
def test_heads(hq, hkv, head_dim):
    cfg = config("px", 5, hq, hkv, head_dim, 51)
    check(cfg, [330, 300, 390, 500, 290], [0, 3, 1, 0, 2], [0, 0, 0, -1, 0], [280])
    check(cfg, [330, 300, 390, 500, 290], [0] * 5, [0] * 5, [257])


@pytest.mark.parametrize("prefix", [0, 15, 16, 17, 127, 128, 129, 144, 1000])
def test_prefix_lengths(prefix):
    cfg = config("px", 3, 8, 2, 128, 52)
    check(cfg, [prefix + 1, prefix + 40, prefix + 200], [0, 3, 2], [0, 0, 0], [prefix])


def test_several_groups_in_any_order():
    rng = np.random.default_rng(5)
    group = rng.integers(-1, 4, 23)
    prefix = [700, 64, 333, 16]
    sl = [(prefix[g] // 16 * 16 if g >= 0 else 0) + int(rng.integers(9, 300)) for g in group]
    gamma = rng.integers(0, 8, 23)
    check(config("px", 23, 16, 2, 128, 53), sl, gamma, group, prefix)
    check(config("px", 23, 16, 2, 64, 53), sl, gamma, group, prefix, gmax=8, padded=True)


def test_groups_of_one_none_and_all():
    cfg = config("px", 4, 8, 2, 128, 54)
    check(cfg, [400, 500, 300, 200], [1, 2, 0, 3], [0, 1, 2, 3], [390, 100, 200, 0])
    check(cfg, [400, 500, 300, 200], [1, 2, 0, 3], [-1] * 4, [390])
    check(cfg, [400, 401, 402, 403], [1, 2, 0, 3], [1, 1, 1, 1], [77, 390])


def test_members_that_begin_inside_the_prefix():
    """Too short for the prefix, exactly behind it, and its block across the prefix's end."""
    cfg = config("px", 5, 8, 2, 128, 55)
    check(cfg, [20, 321, 320, 330, 400], [2, 0, 0, 15, 3], [0] * 5, [320])


@pytest.mark.parametrize("gmax,hq", [(15, 8), (16, 8), (40, 8), (8, 32)])
def test_rows_on_both_sides_of_a_tile(gmax, hq):
    cfg = config("px", 6, hq, 1, 128, 56)
    check(cfg, [600, 555, 590, 700, 800, 610], [gmax, 0, gmax // 2, gmax, 1, gmax], [0, 0, 1, 0, 1, 0], [500, 480], gmax)


def test_long_prefix_few_and_many_rows():
    check(config("px", 2, 8, 2, 128, 57), [9100, 9050], [0, 0], [0, 0], [9000])
    rng = np.random.default_rng(6)
    check(config("px", 40, 16, 2, 64, 57), 2048 + rng.integers(5, 90, 40), rng.integers(0, 5, 40), [0] * 40, [2048])


def test_peaked_rows():
    check(config("px", 4, 8, 2, 128, 58, q_scale=6.0), [700, 900, 650, 800], [4, 2, 0, 4], [0] * 4, [620])


def test_device_detected_conditions():
    cfg = config("px", 6, 8, 2, 128, 59)
    good, cu = np.array([300, 300, 300, 300, 300, 300], np.int32), np.arange(0, 19, 3, dtype=np.int32)
    group = [0, 0, 1, 1, 0, 0]
    kv, q = build(cfg, good, group, [160, 200]), synth.make_q(cfg, 18)
    sl, g = [300, 300, 300, 300, 2, 300], [2, 2, 2, 2, 2, 9]
    o, lse, status = attend(cfg, kv, q, sl, g, cu, 2, [0, 0, 7, -2, 0, 0], [160, -5])
    assert status == sv.SV_DEV_BAD_LEN | sv.SV_DEV_BAD_GAMMA
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, good, [2] * 6, cu, 2, 128 ** -0.5)
    attn_close(o, lse, *ref, np.r_[0:12, 15:18])
    assert (o[12:15] == 7.0).all()
    # a prefix beyond the table's row is not shared
    o, lse, status = attend(cfg, kv, q, good, [2] * 6, cu, 2, group, [10 ** 6, 200])
    assert status == sv.SV_DEV_BAD_LEN
    attn_close(o, lse, *ref, np.arange(18))
    table = kv.block_table.copy()
    table[2, 14] = -1                                                         # behind the prefix: that sequence alone
    o, lse, status = attend(cfg, kv, q, good, [2] * 6, cu, 2, group, [160, 200], table=table)
    assert status == sv.SV_DEV_BAD_PAGE
    attn_close(o, lse, *ref, np.r_[0:6, 9:18])


def test_graph_replay_with_other_lengths():
    cfg = config("px", 3, 8, 2, 128, 60)
    group, prefix = [0, 0, 0], [512]
    big = np.array([700, 800, 600], np.int32)
    kv, cu = build(cfg, big, group, prefix), np.array([0, 3, 6, 9], np.int32)
    q = synth.make_q(cfg, 9)
    pool, qd = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q)
    o, lse = torch.zeros_like(qd), torch.zeros((9, 8), device=DEV)
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    ws = workspace(sv.spec_verify_attn_prefix_workspace_bytes(3, 2, 8, 2, 128, 1))
    sl, gp = i32(big), i32(group)
    args = (qd, o, pool, i32(kv.block_table), sl, i32([2, 2, 2]), i32(cu), 2, 800, gp, i32(prefix), ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sv.spec_verify_attn_prefix(*args, lse=lse)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_verify_attn_prefix(*args, lse=lse)
    for lengths, groups in (([650, 790, 530], [0, 0, 0]), ([700, 515, 520], [0, -1, 0]), ([700, 800, 600], [-1, -1, -1])):
        sl.copy_(i32(lengths))
        gp.copy_(i32(groups))
        graph.replay()
        torch.cuda.synchronize()
        ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, lengths, [2] * 3, cu, 2, 128 ** -0.5)
        attn_close(f64(o), lse.cpu().numpy().astype(np.float64), *ref, np.arange(9))
