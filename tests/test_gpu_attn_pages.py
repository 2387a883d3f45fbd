"""spec_verify_attn_pages on the GPU against the float64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import attn_close, config, f64, lists_to_arrays, status_word

pytestmark = pytest.mark.gpu


def random_lists(rng, sl, gamma, hkv, share, shuffle=False, every=False):
    """Pages with random row masks; every: each row has its own position's page too."""
    lists = []
    for b, (L, g) in enumerate(zip(sl, gamma)):
        heads = []
        for _ in range(hkv):
            n = (L + 15) // 16
            mask = np.zeros(n, object)
            for i in range(g + 1):
                pick = rng.random(n) < share
                if every:
                    pick[(L - g - 1 + i) // 16] = True
                for p in np.nonzero(pick)[0]:
                    mask[p] |= 1 << i
            pages = [int(p) for p in range(n) if mask[p]]
            if shuffle:
                pages = [int(p) for p in rng.permutation(pages)]
            heads.append((pages, [int(mask[p]) for p in pages]))
        lists.append(heads)
    return lists


def attend(cfg, kv, q, sl, gamma, cu, gmax, arrays, most=None, lse=True, pools=None, table=None):
    B = len(sl)
    k, v = pools if pools is not None else (dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    pool = sv.spec_kv_pool_register(k, v)
    qd = dev_bf16(q)
    o, ls = torch.full_like(qd, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    status = status_word()
    most = most or int(max(sl))
    ws = workspace(sv.spec_verify_attn_pages_workspace_bytes(B, gmax, cfg.hq, cfg.hkv, cfg.head_dim))
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    table = kv.block_table if table is None else table
    table = np.pad(table, ((0, 0), (0, max(0, (most + 15) // 16 - table.shape[1]))), constant_values=-1)
    sv.spec_verify_attn_pages(qd, o, pool, i32(table), i32(sl), i32(gamma), i32(cu), gmax, most, dev(arrays[0]),
                              dev(arrays[1].view(np.int64)), dev(arrays[2]), ws, lse=ls if lse else None, device_status=status)
    torch.cuda.synchronize()
    return f64(o), ls.cpu().numpy().astype(np.float64), int(status.item())


def check(cfg, sl, gamma, gmax=None, share=0.4, seed=1, padded=False, shuffle=False, every=False, slot_major=False, width=None):
    sl, gamma = np.asarray(sl, np.int32), np.asarray(gamma, np.int32)
    gmax = int(gamma.max()) if gmax is None else gmax
    rng = np.random.default_rng(seed)
    cu, _ = synth.padded_offsets(len(sl), gmax) if padded else synth.prefix(gamma)
    kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, int(cu[-1]))
    lists = random_lists(rng, sl, gamma, cfg.hkv, share, shuffle, every)
    arrays = lists_to_arrays(lists, width or max(1, max(len(p) for s in lists for p, _ in s)), fill_page=10 ** 6)
    pools = tuple(dev_bf16(np.ascontiguousarray(x.transpose(0, 2, 1, 3))).permute(0, 2, 1, 3) for x in (kv.k_pool, kv.v_pool)) if slot_major else None
    o, lse, status = attend(cfg, kv, q, sl, gamma, cu, gmax, arrays, pools=pools)
    assert status == 0
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, cfg.hkv, cfg.head_dim ** -0.5, *arrays)
    rows = np.concatenate([np.arange(cu[b], cu[b] + gamma[b] + 1) for b in range(len(sl))])
    attn_close(o, lse, *ref, rows)
    rest = np.setdiff1d(np.arange(q.shape[0]), rows)
    assert (o[rest] == 7.0).all() and (lse[rest] == 7.0).all()
    return ref


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (24, 2), (7, 1), (128, 1)])
def test_heads_single_tokens_and_blocks(hq, hkv, head_dim):
    cfg = config("ap", 3, hq, hkv, head_dim, 31)
    check(cfg, [400, 17, 1000], [0, 0, 0])
    check(cfg, [400, 17, 1000], [2, 5, 1], every=True)


@pytest.mark.parametrize("sl", [[1], [15], [16], [17], [64], [65], [127], [128], [129], [1025]])
def test_lengths(sl):
    check(config("ap", 1, 8, 2, 128, 32), sl, [0], share=1.0)
    check(config("ap", 1, 8, 2, 128, 32), sl, [min(sl[0] - 1, 4)], share=0.7)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("gmax,hq", [(15, 8), (16, 8), (31, 8), (32, 8), (63, 8), (40, 16)])
def test_rows_on_both_sides_of_a_tile(gmax, hq, head_dim):
    """One row tile, one and a part, two, and several pairs for a list."""
    cfg = config("ap", 3, hq, 1, head_dim, 33)
    check(cfg, [700, 300, 90], [gmax, 0, gmax // 2], gmax, share=0.5)


def test_ragged_batch_padded_slabs_any_order():
    rng = np.random.default_rng(8)
    sl, g = rng.integers(20, 1500, 13), rng.integers(0, 9, 13)
    check(config("ap", 13, 16, 4, 128, 34), sl, g, 12, share=0.3, padded=True, shuffle=True)
    check(config("ap", 13, 16, 4, 64, 34), sl, g, 8, share=0.3, shuffle=True, slot_major=True)


def test_rows_and_lists_without_keys():
    ref = check(config("ap", 4, 8, 2, 128, 35), [300, 20, 90, 33], [3, 2, 0, 7], share=0.03, width=40)
    assert (ref[2] == -np.inf).any() and np.isfinite(ref[2]).any()
    check(config("ap", 2, 8, 2, 128, 35), [300, 20], [3, 2], share=0.0)


def test_pages_behind_a_row_are_not_read():
    """A listed page with keys behind the row's position, masked for it all the same."""
    cfg = config("ap", 1, 4, 1, 128, 36)
    sl, g, cu = [40], [20], np.array([0, 21], np.int32)
    kv, q = synth.make_kv(cfg, np.array(sl, np.int32)), synth.make_q(cfg, 21)
    arrays = lists_to_arrays([[([1, 2], [2 ** 21 - 1] * 2)]], 2)
    o, lse, status = attend(cfg, kv, q, sl, g, cu, 20, arrays)
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, 1, 128 ** -0.5, *arrays)
    assert status == 0
    attn_close(o, lse, *ref, np.arange(21))


def test_large_scores_and_masked_giants():
    """Peaked rows; the largest score of a page that a row does not read must not reach it."""
    cfg = config("ap", 2, 8, 2, 128, 37, q_scale=6.0)
    check(cfg, [900, 500], [4, 4], share=0.3)
    cfg = config("ap", 1, 4, 1, 64, 38)
    sl, g, cu = [128], [1], np.array([0, 2], np.int32)
    kv, q = synth.make_kv(cfg, np.array(sl, np.int32)), synth.make_q(cfg, 2)
    kv.k_pool[kv.block_table[0, 3]] = synth.bf16_bits(np.float32(1e20)[None])[0]
    arrays = lists_to_arrays([[([0, 3, 5], [3, 2, 3])]], 3)
    o, lse, _ = attend(cfg, kv, q, sl, g, cu, 1, arrays, lse=True)
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, 1, 0.125, *arrays)
    attn_close(o, lse, *ref, [0])


def test_many_pairs_and_few_long_ones():
    """More pairs than blocks, and lists split over many blocks."""
    rng = np.random.default_rng(9)
    check(config("ap", 96, 8, 8, 64, 39), rng.integers(16, 200, 96), rng.integers(0, 4, 96), 3, share=0.5)
    check(config("ap", 1, 8, 2, 128, 39), [30000], [1], share=0.9)
    check(config("ap", 1, 64, 2, 128, 39), [9000], [8], share=0.5)


def test_device_detected_conditions():
    cfg = config("ap", 5, 8, 2, 128, 40)
    good = np.array([200, 300, 200, 200, 200], np.int32)
    kv, cu = synth.make_kv(cfg, good), np.array([0, 3, 6, 9, 12, 15], np.int32)
    q = synth.make_q(cfg, 15)
    lists = random_lists(np.random.default_rng(2), good, [2] * 5, 2, 0.8)
    arrays = lists_to_arrays(lists, 20)
    sl, g = [200, 2, 200, 200, 200], [2, 2, 9, 2, 2]                         # shorter than its block; gamma taken as 2
    arrays[0][3, 0, 1], arrays[0][3, 1, 0] = 13, -4                          # outside the sequence's 13 pages
    arrays[2][4, 0] = 99                                                     # more entries than the list has
    o, lse, status = attend(cfg, kv, q, sl, g, cu, 2, arrays, most=300)
    assert status == sv.SV_DEV_BAD_GAMMA | sv.SV_DEV_BAD_LEN | sv.SV_DEV_BAD_PAGE
    assert (o[3:6] == 7.0).all()
    arrays[1][3, 0, 1] = arrays[1][3, 1, 0] = 0                              # for the oracle: not read
    arrays[0][3, 0, 1] = arrays[0][3, 1, 0] = 0
    arrays[2][4, 0] = 20
    arrays[0][arrays[0] < 0] = 0
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, good, [2] * 5, cu, 2, 128 ** -0.5, *arrays)
    attn_close(o, lse, *ref, np.r_[0:3, 6:15])


def test_bad_page_ids_leave_other_sequences_alone():
    cfg = config("ap", 3, 8, 2, 128, 41)
    sl, g = np.array([200, 300, 250], np.int32), [1, 1, 1]
    kv, cu = synth.make_kv(cfg, sl), np.array([0, 2, 4, 6], np.int32)
    q = synth.make_q(cfg, 6)
    arrays = lists_to_arrays(random_lists(np.random.default_rng(3), sl, g, 2, 1.0), 19)
    table = kv.block_table.copy()
    table[1, 2], table[1, 5] = -1, kv.k_pool.shape[0] + 5
    o, lse, status = attend(cfg, kv, q, sl, g, cu, 1, arrays, table=table)
    assert status == sv.SV_DEV_BAD_PAGE
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, 2, 128 ** -0.5, *arrays)
    attn_close(o, lse, *ref, [0, 1, 4, 5])


def test_all_pages_equal_the_verify_attention_within_roundings():
    cfg = config("ap", 4, 16, 4, 128, 42)
    sl, g = np.array([900, 64, 333, 2000], np.int32), np.array([4, 0, 8, 3], np.int32)
    check(cfg, sl, g, 8, share=1.0)


def test_two_graphs_and_a_side_stream():
    cfg = config("ap", 2, 8, 2, 128, 43)
    sl, g, cu = np.array([900, 400], np.int32), np.array([1, 2], np.int32), np.array([0, 2, 5], np.int32)
    kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, 5)
    arrays = [lists_to_arrays(random_lists(np.random.default_rng(s), sl, g, 2, 0.5), 60, fill_page=0) for s in (1, 2)]
    pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    qd = dev_bf16(q)
    ws = workspace(sv.spec_verify_attn_pages_workspace_bytes(2, 2, 8, 2, 128))
    fixed = [dev(kv.block_table), dev(sl), dev(g), dev(cu)]
    outs, graphs, keep = [], [], []
    side = torch.cuda.Stream()
    for a in arrays:
        o, lse = torch.zeros_like(qd), torch.zeros((5, 8), device=DEV)
        lists = [dev(a[0]), dev(a[1].view(np.int64)), dev(a[2])]
        keep.append(lists)
        call = lambda o=o, lse=lse, lists=lists: sv.spec_verify_attn_pages(qd, o, pool, *fixed, 2, 900, *lists, ws, lse=lse)  # noqa: E731
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        o.zero_()
        outs.append((o, lse))
        graphs.append(graph)
    for k in (0, 1, 0):                                                       # one workspace, one after the other
        graphs[k].replay()
    torch.cuda.synchronize()
    for (o, lse), a in zip(outs, arrays):
        ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, 2, 128 ** -0.5, *a)
        attn_close(f64(o), lse.cpu().numpy().astype(np.float64), *ref, np.arange(5))
