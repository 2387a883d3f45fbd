"""spec_page_select on the GPU against the oracle: lists and masks are whole numbers and have to be equal."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import config, lists_to_arrays, masks_of, status_word

pytestmark = pytest.mark.gpu


def random_bounds(rng, n, hkv, D, few=False):
    hi = 2 if few else 128
    a, b = rng.integers(-hi + 1, hi, (n, hkv, D)), rng.integers(-hi + 1, hi, (n, hkv, D))
    scales = np.full((n, hkv), 0.5, np.float32) if few else rng.uniform(0.005, 0.02, (n, hkv)).astype(np.float32)
    return np.stack([np.maximum(a, b), np.minimum(a, b)], 2).astype(np.int8), scales


def setup(cfg, sl, gamma, gmax, seed, few=False, padded=False):
    rng = np.random.default_rng(seed)
    need = (np.asarray(sl) + 15) // 16
    n = int(need.sum()) + 3
    perm, at, table = rng.permutation(n).astype(np.int32), 0, np.full((len(sl), int(need.max())), -1, np.int32)
    for b, m in enumerate(need):
        table[b, :m] = perm[at:at + m]
        at += m
    cu, _ = synth.padded_offsets(len(sl), gmax) if padded else synth.prefix(np.asarray(gamma, np.int32))
    q = synth.make_q(cfg, int(cu[-1]))
    bounds, scales = random_bounds(rng, n, cfg.hkv, cfg.head_dim, few)
    return table, cu, q, bounds, scales


def select_gpu(cfg, q, bounds, scales, table, sl, gamma, cu, gmax, n_select, n_first, n_last, most=None, width=None):
    B = len(sl)
    most = most or int(max(sl))
    width = width or min((most + 15) // 16, (gmax + 1) * n_select)
    out = (torch.full((B, cfg.hkv, width), -7, dtype=torch.int32, device=DEV), torch.full((B, cfg.hkv, width), 5, dtype=torch.int64, device=DEV),
           torch.full((B, cfg.hkv), -3, dtype=torch.int32, device=DEV))
    status = status_word()
    ws = workspace(sv.spec_page_select_workspace_bytes(B, gmax, cfg.hkv, most))
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    sv.spec_page_select(dev_bf16(q), dev(bounds), dev(scales), i32(table), i32(sl), i32(gamma), i32(cu), gmax, most, n_select, n_first, n_last, *out,
                        ws, device_status=status)
    torch.cuda.synchronize()
    return out[0].cpu().numpy(), masks_of(out[1]), out[2].cpu().numpy(), int(status.item())


def check(cfg, sl, gamma, gmax, n_select, n_first, n_last, seed=1, few=False, padded=False, most=None):
    table, cu, q, bounds, scales = setup(cfg, sl, gamma, gmax, seed, few, padded)
    if most:
        table = np.pad(table, ((0, 0), (0, max(0, (most + 15) // 16 - table.shape[1]))), constant_values=-1)
    pl, rm, n, status = select_gpu(cfg, q, bounds, scales, table, sl, gamma, cu, gmax, n_select, n_first, n_last, most)
    assert status == 0
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, sl, gamma, cu, n_select, n_first, n_last), pl.shape[2])
    np.testing.assert_array_equal(n, ref[2])
    used = np.arange(pl.shape[2]) < n[..., None]
    np.testing.assert_array_equal(np.where(used, pl, -1), ref[0])
    np.testing.assert_array_equal(np.where(used, rm, 0), ref[1])
    assert (pl[~used] == -7).all() and (rm[~used] == 5).all()                  # entries behind the lists stay


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (24, 2), (7, 1), (3, 3), (128, 1)])
def test_heads(hq, hkv, head_dim):
    check(config("ps", 3, hq, hkv, head_dim, 11), [700, 33, 1500], [2, 0, 1], 2, 9, 1, 2)


@pytest.mark.parametrize("n_select,n_first,n_last", [(1, 0, 1), (2, 1, 1), (16, 0, 1), (16, 4, 8), (12, 4, 8), (64, 1, 4), (500, 1, 1)])
def test_counts(n_select, n_first, n_last):
    check(config("ps", 4, 8, 2, 128, 12), [1, 2048, 16, 901], [0, 3, 5, 4], 5, n_select, n_first, n_last)


def test_ragged_batch_with_padded_slabs_and_wide_bounds():
    rng = np.random.default_rng(3)
    sl, g = rng.integers(20, 2100, 9), rng.integers(0, 17, 9)
    check(config("ps", 9, 16, 2, 128, 13), sl, g, 16, 24, 1, 2, padded=True)
    check(config("ps", 9, 16, 2, 128, 13), sl, g, 16, 24, 1, 2, most=20000)    # warps per row for 1250 pages


@pytest.mark.parametrize("length", [127 * 16, 128 * 16, 128 * 16 + 1, 129 * 16, 257 * 16 - 5])
def test_lengths_around_tiles(length):
    check(config("ps", 1, 8, 2, 64, 14), [length], [1], 1, 10, 1, 1)


@pytest.mark.parametrize("length,gamma", [(40000, 0), (40000, 6), (300007, 0), (300007, 8)])
def test_long_contexts(length, gamma):
    """More pages than a row's warps hold, with ties among them."""
    check(config("ps", 1, 2, 1, 64, 15), [length], [gamma], gamma, 40, 1, 2)
    check(config("ps", 1, 2, 1, 64, 15), [length], [gamma], gamma, 40, 1, 2, few=True)


@pytest.mark.parametrize("gamma", [0, 3, 16])
def test_ties_take_the_lower_page(gamma):
    check(config("ps", 2, 2, 2, 64, 16), [3000, 1111], [gamma, gamma], gamma, 30, 2, 3, few=True)
    cfg = config("ps", 1, 2, 2, 64, 16)
    table, cu, q, bounds, scales = setup(cfg, [2000], [gamma], gamma, 1)
    bounds[:], scales[:] = bounds[0], scales[0]                                # all alike
    pl, rm, n, _ = select_gpu(cfg, q, bounds, scales, table, [2000], [gamma], cu, gamma, 11, 0, 1)
    first = (2000 - gamma - 1) // 16                                           # the first row's own page
    assert pl[0, 0, :10].tolist() == list(range(10)) and (rm[0, :, :10] == np.uint64(2 ** (gamma + 1) - 1)).all()
    assert pl[0, 0, 10:n[0, 0]].tolist() == list(range(first, 125))


def test_largest_blocks_and_zero_queries():
    check(config("ps", 2, 8, 1, 128, 17), [1500, 1100], [63, 40], 63, 20, 1, 1)
    cfg = config("ps", 1, 4, 1, 64, 18)
    table, cu, q, bounds, scales = setup(cfg, [900], [2], 2, 1)
    q[1] = 0                                                                   # scores of 0: the lowest pages
    pl, rm, n, status = select_gpu(cfg, q, bounds, scales, table, [900], [2], cu, 2, 8, 1, 1)
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, [900], [2], cu, 8, 1, 1), pl.shape[2])
    assert status == 0 and (np.where(np.arange(pl.shape[2]) < n[..., None], pl, -1) == ref[0]).all()


def test_block_rows_read_what_single_tokens_would():
    """Row i of a block chooses as the same position does alone, with the bounds as they were then."""
    cfg = config("ps", 1, 8, 2, 128, 19)
    table, cu, q, bounds, scales = setup(cfg, [1999], [9], 9, 2)
    pl, rm, n, _ = select_gpu(cfg, q, bounds, scales, table, [1999], [9], cu, 9, 20, 1, 1)
    for i in range(10):
        p1, m1, n1, _ = select_gpu(cfg, q[i:i + 1], bounds, scales, table, [1990 + i], [0], [0, 1], 0, 20, 1, 1)
        for h in range(2):
            mine = pl[0, h, :n[0, h]][(rm[0, h, :n[0, h]] >> np.uint64(i)) & np.uint64(1) == 1]
            np.testing.assert_array_equal(mine, p1[0, h, :n1[0, h]])


def test_device_detected_conditions():
    cfg = config("ps", 5, 8, 2, 128, 20)
    sl, g = [800, 3, 800, 900, 800], [2, 4, 77, 1, 1]
    table, cu, q, bounds, scales = setup(cfg, [800, 800, 800, 900, 800], [2, 4, 4, 1, 1], 4, 1)
    table[4, 7], table[4, 9] = -1, 10 ** 6
    pl, rm, n, status = select_gpu(cfg, q, bounds, scales, table, sl, g, cu, 4, 10, 1, 1, most=890, width=50)
    assert status == sv.SV_DEV_BAD_LEN | sv.SV_DEV_BAD_GAMMA | sv.SV_DEV_BAD_PAGE
    assert (n[1] == 0).all() and (n[3] == 0).all()                             # shorter than its block; beyond max_seq_len
    ref = oracle.page_select(q, bounds, scales, table, [800, 800, 800], [2, 4, 4], cu, 10, 1, 1)
    for b in (0, 2):                                                           # gamma 77 is taken as 4
        for h in range(2):
            assert (pl[b, h, :n[b, h]].tolist(), rm[b, h, :n[b, h]].tolist()) == (ref[b][h][0], ref[b][h][1])


def test_graph_replay_and_side_stream():
    cfg = config("ps", 3, 8, 2, 128, 21)
    sl, g = [700, 1300, 90], [2, 3, 1]
    table, cu, q, bounds, scales = setup(cfg, sl, g, 3, 1)
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    args = [dev_bf16(q), dev(bounds), dev(scales), i32(table), i32(sl), i32(g), i32(cu)]
    out = [torch.zeros((3, 2, 60), dtype=torch.int32, device=DEV), torch.zeros((3, 2, 60), dtype=torch.int64, device=DEV),
           torch.zeros((3, 2), dtype=torch.int32, device=DEV)]
    ws = workspace(sv.spec_page_select_workspace_bytes(3, 3, 2, 1300))
    call = lambda: sv.spec_page_select(*args, 3, 1300, 15, 1, 1, *out, ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        first = [t.clone() for t in out]
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    args[4].copy_(i32([650, 1100, 80]))
    graph.replay()
    torch.cuda.synchronize()
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, [650, 1100, 80], g, cu, 15, 1, 1), 60)
    assert (out[2].cpu().numpy() == ref[2]).all()
    used = np.arange(60) < ref[2][..., None]
    np.testing.assert_array_equal(np.where(used, out[0].cpu().numpy(), -1), ref[0])
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, sl, g, cu, 15, 1, 1), 60)
    np.testing.assert_array_equal(first[2].cpu().numpy(), ref[2])


@pytest.mark.parametrize("gamma", [0, 5])
def test_scales_that_are_no_numbers(gamma):
    """Such pages come first, and a row still takes n_select pages."""
    cfg = config("ps", 2, 8, 2, 128, 22)
    sl, g = [1500, 2900], [gamma, gamma]
    table, cu, q, bounds, scales = setup(cfg, sl, g, gamma, 1)
    scales[table[0, [3, 40, 41]]], scales[table[1, 5:60]] = np.nan, -np.nan
    scales[table[0, 50]], scales[table[1, 70]] = np.inf, -np.inf
    bounds[table[1, 5:20]] = 0
    pl, rm, n, status = select_gpu(cfg, q, bounds, scales, table, sl, g, cu, gamma, 20, 1, 1)
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, sl, g, cu, 20, 1, 1), pl.shape[2])
    used = np.arange(pl.shape[2]) < n[..., None]
    assert status == 0 and (n == ref[2]).all()
    np.testing.assert_array_equal(np.where(used, pl, -1), ref[0])
    np.testing.assert_array_equal(np.where(used, rm, 0), ref[1])


def test_more_sequences_than_threads():
    rng = np.random.default_rng(23)
    check(config("ps", 700, 4, 1, 64, 23), rng.integers(5, 400, 700), rng.integers(0, 4, 700), 3, 6, 1, 1)
