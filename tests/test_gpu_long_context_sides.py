"""The long-context calls against one another and against the verify attention: what several of them promise together."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16, workspace
from tests.longctx import config, f64, lists_to_arrays, masks_of
from tests.test_gpu_attn_prefix import build
from tests.test_gpu_page_select import select_gpu, setup

pytestmark = pytest.mark.gpu


def bounds_of(pool, table, length, n, hkv, head_dim):
    """Bounds of a cache of one sequence while it had `length` tokens."""
    b, s = torch.zeros((n, hkv, 2, head_dim), dtype=torch.int8, device=DEV), torch.zeros((n, hkv), device=DEV)
    one = lambda x: dev(np.array([x], np.int32))  # noqa: E731
    sv.spec_page_bounds_update(pool, b, s, dev(table), one(length), first=one(0), max_new=length)
    return b.cpu().numpy(), s.cpu().numpy()


@pytest.mark.parametrize("n_last", [1, 3])
@pytest.mark.parametrize("length,gamma", [(1999, 9), (1616, 40), (1601, 16)])
def test_rows_of_a_block_choose_as_tokens_did_with_the_bounds_of_their_time(length, gamma, n_last):
    """The block's own keys, behind a row, change nothing for it: the bounds of the whole block against those of a cache that ends
    with the row's position."""
    cfg = config("ls", 1, 8, 2, 128, 130)
    kv, q = synth.make_kv(cfg, np.array([length], np.int32)), synth.make_q(cfg, gamma + 1)
    k = synth.bf16_to_f32(kv.k_pool)
    k[kv.block_table[0, (length - gamma - 1) // 16:]] *= 50.0              # the block's pages would win every comparison
    kv = synth.KVState(synth.bf16_bits(k), kv.v_pool, kv.block_table, kv.strides)
    n = kv.k_pool.shape[0]
    pool = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool))
    whole = bounds_of(pool, kv.block_table, length, n, 2, 128)
    pl, rm, m, status = select_gpu(cfg, q, *whole, kv.block_table, [length], [gamma], [0, gamma + 1], gamma, 20, 1, n_last)
    assert status == 0
    for i in range(gamma + 1):
        end = length - gamma + i
        then = bounds_of(pool, kv.block_table, end, n, 2, 128)
        p1, m1, n1, status = select_gpu(cfg, q[i:i + 1], *then, kv.block_table, [end], [0], [0, 1], 0, 20, 1, n_last)
        assert status == 0 and (m1[0, 0, :20] == 1).all()
        for h in range(2):
            mine = pl[0, h, :m[0, h]][(rm[0, h, :m[0, h]] >> np.uint64(i)) & np.uint64(1) == 1]
            np.testing.assert_array_equal(mine, p1[0, h, :n1[0, h]])


def test_a_side_stream_leaves_whole_lists():
    cfg = config("ls", 3, 8, 2, 128, 131)
    sl, g = [700, 1300, 90], [2, 3, 1]
    table, cu, q, bounds, scales = setup(cfg, sl, g, 3, 1)
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    args = [dev_bf16(q), dev(bounds), dev(scales), i32(table), i32(sl), i32(g), i32(cu)]
    out = [torch.full((3, 2, 60), -7, dtype=torch.int32, device=DEV), torch.full((3, 2, 60), 5, dtype=torch.int64, device=DEV),
           torch.zeros((3, 2), dtype=torch.int32, device=DEV)]
    ws = workspace(sv.spec_page_select_workspace_bytes(3, 3, 2, 1300))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sv.spec_page_select(*args, 3, 1300, 15, 1, 1, *out, ws)
    torch.cuda.synchronize()
    ref = lists_to_arrays(oracle.page_select(q, bounds, scales, table, sl, g, cu, 15, 1, 1), 60)
    used = np.arange(60) < ref[2][..., None]
    np.testing.assert_array_equal(out[2].cpu().numpy(), ref[2])
    np.testing.assert_array_equal(out[0].cpu().numpy(), np.where(used, ref[0], -7))
    np.testing.assert_array_equal(masks_of(out[1]), np.where(used, ref[1], 5))


@pytest.mark.parametrize("hq,hkv,head_dim,gmax", [(16, 4, 128, 8), (64, 8, 128, 16), (12, 12, 64, 0), (8, 1, 64, 3)])
def test_all_pages_and_shared_prefixes_are_the_verify_attention(hq, hkv, head_dim, gmax):
    """The three attentions of one batch.  Each is off by at most what its arithmetic allows (2^-8 (|o| + mag) and float32 parts
    below 4e-5 mag, the log-sum-exp 1e-5), so two of them by twice that."""
    cfg = config("ls", 5, hq, hkv, head_dim, 132)
    gamma = np.minimum(np.array([4, 0, 8, 3, 16], np.int32), gmax)
    sl, group = np.array([900, 330, 420, 2000, 351], np.int32), [0, 0, 0, -1, 0]
    cu, _ = synth.prefix(gamma)
    kv, q = build(cfg, sl, group, [320]), synth.make_q(cfg, int(cu[-1]))
    pool, qd = sv.spec_kv_pool_register(dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)), dev_bf16(q)
    common = (pool, dev(kv.block_table), dev(sl), dev(gamma), dev(cu), gmax, 2000)
    lists = lists_to_arrays([[(list(range((n + 15) // 16)), [2 ** (int(g) + 1) - 1] * ((n + 15) // 16))] * hkv for n, g in zip(sl, gamma)], 125)
    outs = [(torch.zeros_like(qd), torch.zeros(q.shape[:2], device=DEV)) for _ in range(3)]
    i32 = lambda a: dev(np.asarray(a, np.int32))  # noqa: E731
    ws = [workspace(n) for n in (sv.spec_verify_attn_workspace_bytes(5, gmax, hq, hkv, head_dim, 2000),
                                 sv.spec_verify_attn_pages_workspace_bytes(5, gmax, hq, hkv, head_dim),
                                 sv.spec_verify_attn_prefix_workspace_bytes(5, gmax, hq, hkv, head_dim, 1))]
    sv.spec_verify_attn(qd, outs[0][0], *common, ws[0], lse=outs[0][1])
    sv.spec_verify_attn_pages(qd, outs[1][0], *common, dev(lists[0]), dev(lists[1].view(np.int64)), dev(lists[2]), ws[1], lse=outs[1][1])
    sv.spec_verify_attn_prefix(qd, outs[2][0], *common, i32(group), i32([320]), ws[2], lse=outs[2][1])
    torch.cuda.synchronize()
    ro, mag, rl = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, hkv, head_dim ** -0.5)
    allowed = 2.0 ** -8 * (np.abs(ro) + mag) + 4.6e-5 * mag + 1e-30
    dense, dense_lse = f64(outs[0][0]), outs[0][1].cpu().numpy().astype(np.float64)
    for o, lse in outs[1:]:
        assert (np.abs(f64(o) - dense) <= 2 * allowed).all()
        assert np.abs(np.expm1(lse.cpu().numpy().astype(np.float64) - dense_lse)).max() <= 2.1e-5
    assert (np.abs(dense - ro) <= allowed).all() and np.abs(np.expm1(dense_lse - rl)).max() <= 1e-5


def test_parameter_structs_hold_what_the_calls_pack():
    """The structs for callers of the C entry points, and the bytes that the binding's calls hand over in their place."""
    i32 = lambda *n: torch.ones(n, dtype=torch.int32, device=DEV)  # noqa: E731
    index, b16 = torch.cuda.current_device(), torch.ones((4, 2, 16, 64), dtype=torch.bfloat16, device=DEV)
    pool = sv.spec_kv_pool_register(b16, torch.ones_like(b16))
    bounds, scales, q = torch.ones((4, 2, 2, 64), dtype=torch.int8, device=DEV), torch.ones((4, 2), device=DEV), torch.ones((6, 8, 64), dtype=torch.bfloat16, device=DEV)
    lists = i32(2, 2, 5), torch.ones((2, 2, 5), dtype=torch.int64, device=DEV), i32(2, 2)
    for struct, args, pack, a, kw in (
            (sv.page_bounds_params, sv._page_bounds_args, sv._pack_page_bounds, (pool, bounds, scales, i32(2, 5), i32(2)), dict(gamma=i32(2), max_new=3)),
            (sv.page_bounds_params, sv._page_bounds_args, sv._pack_page_bounds, (pool, bounds, scales, i32(2, 5), i32(2)), dict(first=i32(2), device_status=i32(1))),
            (sv.page_select_params, sv._page_select_args, sv._pack_page_select,
             (q, bounds, scales, i32(2, 5), i32(2), i32(2), i32(3), 2, 80, 4, 1, 2, *lists), dict(device_status=i32(1)))):
        p = struct(*a, **kw)
        assert bytes(p) == pack(*args(index, *a, **kw))
    torch.cuda.synchronize()
