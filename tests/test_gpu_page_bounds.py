"""spec_page_bounds_update on the GPU against the oracle, whole arrays for equality."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, dev, dev_bf16
from tests.longctx import config, status_word

pytestmark = pytest.mark.gpu


def check(cfg, seq_len, first=None, gamma=None, max_new=None, slot_major=False, k_bits=None, kv=None):
    sl = np.asarray(seq_len, np.int32)
    kv = kv if kv is not None else synth.make_kv(cfg, np.maximum(sl, 1))
    k_bits = kv.k_pool if k_bits is None else k_bits
    start = np.asarray(first, np.int32) if first is not None else sl - (np.asarray(gamma, np.int32) + 1)
    n = k_bits.shape[0]
    rng = np.random.default_rng(1)
    old = rng.integers(-128, 128, (n, cfg.hkv, 2, cfg.head_dim)).astype(np.int8), rng.random((n, cfg.hkv)).astype(np.float32)
    k = dev_bf16(np.ascontiguousarray(k_bits.transpose(0, 2, 1, 3))).permute(0, 2, 1, 3) if slot_major else dev_bf16(k_bits)
    pool = sv.spec_kv_pool_register(k, k)
    bounds, scales, status = dev(old[0]), dev(old[1]), status_word()
    most = max_new or max(1, int((sl - start).max()))
    sv.spec_page_bounds_update(pool, bounds, scales, dev(kv.block_table), dev(sl), gamma=None if gamma is None else dev(np.asarray(gamma, np.int32)),
                               first=None if first is None else dev(np.asarray(first, np.int32)), max_new=most, device_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    ref = oracle.page_bounds_update(k_bits, kv.strides, kv.block_table, sl, start, *old)
    np.testing.assert_array_equal(bounds.cpu().numpy(), ref[0])
    np.testing.assert_array_equal(scales.cpu().numpy(), ref[1])
    return ref


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("slot_major", [False, True])
def test_prompts_and_blocks(head_dim, slot_major):
    cfg = config("pb", 6, 4, 3, head_dim, 91)
    sl = [1, 16, 17, 333, 48, 250]
    check(cfg, sl, first=[0] * 6, slot_major=slot_major)
    check(cfg, sl, first=[0, 15, 16, 100, 48, 0], slot_major=slot_major)           # 48 = the length: nothing new
    check(cfg, sl, gamma=[0, 4, 16, 16, 15, 1], max_new=17, slot_major=slot_major)
    check(cfg, sl, gamma=[0, 0, 0, 0, 0, 0], max_new=1, slot_major=slot_major)


def test_absent_sequences_and_wider_grid():
    cfg = config("pb0", 3, 4, 2, 128, 92)
    check(cfg, [0, 20, 0], first=[0, 3, 0], max_new=5000)


def test_extreme_keys():
    """Zeros, one large channel, subnormal and largest values, halves between two steps."""
    cfg = config("pbx", 1, 2, 2, 128, 93)
    kv = synth.make_kv(cfg, np.array([80], np.int32))
    k = synth.bf16_to_f32(kv.k_pool).copy()
    at = kv.block_table[0]
    k[at[0]] = 0.0
    k[at[1], :, :, 5] = 30000.0
    k[at[2]] = 0.0
    k[at[2], :, 3, 7] = 1e-39                                                    # a subnormal number
    k[at[3], 0] = 3.3e38
    k[at[3], 1, :, ::2] = -3.3e38
    k[at[4]] = np.arange(128) - 63.5                                             # steps of 1/2
    k[at[4], :, :, 0] = -127.0
    check(cfg, [80], first=[0], k_bits=synth.bf16_bits(k), kv=kv)


def test_random_walk_of_blocks_follows_the_cache():
    """Blocks appended and partly rejected: what the last update of a page saw is what counts."""
    cfg = config("pbw", 2, 4, 2, 64, 94)
    kv = synth.make_kv(cfg, np.array([400, 400], np.int32))
    rng = np.random.default_rng(7)
    k = dev_bf16(kv.k_pool)
    pool = sv.spec_kv_pool_register(k, k)
    n = kv.k_pool.shape[0]
    bounds, scales = torch.zeros((n, 2, 2, 64), dtype=torch.int8, device=DEV), torch.zeros((n, 2), device=DEV)
    ref = bounds.cpu().numpy(), scales.cpu().numpy()
    length = np.array([5, 90], np.int32)
    sv.spec_page_bounds_update(pool, bounds, scales, dev(kv.block_table), dev(length), first=dev(np.zeros(2, np.int32)), max_new=90)
    ref = oracle.page_bounds_update(kv.k_pool, kv.strides, kv.block_table, length, [0, 0], *ref)
    for _ in range(6):
        gamma = rng.integers(0, 9, 2).astype(np.int32)
        length = (length + gamma + 1).astype(np.int32)
        sv.spec_page_bounds_update(pool, bounds, scales, dev(kv.block_table), dev(length), gamma=dev(gamma), max_new=9)
        ref = oracle.page_bounds_update(kv.k_pool, kv.strides, kv.block_table, length, length - gamma - 1, *ref)
        length = (length - rng.integers(0, gamma + 1)).astype(np.int32)          # the rejected part of the block
    torch.cuda.synchronize()
    np.testing.assert_array_equal(bounds.cpu().numpy(), ref[0])
    np.testing.assert_array_equal(scales.cpu().numpy(), ref[1])


def test_device_detected_conditions():
    cfg = config("pbc", 6, 2, 2, 128, 95)
    sl = np.array([40, 40, 40, 40, 4000, 40], np.int32)
    kv = synth.make_kv(cfg, np.full(6, 40, np.int32))
    table = kv.block_table.copy()
    table[5, 1], table[5, 2] = -1, kv.k_pool.shape[0]
    first = np.array([0, -1, 30, 7, 3990, 0], np.int32)                        # -1, and 33 positions where 40 are allowed
    k = dev_bf16(kv.k_pool)
    pool = sv.spec_kv_pool_register(k, k)
    n = kv.k_pool.shape[0]
    zero = np.zeros((n, 2, 2, 128), np.int8), np.zeros((n, 2), np.float32)
    bounds, scales, status = dev(zero[0]), dev(zero[1]), status_word()
    sv.spec_page_bounds_update(pool, bounds, scales, dev(table), dev(sl), first=dev(first), max_new=40, device_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == sv.SV_DEV_BAD_LEN | sv.SV_DEV_BAD_PAGE
    fine = [0, 2, 3, 5]
    ok_table = table[fine].copy()
    ok_table[3, 1:] = ok_table[3, 0]                                           # checked apart below
    ref = oracle.page_bounds_update(kv.k_pool, kv.strides, ok_table[:3], sl[fine][:3], first[fine][:3], *zero)
    ref = oracle.page_bounds_update(kv.k_pool, kv.strides, ok_table[3:], [16], [0], *ref)
    np.testing.assert_array_equal(bounds.cpu().numpy(), ref[0])
    np.testing.assert_array_equal(scales.cpu().numpy(), ref[1])
    status = status_word()
    sv.spec_page_bounds_update(pool, bounds, scales, dev(kv.block_table), dev(np.full(6, 40, np.int32)), gamma=dev(np.array([-1, 9, 3, 0, 0, 0], np.int32)),
                               max_new=4, device_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == sv.SV_DEV_BAD_GAMMA
