"""Pins of the long-context oracles (bounds of a page's keys, choice of pages, attention over listed pages): by hand, against
properties, and against independent restatements."""
import numpy as np
import pytest
from scipy.special import logsumexp

import oracle
from paper_2504_00030_b200 import synth


def cfg_of(**kw):
    base = dict(name="lc", batch=3, hq=8, hkv=2, head_dim=64, vocab=100, ctx_lo=40, ctx_hi=200, gamma_lo=0, gamma_hi=4, gamma_max=4,
                temperature=1.0, sigma_noise=1.0, seed=5)
    return synth.VerifyConfig(**{**base, **kw})


def test_bounds_by_hand():
    k = np.zeros((2, 1, 16, 64), np.float32)
    k[1, 0, 0, :4] = [1.0, -2.0, 127.0, 0.5]
    k[1, 0, 1, :4] = [3.0, -8.0, 1.0, 1.5]
    k[1, 0, 2, :4] = 1e6                                        # beyond the length: not looked at
    strides = [16 * 64, 16 * 64, 64, 1]
    bounds, scales = oracle.page_bounds_update(synth.bf16_bits(k), strides, [[1]], [2], [0], np.full((2, 1, 2, 64), 9, np.int8),
                                               np.full((2, 1), 7.0, np.float32))
    assert scales[1, 0] == 1.0 and scales[0, 0] == 7.0 and (bounds[0] == 9).all()
    assert bounds[1, 0, 0, :5].tolist() == [3, -2, 127, 2, 0] and bounds[1, 0, 1, :5].tolist() == [1, -8, 1, 0, 0]      # halves to even


def test_bounds_only_the_pages_from_first_on():
    cfg = cfg_of(batch=1)
    kv = synth.make_kv(cfg, np.array([100], np.int32))
    new = np.full((kv.k_pool.shape[0], 2, 2, 64), 3, np.int8), np.full((kv.k_pool.shape[0], 2), 3.0, np.float32)
    bounds, _ = oracle.page_bounds_update(kv.k_pool, kv.strides, kv.block_table, [100], [47], *new)
    touched = [(bounds[p] != 3).any() for p in kv.block_table[0]]
    assert touched == [False] * 2 + [True] * 5


def test_score_bounds_every_key_of_the_page():
    """Up to the roundings to 8 bits (half a step of the query and of the bound), no key of a page gives more than its score."""
    cfg = cfg_of(batch=1)
    kv = synth.make_kv(cfg, np.array([160], np.int32))
    n = kv.k_pool.shape[0]
    bounds, scales = oracle.page_bounds_update(kv.k_pool, kv.strides, kv.block_table, [160], [0], np.zeros((n, 2, 2, 64), np.int8),
                                               np.zeros((n, 2), np.float32))
    q = synth.make_q(cfg, 1)[0, :4]
    score, _ = oracle.page_choice(q, bounds, scales, 0, kv.block_table[0], 10, 5, 1, 1)
    qf = synth.bf16_to_f32(q).astype(np.float64)
    qs = np.abs(qf).max() / 127
    for p in range(10):
        k = synth.bf16_to_f32(kv.k_pool[kv.block_table[0, p], 0]).astype(np.float64)
        s = float(scales[kv.block_table[0, p], 0])
        # |q k - qi Mi qs s| <= |q| s / 2 + 127 s qs / 2 for each dim, and the like for the minimum
        slack = (np.abs(qf).sum(1) * s / 2 + 64 * 127 * s * qs / 2).max()
        assert (qf @ k.T).max() <= score[p] * qs + slack


def test_choice_fixed_pages_ties_and_short_contexts():
    bounds = np.zeros((12, 1, 2, 64), np.int8)
    scales = np.ones((12, 1), np.float32)
    bounds[:, 0, 0, 0] = [5, 9, 1, 7, 7, 7, 2, 7, 0, 0, 0, 0]
    bounds[:, 0, 1, 0] = bounds[:, 0, 0, 0]
    q = synth.bf16_bits(np.eye(1, 64, dtype=np.float32))
    table = np.arange(12, dtype=np.int32)
    take = lambda *a: np.nonzero(oracle.page_choice(q, bounds, scales, 0, table, *a)[1])[0].tolist()  # noqa: E731
    assert take(12, 5, 0, 1) == [1, 3, 4, 5, 11]                # three of the four sevens, the lower pages
    assert take(12, 5, 1, 2) == [0, 1, 3, 10, 11]
    assert take(12, 3, 1, 2) == [0, 10, 11]
    assert take(4, 5, 1, 2) == [0, 1, 2, 3] and take(1, 5, 1, 2) == [0]
    assert take(12, 12, 0, 1) == list(range(12))


@pytest.mark.parametrize("group", [1, 4])
def test_scores_against_numpy(group):
    rng = np.random.default_rng(4)
    a, b = (rng.integers(-127, 128, (9, 2, 64)) for _ in range(2))
    bounds = np.stack([np.maximum(a, b), np.minimum(a, b)], 2).astype(np.int8)
    scales = rng.uniform(0.01, 0.02, (9, 2)).astype(np.float32)
    q = synth.bf16_bits(rng.standard_normal((group, 64)).astype(np.float32))
    qf = synth.bf16_to_f32(q)
    qi = np.clip(np.rint(qf / np.float32(np.abs(qf).max() * np.float32(1 / 127))), -127, 127).astype(np.int64)
    table = rng.permutation(9).astype(np.int32)
    bd = bounds[table, 1].astype(np.int64)
    want = np.maximum(qi[:, None] * bd[None, :, 0], qi[:, None] * bd[None, :, 1]).sum(-1).max(0).astype(np.float32) * scales[table, 1]
    score, chosen = oracle.page_choice(q, bounds, scales, 1, table, 9, 4, 0, 1)
    np.testing.assert_array_equal(score, want)
    assert set(np.nonzero(chosen)[0]) == {8} | set(np.argsort(-want[:8], kind="stable")[:3])


def test_attention_over_all_pages_is_the_verify_attention():
    cfg = cfg_of()
    sl, g = synth.draw_lengths(cfg)
    cu, _ = synth.prefix(g)
    kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, int(cu[-1]))
    ref = oracle.verify_attn(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, cfg.hq, cfg.hkv, 16, 0.125)
    width = kv.block_table.shape[1]
    lists = np.tile(np.arange(width, dtype=np.int32)[::-1], (3, 2, 1))                  # any order
    n = np.repeat(((sl + 15) // 16)[:, None], 2, 1)
    lists = np.stack([np.stack([np.pad(np.arange(m, dtype=np.int32)[::-1], (0, width - m))] * 2) for m in n[:, 0]])
    for args in ((), (lists, np.full(lists.shape, 31, np.uint64), n)):
        o, mag, lse = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, cfg.hkv, 0.125, *args)
        np.testing.assert_allclose(o, ref[0], atol=1e-12)
        np.testing.assert_allclose(lse, ref[1], atol=1e-12)
        assert (np.abs(o) <= mag + 1e-12).all()


def test_attention_over_listed_pages_against_numpy():
    cfg = cfg_of(batch=1)
    sl, g, cu = np.array([75], np.int32), np.array([2], np.int32), np.array([0, 3], np.int32)
    kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, 3)
    lists = np.array([[[0, 2, 4], [4, 1, 0]]], np.int32)
    masks = np.array([[[0b001, 0b101, 0b111], [0b110, 0b011, 0]]], np.uint64)
    o, _, lse = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, g, cu, 2, 0.25, lists, masks, [[3, 2]])
    k, v, qf = (synth.bf16_to_f32(x).astype(np.float64) for x in (kv.k_pool[kv.block_table[0, :5]], kv.v_pool[kv.block_table[0, :5]], q))
    for i in range(3):
        for h in range(8):
            pages = [int(p) for p, m in zip(lists[0, h // 4][:3 - h // 4], masks[0, h // 4]) if int(m) >> i & 1]
            at = [t for p in pages for t in range(p * 16, p * 16 + 16) if t <= 72 + i]
            if not at:
                assert (o[i, h] == 0).all() and lse[i, h] == -np.inf
                continue
            s = np.array([qf[i, h] @ k[t // 16, h // 4, t % 16] * 0.25 for t in at])
            np.testing.assert_allclose(lse[i, h], logsumexp(s), atol=1e-12)
            np.testing.assert_allclose(o[i, h], np.exp(s - logsumexp(s)) @ np.array([v[t // 16, h // 4, t % 16] for t in at]), atol=1e-12)
