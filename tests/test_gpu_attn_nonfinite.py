"""Attention over listed pages and behind shared prefixes with queries that are no numbers or infinite: the rows that the
float64 oracle makes NaN are NaN, in the output and in the log-sum-exp, wherever a block's share of the work ends; all other
rows are as if those queries were not there."""
import numpy as np
import pytest

import oracle
from paper_2504_00030_b200 import synth
from tests import test_gpu_attn_pages as pages
from tests import test_gpu_attn_prefix as prefixes
from tests.longctx import attn_close, config, lists_to_arrays

pytestmark = pytest.mark.gpu

NAN, INF = 0x7fc0, 0x7f80


def spoil(rng, q, kv):
    """Every sixth row and head gets a NaN or +inf.  Dim 3 of the keys is +1 and -1 by turns, so that a query infinite there
    has +inf among its scores on any page that it sees."""
    kv.k_pool[:, :, 0::2, 3], kv.k_pool[:, :, 1::2, 3] = synth.bf16_bits(np.array([1.0, -1.0], np.float32))
    pick = rng.random(q.shape[:2]) < 1 / 6
    pick.reshape(-1)[0] = True
    r, h = np.nonzero(pick)
    infinite = rng.random(len(r)) < 0.5
    q[r[infinite], h[infinite], 3] = INF
    q[r[~infinite], h[~infinite], rng.integers(0, q.shape[2], (~infinite).sum())] = NAN


def same(o, lse, ref, rows):
    """NaN where the oracle has it; the rest within the tolerance of the arithmetic."""
    ro, mag, rl = ref
    bad = np.isnan(rl[rows])
    assert bad.any() and not bad.all()
    assert (np.isnan(o[rows]) == bad[..., None]).all(), "outputs"
    assert (np.isnan(lse[rows]) == bad).all(), "log-sum-exps"
    keep = lambda a: np.where(np.isnan(rl).reshape(rl.shape + (1,) * (a.ndim - 2)), 0.0, a)  # noqa: E731
    attn_close(keep(o), keep(lse), keep(ro), keep(mag), keep(rl), rows)


def over_pages(cfg, sl, gamma, share):
    rng = np.random.default_rng(cfg.seed)
    sl, gamma = np.asarray(sl, np.int32), np.asarray(gamma, np.int32)
    cu, _ = synth.prefix(gamma)
    kv, q = synth.make_kv(cfg, sl), synth.make_q(cfg, int(cu[-1]))
    spoil(rng, q, kv)
    lists = pages.random_lists(rng, sl, gamma, cfg.hkv, share)
    arrays = lists_to_arrays(lists, max(1, max(len(p) for s in lists for p, _ in s)))
    o, lse, status = pages.attend(cfg, kv, q, sl, gamma, cu, int(gamma.max()), arrays)
    assert status == 0
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, cfg.hkv, cfg.head_dim ** -0.5, *arrays)
    same(o, lse, ref, np.arange(int(cu[-1])))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("hq,gmax", [(4, 3), (16, 7), (32, 16)])
def test_lists_in_whole_pairs_and_split(hq, gmax, head_dim):
    """From 8 to 544 rows to a kv head (queries brought ahead, one row tile, two, several pairs): many short lists, then few long ones."""
    rng = np.random.default_rng(81)
    over_pages(config("nf", 160, hq, hq // 2 if hq == 4 else 4, head_dim, 81), rng.integers(gmax + 1, 150, 160), rng.integers(0, gmax + 1, 160), 0.5)
    over_pages(config("nf", 2, hq, 1, head_dim, 82), [9000, 700], [gmax, 0], 0.5)


def test_rows_without_keys_stay_zeros():
    over_pages(config("nf", 12, 8, 2, 128, 83), [200] * 12, [3] * 12, 0.05)


def behind_prefixes(cfg, sl, gamma, group, prefix):
    sl, gamma = np.asarray(sl, np.int32), np.asarray(gamma, np.int32)
    cu, _ = synth.prefix(gamma)
    kv, q = prefixes.build(cfg, sl, group, prefix), synth.make_q(cfg, int(cu[-1]))
    spoil(np.random.default_rng(cfg.seed), q, kv)
    o, lse, status = prefixes.attend(cfg, kv, q, sl, gamma, cu, int(gamma.max()), group, prefix)
    assert status == 0
    ref = oracle.attn_pages(q, kv.k_pool, kv.v_pool, kv.strides, kv.block_table, sl, gamma, cu, cfg.hkv, cfg.head_dim ** -0.5)
    same(o, lse, ref, np.arange(int(cu[-1])))


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("gmax", [0, 3, 17])
def test_prefixes_in_whole_pairs_and_split(gmax, head_dim):
    rng = np.random.default_rng(84)
    cfg = config("nf", 80, 16, 8, head_dim, 84)
    group, prefix = np.arange(80) // 2, [int(n) * 16 for n in rng.integers(1, 9, 40)]
    gamma = rng.integers(0, gmax + 1, 80)
    gamma[0] = gmax
    behind_prefixes(cfg, [prefix[g] + int(gamma[b]) + 1 + int(rng.integers(0, 60)) for b, g in enumerate(group)], gamma, group, prefix)
    behind_prefixes(config("nf", 3, 8, 2, head_dim, 85), [5000, 5300, 400], [gmax, 0, gmax], [0, 0, -1], [4096])
