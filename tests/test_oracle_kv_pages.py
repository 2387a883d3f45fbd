"""The oracle's page update against hand-worked cases and invariants: no page is lost or held twice, a pass there and back
restores the counts, rows name the slot that the block table names."""
import numpy as np
import pytest

import oracle


def new_pool(batch, stride, n_pages, rng):
    return (np.full((batch, stride), -1, np.int32), np.zeros(batch, np.int32), rng.permutation(n_pages).astype(np.int32), n_pages)


def test_hand_worked_case():
    table = np.array([[4, 7, -1], [2, -1, -1], [-1, -1, -1]], np.int32)
    held = np.array([2, 1, 0], np.int32)
    free = np.array([0, 1, 3, 5, 9, 9, 9, 9], np.int32)          # four free pages; what lies above is scratch
    # sequence 0 shrinks to one page (gives 7 back), 1 grows to three (takes 7, then 5), 2 appears with one page (takes 3)
    bt, h, fl, nf, slot, pos, cond = oracle.kv_pages_update([16, 48, 3], table, held, free, 4, 7, [0, 1, 2], [0, 1, 3, 6], 2)
    assert cond == 0 and nf == 2
    assert bt.tolist() == [[4, -1, -1], [2, 7, 5], [3, -1, -1]]
    assert h.tolist() == [1, 3, 1]
    assert fl.tolist() == [0, 1, 3, 5, 7, 9, 9, 9]
    assert pos.tolist() == [15, 46, 47, 0, 1, 2, -1]
    assert slot.tolist() == [4 * 16 + 15, 5 * 16 + 14, 5 * 16 + 15, 48, 49, 50, -1]


def test_out_of_pages_stops_the_acquisition():
    table, held, free, n = new_pool(4, 4, 8, np.random.default_rng(0))
    bt, h, fl, nf, slot, pos, cond = oracle.kv_pages_update([48, 64, 48, 16], table, held, free, n, 4, [0] * 4, [0, 1, 2, 3, 4], 0)
    assert cond == 64 and h.tolist() == [3, 4, 0, 0] and nf == 1            # 3 and 4 fit, 3 does not, nor the one behind it
    assert (slot[:2] >= 0).all() and (slot[2:] == -1).all() and (pos[2:] == -1).all()


@pytest.mark.parametrize("seed", range(4))
def test_pages_are_neither_lost_nor_shared(seed):
    rng = np.random.default_rng(seed)
    B, stride, n_pages = 13, 9, 80
    bt, held, fl, nf = new_pool(B, stride, n_pages, rng)
    for step in range(40):
        length = rng.integers(0, stride * 16 + 1, B).astype(np.int32)
        length[rng.random(B) < 0.2] = 0
        gamma = rng.integers(0, 5, B).astype(np.int32)
        cu = np.concatenate([[0], np.cumsum(gamma + 1)]).astype(np.int32)
        bt, held, fl, nf, slot, pos, cond = oracle.kv_pages_update(length, bt, held, fl, nf, int(cu[-1]), gamma, cu, 4)
        mine = [bt[b, :held[b]].tolist() for b in range(B)]
        every = sum(mine, []) + fl[:nf].tolist()
        assert sorted(every) == list(range(n_pages))
        assert all((bt[b, held[b]:] == -1).all() for b in range(B))
        for b in range(B):
            got = held[b] * 16 >= length[b]
            for i in range(gamma[b] + 1):
                p = length[b] - gamma[b] - 1 + i
                if got and length[b] > gamma[b]:
                    assert pos[cu[b] + i] == p and slot[cu[b] + i] == mine[b][p // 16] * 16 + p % 16
                else:
                    assert pos[cu[b] + i] == -1 and slot[cu[b] + i] == -1


def test_conditions():
    table, held, free, n = new_pool(2, 2, 8, np.random.default_rng(1))
    assert oracle.kv_pages_update([33, 1], table, held, free, n)[6] == 32            # beyond the table row
    assert oracle.kv_pages_update([-1, 1], table, held, free, n)[6] == 32
    assert oracle.kv_pages_update([1, 1], table, [3, 0], free, n)[6] == 32
    assert oracle.kv_pages_update([1, 1], table, held, free, 9)[6] == 2
    assert oracle.kv_pages_update([1, 1], table, held, free, n, 4, [1, 0], [0, 2, 4], 1)[6] == 32     # shorter than its block
    assert oracle.kv_pages_update([4, 4], table, held, free, n, 4, [3, -1], [0, 2, 4], 1)[6] == 1
