"""spec_kv_pages_update against the oracle's sequential walk: every array of the state and both row arrays, whole."""
import ctypes as C
import threading

import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from tests.harness import DEV, dev


def new_state(B, stride, n_pages, seed):
    rng = np.random.default_rng(seed)
    return [np.full((B, stride), -1, np.int32), np.zeros(B, np.int32), rng.permutation(n_pages).astype(np.int32), n_pages]


def upload(state):
    return dev(state[0]), dev(state[1]), dev(state[2]), dev(np.array([state[3]], np.int32))


def step_both(d_state, state, length, gamma=None, cu=None, gamma_max=0, n_rows=0, stream=None, want=("slot_map", "positions")):
    """One update on the device and by the oracle; asserts that they agree.  Returns the oracle's new state and rows."""
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    slot = torch.full((n_rows,), -9, dtype=torch.int64, device=DEV) if n_rows and "slot_map" in want else None
    pos = torch.full((n_rows,), -9, dtype=torch.int32, device=DEV) if n_rows and "positions" in want else None
    sv.spec_kv_pages_update(dev(np.asarray(length, np.int32)), *d_state, dev(np.asarray(gamma, np.int32)) if gamma is not None else None,
                            dev(np.asarray(cu, np.int32)) if cu is not None else None, gamma_max, slot, pos, status, stream)
    torch.cuda.synchronize()
    bt, held, fl, nf, r_slot, r_pos, cond = oracle.kv_pages_update(length, *state, n_rows, gamma, cu, gamma_max)
    np.testing.assert_array_equal(d_state[0].cpu().numpy(), bt)
    np.testing.assert_array_equal(d_state[1].cpu().numpy(), held)
    np.testing.assert_array_equal(d_state[2].cpu().numpy(), fl)
    assert int(d_state[3].item()) == nf
    if slot is not None:
        np.testing.assert_array_equal(slot.cpu().numpy(), r_slot)
    if pos is not None:
        np.testing.assert_array_equal(pos.cpu().numpy(), r_pos)
    assert int(status.item()) == cond
    return [bt, held, fl, nf], r_slot, r_pos, cond


# ------------------------------------------------------------------------------------------------ refusals (no device needed)
def good_params():
    p = sv.KvPagesParams()
    p.seq_len = p.block_table = p.n_held = p.free_list = p.n_free = p.gamma = p.cu_q = p.slot_map = p.positions = 4096
    p.batch, p.block_table_stride, p.n_pages, p.page_size, p.gamma_max, p.n_rows = 2, 4, 8, 16, 3, 8
    return p


@pytest.mark.parametrize("field,value,status", [
    ("seq_len", None, sv.SV_EINVAL), ("block_table", None, sv.SV_EINVAL), ("n_held", None, sv.SV_EINVAL), ("free_list", None, sv.SV_EINVAL),
    ("n_free", None, sv.SV_EINVAL), ("batch", 0, sv.SV_EINVAL), ("block_table_stride", 0, sv.SV_EINVAL), ("n_pages", 0, sv.SV_EINVAL),
    ("gamma_max", -1, sv.SV_EINVAL), ("n_rows", -1, sv.SV_EINVAL), ("n_rows", 0, sv.SV_EINVAL), ("gamma", None, sv.SV_EINVAL), ("cu_q", None, sv.SV_EINVAL),
    ("page_size", 32, sv.SV_EUNSUPPORTED), ("n_pages", 1 << 30, sv.SV_EUNSUPPORTED), ("n_rows", 1 << 31, sv.SV_EUNSUPPORTED),
    ("block_table_stride", 1 << 30, sv.SV_EUNSUPPORTED)])
def test_refused_before_any_launch(field, value, status):
    p = good_params()
    setattr(p, field, value)
    assert sv.load().spec_kv_pages_update(C.byref(p), None) == status
    assert sv.load().spec_kv_pages_update(None, None) == sv.SV_EINVAL


def test_binding_refuses_host_tensors():
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        sv.spec_kv_pages_update(i, i.reshape(2, 1), i, i, i[:1])


@pytest.mark.gpu
def test_binding_refuses_mismatched_shapes():
    B, S = 3, 4
    length, held, fl, nf = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B, B, 8, 1))
    table = torch.zeros((B, S), dtype=torch.int32, device=DEV)
    cu, rows = torch.zeros(B + 1, dtype=torch.int32, device=DEV), torch.zeros(6, dtype=torch.int64, device=DEV)
    for bad in (dict(block_table=table[:2]), dict(n_held=held[:2]), dict(gamma=held[:2], cu_q=cu, slot_map=rows), dict(gamma=held, cu_q=cu[:3], slot_map=rows),
                dict(gamma=held, cu_q=cu, slot_map=rows, positions=held), dict(block_table=table[:, :2]), dict(free_list=fl.long()), dict(block_table=table[0])):
        a = dict(seq_len=length, block_table=table, n_held=held, free_list=fl, n_free=nf)
        a.update(bad)
        with pytest.raises(ValueError):
            sv.spec_kv_pages_update(**a)
    with pytest.raises(sv.SpecVerifyError):
        sv.spec_kv_pages_update(length, table, held, fl, nf, slot_map=rows)         # rows without gamma / cu_q
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ against the oracle
@pytest.mark.gpu
@pytest.mark.parametrize("B,stride,gamma_max", [(1, 1, 0), (1, 300, 8), (2, 3, 64), (31, 9, 4), (128, 40, 16), (384, 30, 4), (385, 30, 4), (512, 300, 4), (513, 300, 4), (1024, 5, 2),
                                                (1025, 6, 2), (3000, 4, 1)])
def test_random_walk(B, stride, gamma_max):
    rng = np.random.default_rng([B, stride])
    n_pages = max(2, B * stride * 2 // 3)                       # some steps run out of pages
    state = new_state(B, stride, n_pages, B)
    d_state = upload(state)
    seen = 0
    for step in range(6):
        length = rng.integers(0, stride * 16 + 1, B)
        length[rng.random(B) < 0.2] = 0
        if step == 3:
            length[:] = stride * 16
        if step == 4:
            length[:] = 0
        gamma = rng.integers(0, gamma_max + 1, B)
        if step % 2:
            cu = np.arange(B + 1) * (gamma_max + 1)             # row slabs of one size
        else:
            cu = np.concatenate([[0], np.cumsum(gamma + 1)])
        n_rows = int(cu[-1]) + (5 if step == 2 else 0)
        state, slot, pos, cond = step_both(d_state, state, length, gamma, cu, gamma_max, n_rows)
        seen |= cond
        ids = np.concatenate([state[0][state[0] >= 0], state[2][:state[3]]])
        assert sorted(ids.tolist()) == list(range(n_pages))
    assert bool(seen & 64) == (n_pages < B * stride)          # step 3 asks for every column


@pytest.mark.gpu
def test_one_long_sequence_and_an_admission_of_many_pages():
    state = new_state(3, 70000, 200000, 5)
    d_state = upload(state)
    for length in ([1, 70000 * 16, 17], [1000000, 5, 0], [70000 * 16, 70000 * 16, 60000 * 16], [0, 0, 0]):
        state, *_ = step_both(d_state, state, length, [0, 4, 16], [0, 1, 6, 23], 16, 23)


@pytest.mark.gpu
@pytest.mark.parametrize("want", [(), ("slot_map",), ("positions",)])
def test_rows_are_optional(want):
    state = new_state(5, 8, 30, 6)
    d_state = upload(state)
    if want:
        step_both(d_state, state, [5, 20, 128, 0, 33], [4, 0, 3, 2, 1], [0, 5, 6, 10, 13, 15], 4, 15, want=want)
    else:
        step_both(d_state, state, [5, 20, 128, 0, 33])


@pytest.mark.gpu
def test_conditions_leave_the_others_alone():
    state = new_state(6, 4, 40, 7)
    state[1][4] = 9                                             # more pages than its row has columns
    d_state = upload(state)
    state, slot, pos, cond = step_both(d_state, state, [65, -3, 40, 2, 16, 64], [1, 1, 9, 3, 0, 2], [0, 2, 4, 8, 12, 13, 16], 3, 16)
    assert cond == sv.SV_DEV_BAD_LEN | sv.SV_DEV_BAD_GAMMA
    assert state[1].tolist() == [0, 0, 3, 1, 9, 4]
    assert (slot[4:8] >= 0).all() and (slot[13:16] >= 0).all() and (slot[:4] == -1).all() and (slot[8:13] == -1).all()


@pytest.mark.gpu
def test_bad_counts_and_bad_table_entries():
    state = new_state(3, 4, 10, 8)
    state[3] = 14                                               # more free pages than the pool has
    d_state = upload(state)
    state, *_, cond = step_both(d_state, state, [16, 0, 20], [0, 0, 0], [0, 1, 2, 3], 0, 3)
    assert cond == sv.SV_DEV_BAD_PAGE
    state = [np.array([[99, -5, 3, -1], [1, 2, -1, -1]], np.int32), np.array([3, 2], np.int32), np.array([0, 4, 5, 6], np.int32), 3]
    d_state = upload(state)
    # four pages in all: 99 is no page of the pool, and what is given back does not fit the stack
    state, slot, pos, cond = step_both(d_state, state, [16, 0], [3, 0], [0, 4, 5], 3, 5)
    assert cond == sv.SV_DEV_BAD_PAGE and (slot[:4] == -1).all() and state[3] == 4


@pytest.mark.gpu
def test_on_another_stream_and_replayed_from_a_graph():
    rng = np.random.default_rng(9)
    B, stride, gmax = 40, 12, 4
    state = new_state(B, stride, B * stride, 9)
    d_state = upload(state)
    length, gamma, cu = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B, B, B + 1))
    slot, pos = torch.zeros(B * (gmax + 1), dtype=torch.int64, device=DEV), torch.zeros(B * (gmax + 1), dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call = lambda s=None: sv.spec_kv_pages_update(length, *d_state, gamma, cu, gmax, slot, pos, status, s)  # noqa: E731
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        ln, g = rng.integers(gmax + 1, stride * 16 + 1, B), rng.integers(0, gmax + 1, B)
        cq = np.concatenate([[0], np.cumsum(g + 1)])
        for t, a in ((length, ln), (gamma, g), (cu, cq)):
            t.copy_(dev(a.astype(np.int32)))
        torch.cuda.synchronize()
        if step % 2:
            call(side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        bt, held, fl, nf, r_slot, r_pos, cond = oracle.kv_pages_update(ln, *state, slot.numel(), g, cq, gmax)
        state = [bt, held, fl, nf]
        np.testing.assert_array_equal(d_state[0].cpu().numpy(), bt)
        np.testing.assert_array_equal(d_state[2].cpu().numpy(), fl)
        np.testing.assert_array_equal(slot.cpu().numpy(), r_slot)
        np.testing.assert_array_equal(pos.cpu().numpy(), r_pos)
        assert int(status.item()) == cond == 0


@pytest.mark.gpu
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("B", [300, 700, 5000])
def test_behind_the_controller_step_after_step(B, graph):
    """Lengths that the controller writes directly in front of each call, one step after the other with nothing in between."""
    rng = np.random.default_rng(B)
    gmax, steps, stride = 4, 12, 12
    cfg = sv.GammaConfig(0.5, 2.0, 1, gmax, sv.SV_GT_PROPOSED)
    g0 = rng.integers(1, gmax + 1, B).astype(np.int32)
    first = (rng.integers(1, 60, B) + g0 + 1).astype(np.int32)
    accepted = [rng.integers(0, 2, B).astype(np.int32) for _ in range(steps)]
    n_pages = B * stride
    state = new_state(B, stride, n_pages, B)
    d_state = upload(state)
    cq, cd = np.concatenate([[0], np.cumsum(g0 + 1)]).astype(np.int32), np.concatenate([[0], np.cumsum(g0)]).astype(np.int32)
    g, sl, d_cq, d_cd, gbar = dev(g0), dev(first), dev(cq), dev(cd), dev(g0.astype(np.float64))
    d_acc = [dev(a) for a in accepted]
    n_rows = B * (gmax + 1)
    slot, pos = torch.zeros(n_rows, dtype=torch.int64, device=DEV), torch.zeros(n_rows, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def loop():
        for a in d_acc:
            sv.gamma_tune_update(a, gbar, g, sl, d_cq, d_cd, cfg, device_status=status)
            sv.spec_kv_pages_update(sl, *d_state, g, d_cq, gmax, slot, pos, status)

    torch.cuda.synchronize()
    if graph:
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            loop()
        captured.replay()
    else:
        loop()
    torch.cuda.synchronize()
    o_g, o_sl, o_gbar = g0, first, g0.astype(np.float64)
    for a in accepted:
        o_gbar, o_g, o_sl, o_cq, o_cd = oracle.gamma_tune_update(a, o_gbar, o_g, o_sl, 0.5, 2.0, 1, gmax)
        *state, r_slot, r_pos, cond = oracle.kv_pages_update(o_sl, *state, n_rows, o_g, o_cq, gmax)
        assert cond == 0
    for d, r in zip(d_state, state):
        np.testing.assert_array_equal(d.cpu().numpy().reshape(-1), np.asarray(r).reshape(-1))
    np.testing.assert_array_equal(slot.cpu().numpy(), r_slot)
    np.testing.assert_array_equal(pos.cpu().numpy(), r_pos)
    assert int(status.item()) == 0


@pytest.mark.gpu
def test_batches_of_different_sizes_from_several_host_threads():
    """Threads of one process with states of their own, whose prefix sums take more shared memory than a kernel may have by default."""
    sizes, steps, stride = (8000, 3000, 5500), 600, 3
    runs, statuses = [], [[] for _ in sizes]
    for B in sizes:
        rng = np.random.default_rng(B)
        lengths = [rng.integers(0, stride * 16 + 1, B).astype(np.int32) for _ in range(2)]
        state = new_state(B, stride, B * stride, B)
        d_state, d_len, cond = upload(state), [dev(a) for a in lengths], torch.zeros(1, dtype=torch.int32, device=DEV)
        runs.append((lengths, state, d_state, d_len, cond, [sv.kv_pages_params(a, *d_state, device_status=cond) for a in d_len], torch.cuda.Stream()))
    torch.cuda.synchronize()
    lib, start = sv.load(), threading.Barrier(len(sizes))

    def worker(k):
        torch.cuda.set_device(DEV)
        params, stream = runs[k][5], runs[k][6]
        start.wait()
        for step in range(steps):
            statuses[k].append(lib.spec_kv_pages_update(C.byref(params[step % 2]), stream.cuda_stream))
            if statuses[k][-1] != sv.SV_OK:
                return

    threads = [threading.Thread(target=worker, args=(k,)) for k in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert [set(s) for s in statuses] == [{sv.SV_OK}] * len(sizes)
    for lengths, state, d_state, _, cond, _, _ in runs:
        for step in range(steps):
            *state, _, _, o_cond = oracle.kv_pages_update(lengths[step % 2], *state)
            assert o_cond == 0
        for d, r in zip(d_state, state):
            np.testing.assert_array_equal(d.cpu().numpy().reshape(-1), np.asarray(r).reshape(-1))
        assert int(cond.item()) == 0
