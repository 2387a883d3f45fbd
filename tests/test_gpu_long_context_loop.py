"""The long-context calls together, as a decoding loop uses them: a draft block's keys are appended, the bounds of their
pages brought up to date, pages chosen, and the block attends over them; and blocks behind a shared prompt."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, bits_of, dev, dev_bf16, workspace
from tests.longctx import attn_close, config, f64, lists_to_arrays, masks_of, status_word
from tests.test_gpu_attn_prefix import build

pytestmark = pytest.mark.gpu
SELECT = (12, 1, 2)


class Loop:
    """Device state of a batch at most `most` tokens long; step() is what is captured."""

    def __init__(self, cfg, most, gmax, group=None, prefix=None):
        B = cfg.batch
        self.cfg, self.most, self.gmax, self.group = cfg, most, gmax, group
        kv = build(cfg, [most] * B, group if group is not None else [-1] * B, prefix or [16])
        self.table, self.strides = kv.block_table, kv.strides
        self.k, self.v = dev_bf16(kv.k_pool), dev_bf16(kv.v_pool)
        self.pool = sv.spec_kv_pool_register(self.k, self.v)
        n = kv.k_pool.shape[0]
        self.bounds, self.scales = torch.zeros((n, cfg.hkv, 2, cfg.head_dim), dtype=torch.int8, device=DEV), torch.zeros((n, cfg.hkv), device=DEV)
        cu, _ = synth.padded_offsets(B, gmax)                              # a slab of gmax + 1 rows for each sequence
        self.cu, rows = cu, int(cu[-1])
        self.d_table, self.d_cu = dev(kv.block_table), dev(cu)
        self.sl, self.gamma = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
        self.q = torch.zeros((rows, cfg.hq, cfg.head_dim), dtype=torch.bfloat16, device=DEV)
        self.k_new, self.v_new = (torch.zeros((rows, cfg.hkv, cfg.head_dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        self.o, self.lse = torch.zeros_like(self.q), torch.zeros(rows, cfg.hq, device=DEV)
        self.status = status_word()
        width = min((most + 15) // 16, (gmax + 1) * SELECT[0])
        self.lists = (torch.zeros((B, cfg.hkv, width), dtype=torch.int32, device=DEV), torch.zeros((B, cfg.hkv, width), dtype=torch.int64, device=DEV),
                      torch.zeros((B, cfg.hkv), dtype=torch.int32, device=DEV))
        if group is not None:
            self.d_group, self.d_prefix = dev(np.asarray(group, np.int32)), dev(np.asarray(prefix, np.int32))
            self.ws = workspace(sv.spec_verify_attn_prefix_workspace_bytes(B, gmax, cfg.hq, cfg.hkv, cfg.head_dim, len(prefix)))
        else:
            self.ws_select = workspace(sv.spec_page_select_workspace_bytes(B, gmax, cfg.hkv, most))
            self.ws = workspace(sv.spec_verify_attn_pages_workspace_bytes(B, gmax, cfg.hq, cfg.hkv, cfg.head_dim))

    def prompt(self, lengths):
        lengths = np.asarray(lengths, np.int32)
        sv.spec_page_bounds_update(self.pool, self.bounds, self.scales, self.d_table, dev(lengths), first=torch.zeros_like(self.sl),
                                   max_new=int(lengths.max()), device_status=self.status)

    def block(self, lengths, gamma, seed):
        """The next draft block's inputs; lengths include it."""
        self.sl.copy_(dev(np.asarray(lengths, np.int32)))
        self.gamma.copy_(dev(np.asarray(gamma, np.int32)))
        rng = np.random.default_rng(seed)
        for t in (self.q, self.k_new, self.v_new):
            t.copy_(dev_bf16(synth.bf16_bits(rng.standard_normal(tuple(t.shape)).astype(np.float32))))

    def step(self):
        common = (self.d_table, self.sl, self.gamma, self.d_cu, self.gmax)
        sv.spec_kv_append(self.k_new, self.v_new, self.pool, *common, device_status=self.status)
        if self.group is not None:
            sv.spec_verify_attn_prefix(self.q, self.o, self.pool, *common, self.most, self.d_group, self.d_prefix, self.ws, lse=self.lse,
                                       device_status=self.status)
            return
        sv.spec_page_bounds_update(self.pool, self.bounds, self.scales, self.d_table, self.sl, gamma=self.gamma, max_new=self.gmax + 1,
                                   device_status=self.status)
        sv.spec_page_select(self.q, self.bounds, self.scales, *common, self.most, *SELECT, *self.lists, self.ws_select, device_status=self.status)
        sv.spec_verify_attn_pages(self.q, self.o, self.pool, *common, self.most, *self.lists, self.ws, lse=self.lse, device_status=self.status)

    def snapshot(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        return [t.clone() for t in (self.k, self.v, self.bounds, self.scales, *self.lists, self.o, self.lse)]

    def check(self, before, lengths, gamma):
        """A step from the state `before` (numpy: k, v, bounds, scales) against the oracle; the state after it."""
        cfg, (k, v, bounds, scales) = self.cfg, before
        sl, g = np.asarray(lengths, np.int32), np.asarray(gamma, np.int32)
        q = bits_of(self.q)
        k, v = oracle.kv_append(bits_of(self.k_new), bits_of(self.v_new), k, v, self.strides, self.table, sl, g, self.cu, 16)
        np.testing.assert_array_equal(bits_of(self.k), k)
        np.testing.assert_array_equal(bits_of(self.v), v)
        arrays = ()
        if self.group is None:
            bounds, scales = oracle.page_bounds_update(k, self.strides, self.table, sl, sl - g - 1, bounds, scales)
            np.testing.assert_array_equal(self.bounds.cpu().numpy(), bounds)
            np.testing.assert_array_equal(self.scales.cpu().numpy(), scales)
            arrays = lists_to_arrays(oracle.page_select(q, bounds, scales, self.table, sl, g, self.cu, *SELECT), self.lists[0].shape[2])
            used = np.arange(arrays[0].shape[2]) < arrays[2][..., None]
            np.testing.assert_array_equal(self.lists[2].cpu().numpy(), arrays[2])
            np.testing.assert_array_equal(np.where(used, self.lists[0].cpu().numpy(), -1), arrays[0])
            np.testing.assert_array_equal(np.where(used, masks_of(self.lists[1]), 0), arrays[1])
        ref = oracle.attn_pages(q, k, v, self.strides, self.table, sl, g, self.cu, cfg.hkv, cfg.head_dim ** -0.5, *arrays)
        rows = np.concatenate([np.arange(self.cu[b], self.cu[b] + g[b] + 1) for b in range(len(sl))])
        attn_close(f64(self.o), self.lse.cpu().numpy().astype(np.float64), *ref, rows)
        return k, v, bounds, scales

    def state(self):
        torch.cuda.synchronize()
        return bits_of(self.k), bits_of(self.v), self.bounds.cpu().numpy(), self.scales.cpu().numpy()


def captured(loop):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.step()
    return graph


def blocks(rng, lengths, gmax, n):
    """n draft blocks, each behind an accepted part of the one before."""
    lengths = np.asarray(lengths)
    for _ in range(n):
        gamma = rng.integers(0, gmax + 1, len(lengths))
        yield lengths + gamma + 1, gamma
        lengths = lengths + rng.integers(1, gamma + 2)


@pytest.mark.parametrize("hq,hkv,head_dim,gmax", [(8, 2, 128, 4), (16, 1, 64, 9), (4, 4, 128, 0)])
def test_blocks_over_chosen_pages(hq, hkv, head_dim, gmax):
    """Eager steps and replays of one captured step, the lengths on the device; a block is redone over a rejected one's slots."""
    rng = np.random.default_rng(61)
    loop = Loop(config("lc", 4, hq, hkv, head_dim, 61), 1400, gmax)
    start = [1200, 300, 17, 640]
    loop.prompt(start)
    state = loop.state()
    graph = None
    for n, (lengths, gamma) in enumerate(blocks(rng, start, gmax, 6)):
        loop.block(lengths, gamma, n)
        if n < 2:
            loop.step()
        else:
            graph = graph or captured(loop)
            graph.replay()
        loop.snapshot()
        state = loop.check(state, lengths, gamma)


def test_blocks_behind_a_shared_prompt():
    rng = np.random.default_rng(62)
    loop = Loop(config("lc", 7, 16, 2, 128, 62), 1100, 5, [0, 0, -1, 1, 0, 1, 0], [800, 330])
    start = [805, 900, 400, 340, 850, 333, 801]
    state = loop.state()
    graph = None
    for n, (lengths, gamma) in enumerate(blocks(rng, start, 5, 5)):
        loop.block(lengths, gamma, n)
        if n < 2:
            loop.step()
        else:
            graph = graph or captured(loop)
            graph.replay()
        loop.snapshot()
        state = loop.check(state, lengths, gamma)


def test_two_loops_on_two_streams():
    """Calls that are under way at once, each with its own workspaces, give the bits that they give alone."""
    loops = [Loop(config("lc", 24, 16, 2, 128, 63 + i), 1400, 4) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in loops]
    lengths = np.random.default_rng(63).integers(600, 1400, 24)
    gamma = np.arange(24) % 5
    alone = []
    for loop in loops:
        loop.prompt(lengths - gamma - 1)
        loop.block(lengths, gamma, 1)
        loop.step()
        alone.append(loop.snapshot())
        loop.o.zero_()
        loop.lse.zero_()
    torch.cuda.synchronize()
    for _ in range(4):
        for loop, stream in zip(loops, streams):
            with torch.cuda.stream(stream):
                loop.step()
    for loop, first in zip(loops, alone):
        for a, b in zip(loop.snapshot(), first):
            assert torch.equal(a, b)
