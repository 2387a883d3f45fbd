"""The verify step with everything around it on the device: prompts admitted into an empty paged cache, then steps of pages ->
norm, rotation and append -> attention -> penalties and masks -> accept -> counts -> controller, enqueued call by call or
replayed from a graph, nothing read back in between.  Every call's outputs of every step against the oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, AcceptOut, attn_allowed, bits_of, compare_accept, dev, dev_bf16, workspace
from tests.test_gpu_logits_adjust import F32 as LOGIT_F32
from tests.test_gpu_rope_append import near

pytestmark = pytest.mark.gpu


def heads(cfg, n, step):
    w = (cfg.hq + 2 * cfg.hkv) * cfg.head_dim
    return synth.normal_bf16_bits(cfg.seed, 70, n * w, 1.0, step).reshape(n, w)


@pytest.mark.parametrize("graph", [False, True])
def test_loop_from_empty_cache(graph):
    cfg = synth.VerifyConfig("loop", 5, 8, 2, 128, 3001, 1, 1, 4, 4, 6, 0.8, 0.7, seed=77)
    B, gmax, V, D, hq, hkv, steps = cfg.batch, cfg.gamma_max, cfg.vocab, cfg.head_dim, cfg.hq, cfg.hkv, 5
    rng = np.random.default_rng(3)
    prompt = np.array([3, 40, 17, 16, 129], np.int32)
    stride, n_pages = 20, 64
    strides = (hkv * 16 * D, 16 * D, D, 1)
    inv = 10000.0 ** (-np.arange(D // 2) / (D // 2))
    qw, kw = (synth.bf16_to_f32(synth.bf16_bits(rng.uniform(0.6, 1.4, D).astype(np.float32))) for _ in range(2))
    split = [hq * D, hkv * D, hkv * D]

    # ---- device state
    k_pool, v_pool = (torch.zeros((n_pages, hkv, 16, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pool = sv.spec_kv_pool_register(k_pool, v_pool)
    table, held = torch.full((B, stride), -1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    free = rng.permutation(n_pages).astype(np.int32)
    free_list, n_free = dev(free), torch.full((1,), n_pages, dtype=torch.int32, device=DEV)
    counts = torch.full((B, (V + 7) // 8 * 8), 5, dtype=torch.int16, device=DEV)              # leftovers of earlier requests
    d_inv, d_qw, d_kw = dev(inv), dev(qw).to(torch.bfloat16), dev(kw).to(torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rep, freq, pres = (rng.uniform(a, b, B).astype(np.float32) for a, b in ((1.0, 1.3), (0.0, 0.3), (0.0, 0.3)))
    d_rep, d_freq, d_pres = dev(rep), dev(freq), dev(pres)

    # ---- prompts: all their positions are rows of one call
    n_prompt = int(prompt.sum())
    cu_p = np.concatenate([[0], np.cumsum(prompt)]).astype(np.int32)
    qkv_p, ptoks = heads(cfg, n_prompt, 99), rng.integers(0, V, n_prompt).astype(np.int32)
    slots_p, pos_p = torch.zeros(n_prompt, dtype=torch.int64, device=DEV), torch.zeros(n_prompt, dtype=torch.int32, device=DEV)
    sv.spec_kv_pages_update(dev(prompt), table, held, free_list, n_free, dev(prompt - 1), dev(cu_p), int(prompt.max()), slots_p, pos_p, status)
    q, k, v = (x.unflatten(1, (-1, D)) for x in dev_bf16(qkv_p).split(split, 1))
    sv.spec_rope_append(q, k, v, torch.empty((n_prompt, hq, D), dtype=torch.bfloat16, device=DEV), pool, pos_p, slots_p, d_inv, d_qw, d_kw, device_status=status)
    sv.spec_token_counts_update(counts, V, dev(ptoks), dev(cu_p), int(prompt.max()), torch.ones(B, dtype=torch.int32, device=DEV), True, status)
    torch.cuda.synchronize()
    ref = [np.full((B, stride), -1, np.int32), np.zeros(B, np.int32), free, n_pages]
    *ref, r_slots, r_pos, cond = oracle.kv_pages_update(prompt, *ref, n_prompt, prompt - 1, cu_p, int(prompt.max()))
    assert cond == 0 and int(status.item()) == 0
    np.testing.assert_array_equal(slots_p.cpu().numpy(), r_slots)
    np.testing.assert_array_equal(pos_p.cpu().numpy(), np.concatenate([np.arange(n) for n in prompt]))
    _, k_h, v_h = np.split(qkv_p.reshape(n_prompt, -1, D), [hq, hq + hkv], 1)
    near(bits_of(k_pool)[r_slots // 16, :, r_slots % 16], *oracle.norm_rotate(k_h, r_pos, inv, kw))
    np.testing.assert_array_equal(bits_of(v_pool)[r_slots // 16, :, r_slots % 16], v_h)
    r_counts = oracle.token_counts_update(np.full(tuple(counts.shape), 5, np.int16), V, ptoks, cu_p[:-1], prompt, np.ones(B, np.int32), True)
    np.testing.assert_array_equal(counts.cpu().numpy(), r_counts)

    # ---- the steps' buffers (row slabs of one size, so that a graph can hold their addresses)
    gcfg = sv.GammaConfig(0.5, 2.0, 1, gmax, sv.SV_GT_PROPOSED, True)
    cu_q, cu_d = synth.padded_offsets(B, gmax)
    n_q, n_d, words = int(cu_q[-1]), int(cu_d[-1]), (V + 31) // 32
    full = np.full(B, gmax, np.int32)
    inputs = [synth.make_logits(cfg, full, cu_q, cu_d, step=t) for t in range(steps)]
    qkvs = [heads(cfg, n_q, t) for t in range(steps)]
    masks = rng.integers(0, 2 ** 32, (steps, n_q, words), dtype=np.uint32) | rng.integers(0, 2 ** 32, (steps, n_q, words), dtype=np.uint32)
    masks[:, ::3] = 0xffffffff
    max_len = int(prompt.max()) + (steps + 1) * (gmax + 1)
    gbar, g = torch.zeros(B, dtype=torch.float64, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    d_cq, d_cd = (torch.zeros(B + 1, dtype=torch.int32, device=DEV) for _ in range(2))
    sv.gamma_tune_init(gbar, g, d_cq, d_cd, gcfg, 3)
    sl = dev(prompt) + g + 1
    qkv = torch.zeros((n_q, sum(split)), dtype=torch.bfloat16, device=DEV)
    q_in, k_in, v_in = (x.unflatten(1, (-1, D)) for x in qkv.split(split, 1))
    q_rot, o = torch.zeros((n_q, hq, D), dtype=torch.bfloat16, device=DEV), torch.zeros((n_q, hq, D), dtype=torch.bfloat16, device=DEV)
    slots, pos = torch.zeros(n_q, dtype=torch.int64, device=DEV), torch.zeros(n_q, dtype=torch.int32, device=DEV)
    tl, dl = torch.zeros((n_q, V), device=DEV), torch.zeros((n_d, V), device=DEV)
    x, ua, us = torch.zeros(n_d, dtype=torch.int32, device=DEV), torch.zeros(n_d, device=DEV), torch.zeros(B, device=DEV)
    mask = torch.zeros((n_q, words), dtype=torch.int32, device=DEV)
    n_acc, toks = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros((B, gmax + 1), dtype=torch.int32, device=DEV)
    ws_a = workspace(sv.spec_verify_attn_workspace_bytes(B, gmax, hq, hkv, D, max_len))
    ws_s = workspace(sv.spec_accept_sample_workspace_bytes(B, gmax, V))

    def step():
        sv.spec_kv_pages_update(sl, table, held, free_list, n_free, g, d_cq, gmax, slots, pos, status)
        sv.spec_rope_append(q_in, k_in, v_in, q_rot, pool, pos, slots, d_inv, d_qw, d_kw, device_status=status)
        sv.spec_verify_attn(q_rot, o, pool, table, sl, g, d_cq, gmax, max_len, ws_a, device_status=status)
        sv.spec_logits_adjust(tl, tl, g, d_cq, d_cd, gmax, x, counts, d_rep, d_freq, d_pres, mask=mask, device_status=status)
        sv.spec_accept_sample(tl, dl, x, ua, us, cfg.temperature, g, d_cq, d_cd, gmax, n_acc, toks, ws_s, device_status=status)
        sv.spec_token_counts_update(counts, V, toks, device_status=status)
        before = (g.clone(), sl.clone())
        sv.gamma_tune_update(n_acc, gbar, g, sl, d_cq, d_cd, gcfg, device_status=status)
        return before

    captured = None
    if graph:
        keep = [t.clone() for t in (table, held, free_list, n_free, counts, gbar, g, sl, d_cq, d_cd, k_pool, v_pool)]
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()                                             # first calls outside the capture
        side.synchronize()
        for t, c in zip((table, held, free_list, n_free, counts, gbar, g, sl, d_cq, d_cd, k_pool, v_pool), keep):
            t.copy_(c)
        status.zero_()
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            b_g, b_sl = step()
    moved = 0
    for t in range(steps):
        li = inputs[t]
        for d, s in ((tl, li.target_logits), (dl, li.draft_logits), (x, li.draft_tokens), (ua, li.u_accept), (us, li.u_sample), (mask, masks[t].view(np.int32))):
            d.copy_(dev(s))
        qkv.copy_(dev_bf16(qkvs[t]))
        if graph:
            captured.replay()
        else:
            b_g, b_sl = step()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        gam, length = b_g.cpu().numpy(), b_sl.cpu().numpy()
        # pages, slots, positions
        held_before = ref[1]
        *ref, r_slots, r_pos, cond = oracle.kv_pages_update(length, *ref, n_q, gam, cu_q, gmax)
        assert cond == 0
        moved += int((ref[1] != held_before).sum())
        np.testing.assert_array_equal(table.cpu().numpy(), ref[0])
        np.testing.assert_array_equal(held.cpu().numpy(), ref[1])
        np.testing.assert_array_equal(free_list.cpu().numpy(), ref[2])
        np.testing.assert_array_equal(slots.cpu().numpy(), r_slots)
        np.testing.assert_array_equal(pos.cpu().numpy(), r_pos)
        # queries and the cache
        used = r_slots >= 0
        q_h, k_h, v_h = np.split(qkvs[t].reshape(n_q, -1, D), [hq, hq + hkv], 1)
        near(bits_of(q_rot)[used], *(a[used] for a in oracle.norm_rotate(q_h, r_pos, inv, qw)))
        kb, vb, at = bits_of(k_pool), bits_of(v_pool), r_slots[used]
        near(kb[at // 16, :, at % 16], *(a[used] for a in oracle.norm_rotate(k_h, r_pos, inv, kw)))
        np.testing.assert_array_equal(vb[at // 16, :, at % 16], v_h[used])
        # attention over what is in the cache
        o_ref, _ = oracle.verify_attn(bits_of(q_rot), kb, vb, strides, ref[0], length, gam, cu_q, hq, hkv, 16, float(np.float32(D ** -0.5)))
        got = synth.bf16_to_f32(bits_of(o)).astype(np.float64)
        assert (np.abs(got - o_ref)[used] <= attn_allowed(o_ref)[used]).all()
        # logits
        adj, mag = oracle.logits_adjust(li.target_logits, gam, cu_q, cu_d, None, li.draft_tokens, r_counts, rep, freq, pres, mask=masks[t])
        got = tl.cpu().numpy()
        np.testing.assert_array_equal(got[~used], li.target_logits[~used])
        inf = np.isinf(adj[used])
        np.testing.assert_array_equal(got[used][inf], adj[used][inf])
        assert (np.abs(got[used][~inf] - adj[used][~inf]) <= (mag[used] * LOGIT_F32)[~inf]).all()
        # accept on the device's logits, counts, controller
        out = AcceptOut(n_acc.cpu().numpy(), toks.cpu().numpy(), None, None, None, 0, 0)
        compare_accept(out, synth.LogitInputs(got, li.draft_logits, li.draft_tokens, li.u_accept, li.u_sample), cfg.temperature, gam, cu_q, cu_d, gmax)
        r_counts = oracle.token_counts_update(r_counts, V, out.out_tokens, np.arange(B) * (gmax + 1), [gmax + 1] * B)
        np.testing.assert_array_equal(counts.cpu().numpy(), r_counts)
        np.testing.assert_array_equal(sl.cpu().numpy(), length - (gam + 1) + (out.n_accepted + 1) + (g.cpu().numpy() + 1))
    assert moved > 0


def test_draft_rows_then_the_step():
    """Drafting with the sequence's penalties (one row per sequence and drafting step), each row with the drafts so far in its
    history: the draft-side rows equal the oracle's, and the drafted tokens are the ones that rows drew."""
    B, V, gmax, T = 3, 2048, 5, 0.9
    rng = np.random.default_rng(4)
    counts = rng.integers(0, 3, (B, V)).astype(np.int16) * (rng.random((B, V)) < 0.05).astype(np.int16)
    gamma = np.array([5, 2, 4], np.int32)
    cu_d = np.concatenate([[0], np.cumsum(gamma)]).astype(np.int32)
    pen = dict(repetition=np.full(B, 1.5, np.float32), presence=np.full(B, 0.7, np.float32))
    d = {k: dev(v) for k, v in pen.items()}
    d_counts, d_gamma, d_cd = dev(counts), dev(gamma), dev(cu_d)
    n_dr, active = torch.zeros(B, dtype=torch.int32, device=DEV), torch.ones(B, dtype=torch.int32, device=DEV)
    toks, status = torch.full((int(cu_d[-1]),), -1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = workspace(sv.spec_draft_step_workspace_bytes(B, V))
    r_n, r_active, r_toks, r_top = np.zeros(B, np.int32), np.ones(B, np.int32), np.full(int(cu_d[-1]), -1, np.int32), np.zeros(int(cu_d[-1]))
    for step in range(gmax):
        rows, u = (rng.standard_normal((B, V)) * 3).astype(np.float32), rng.random(B).astype(np.float32)
        x = dev(rows)
        sv.spec_logits_adjust(x, x, None, None, d_cd, gmax, toks, d_counts, n_drafted=n_dr, active=active, device_status=status, **d)
        sv.spec_draft_step(x, T, 0.0, dev(u), d_gamma, d_cd, gmax, n_dr, active, toks, ws, device_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        adj, mag = oracle.logits_adjust(rows, cu_d=cu_d, n_drafted=r_n, draft_tokens=r_toks, counts=counts, **pen)
        got = x.cpu().numpy()
        on = r_active != 0
        np.testing.assert_array_equal(got[~on], rows[~on])
        assert (np.abs(got - adj)[on] <= (mag * LOGIT_F32)[on]).all()
        alt, flag, _ = oracle.draft_step(got, T, 0.0, u, gamma, cu_d, r_n, r_active, r_toks, r_top)
        dev_toks = toks.cpu().numpy()
        for b in np.flatnonzero(on):
            i = cu_d[b] + r_n[b] - 1
            if dev_toks[i] != r_toks[i]:
                assert flag[b] and dev_toks[i] == alt[b]
                r_toks[i] = dev_toks[i]
        np.testing.assert_array_equal(n_dr.cpu().numpy(), r_n)
        np.testing.assert_array_equal(active.cpu().numpy(), r_active)
    assert r_n.tolist() == gamma.tolist()


def test_parameter_structs_hold_what_the_calls_pack():
    """The structs for callers of the C entry points, and the bytes that the binding's calls hand over in their place."""
    i32 = lambda *n: torch.ones(n, dtype=torch.int32, device=DEV)  # noqa: E731
    b16 = lambda *n: torch.ones(n, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    index, rows = torch.cuda.current_device(), torch.ones(6, dtype=torch.int64, device=DEV)
    pool = sv.spec_kv_pool_register(b16(4, 2, 16, 64), b16(4, 2, 16, 64))
    counts, x, f = torch.ones((2, 104), dtype=torch.int16, device=DEV), torch.ones((6, 100), device=DEV), torch.ones(2, device=DEV)
    freqs = torch.ones(32, dtype=torch.float64, device=DEV)
    q, k, v = b16(6, 8 * 64).unflatten(1, (8, 64)).split([4, 2, 2], 1)
    for struct, args, pack, a, kw in (
            (sv.kv_pages_params, sv._kv_pages_args, sv._pack_kv_pages, (i32(2), i32(2, 5), i32(2), i32(9), i32(1), i32(2), i32(3), 2, rows, i32(6), i32(1)), {}),
            (sv.rope_append_params, sv._rope_append_args, sv._pack_rope_append, (q, k, v, b16(6, 4, 64), pool, i32(6), rows, freqs, b16(64), b16(64), 1e-5, True),
             dict(rope_scale=0.5, device_status=i32(1))),
            (sv.logits_adjust_params, sv._logits_adjust_args, sv._pack_logits_adjust, (x, torch.ones_like(x), i32(2), i32(3), i32(3), 2, i32(4), counts, f, f, f),
             dict(bias_tokens=i32(2, 3), bias_values=torch.ones((2, 3), device=DEV), n_bias=i32(2), mask=i32(6, 4), active=i32(2))),
            (sv.token_counts_params, sv._token_counts_args, sv._pack_token_counts, (counts, 100, i32(7), i32(3), 5, i32(2), True, i32(1)), {})):
        p = struct(*a, **kw)
        assert bytes(p) == pack(*args(index, *a, **kw))
    torch.cuda.synchronize()
