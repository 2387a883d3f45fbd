"""Shared helpers of the long-context GPU tests."""
from __future__ import annotations

import numpy as np
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, bits_of, dev, dev_bf16, workspace


def config(name, batch, hq, hkv, head_dim, seed, q_scale=1.0):
    return synth.VerifyConfig(name, batch, hq, hkv, head_dim, 100, 1, 1, 0, 0, 0, 1.0, 1.0, q_scale=q_scale, seed=seed)


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def attn_close(o_gpu, lse_gpu, o, mag, lse, rows):
    """What the arithmetic allows, element by element.  The output is rounded to bf16 (2^-8 |o|), the weights of the second
    product are (2^-8 of each, at most 2^-8 mag where mag is the attention over |v|), and the float32 parts -- scores of
    up to 128 products, 2^-22 of an exponential, sums -- stay below 1e-5 relative, which is what the log-sum-exp is held to."""
    allowed = (2.0 ** -8 * (np.abs(o) + mag) + 2.0 ** -16 * mag + 3e-5 * mag + 1e-30)[rows]
    diff = np.abs(o_gpu[rows] - o[rows])
    assert (diff <= allowed).all(), f"off by {np.max(diff / allowed)} of what is allowed"
    if lse_gpu is not None:
        a, b = lse_gpu[rows], lse[rows]
        assert ((a == -np.inf) == (b == -np.inf)).all()
        ok = np.isfinite(b)
        if ok.any():
            assert np.abs(np.expm1(a[ok] - b[ok])).max() <= 1e-5


def f64(t):
    return synth.bf16_to_f32(bits_of(t)).astype(np.float64)


def masks_of(t):
    return t.cpu().numpy().view(np.uint64)


def lists_to_arrays(lists, width, fill_page=-1):
    """[batch][hkv] of (pages, masks) -> page_list, row_mask, n_list."""
    B, H = len(lists), len(lists[0])
    pl, rm, n = np.full((B, H, width), fill_page, np.int32), np.zeros((B, H, width), np.uint64), np.zeros((B, H), np.int32)
    for b in range(B):
        for h in range(H):
            pages, masks = lists[b][h]
            n[b, h] = len(pages)
            pl[b, h, :len(pages)], rm[b, h, :len(pages)] = pages, masks
    return pl, rm, n
