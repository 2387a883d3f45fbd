"""spec_logits_adjust and spec_token_counts_update against the oracle; rows and padding that belong to nobody stay as they were."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from tests.harness import DEV, dev

FILL = 77.0
# float32 errors relative to the sum of the terms' magnitudes: 1 / repetition and its product (two half-ulps, 2^-23),
# frequency * count, + presence, + bias, the last addition (a half-ulp each): below 2^-22.
F32 = 2.0 ** -22


def make_case(B, V, gmax, seed, bf16=False, penal=True, bias=0, mask=False, draft=False, pad_rows=0, gamma=None, stride=None, which="rfp"):
    rng = np.random.default_rng([seed, B, V])
    c = dict(B=B, V=V, gmax=gmax, bf16=bf16, draft=draft)
    g = rng.integers(0, gmax + 1, B).astype(np.int32) if gamma is None else np.asarray(gamma, np.int32)
    c["gamma"], c["cu_q"], c["cu_d"] = g, np.concatenate([[0], np.cumsum(g + 1)]).astype(np.int32), np.concatenate([[0], np.cumsum(g)]).astype(np.int32)
    n = B if draft else int(c["cu_q"][-1]) + pad_rows
    c["n_rows"], c["stride"] = n, stride or V
    x = (rng.standard_normal((n, V)) * 3).astype(np.float32)
    if bf16:
        x = torch.from_numpy(x).to(torch.bfloat16).float().numpy()
    c["x"] = x
    c["n_drafted"] = rng.integers(0, g + 1).astype(np.int32) if draft else None
    c["tokens"] = np.minimum((rng.random(max(1, int(g.sum()))) ** 4 * V).astype(np.int32), V - 1)
    c["kw"] = {}
    if penal:
        cs = (V + 7) // 8 * 8
        cnt = np.zeros((B, cs), np.int16)
        for b in range(B):
            t = np.minimum((rng.random(60) ** 4 * V).astype(np.int64), V - 1)
            np.add.at(cnt[b], t, 1)
            t = np.minimum((rng.random(60) ** 2 * V).astype(np.int64), V - 1)
            cnt[b, t] |= np.int16(-32768)
        cnt[:, V:] = 0x1234                              # behind the vocabulary: not read into anything
        c["kw"]["counts"] = cnt
        names = dict(r="repetition", f="frequency", p="presence")
        for k in which:
            lo, hi = dict(r=(0.8, 1.5), f=(-0.3, 0.6), p=(-0.2, 0.7))[k]
            c["kw"][names[k]] = rng.uniform(lo, hi, B).astype(np.float32)
    if bias:
        c["kw"]["bias_tokens"] = rng.integers(0, V, (B, bias)).astype(np.int32)
        c["kw"]["bias_values"] = rng.uniform(-30, 30, (B, bias)).astype(np.float32)
        c["kw"]["n_bias"] = rng.integers(0, bias + 1, B).astype(np.int32)
    if mask:
        m = rng.integers(0, 2 ** 32, (n, (V + 31) // 32 + 1), dtype=np.uint32)
        kind = rng.integers(0, 4, n)
        m[kind == 0] = 0xffffffff
        m[kind == 1] &= rng.integers(0, 2 ** 32, m[kind == 1].shape, dtype=np.uint32) & rng.integers(0, 2 ** 32, m[kind == 1].shape, dtype=np.uint32)
        m[kind == 2] = 0                                 # nothing allowed
        c["kw"]["mask"] = m
    return c


def gpu_args(c):
    kw = {}
    for k, v in c["kw"].items():
        kw["token_counts" if k == "counts" else k] = dev(v.view(np.int32) if k == "mask" else v)
    if c["draft"]:
        kw["n_drafted"] = dev(c["n_drafted"])
    return (dev(c["gamma"]), dev(c["cu_q"]), dev(c["cu_d"]), c["gmax"], dev(c["tokens"])), kw


def logits_of(c, fill=FILL):
    """[n_rows, V] view of a buffer with the case's row stride; the padding holds `fill`."""
    buf = torch.full((c["n_rows"], c["stride"]), fill, device=DEV, dtype=torch.bfloat16 if c["bf16"] else torch.float32)
    buf[:, :c["V"]] = dev(c["x"]).to(buf.dtype)
    return buf


def run(c, inplace=False, stream=None, active=None):
    buf = logits_of(c)
    out = buf if inplace else torch.full_like(buf, FILL)
    args, kw = gpu_args(c)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    x = buf[:, :c["V"]]
    sv.spec_logits_adjust(x, x if inplace else out[:, :c["V"]], *args, **kw, active=active, device_status=status, stream=stream)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64), int(status.item())


def check(c, got, inplace=False, skipped=()):
    V = c["V"]
    ref, mag = oracle.logits_adjust(c["x"], c["gamma"], c["cu_q"], c["cu_d"], c["n_drafted"], c["tokens"], **c["kw"])
    for b in skipped:
        rows = [b] if c["draft"] else range(c["cu_q"][b], c["cu_q"][b + 1])
        ref[rows] = np.nan
    used = ~np.isnan(ref).all(1) if c["n_rows"] else np.zeros(0, bool)
    assert (got[:, V:] == FILL).all()                    # between the vocabulary and the stride
    if inplace:
        np.testing.assert_array_equal(got[~used, :V], c["x"][~used])
    else:
        assert (got[~used] == FILL).all()
    g, r, m = got[used, :V], ref[used], mag[used]
    inf = ~np.isfinite(r)
    np.testing.assert_array_equal(g[inf], r[inf])
    g, r, m = g[~inf], r[~inf], m[~inf]
    allowed = m * F32 + (np.abs(r) + m * F32) * (2.0 ** -8 if c["bf16"] else 0.0) + 1e-300
    err = np.abs(g - r)
    assert (err <= allowed).all(), float((err / allowed).max())


# ------------------------------------------------------------------------------------------------ refusals (no device needed)
def good_params():
    p = sv.LogitsAdjustParams()
    base = 1 << 20
    p.logits, p.out = base, base + (1 << 18)
    p.row_stride = p.out_stride = 1000
    p.n_rows, p.vocab, p.batch, p.gamma_max = 4, 1000, 2, 1
    p.gamma = p.cu_q = p.cu_d = p.draft_tokens = p.token_counts = p.repetition = p.bias_tokens = p.bias_values = p.n_bias = p.mask = 4096
    p.n_d_rows, p.count_stride, p.bias_stride, p.mask_stride = 2, 1000, 3, 32
    return p


@pytest.mark.parametrize("field,value,status", [
    ("logits", None, sv.SV_EINVAL), ("out", None, sv.SV_EINVAL), ("batch", 0, sv.SV_EINVAL), ("vocab", 0, sv.SV_EINVAL), ("n_rows", 0, sv.SV_EINVAL),
    ("gamma_max", -1, sv.SV_EINVAL), ("row_stride", 999, sv.SV_EINVAL), ("out_stride", 999, sv.SV_EINVAL), ("gamma", None, sv.SV_EINVAL), ("cu_q", None, sv.SV_EINVAL),
    ("cu_d", None, sv.SV_EINVAL), ("draft_tokens", None, sv.SV_EINVAL), ("token_counts", None, sv.SV_EINVAL), ("count_stride", 992, sv.SV_EINVAL),
    ("n_d_rows", -1, sv.SV_EINVAL), ("bias_tokens", None, sv.SV_EINVAL), ("bias_values", None, sv.SV_EINVAL), ("n_bias", None, sv.SV_EINVAL), ("bias_stride", 0, sv.SV_EINVAL),
    ("mask_stride", 31, sv.SV_EINVAL), ("gamma_max", 65, sv.SV_EUNSUPPORTED), ("bias_stride", (1 << 30) + 1, sv.SV_EUNSUPPORTED), ("vocab", (1 << 30) + 1, sv.SV_EINVAL), ("token_counts", 4100, sv.SV_EALIGN),
    ("count_stride", 1004, sv.SV_EALIGN), ("logits", (1 << 20) + 2, sv.SV_EALIGN), ("out", (1 << 20) + 16, sv.SV_EINVAL), ("out", (1 << 20) - 16, sv.SV_EINVAL),
    ("out", (1 << 20) + 4000 * 3 + 3999 // 4 * 4, sv.SV_EINVAL)])
def test_refused_before_any_launch(field, value, status):
    p = good_params()
    setattr(p, field, value)
    assert sv.load().spec_logits_adjust(C.byref(p), None) == status
    assert sv.load().spec_logits_adjust(None, None) == sv.SV_EINVAL


def test_draft_rows_need_a_row_per_sequence_and_nothing_to_do_is_nothing():
    p = good_params()
    p.n_drafted, p.gamma, p.cu_q, p.n_rows = 4096, None, None, 1
    assert sv.load().spec_logits_adjust(C.byref(p), None) == sv.SV_EINVAL
    p = good_params()
    p.out = p.logits
    p.repetition = p.bias_tokens = p.bias_values = p.n_bias = p.mask = None
    assert sv.load().spec_logits_adjust(C.byref(p), None) == sv.SV_OK


@pytest.mark.parametrize("field,value,status", [
    ("token_counts", None, sv.SV_EINVAL), ("batch", 0, sv.SV_EINVAL), ("vocab", 0, sv.SV_EINVAL), ("max_tokens", -1, sv.SV_EINVAL), ("count_stride", 90, sv.SV_EINVAL),
    ("tokens", None, sv.SV_EINVAL), ("token_stride", 3, sv.SV_EINVAL), ("token_counts", 4104, sv.SV_EALIGN), ("count_stride", 100, sv.SV_EALIGN),
    ("max_tokens", 0, sv.SV_OK)])
def test_counts_refusals(field, value, status):
    p = sv.TokenCountsParams()
    p.token_counts = p.tokens = 4096
    p.count_stride, p.vocab, p.batch, p.token_stride, p.max_tokens = 104, 100, 2, 4, 4
    setattr(p, field, value)
    assert sv.load().spec_token_counts_update(C.byref(p), None) == status
    assert sv.load().spec_token_counts_update(None, None) == sv.SV_EINVAL


@pytest.mark.gpu
def test_binding_refusals():
    c = make_case(3, 100, 2, 1, bias=4, mask=True)
    x = logits_of(c)
    args, kw = gpu_args(c)
    g, cq, cd, gm, tk = args
    good = dict(logits=x, out=torch.zeros_like(x), gamma=g, cu_q=cq, cu_d=cd, gamma_max=gm, draft_tokens=tk, **kw)
    for bad in (dict(out=x[:, :50]), dict(out=torch.zeros_like(x).double()), dict(gamma=g[:2]), dict(cu_q=cq[:3]), dict(repetition=kw["repetition"][:1]),
                dict(token_counts=kw["token_counts"][:, :96]), dict(token_counts=kw["token_counts"].int()), dict(bias_values=kw["bias_values"][:, :2]),
                dict(mask=kw["mask"][:, :3]), dict(mask=kw["mask"][:1]), dict(logits=x.t()), dict(logits=x.half()), dict(active=g[:1]), dict(n_drafted=g[:2]),
                dict(logits=x.cpu())):
        with pytest.raises(ValueError):
            sv.spec_logits_adjust(**{**good, **bad})
    with pytest.raises(ValueError):
        sv.spec_token_counts_update(kw["token_counts"], 200)
    with pytest.raises(ValueError):
        sv.spec_token_counts_update(kw["token_counts"], 100, tk.reshape(1, -1))
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ against the oracle
SHAPES = [(1, 1, 0), (1, 7, 3), (2, 100, 64), (3, 1003, 5), (5, 4096, 16), (4, 4100, 4), (2, 32000, 8), (9, 2049, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,V,gmax", SHAPES)
def test_everything_together(B, V, gmax, bf16):
    for draft in (False, True):
        for inplace in (False, True):
            c = make_case(B, V, gmax, 1, bf16=bf16, bias=12, mask=True, draft=draft, pad_rows=0 if draft else 3)
            got, status = run(c, inplace)
            assert status == 0
            check(c, got, inplace)


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("penal,bias,mask", [(True, 0, False), (False, 5, False), (False, 0, True), (True, 5, False), (True, 0, True), (False, 5, True), (False, 0, False)])
def test_each_part_alone(penal, bias, mask, bf16):
    for draft in (False, True):
        for inplace in (False, True):
            c = make_case(6, 5003, 7, 2, bf16=bf16, penal=penal, bias=bias, mask=mask, draft=draft)
            got, status = run(c, inplace)
            assert status == 0
            check(c, got, inplace)
    for which in ("r", "f", "p", "rf", "rp", "fp"):
        if penal:
            c = make_case(3, 1030, 7, 3, bf16=bf16, bias=bias, mask=mask, which=which)
            got, _ = run(c)
            check(c, got)


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V,stride", [(1000, 1008), (1001, 1024), (1000, 1003), (999, 1001)])
def test_strides_and_alignments(V, stride, bf16):
    for inplace in (False, True):
        c = make_case(3, V, 5, 4, bf16=bf16, bias=6, mask=True, stride=stride)
        got, status = run(c, inplace)
        assert status == 0
        check(c, got, inplace)


@pytest.mark.gpu
def test_a_draft_that_repeats_and_saturated_counts():
    c = make_case(2, 300, 16, 5, gamma=[16, 9])
    c["tokens"][:] = 123
    c["kw"]["counts"][0, 123], c["kw"]["counts"][1, 123] = 32767, -1
    got, status = run(c)
    assert status == 0
    check(c, got)


@pytest.mark.gpu
def test_infinities_and_nan():
    c = make_case(1, 64, 3, 6, mask=True, bias=3, gamma=[3])
    c["x"][:, 0:4] = [np.inf, -np.inf, np.nan, 0.0]
    c["kw"]["mask"][:] = 0xffffffff
    c["kw"]["mask"][1, 0] = 0xfffffff0                  # the special ones masked in one row
    c["kw"]["counts"][0, :4] = [2, 1, 1, 1]
    c["kw"]["bias_tokens"][:], c["kw"]["bias_values"][:], c["kw"]["n_bias"][:] = [[9, 10, 11]], [[-np.inf, np.inf, 1.0]], 3
    got, status = run(c)
    ref, _ = oracle.logits_adjust(c["x"], c["gamma"], c["cu_q"], c["cu_d"], None, c["tokens"], **c["kw"])
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref))
    assert (got[1, :4] == -np.inf).all()
    special = ~np.isfinite(ref) & ~np.isnan(ref)
    np.testing.assert_array_equal(got[special], ref[special])
    assert (got[:, 9] == -np.inf).all() and (got[:, 10] == np.inf).all()


@pytest.mark.gpu
def test_a_bias_list_that_names_a_token_twice():
    c = make_case(2, 700, 2, 7, penal=False, bias=8)
    c["kw"]["bias_tokens"][:] = [[5, 5, 600, 5, 7, 600, 5, 8]] * 2
    c["kw"]["n_bias"][:] = [8, 4]
    for _ in range(3):
        got, status = run(c)
        assert status == 0
        check(c, got)


@pytest.mark.gpu
@pytest.mark.parametrize("draft", [False, True])
def test_inactive_sequences_are_left(draft):
    c = make_case(4, 515, 3, 8, mask=True, draft=draft)
    for inplace in (False, True):
        got, status = run(c, inplace, active=dev(np.array([1, 0, 5, 0], np.int32)))
        assert status == 0
        check(c, got, inplace, skipped=(1, 3))


@pytest.mark.gpu
def test_bad_inputs_are_reported_and_do_not_spread():
    c = make_case(4, 512, 3, 9, bias=4, gamma=[2, 3, 1, 2])
    good = run(c)[0]
    bad = {**c, "kw": {k: v.copy() for k, v in c["kw"].items()}, "tokens": c["tokens"].copy(), "gamma": c["gamma"].copy()}
    bad["tokens"][c["cu_d"][1]] = 512
    bad["kw"]["bias_tokens"][0, 0], bad["kw"]["n_bias"][0] = -4, 2
    got, status = run(bad)
    assert status == sv.SV_DEV_BAD_TOKEN
    rows = slice(c["cu_q"][2], c["cu_q"][4])
    np.testing.assert_array_equal(got[rows], good[rows])
    check(bad, got)                                     # the oracle leaves such tokens out
    bad = {**c, "gamma": c["gamma"].copy()}
    bad["gamma"][3] = 70
    got, status = run(bad)                              # clamped to gamma_max = 3: one row more than the buffer has
    assert status == sv.SV_DEV_BAD_GAMMA | sv.SV_DEV_BAD_LEN
    np.testing.assert_array_equal(got[:c["cu_q"][3]], good[:c["cu_q"][3]])
    assert (got[c["cu_q"][3]:] == FILL).all()
    bad = {**c, "kw": {**c["kw"], "n_bias": np.array([0, 99, 1, -1], np.int32)}}
    got, status = run(bad)
    assert status == sv.SV_DEV_BAD_LEN
    check({**c, "kw": {**c["kw"], "n_bias": np.array([0, 4, 1, 0], np.int32)}}, got)
    bad = {**c, "tokens": c["tokens"][:5]}              # the last sequence's drafts are not there
    assert run(bad)[1] == sv.SV_DEV_BAD_LEN


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets():
    """Row stride that takes the last rows past 2^31 elements (bf16), one sequence."""
    V, stride = 1024, (1 << 30) + 4096
    c = make_case(1, V, 2, 10, bf16=True, mask=True, bias=3, gamma=[2], stride=V)
    flat = torch.zeros(2 * stride + V, dtype=torch.bfloat16, device=DEV)
    x = flat.as_strided((3, V), (stride, 1))
    x.copy_(dev(c["x"]))
    args, kw = gpu_args(c)
    sv.spec_logits_adjust(x, x, *args, **kw)
    torch.cuda.synchronize()
    check(c, x.float().cpu().numpy().astype(np.float64), True)


# ------------------------------------------------------------------------------------------------ counts
def counts_both(counts, V, tokens, first, n, d_tokens, reset=None, prompt=False, cu=None, most=None, stream=None):
    d = dev(counts)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    sv.spec_token_counts_update(d, V, d_tokens, dev(np.asarray(cu, np.int32)) if cu is not None else None, most, dev(np.asarray(reset, np.int32)) if reset is not None else None,
                                prompt, status, stream)
    torch.cuda.synchronize()
    ref = oracle.token_counts_update(counts, V, tokens, first, n, reset, prompt)
    np.testing.assert_array_equal(d.cpu().numpy(), ref)
    return ref, int(status.item())


@pytest.mark.gpu
@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("with_reset", [False, True])
@pytest.mark.parametrize("B,V,W", [(1, 1, 1), (3, 1001, 17), (128, 32000, 17), (2, 70001, 65), (5, 50257, 3000), (1, 128256, 8192)])
def test_counts_padded_and_packed(B, V, W, prompt, with_reset):
    rng = np.random.default_rng([B, V, W])
    cs = (V + 7) // 8 * 8 + 8
    counts = rng.integers(-32768, 32768, (B, cs)).astype(np.int16)
    tokens = np.minimum((rng.random((B, W)) ** 5 * V).astype(np.int32), V - 1)
    n = rng.integers(0, W + 1, B)
    reset = (rng.random(B) < 0.6).astype(np.int32) if with_reset else None
    padded = np.where(np.arange(W) < n[:, None], tokens, -1).astype(np.int32)
    kw = dict(reset=reset, prompt=prompt)
    ref, status = counts_both(counts, V, padded, np.arange(B) * W, [W] * B, dev(padded), **kw)
    assert status == 0
    wide = torch.full((B, W + 3), 5, dtype=torch.int32, device=DEV)          # rows of a wider buffer
    wide[:, :W] = dev(padded)
    counts_both(counts, V, padded, np.arange(B) * W, [W] * B, wide[:, :W], **kw)
    packed = np.concatenate([tokens[b, :n[b]] for b in range(B)] + [np.zeros(1, np.int32)])[:max(1, int(n.sum()))]
    cu = np.concatenate([[0], np.cumsum(n)])
    ref2, status = counts_both(counts, V, packed, cu[:-1], n, dev(packed), cu=cu, most=W, **kw)
    assert status == 0
    np.testing.assert_array_equal(ref, ref2)


@pytest.mark.gpu
def test_counts_saturate_and_neighbours_share_a_word():
    V = 40
    counts = np.zeros((3, V), np.int16)
    counts[0, 6], counts[0, 7], counts[1, 6], counts[2, 7] = 32760, 32767, -9, -1
    tokens = np.tile(np.array([6, 7], np.int32), (3, 100))
    for reset in (None, [0, 0, 0]):
        ref, status = counts_both(counts, V, tokens, [0, 200, 400], [200] * 3, dev(tokens), reset=reset)
        assert status == 0
        assert ref[0, 6] == 32767 and ref[0, 7] == 32767 and ref[1, 6] == -1 and ref[2, 7] == -1 and ref[2, 6] == 100


@pytest.mark.gpu
@pytest.mark.parametrize("prompt", [False, True])
def test_counts_prompts_of_every_alignment(prompt):
    """Short prompts from every boundary, with tokens outside the vocabulary at every place of a group of four."""
    V, top = 40000, 2 ** 31 - 1
    n = np.asarray([k for k in range(14) for _ in range(3)])
    cu = np.concatenate([[0], np.cumsum(n)])
    rng = np.random.default_rng(3)
    for odd in (0, 1):                                  # without and with what is to be reported
        flat = rng.integers(0, V, int(cu[-1])).astype(np.int32)
        flat[rng.random(flat.size) < 0.3] = V - 1
        flat[rng.random(flat.size) < 0.2] = -1
        if odd:
            flat[::5] = rng.choice([-2, V, V + 1, top, -top - 1, 32768 - 65536], flat[::5].size)
        counts = rng.integers(-32768, 32768, (n.size, V)).astype(np.int16)
        reset = (np.arange(n.size) % 4 != 0).astype(np.int32)
        for shift in range(4):
            d_tokens = torch.zeros(flat.size + 4, dtype=torch.int32, device=DEV)[shift:shift + flat.size]
            d_tokens.copy_(dev(flat))
            _, status = counts_both(counts, V, flat, cu[:-1], n, d_tokens, reset=reset, prompt=prompt, cu=cu, most=13)
            assert status == (4 if odd else 0)


@pytest.mark.gpu
def test_counts_conditions_and_reset_alone():
    V = 100
    counts = np.arange(4 * 104, dtype=np.int16).reshape(4, 104)
    tokens = np.array([[3, -2, 100, 7]] * 4, np.int32)
    ref, status = counts_both(counts, V, tokens, np.arange(4) * 4, [4] * 4, dev(tokens))
    assert status == sv.SV_DEV_BAD_TOKEN
    flat = tokens[:, 0].copy()
    for cu, n in (([0, 1, 9, 2, 3], [1, 0, 0, 1]), ([0, 4, 4, 4, 4], [0, 0, 0, 0]), ([-1, 1, 2, 3, 4], [0, 1, 1, 1])):
        _, status = counts_both(counts, V, flat, np.clip(cu[:4], 0, 3), n, dev(flat), cu=cu, most=3)
        assert status == sv.SV_DEV_BAD_LEN
    ref, status = counts_both(counts, V, flat, [0] * 4, [0] * 4, None, reset=[1, 0, 0, 1])
    assert status == 0 and (ref[[0, 3], :V] == 0).all() and (ref[0, V:] == counts[0, V:]).all()


@pytest.mark.gpu
def test_on_another_stream_and_replayed_from_a_graph():
    c = make_case(3, 1500, 4, 11, bias=4, mask=True)
    got, status = run(c, stream=torch.cuda.Stream())
    assert status == 0
    check(c, got)
    x = torch.zeros((c["n_rows"], c["V"]), device=DEV)
    out = torch.full_like(x, FILL)
    args, kw = gpu_args(c)
    kw["token_counts"] = torch.zeros_like(kw["token_counts"])
    emitted = torch.full((3, 5), -1, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_token_counts_update(kw["token_counts"], c["V"], emitted)
        sv.spec_logits_adjust(x, out, *args, **kw)
    x.copy_(dev(c["x"]))
    counts = np.zeros_like(c["kw"]["counts"])
    rng = np.random.default_rng(0)
    for step in range(3):                               # the counts of earlier replays are there
        t = rng.integers(-1, c["V"], (3, 5)).astype(np.int32)
        emitted.copy_(dev(t))
        graph.replay()
        torch.cuda.synchronize()
        counts = oracle.token_counts_update(counts, c["V"], t, [0, 5, 10], [5] * 3)
        np.testing.assert_array_equal(kw["token_counts"].cpu().numpy(), counts)
        check({**c, "kw": {**c["kw"], "counts": counts}}, out.cpu().numpy().astype(np.float64))


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("V", [1, 3, 9, 1000, 2053, 9001])
def test_logits_and_out_that_lie_differently(V, bf16):
    """Every pair of offsets from a 16-byte boundary: bases and strides of their own for logits and out."""
    c = make_case(2, V, 4, 12, bf16=bf16, bias=5, mask=True, gamma=[4, 3])
    n, dt = c["n_rows"], torch.bfloat16 if bf16 else torch.float32
    args, kw = gpu_args(c)
    for off_in, off_out, gap_in, gap_out in ((1, 0, 0, 0), (0, 3, 1, 7), (5, 2, 3, 0), (7, 7, 2, 2), (2, 5, 0, 9)):
        si, so = V + gap_in, V + gap_out
        x = torch.full((off_in + n * si + 16,), FILL, device=DEV, dtype=dt)[off_in:off_in + n * si].unflatten(0, (n, si))[:, :V]
        whole = torch.full((off_out + n * so + 16,), FILL, device=DEV, dtype=dt)
        out = whole[off_out:off_out + n * so].unflatten(0, (n, so))[:, :V]
        x.copy_(dev(c["x"]))
        sv.spec_logits_adjust(x, out, *args, **kw)
        torch.cuda.synchronize()
        check({**c, "stride": V}, out.float().cpu().numpy().astype(np.float64))
        out.fill_(FILL)
        assert bool((whole == FILL).all())              # nothing in front of, between or behind the rows
        sv.spec_logits_adjust(x, x, *args, **kw)
        torch.cuda.synchronize()
        check({**c, "stride": V}, x.float().cpu().numpy().astype(np.float64), True)


@pytest.mark.gpu
def test_a_bias_list_longer_than_a_block_takes_at_a_time():
    c = make_case(2, 6000, 2, 13, bias=2500)
    c["kw"]["n_bias"][:] = [2500, 1100]
    c["kw"]["bias_tokens"][:, 2000:2040] = c["kw"]["bias_tokens"][:, :40]      # named again by a later part
    got, status = run(c)
    assert status == 0
    check(c, got)


# Shapes that give a block several rows on 148 multiprocessors, by the 592 blocks that the rows are dealt out over: all rows of a
# sequence (the ring of four stages comes around), and two to five rows with several blocks along a sequence.
BLOCKS_OF_ROWS = [(600, 1000, 8, 1000), (600, 1001, 8, 1001), (600, 1003, 8, 1008), (100, 1000, 8, 1000), (150, 1002, 8, 1002), (220, 9001, 8, 9001), (220, 9000, 8, 9008),
                  (700, 104, 64, 104), (700, 101, 64, 101)]


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("B,V,gmax,stride", BLOCKS_OF_ROWS)
def test_blocks_of_several_rows(B, V, gmax, stride, inplace, bf16):
    """Drafts join the history from row to row, some of them twice, and one where nothing else changes an element near it."""
    for penal, bias, mask in ((True, 12, True), (True, 0, False), (False, 5, False), (False, 0, True)):
        c = make_case(B, V, gmax, 14, bf16=bf16, penal=penal, bias=bias, mask=mask, pad_rows=3, stride=stride)
        far = V - 3                                     # in the last unit or next to it, with neighbours that nothing touches
        for b in range(B):
            lo, hi = c["cu_d"][b], c["cu_d"][b + 1]
            if hi - lo >= 2:
                c["tokens"][hi - 2] = far if b % 2 else c["tokens"][lo]
        if penal:
            c["kw"]["counts"][:, V - 16:V] = 0
        if bias:
            c["kw"]["bias_tokens"] %= V - 16
        got, status = run(c, inplace)
        assert status == 0
        check(c, got, inplace)
