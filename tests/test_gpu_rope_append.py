"""spec_rope_append against the oracle: queries, and the pools whole, so that a write to a wrong place is caught too."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

import oracle
from paper_2504_00030_b200 import binding as sv
from paper_2504_00030_b200 import synth
from tests.harness import DEV, bits_of, dev, dev_bf16

# float32 error of an element next to the pair it comes from: the sum of D <= 128 squares (relative at most 2^-24 * (16 + 4)
# in its lane-and-tree order), its root and the products with root and weight (2^-21 for rsqrt's two ulps and three products), the
# angle below half a turn rounded once (pi * 2^-24) and sine and cosine (two ulps): together below 2^-19.
F32 = 2.0 ** -19


def make_case(n, hq, hkv, D, rot, seed, norm="both", w32=False, interleaved=False, axes=1, far=5000, pad=0.0, scale=1.0, eps=1e-6, x_scale=1.5):
    rng = np.random.default_rng([seed, n, hq, D])
    c = dict(n=n, hq=hq, hkv=hkv, D=D, interleaved=interleaved, scale=scale, eps=eps)
    c["qkv"] = synth.bf16_bits((rng.standard_normal((n, (hq + 2 * hkv) * D)) * x_scale).astype(np.float32))
    c["inv"] = 10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))
    c["pos"] = rng.integers(0, far, (axes, n) if axes > 1 else n).astype(np.int32)
    c["axis"] = rng.integers(0, axes, rot // 2).astype(np.uint8) if axes > 1 else None
    w = lambda: (lambda v: v if w32 else synth.bf16_to_f32(synth.bf16_bits(v)))(rng.uniform(0.5, 1.5, D).astype(np.float32))  # noqa: E731
    c["qw"] = w() if norm in ("both", "q") else None
    c["kw"] = w() if norm in ("both", "k") else None
    c["w32"] = w32
    c["n_pages"] = (n + 15) // 16 + 3
    c["slots"] = rng.permutation(c["n_pages"] * 16)[:n].astype(np.int64)
    c["slots"][rng.random(n) < pad] = -1
    c["pool_k"], c["pool_v"] = (synth.bf16_bits(rng.standard_normal((c["n_pages"], hkv, 16, D)).astype(np.float32)) for _ in range(2))
    return c


def views(t, c):
    hq, hkv, D = c["hq"], c["hkv"], c["D"]
    return (x.unflatten(1, (-1, D)) for x in t.split([hq * D, hkv * D, hkv * D], 1))


def call(c, qkv=None, pools=None, q_out=None, stream=None, status=None):
    qkv = dev_bf16(c["qkv"]) if qkv is None else qkv
    q, k, v = views(qkv, c)
    kp, vp = pools if pools is not None else (dev_bf16(c["pool_k"]), dev_bf16(c["pool_v"]))
    pool = sv.spec_kv_pool_register(kp, vp)
    q_out = dev_bf16(np.full((c["n"], c["hq"], c["D"]), 0x4242, np.uint16)) if q_out is None else q_out
    w = lambda x: None if x is None else dev(x) if c["w32"] else dev(x).to(torch.bfloat16)  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
    sv.spec_rope_append(q, k, v, q_out, pool, dev(c["pos"]), dev(c["slots"]), dev(c["inv"]) if len(c["inv"]) else None, w(c["qw"]), w(c["kw"]), c["eps"],
                        c["interleaved"], dev(c["axis"]) if c["axis"] is not None else None, c["scale"], status, stream)
    torch.cuda.synchronize()
    return q_out, kp, vp, int(status.item())


def near(got_bits, z, mag):
    got = synth.bf16_to_f32(got_bits).astype(np.float64)
    err = np.abs(got - z)
    # one rounding to bf16 (2^-8 of the value, or half the smallest subnormal step) of a float32 result
    allowed = np.abs(z) * 2.0 ** -8 + mag * F32 * (1 + 2.0 ** -8) + 2.0 ** -134
    assert (err <= allowed).all(), float((err / np.maximum(allowed, 1e-300)).max())


def check(c, out):
    q_out, kp, vp, status = out
    hq, hkv, D = c["hq"], c["hkv"], c["D"]
    q, k, v = np.split(c["qkv"].reshape(c["n"], -1, D), [hq, hq + hkv], 1)
    args = (c["pos"], c["inv"])
    kw = dict(eps=c["eps"], interleaved=c["interleaved"], freq_axis=c["axis"], scale=c["scale"])
    used = (c["slots"] >= 0) & (c["slots"] < c["n_pages"] * 16)
    got = bits_of(q_out)
    near(got[used], *(a[used] for a in oracle.norm_rotate(q, *args, weight=c["qw"], **kw)))
    assert (got[~used] == 0x4242).all()
    page, at = c["slots"][used] // 16, c["slots"][used] % 16
    kb, vb = bits_of(kp), bits_of(vp)
    near(kb[page, :, at], *(a[used] for a in oracle.norm_rotate(k, *args, weight=c["kw"], **kw)))
    np.testing.assert_array_equal(vb[page, :, at], v[used])
    touched = np.zeros((c["n_pages"], 16), bool)
    touched[page, at] = True
    np.testing.assert_array_equal(kb.transpose(0, 2, 1, 3)[~touched], c["pool_k"].transpose(0, 2, 1, 3)[~touched])
    np.testing.assert_array_equal(vb.transpose(0, 2, 1, 3)[~touched], c["pool_v"].transpose(0, 2, 1, 3)[~touched])
    return status


# ------------------------------------------------------------------------------------------------ refusals (no device needed)
def good_params(pool):
    p = sv.RopeAppendParams()
    p.q, p.k_new, p.v_new, p.q_out, p.slot_map, p.positions, p.inv_freq = (4096 * 16 * (i + 1) for i in range(7))
    p.pool, p.hq, p.n_rows, p.n_axes, p.rot_dim, p.rope_scale, p.eps = pool, 2, 3, 1, 64, 1.0, 1e-6
    p.q_stride, p.k_stride, p.v_stride = 128, 64, 64
    return p


def host_pool(D=64, hkv=1):
    """A pool handle over addresses that nothing reads; head_dim 64 / 128 need the driver's tensor maps."""
    h = C.c_void_p()
    st = (C.c_int64 * 4)(hkv * 16 * D, 16 * D, D, 1)
    assert sv.load().spec_kv_pool_register(1 << 20, 1 << 21, 4, 16, hkv, D, st, C.byref(h)) == sv.SV_OK
    return h


@pytest.mark.parametrize("field,value,status", [
    ("pool", None, sv.SV_EINVAL), ("q", None, sv.SV_EINVAL), ("k_new", None, sv.SV_EINVAL), ("v_new", None, sv.SV_EINVAL), ("q_out", None, sv.SV_EINVAL),
    ("slot_map", None, sv.SV_EINVAL), ("positions", None, sv.SV_EINVAL), ("inv_freq", None, sv.SV_EINVAL), ("hq", 0, sv.SV_EINVAL), ("n_rows", -1, sv.SV_EINVAL),
    ("n_axes", 0, sv.SV_EINVAL), ("rot_dim", -16, sv.SV_EINVAL), ("rot_dim", 112, sv.SV_EINVAL), ("eps", -1.0, sv.SV_EINVAL), ("eps", float("nan"), sv.SV_EINVAL),
    ("q_stride", 80, sv.SV_EINVAL), ("k_stride", 40, sv.SV_EINVAL), ("v_stride", 0, sv.SV_EINVAL), ("rot_dim", 24, sv.SV_EUNSUPPORTED),
    ("n_rows", 1 << 31, sv.SV_EUNSUPPORTED), ("q", 4096 * 16 + 8, sv.SV_EALIGN), ("q_weight", 4100, sv.SV_EALIGN), ("k_weight", 4100, sv.SV_EALIGN),
    ("q_stride", 196, sv.SV_EALIGN), ("k_stride", 100, sv.SV_EALIGN), ("v_stride", 100, sv.SV_EALIGN), ("q_out", 4096 * 16 + 64, sv.SV_EINVAL),
    ("q_out", 4096 * 32 + 128, sv.SV_EINVAL), ("q_out", 4096 * 48 - 256, sv.SV_EINVAL)])
def test_refused_before_any_launch(field, value, status):
    pool = host_pool(96)
    p = good_params(pool)
    p.rot_dim, p.q_stride, p.k_stride, p.v_stride = 96, 192, 96, 96
    setattr(p, field, value)
    assert sv.load().spec_rope_append(C.byref(p), None) == status
    assert sv.load().spec_rope_append(None, None) == sv.SV_EINVAL
    sv.load().spec_kv_pool_release(pool)


def test_odd_head_dim_is_refused_and_no_rows_is_nothing():
    pool = host_pool(40)
    p = good_params(pool)
    p.rot_dim = 16
    assert sv.load().spec_rope_append(C.byref(p), None) == sv.SV_EUNSUPPORTED
    sv.load().spec_kv_pool_release(pool)
    pool = host_pool(96)
    p = good_params(pool)
    p.q_stride, p.k_stride, p.v_stride, p.n_rows, p.q = 192, 96, 96, 0, None
    assert sv.load().spec_rope_append(C.byref(p), None) == sv.SV_OK
    sv.load().spec_kv_pool_release(pool)


@pytest.mark.gpu
def test_binding_refusals():
    c = make_case(4, 2, 1, 64, 64, 1)
    qkv = dev_bf16(c["qkv"])
    q, k, v = views(qkv, c)
    pool = sv.spec_kv_pool_register(dev_bf16(c["pool_k"]), dev_bf16(c["pool_v"]))
    good = dict(q=q, k_new=k, v_new=v, q_out=torch.zeros_like(q).contiguous(), pool=pool, positions=dev(c["pos"]), slot_map=dev(c["slots"]), inv_freq=dev(c["inv"]))
    for bad in (dict(q=q[:3]), dict(k_new=k[:, :, :32]), dict(v_new=v.float()), dict(q_out=good["q_out"][:2]), dict(positions=dev(c["pos"][:3])),
                dict(slot_map=dev(c["slots"]).int()), dict(inv_freq=dev(c["inv"]).float()), dict(freq_axis=torch.zeros(5, dtype=torch.uint8, device=DEV)),
                dict(q_weight=torch.zeros(32, dtype=torch.bfloat16, device=DEV)), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(q=q.cpu()),
                dict(q_weight=torch.ones(64, device=DEV), k_weight=torch.ones(64, dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(ValueError):
            sv.spec_rope_append(**{**good, **bad})
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ against the oracle
@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 17, 300])
@pytest.mark.parametrize("hq,hkv,D,rot", [(12, 12, 64, 64), (32, 8, 128, 128), (64, 8, 128, 128), (7, 1, 96, 96), (5, 5, 80, 48), (3, 1, 16, 16), (4, 2, 48, 32),
                                          (1, 1, 112, 16), (6, 2, 128, 0)])
def test_shapes(n, hq, hkv, D, rot):
    c = make_case(n, hq, hkv, D, rot, 1, pad=0.2 if n > 2 else 0.0)
    assert check(c, call(c)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,hq,hkv,D,rot", [(4800, 1, 1, 128, 128), (4801, 1, 1, 112, 64), (5002, 4, 1, 64, 64), (5007, 2, 1, 48, 16), (16381, 8, 1, 128, 128),
                                            (9001, 1, 2, 16, 16), (16380, 16, 4, 64, 48), (7003, 3, 1, 80, 0)])
def test_many_rows_of_few_heads(n, hq, hkv, D, rot):
    """Enough rows to fill the GPU several times over, so that a warp takes more than one; whole groups of them are padding."""
    for k in range(4):
        c = make_case(n, hq, hkv, D, rot, 5 + k, norm=("both", "none", "q", "k")[k], w32=k == 3, interleaved=k % 2 == 1, axes=1 + k, far=70000,
                      pad=(0.0, 0.9, 0.3, 0.02)[k], scale=1.0 - 0.1 * k)
        c["slots"][n // 2:n // 2 + 40] = -1
        if k == 2:
            c["slots"][n - 1] = c["n_pages"] * 16
        assert check(c, call(c)) == (sv.SV_DEV_BAD_PAGE if k == 2 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["none", "q", "k", "both"])
@pytest.mark.parametrize("w32", [False, True])
def test_norms_and_pairings(interleaved, norm, w32):
    for D, rot in ((128, 128), (128, 64), (64, 32), (96, 80)):
        c = make_case(23, 6, 3, D, rot, 2, norm=norm, w32=w32, interleaved=interleaved, eps=1e-5, scale=1.1)
        assert check(c, call(c)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("far", [2, 131072, 1 << 24, 2 ** 31 - 1])
def test_far_positions_and_axes(far):
    for axes in (1, 3, 4):
        c = make_case(65, 4, 2, 128, 128, 3, axes=axes, far=far, interleaved=axes == 3)
        assert check(c, call(c)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("x_scale,eps", [(0.0, 1e-6), (1e-18, 1e-6), (1e18, 1e-6), (3e-3, 0.0)])
def test_extreme_magnitudes(x_scale, eps):
    c = make_case(9, 4, 2, 128, 128, 4, x_scale=x_scale, eps=eps)
    assert check(c, call(c)) == 0


@pytest.mark.gpu
def test_an_axis_beyond_the_last_is_the_last():
    c = make_case(12, 4, 2, 64, 64, 5, axes=2)
    c["axis"][:] = 200
    out = call(c)
    c["axis"][:] = 1
    assert check(c, out) == 0


@pytest.mark.gpu
def test_bad_slots_are_skipped():
    c = make_case(40, 4, 2, 64, 64, 6)
    c["slots"][3], c["slots"][17], c["slots"][20] = c["n_pages"] * 16, 1 << 40, -(1 << 40)
    assert check(c, call(c)) == sv.SV_DEV_BAD_PAGE


@pytest.mark.gpu
def test_in_place_contiguous_heads_and_a_slot_major_pool():
    c = make_case(50, 8, 4, 128, 128, 7)
    D = 128
    q, k, v = (x.contiguous() for x in views(dev_bf16(c["qkv"]), c))
    kp, vp = (dev_bf16(np.ascontiguousarray(c[x].transpose(0, 2, 1, 3))).permute(0, 2, 1, 3) for x in ("pool_k", "pool_v"))
    pool = sv.spec_kv_pool_register(kp, vp)
    sv.spec_rope_append(q, k, v, q, pool, dev(c["pos"]), dev(c["slots"]), dev(c["inv"]), dev(c["qw"]).to(torch.bfloat16), dev(c["kw"]).to(torch.bfloat16), c["eps"])
    torch.cuda.synchronize()
    assert check(c, (q, kp, vp, 0)) == 0
    assert D == c["D"]


@pytest.mark.gpu
def test_overlapping_output_is_refused():
    c = make_case(5, 4, 1, 64, 64, 8)
    buf = torch.zeros((6, 4, 64), dtype=torch.bfloat16, device=DEV)
    k = torch.zeros((5, 1, 64), dtype=torch.bfloat16, device=DEV)
    pool = sv.spec_kv_pool_register(dev_bf16(c["pool_k"]), dev_bf16(c["pool_v"]))
    with pytest.raises(sv.SpecVerifyError):
        sv.spec_rope_append(buf[:5], k, k, buf[1:], pool, dev(c["pos"]), dev(c["slots"]), dev(c["inv"]))
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """A pool of more than 2^31 elements and a row stride that takes the last row past 2^31 elements."""
    c = make_case(3, 2, 1, 128, 128, 9)
    n_pages = (1 << 31) // (16 * 128) + 40
    kp, vp = (torch.zeros((n_pages, 1, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    c["slots"] = np.array([5, n_pages * 16 - 1, (n_pages - 20) * 16 + 3], np.int64)
    wide = (1 << 30) + 4096 * 8
    flat = torch.zeros(2 * wide + 4 * 128, dtype=torch.bfloat16, device=DEV)
    rows = flat.as_strided((3, 4 * 128), (wide, 1))
    rows.copy_(dev_bf16(c["qkv"]))
    q, k, v = views(rows, c)
    pool = sv.spec_kv_pool_register(kp, vp)
    q_out = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=DEV)
    sv.spec_rope_append(q, k, v, q_out, pool, dev(c["pos"]), dev(c["slots"]), dev(c["inv"]), dev(c["qw"]).to(torch.bfloat16), dev(c["kw"]).to(torch.bfloat16), c["eps"])
    torch.cuda.synchronize()
    args, kw = (c["pos"], c["inv"]), dict(eps=c["eps"])
    bq, bk, bv = np.split(c["qkv"].reshape(3, -1, 128), [2, 3], 1)
    near(bits_of(q_out), *oracle.norm_rotate(bq, *args, weight=c["qw"], **kw))
    at = torch.from_numpy(c["slots"]).to(DEV)
    near(bits_of(kp[at // 16, :, at % 16]), *oracle.norm_rotate(bk, *args, weight=c["kw"], **kw))
    np.testing.assert_array_equal(bits_of(vp[at // 16, :, at % 16]), bv)
    assert int(torch.count_nonzero(vp.view(torch.int16))) == np.count_nonzero(bv)


@pytest.mark.gpu
def test_on_another_stream_and_replayed_from_a_graph():
    c = make_case(33, 8, 2, 128, 128, 10, pad=0.3)
    side = torch.cuda.Stream()
    assert check(c, call(c, stream=side)) == 0
    qkv, kp, vp = torch.zeros((33, 12 * 128), dtype=torch.bfloat16, device=DEV), dev_bf16(c["pool_k"]), dev_bf16(c["pool_v"])
    q, k, v = views(qkv, c)
    pool = sv.spec_kv_pool_register(kp, vp)
    q_out = dev_bf16(np.full((33, 8, 128), 0x4242, np.uint16))
    pos, slots, inv, qw, kw = dev(c["pos"]), dev(c["slots"]), dev(c["inv"]), dev(c["qw"]).to(torch.bfloat16), dev(c["kw"]).to(torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sv.spec_rope_append(q, k, v, q_out, pool, pos, slots, inv, qw, kw, c["eps"])
    qkv.copy_(dev_bf16(c["qkv"]))
    graph.replay()
    torch.cuda.synchronize()
    assert check(c, (q_out, kp, vp, 0)) == 0


@pytest.mark.gpu
def test_no_rows_is_nothing():
    c = make_case(16, 4, 2, 64, 64, 11)
    pool = sv.spec_kv_pool_register(dev_bf16(c["pool_k"]), dev_bf16(c["pool_v"]))
    q, k, v = views(dev_bf16(c["qkv"]), c)
    before = sv.sv_launch_count()
    sv.spec_rope_append(q[:0], k[:0], v[:0], torch.zeros((0, 4, 64), dtype=torch.bfloat16, device=DEV), pool, dev(c["pos"])[:0], dev(c["slots"])[:0], dev(c["inv"]))
    assert sv.sv_launch_count() == before


@pytest.mark.gpu
@pytest.mark.parametrize("n,hq,hkv,D,rot", [(2300, 32, 8, 128, 128), (2400, 32, 8, 128, 64), (2300, 64, 8, 64, 64), (4700, 33, 5, 96, 96), (3000, 24, 24, 96, 48),
                                            (2350, 36, 12, 48, 32), (2368, 40, 9, 64, 16), (1200, 64, 8, 128, 128), (4700, 20, 6, 80, 80)])
def test_many_rows_of_many_heads(n, hq, hkv, D, rot):
    """Enough rows that a warp takes 6 to 13 rounds of one, from queries on to keys and to values, the last of each kind a part of a
    round: on 148 multiprocessors the ring of copies comes around more than once."""
    for k in range(2):
        c = make_case(n, hq, hkv, D, rot, 9 + k, norm=("both", "k")[k], w32=k == 1, interleaved=k == 1, axes=1 + 2 * k, far=70000, pad=(0.0, 0.2)[k],
                      scale=1.0 - 0.1 * k)
        c["slots"][n // 2:n // 2 + 20] = -1
        assert check(c, call(c)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n,hq,hkv,D,rot", [(2300, 32, 8, 128, 128), (4700, 33, 5, 96, 64), (5002, 4, 1, 64, 64), (16381, 8, 1, 128, 128)])
def test_in_place_where_copies_run_ahead_of_the_stores(n, hq, hkv, D, rot):
    """Many rounds a warp, and several rows a warp, with the queries turned where they are: padding rows stay as they were."""
    c = make_case(n, hq, hkv, D, rot, 12, pad=0.1, interleaved=hq == 33)
    q, k, v = (x.contiguous() for x in views(dev_bf16(c["qkv"]), c))
    kp, vp = dev_bf16(c["pool_k"]), dev_bf16(c["pool_v"])
    w = [dev(c[x]).to(torch.bfloat16) for x in ("qw", "kw")]
    sv.spec_rope_append(q, k, v, q, sv.spec_kv_pool_register(kp, vp), dev(c["pos"]), dev(c["slots"]), dev(c["inv"]), *w, c["eps"], c["interleaved"])
    torch.cuda.synchronize()
    padding = c["slots"] < 0
    np.testing.assert_array_equal(bits_of(q)[padding], c["qkv"].reshape(n, -1, D)[padding, :hq])
    q[dev(padding)] = dev_bf16(np.full((1, hq, D), 0x4242, np.uint16))       # what check expects of rows that are left alone
    assert check(c, (q, kp, vp, 0)) == 0


@pytest.mark.parametrize("k_at,v_at", [(0, 0), (-1, 0), (0, -1)])
def test_binding_refuses_a_pool_of_another_device(k_at, v_at):
    """Host tensors (device index -1) stand for those of the current device: the pool's memory lies on another one."""
    c = make_case(4, 2, 1, 64, 64, 1)
    q, k, v = views(torch.from_numpy(c["qkv"].view(np.int16)).view(torch.bfloat16), c)
    at = lambda i: types.SimpleNamespace(get_device=lambda: i)  # noqa: E731
    pool = types.SimpleNamespace(hkv=1, head_dim=64, handle=C.c_void_p(4096), k_pool=at(-1), v_pool=at(-1))
    args = (-1, q, k, v, torch.zeros_like(q).contiguous(), pool, torch.from_numpy(c["pos"]), torch.from_numpy(c["slots"]), torch.from_numpy(c["inv"]))
    assert 4096 in sv._rope_append_args(*args)
    pool.k_pool, pool.v_pool = at(k_at), at(v_at)
    with pytest.raises(ValueError, match="pool"):
        sv._rope_append_args(*args)


def test_binding_refuses_a_released_pool():
    c = make_case(4, 2, 1, 64, 64, 1)
    q, k, v = views(torch.from_numpy(c["qkv"].view(np.int16)).view(torch.bfloat16), c)
    here = types.SimpleNamespace(get_device=lambda: -1)
    pool = types.SimpleNamespace(hkv=1, head_dim=64, handle=None, k_pool=here, v_pool=here)
    with pytest.raises(ValueError, match="pool"):
        sv._rope_append_args(-1, q, k, v, torch.zeros_like(q).contiguous(), pool, torch.from_numpy(c["pos"]), torch.from_numpy(c["slots"]), torch.from_numpy(c["inv"]))


@pytest.mark.parametrize("hq,hkv", [((1 << 20) + 1, 1), (1 << 28, 1), (2, (1 << 20) + 1)])
def test_more_heads_than_32_bit_offsets_reach_are_refused(hq, hkv):
    """Offsets of a head within its row are kept in 32 bits.  (Nothing lies behind these addresses, and nothing is launched.)"""
    pool = host_pool(96, hkv)
    p = good_params(pool)
    p.q, p.k_new, p.v_new, p.q_out = ((i + 1) << 50 for i in range(4))
    p.rot_dim, p.hq, p.q_stride, p.k_stride, p.v_stride = 96, hq, hq * 96, hkv * 96, hkv * 96
    assert sv.load().spec_rope_append(C.byref(p), None) == sv.SV_EUNSUPPORTED
    sv.load().spec_kv_pool_release(pool)
