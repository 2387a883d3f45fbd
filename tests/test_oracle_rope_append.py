"""The oracle's norm and rotation against complex arithmetic in numpy and against properties of the definition."""
import numpy as np
import pytest

import oracle
from paper_2504_00030_b200 import synth


def heads(n, h, D, seed):
    return synth.bf16_bits(np.random.default_rng(seed).standard_normal((n, h, D)).astype(np.float32) * 1.5)


@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (128, 128, True), (96, 48, False), (80, 16, True), (32, 0, False)])
def test_against_complex_products(D, rot, interleaved):
    n, h = 7, 3
    x = heads(n, h, D, D + rot)
    rng = np.random.default_rng(rot)
    w = rng.uniform(0.5, 1.5, D)
    inv = 10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))
    axis = rng.integers(0, 3, rot // 2).astype(np.uint8)
    pos = rng.integers(0, 100000, (3, n)).astype(np.int32)
    z, mag = oracle.norm_rotate(x, pos, inv, w, 1e-5, interleaved, axis, 1.25)
    y = synth.bf16_to_f32(x).astype(np.float64)
    y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + 1e-5) * w
    ref = y.copy()
    a = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    b = a + 1 if interleaved else a + rot // 2
    turn = np.exp(1j * pos[axis, :].T * inv)[:, None, :]
    c = (y[..., a] + 1j * y[..., b]) * turn * 1.25
    ref[..., a], ref[..., b] = c.real, c.imag
    np.testing.assert_allclose(z, ref, rtol=0, atol=1e-11)
    assert (mag + 1e-12 >= np.abs(z)).all()


def test_position_zero_and_lengths():
    x = heads(4, 2, 64, 1)
    inv = 10000.0 ** (-np.arange(32) / 32)
    z0, _ = oracle.norm_rotate(x, np.zeros(4, np.int32), inv)
    np.testing.assert_array_equal(z0, synth.bf16_to_f32(x))                      # no weights, no angle: x itself
    z, _ = oracle.norm_rotate(x, np.array([1, 17, 4000, 2 ** 31 - 1], np.int32), inv)
    np.testing.assert_allclose(np.linalg.norm(z, axis=-1), np.linalg.norm(z0, axis=-1), rtol=1e-12)
    # the product of a query and a key turned by their positions depends on the difference alone
    q, k = heads(1, 1, 64, 2), heads(1, 1, 64, 3)
    dots = [(oracle.norm_rotate(q, np.array([p + 9], np.int32), inv)[0] * oracle.norm_rotate(k, np.array([p], np.int32), inv)[0]).sum()
            for p in (0, 5, 1000)]
    np.testing.assert_allclose(dots, dots[0], rtol=1e-9)
