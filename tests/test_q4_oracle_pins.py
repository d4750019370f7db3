"""Pins of the oracle's 4-bit format and rotation: values written out by hand, and statements that the definition implies (CPU)."""

import numpy as np

from oracle import attention_oracle as A


def block(*first):
    return np.array(list(first) + [0.0] * (16 - len(first)))


def held(x):
    return A.q4_values(*A.q4_hold(x))


def test_numbers_of_the_scale():
    assert len(A.E5M2) == 0x54 and A.E5M2[0x3C] == 1.0 and A.E5M2[0x3D] == 1.25 and A.E5M2[1] == 2.0 ** -16 and A.E5M2[4] == 2.0 ** -14
    assert (np.diff(A.E5M2) > 0).all() and A.E5M2[0x53] == 56.0
    halves = (np.arange(0x54, dtype=np.uint16) << 8).view(np.float16).astype(np.float64)
    assert np.array_equal(halves, A.E5M2)                                 # the upper half of an fp16


def test_blocks_by_hand():
    codes, scales = A.q4_hold(block(120.0, -120.0, 8.0, 24.0, 40.0, -7.9))           # S = 16
    assert scales.tolist() == [0x3C]
    assert codes[:3].tolist() == [15 | 1 << 4, 8 | 10 << 4, 10 | 8 << 4]             # 8 / 16 and 40 / 16 lie between two: the even one
    assert A.q4_hold(block(np.nextafter(120.0, 200.0)))[1].tolist() == [0x3D]        # S = 20
    assert held(block(7.49 * 16))[0] == 112.0
    assert A.q4_hold(block(0.0))[1].tolist() == [0] and (A.q4_hold(block(0.0))[0] == 0x88).all()
    assert held(block(1e5, 6272.0, -1e30))[:3].tolist() == [6272.0, 6272.0, -6272.0] and A.q4_hold(block(6721.0))[1].tolist() == [0x53]
    assert held(block(2.0 ** -13))[0] == 0 and held(block(1.01 * 2.0 ** -13))[0] == 2.0 ** -12
    for bad in (np.nan, np.inf, -np.inf):
        c, e = A.q4_hold(np.concatenate([block(1.0, bad), block(1.0)]))
        assert e[0] == 0x7F and np.isnan(held(np.concatenate([block(1.0, bad), block(1.0)]))[:16]).all() and e[1] != 0x7F


def test_error_is_half_a_step_at_most():
    x = np.random.default_rng(1).standard_normal((500, 128)) * np.exp(np.random.default_rng(2).uniform(-5, 7, (500, 1)))
    _, e = A.q4_hold(x)
    S = np.repeat(16 * A.E5M2[e], 16, axis=-1)
    top = np.abs(x).reshape(500, 8, 16).max(-1)
    assert (np.abs(held(x) - x) <= S / 2).all()
    assert (top <= 120 * A.E5M2[e]).all() and (top > 120 * A.E5M2[e - 1]).all()
    v = held(x).astype(np.float32)
    assert np.array_equal((v.view(np.uint32) & 0xFFFF), np.zeros(v.shape, np.uint32))            # exact in bf16


def test_rotation_by_hand():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    quarter = np.full((1, 2), np.pi / 2)
    assert np.allclose(A.rotate(x, quarter)[0], [[[-3, -4, 1, 2]]])
    assert np.allclose(A.rotate(x, quarter, interleaved=True)[0], [[[-2, 1, -4, 3]]])
    assert np.allclose(A.rotate(x, quarter[:, :1])[0], [[[-2, 1, 3, 4]]])
    assert np.allclose(A.rotate(x, np.zeros((1, 0)), eps=2.5, weight=[1, 1, 1, 2])[0] * np.sqrt(10.0), [[[1, 2, 3, 8]]])
