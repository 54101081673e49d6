"""The definitions in oracle/paged.py against things known by other means."""
import math

import numpy as np

from oracle import mx, paged


def test_angles_of_far_positions():
    # sin and cos of whole numbers of radians, reduced here by hand with 2 pi to 50 digits: 10^9 radians.
    a = paged.angle(1.0, 10 ** 9)
    turns = 10 ** 9 / (2 * math.pi)
    assert abs(a - 2 * math.pi * (turns - math.floor(turns))) < 1e-5
    assert abs(math.sin(a) - 0.545843449448699) < 1e-9   # sin(10^9)
    assert paged.angle(0.5, 2) == 1.0 and paged.angle(1.0, 0) == 0.0


def test_rotation_is_one_of_complex_numbers():
    r = np.random.default_rng(0)
    x = r.standard_normal((2, 5, 64))
    pos = r.integers(-50, 50, (2, 5))
    freq, axis = r.random(8), np.array([0, 1] * 4)
    y = paged.rotate(x, pos, freq, axis)
    z = (x[..., :8] + 1j * x[..., 8:16]) * np.exp(1j * pos[axis].T * freq)
    assert np.allclose(y[..., :8], z.real) and np.allclose(y[..., 8:16], z.imag)
    assert np.array_equal(y[..., 16:], x[..., 16:])
    # Neighbouring channels: the same after the channels change places.
    order = np.concatenate([np.arange(0, 16, 2), np.arange(1, 16, 2), np.arange(16, 64)])
    w = paged.rotate(x, pos, freq, axis, adjacent=True)
    assert np.allclose(w[..., order], paged.rotate(x[..., order], pos, freq, axis))
    assert np.allclose(paged.rotate(y, -pos, freq, axis), x)


def test_places():
    pages = np.array([[3, 1, -1], [0, 9, 2]])
    got = paged.places(pages, 4, 5, start=[2, 3], m=4, count=[3, 99])
    assert got == [(0, 0, 3, 2), (0, 1, 3, 3), (0, 2, 1, 0), (1, 0, 0, 3)]   # page 9 is outside the pool
    assert paged.places(pages, 4, 5, start=[-1, 11], m=2) == [(0, 1, 3, 0), (1, 0, 2, 3)]


def test_tree_attention_of_one_sequence():
    r = np.random.default_rng(1)
    K, V = r.standard_normal((4, 1, 3, 8)), r.standard_normal((4, 1, 3, 8))
    Q, Kt, Vt = r.standard_normal((1, 2, 2, 8)), r.standard_normal((1, 1, 2, 8)), r.standard_normal((1, 1, 2, 8))
    pages = np.array([[2, 0, 1]])
    mask = np.array([[[True, False], [True, True]]])
    got = paged.tree_attention(Q, K, V, pages, 7, Kt, Vt, mask=mask)
    line = np.concatenate([K[2, 0], K[0, 0], K[1, 0, :1]]), np.concatenate([V[2, 0], V[0, 0], V[1, 0, :1]])
    for hq in range(2):
        for i in range(2):
            k, v = (np.concatenate([c, t[0, 0, :i + 1]]) for c, t in zip(line, (Kt, Vt)))
            assert np.allclose(got[0, hq, i], mx.attention(Q[0, hq, i:i + 1], k, v)[0])
    nothing = paged.tree_attention(Q, K, V, pages, 7, Kt, Vt, cache_len=[0], mask=np.zeros_like(mask))
    assert (nothing == 0).all()
