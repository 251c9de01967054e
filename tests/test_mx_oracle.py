"""The plain microscaled reference against facts of the format (CPU)."""
import numpy as np
import pytest

from oracle import microscaled as mx


def test_every_code_under_every_scale_comes_back():
    for byte in range(2, 253):
        n = np.tile(np.arange(16, dtype=np.uint8), 2)[None]
        n[n == 8] = 0
        v = mx.decode(n, np.array([[byte]], dtype=np.uint8))
        code, scale = mx.encode(v.astype(np.float32))
        assert scale[0, 0] == byte and np.array_equal(code, n)


@pytest.mark.parametrize("value,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.0, 7), (7.99, 7),
                                        (0.2500001, 1), (0.7499999, 1), (4.9999995, 6), (5.0000005, 7), (-5.0, 14), (-0.25, 0)])
def test_ties_go_to_the_even_code_and_large_values_saturate(value, code):
    u = np.full((1, 32), 4.0, dtype=np.float32)  # the block's scale is 1
    u[0, 5] = value
    got, scale = mx.encode(u)
    assert scale[0, 0] == 127 and got[0, 5] == code and got[0, 4] == 6


def test_error_of_a_rounding_is_half_a_step():
    u = np.random.default_rng(0).standard_normal((64, 512)).astype(np.float32)
    n, s = mx.encode(u)
    v, unit = mx.decode(n, s), np.repeat(np.exp2(s.astype(np.float64) - 127), 32, axis=1)
    a = np.abs(u) / unit
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert np.all(np.abs(v - u) <= unit * np.where(a <= 6, step / 2, 2.0))


def test_layouts_invert():
    r = np.random.default_rng(1)
    n = r.integers(0, 16, (48, 384)).astype(np.uint8)
    n[n == 8] = 0
    assert np.array_equal(mx.split_nibbles(mx.pack_nibbles(n)), n)
    s = r.integers(0, 255, (48, 12)).astype(np.uint8)
    assert np.array_equal(mx.rows(mx.steps(s)), s)
    t = mx.tiles(mx.pack_nibbles(n))
    assert t[1, 2, 3, 5, 7] == mx.pack_nibbles(n)[16 + 5, 64 * 2 + 16 * 3 + 7]


def test_rotation_is_the_hadamard_matrix():
    from scipy.linalg import hadamard
    x = np.random.default_rng(2).standard_normal((3, 512)).astype(np.float32)
    for b in (1, 2, 32, 256):
        want = (x.reshape(-1, b).astype(np.float64) @ hadamard(b)) / np.sqrt(b)
        # log2 b additions and one product of half a step each, of at most the largest partial sum
        assert np.allclose(mx.fold(x, b).reshape(-1, b), want, atol=2.0 ** -24 * 10 * np.abs(x).max() * np.sqrt(b), rtol=0)
