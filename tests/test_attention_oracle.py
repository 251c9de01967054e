"""The attention oracle and the rotation frequencies against brute force and their defining properties (CPU)."""
import math

import numpy as np
import pytest

from oracle import attention as ref
from tests.attention_util import make_table, native_v, plain_v


def test_attention_is_the_weighted_mean_by_loops():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 4)), rng.standard_normal((5, 4)), rng.standard_normal((5, 4))
    seen = np.array([[1, 1, 0, 0, 1], [0, 0, 0, 0, 0], [0, 1, 0, 0, 0]], dtype=bool)
    out, spread, reach = ref.attention(q, k, v, seen, 0.5)
    for r in range(3):
        w = [math.exp(0.5 * sum(q[r, d] * k[j, d] for d in range(4))) if seen[r, j] else 0.0 for j in range(5)]
        for d in range(4):
            want = sum(w[j] * v[j, d] for j in range(5)) / sum(w) if sum(w) else 0.0
            assert abs(out[r, d] - want) < 1e-14
    assert (out[1] == 0).all() and np.allclose(out[2], v[1], atol=1e-15)
    assert (spread >= np.abs(out) - 1e-15).all() and (reach >= 0).all()


def test_unseen_keys_have_no_effect():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 8)), rng.standard_normal((6, 8)), rng.standard_normal((6, 8))
    seen = np.tile([True, True, False, True, False, True], (2, 1))
    want = ref.attention(q, k, v, seen, 1.0)[0]
    k[2], v[2], k[4], v[4] = np.nan, np.inf, -np.inf, np.nan
    assert np.array_equal(ref.attention(q, k, v, seen, 1.0)[0], want)


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_keeps_norms_and_depends_on_distance(inter):
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((1, 1, 32)), rng.standard_normal((1, 1, 32))
    a = np.arange(200)[:, None] * (10000.0 ** (-np.arange(0, 32, 2) / 32))[None]
    table = np.stack([np.cos(a), np.sin(a)], axis=-1)
    r = lambda z, m: ref.norm_rotate(z, table, np.array([m]), interleaved=inter)[0, 0]  # noqa: E731
    assert abs(np.linalg.norm(r(x, 77)) - np.linalg.norm(x)) < 1e-12
    assert abs(r(x, 10) @ r(y, 4) - r(x, 150) @ r(y, 144)) < 1e-10
    assert np.allclose(r(x, 0), x[0, 0])
    z = ref.norm_rotate(x, None, None, np.full(32, 2.0), 0.0)
    assert abs((z * z).mean() - 4.0) < 1e-12


def test_halves_and_pairs_are_one_rotation_in_two_orders():
    x = np.random.default_rng(3).standard_normal((4, 2, 16))
    table, pos = make_table(9, 16), np.array([0, 3, 8, 1])
    order = np.arange(16).reshape(2, 8).T.reshape(-1)  # halves' pair i at (2i, 2i + 1)
    a = ref.norm_rotate(x, table, pos)[..., order]
    assert np.allclose(a, ref.norm_rotate(x[..., order], table, pos, interleaved=True))


def test_append_page_contract():
    codes = np.zeros((16, 4), dtype=np.int8)
    new = np.array([[1.0, -2.0, 0.5, 0.0]], dtype=np.float32)
    c, s = ref.append_page(new, codes, np.float32(9.0), 0)
    assert s == np.float32(2.0) / np.float32(127) and list(c[0]) == [64, -127, 32, 0]
    c2, s2 = ref.append_page(2 * new, c, s, 1)  # twice as large: the earlier codes are halved, ties to even
    assert s2 == np.float32(4.0) / np.float32(127) and list(c2[0]) == [32, -64, 16, 0] and list(c2[1]) == [64, -127, 32, 0]
    c3, s3 = ref.append_page(new / 4, c2, s2, 2)
    assert s3 == s2 and np.array_equal(c3[:2], c2[:2])
    c4, s4 = ref.append_page(new * np.nan, c3, s3, 3)
    assert np.isnan(s4) and (c4[3] == 0).all() and np.array_equal(c4[:3], c3[:3])


def test_native_value_order_round_trips():
    x = np.arange(2 * 3 * 32 * 16).reshape(2, 3, 32, 16).astype(np.int16)
    n = native_v(x)
    assert n.shape == (2, 3, 2, 16, 16) and n[1, 2, 1, 5, 7] == x[1, 2, 23, 5] and np.array_equal(plain_v(n), x)


def test_frequencies():
    from paper_2609_24433_amd import fq
    f, m = fq.rope_frequencies(64)
    assert m == 1.0 and f.shape == (32,) and f[0] == 1.0 and abs(f[-1].item() - 10000.0 ** (-62 / 64)) < 1e-15
    assert np.allclose(fq.rope_frequencies(64, scaling="linear", factor=4.0)[0], f / 4)
    b, _ = fq.rope_frequencies(64, scaling="base", factor=4.0)
    assert b[0] == 1.0 and abs((f[-1] / b[-1]).item() - 4.0) < 1e-9
    p, m = fq.rope_frequencies(64, scaling="by_parts", factor=4.0, original_length=4096)
    turns = f * 4096 / (2 * math.pi)
    assert np.allclose(p[turns > 32], f[turns > 32]) and np.allclose(p[turns < 1], f[turns < 1] / 4)
    assert (p <= f).all() and (p >= f / 4 * (1 - 1e-12)).all() and abs(m - (1 + 0.1 * math.log(4))) < 1e-15
    with pytest.raises(ValueError):
        fq.rope_frequencies(64, scaling="by_parts", factor=4.0)
    with pytest.raises(ValueError):
        fq.rope_frequencies(64, scaling="other")
