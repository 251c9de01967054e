"""The attention weights of calls with few query rows keep 15 bits and more in the product with the values: a result is
nearer the definition than weights of 8 bits would leave it, where the mean is small beside what it averages."""
import numpy as np
import pytest
import torch

from oracle import attention as ref
from tests.attention_util import bf16, ints, make_cache, sequence, to_device
from tests.gpu_util import flush


def bound(out, spread, reach, D, keys, bits):
    """The output's one rounding, the weights' to `bits` bits, and fp32 scores and sums (oracle.attention.tolerance's)."""
    u = 2.0 ** -24
    return 1.01 * (2.0 ** -8 * np.abs(out) + 2.0 ** -bits * spread) + spread * (2 * (D + 16) * u * reach + (keys + 32) * 2 * u) + 1e-37


SHAPES = [(32, 40), (64, 64), (64, 17), (128, 33), (256, 64)]


def inputs(rng, R, D, S, b=lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()):
    return b(rng.standard_normal((R, D))), b(rng.standard_normal((S, D))), b(rng.standard_normal((S, D)))


@pytest.mark.parametrize("D,S", SHAPES)
def test_the_bound_tells_weights_of_8_bits_apart(D, S):
    """(the definition with its weights rounded to bf16 once, and to two bf16 values)"""
    q, k, v = inputs(np.random.default_rng(D + S), 4, D, S)
    out, spread, reach = ref.attention(q, k, v, np.ones((4, S), dtype=bool), 0.3 / np.sqrt(D))
    p = np.exp(q @ k.T * (0.3 / np.sqrt(D)))
    r = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()  # noqa: E731
    for weights, holds in ((r(p), False), (r(p) + r(p - r(p)), True)):
        got = r(weights @ v / p.sum(axis=1, keepdims=True))
        assert (np.abs(got - out) <= bound(out, spread, reach, D, S, 15)).all() == holds


@pytest.mark.gpu
@pytest.mark.parametrize("D,S", SHAPES)
@pytest.mark.parametrize("n", [1, 5])
def test_weights_over_the_cache(D, S, n):
    from paper_2609_24433_amd import fq
    flush(f"weights cached D={D} S={S} n={n}")
    rng = np.random.default_rng(D + S + n)
    table, kc, ks, vc, vs = make_cache(rng, [S], 16, 2, D, spread=0.5)
    q, qt = bf16(rng.standard_normal((n, 4, D)))
    scale = 0.1 / np.sqrt(D)
    out = fq.cache_attention(qt, to_device(kc, ks, vc, vs), ints(table), ints([0, n]), ints([S]), n, S, scale, False)
    got = out.double().cpu().numpy()
    for h in range(4):
        k, v = sequence(table, kc, ks, 0, S, h // 2), sequence(table, vc, vs, 0, S, h // 2)
        want, spread, reach = ref.attention(q[:, h], k, v, np.ones((n, S), dtype=bool), scale)
        assert (np.abs(got[:, h] - want) <= bound(want, spread, reach, D, S, 16)).all(), h


@pytest.mark.gpu
@pytest.mark.parametrize("D,S", SHAPES)
@pytest.mark.parametrize("n", [1, 5])
def test_weights_over_states(D, S, n):
    from paper_2609_24433_amd import fq
    flush(f"weights states D={D} S={S} n={n}")
    rng = np.random.default_rng(D + S + n)
    q, qt = bf16(rng.standard_normal((2, n, 4, D)))
    k, kt = bf16(rng.standard_normal((2, S, 2, D)))
    v, vt = bf16(rng.standard_normal((2, S, 2, D)))
    scale = 0.3 / np.sqrt(D)
    got = fq.cross_attention(qt, kt, vt, scale=scale).double().cpu().numpy()
    for b in range(2):
        for h in range(4):
            want, spread, reach = ref.attention(q[b, :, h], k[b, :, h // 2], v[b, :, h // 2], np.ones((n, S), dtype=bool), scale)
            assert (np.abs(got[b, :, h] - want) <= bound(want, spread, reach, D, S, 15)).all(), (b, h)
