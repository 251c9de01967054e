"""Single roundings on the GPU: codes with a token scale as values, and the rounding to E2M1 under every scale."""
import numpy as np
import pytest
import torch

from oracle import microscaled as mx
from tests.mx_util import dev, fq

pytestmark = pytest.mark.gpu


def bf16_of_exact(v):
    """fp64 values, normal in bf16, to bf16 with one rounding to nearest, ties to even."""
    m, e = np.frexp(v)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


@pytest.mark.parametrize("bits", [4, 8])
def test_a_value_is_the_fp32_product_rounded_to_bf16(bits):
    """Scales whose product with a code lies beside a tie of bf16, and on it once it is an fp32: two roundings and one differ there,
    and the values are what two give."""
    q = 127 if bits == 8 else 7
    r = np.random.default_rng(bits)
    K = 128
    # codes but powers of two, scales next to (an odd number of half steps of bf16) / code
    c = r.choice([k for k in range(3, q + 1) if k & (k - 1)], 4096)
    tie = (257 + 2 * r.integers(0, 128, c.size)) / 256
    d = (tie / c).astype(np.float32)
    product = c.astype(np.float64) * d.astype(np.float64)
    twice = torch.from_numpy(product.astype(np.float32)).to(torch.bfloat16).double().numpy()
    differ = twice != bf16_of_exact(product)
    assert differ.sum() > 64  # the inputs do tell the two apart
    c, d, twice = c[differ], d[differ], twice[differ]
    codes = np.repeat(c[:, None], K, axis=1).astype(np.int8)
    codes[:, 1::2] *= -1
    raw = codes.view(np.uint8) if bits == 8 else mx.pack_nibbles((codes & 15).astype(np.uint8))
    got = fq().read_codes(dev(raw), dev(d), bits).double().cpu().numpy()
    assert np.array_equal(got, np.where(np.arange(K) % 2, -1.0, 1.0) * twice[:, None])
