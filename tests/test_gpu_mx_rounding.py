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


@pytest.mark.parametrize("sign", [1, -1])
def test_every_scale_rounds_ties_to_the_even_code_and_their_neighbours_to_the_nearest(sign):
    """All scales that a block of finite floats can have, one a row: every middle between two magnitudes, the floats on both sides of
    it, the magnitudes and what saturates, against the rule.  Middles are floats under every scale but the lowest ones, where the
    reference takes the floats that they round to."""
    middles = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    near = np.concatenate([np.nextafter(middles, np.float32(0)), middles, np.nextafter(middles, np.float32(8))])
    others = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 6.5, 7.0, np.nextafter(np.float32(8), np.float32(0))], np.float32)
    values = np.concatenate([near, others]).astype(np.float64)
    assert values.size == 32 and values.max() >= 4  # the largest sets the scale: values are multiples of it
    bytes_ = np.arange(0, 253)
    with np.errstate(over="raise"):
        block = (sign * values[None] * np.exp2(bytes_[:, None] - 127.0)).astype(np.float32)
    r = np.random.default_rng(5)
    u = np.concatenate([block[:, r.permutation(32)] for _ in range(4)], axis=1)  # a value in different lanes and slots
    codes, scales = fq().mx_quant(dev(u), 1)
    want, ws = mx.encode(u)
    assert np.array_equal(ws, np.repeat(bytes_[:, None], 4, axis=1))
    assert np.array_equal(mx.rows(scales.cpu().numpy()), ws)
    got = mx.split_nibbles(codes.cpu().numpy())
    assert np.array_equal(got, want), np.argwhere(got != want)[:4]


@pytest.mark.parametrize("rows", ["bf16", "norm"])
def test_ties_of_bf16_rows_under_every_scale(rows):
    """Middles and their neighbours in bf16 through the rounding of tokens, and through the norm's (rows under gains of 2^k; beside an
    eps of 2^32 the mean square vanishes, and the factor is 2^-16)."""
    middles = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    values = np.concatenate([middles * (1 - 2.0 ** -8), middles, middles * (1 + 2.0 ** -7), [4.0, 6.0, 7.0, 7.96875, 0.5, 1.5, 3.0, 0.0, 2.0, 1.0, 6.5]])
    values = mx.bf16(values.astype(np.float32)) * np.where(np.arange(values.size) % 3, 1, -1).astype(np.float32)
    assert values.size == 32
    bytes_ = np.arange(8, 253)
    if rows == "bf16":
        u = np.tile(values[None] * np.exp2(bytes_[:, None] - 127.0).astype(np.float32), (1, 4)).astype(np.float32)
        assert np.array_equal(mx.bf16(u), u)
        codes, scales = fq().mx_quant(dev(u).to(torch.bfloat16), 1)
        want, ws = mx.encode(u)
    else:
        x = np.tile(values[None], (1, 4))
        want, ws, codes, scales = [], [], [], []
        for byte in range(8, 239, 3):
            gain = np.full(128, 2.0 ** (byte - 127 + 16), np.float32)
            c, s, _ = fq().norm_mx_quant(dev(x).to(torch.bfloat16), dev(gain), 1, eps=2.0 ** 32)
            u = mx.norm(x, gain, 2.0 ** 32)[1]
            assert np.array_equal(u, x * np.float32(2.0 ** (byte - 127)))  # exact: nothing but powers of two
            w, sw = mx.encode(u)
            assert (sw == byte).all()
            want.append(w), ws.append(sw), codes.append(c), scales.append(s)
        want, ws, codes, scales = np.concatenate(want), np.concatenate(ws), torch.cat(codes), torch.cat(scales, dim=1)
    assert np.array_equal(mx.rows(scales.cpu().numpy()), ws)
    got = mx.split_nibbles(codes.cpu().numpy())
    assert np.array_equal(got, want), np.argwhere(got != want)[:4]
