"""The norm's codes and scales through the integer product, against the plain norm, rounding and product."""
import numpy as np
import pytest

from oracle import microscaled as mx
from tests.gpu_util import flush
from tests.mx_util import HALF_BF16, dev, dev_bf16, fq, strided, tokens

pytestmark = pytest.mark.gpu

EPS = 1e-6


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,K,N,b", [(1, 1024, 256, 64), (60, 1024, 256, 64), (130, 896, 272, 128), (300, 2048, 512, 256)])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_then_product(M, K, N, b, bits, residual):
    """The plain side's codes, scales and weights are fp64 values, and its sums of products exact.  The product takes the sum (one
    rounding above 2^24, with 8 bits and 2048 channels), the two scales' product and the product of both in fp32, three half steps of
    2^-24, and rounds to bf16, 2^-8: nothing else is allowed."""
    flush(f"norm, gemm M={M} K={K} N={N} b={b} bits={bits}")
    f = fq()
    r = np.random.default_rng(M + K + bits)
    x, res = tokens(M, K, 1, special=False), tokens(M, K, 2, special=False) if residual else None
    gain = r.uniform(0.5, 1.5, K).astype(np.float32)
    lin = f.QuantLinear(dev((r.standard_normal((N, K)) * 0.02).astype(np.float32)), b, bits)
    codes, delta, _ = f.norm_quant(strided(x), dev(gain), b, bits, None if res is None else dev_bf16(res), EPS)
    y = f.gemm(codes, delta, lin.w_packed, lin.w_scale, N, K, bits).double().cpu().numpy()

    c, d = mx.codes(mx.butterfly(mx.norm(x, gain, EPS, res)[1], b), b, bits)
    w = f.unpack_weights(lin.w_packed, N, K, bits).cpu().numpy().astype(np.float64)
    want = (c.astype(np.float64) @ w.T) * d.astype(np.float64)[:, None] * lin.w_scale.cpu().numpy().astype(np.float64)[None]

    def within(v):
        return np.abs(y - v) <= np.abs(want) * (HALF_BF16 + 2.0 ** -21)

    assert within(want).all(), float((np.abs(y - want) / np.maximum(np.abs(want), 1e-30)).max())
    # what an exchange of rows, columns or channels, or a lost scale, would give is far outside
    others = [np.zeros_like(want), want[:, ::-1], want * 1.02]
    if M > 1:
        others += [want[::-1], want / d[:, None] * np.roll(d, 1)[:, None]]
    others.append((c[:, ::-1].astype(np.float64) @ w.T) * d[:, None] * lin.w_scale.cpu().numpy()[None])
    for v in others:
        assert within(v).mean() < 0.1
