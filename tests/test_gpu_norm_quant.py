"""The norm before a projection on the GPU against the plain reference: the residual stream, codes and scales bit for bit."""
import numpy as np
import pytest
import torch

from oracle import microscaled as mx
from tests.gpu_util import DEV, canonical_codes, flush
from tests.mx_util import dev, dev_bf16, fq, strided, tokens

pytestmark = pytest.mark.gpu

EPS = 1e-6


def rotated(y, b, post=None):
    with np.errstate(all="ignore"):
        u = mx.butterfly(y, b)
        return u if post is None else u * post


def check(x, weight, b, fmt, res=None, post=None, r=1.0, eps=EPS, residual=None, sum_out=None, into=None):
    """x, res: fp32 arrays of bf16 values; residual, sum_out: the tensors to pass."""
    f = fq()
    h, y = mx.norm(x, weight, eps, res)
    xd = strided(x) if into is None else into
    rd = residual if residual is not None else None if res is None else strided(res, 8)
    w, p = dev(weight), None if post is None else dev(post)
    if fmt == "mx":
        codes, scale, total = f.norm_mx_quant(xd, w, b, rd, eps, p, sum_out)
        with np.errstate(all="ignore"):
            u = mx.butterfly(y, b) * mx.root(b)
            u = u if post is None else u * post
        want, ws = mx.encode(u)
        assert np.array_equal(mx.rows(scale.cpu().numpy()), ws)
        assert np.array_equal(mx.split_nibbles(codes.cpu().numpy()), want)
    else:
        bits = int(fmt[1])
        codes, scale, total = f.norm_quant(xd, w, b, bits, rd, eps, r, p, sum_out)
        want, delta = mx.codes(rotated(y, b, post), b, bits, r)
        assert np.array_equal(scale.cpu().numpy(), delta, equal_nan=True), np.argwhere(scale.cpu().numpy() != delta)[:4]
        assert np.array_equal(codes.cpu().numpy(), canonical_codes(want, bits))
    assert np.array_equal(total.float().cpu().numpy(), h, equal_nan=True)
    return codes, scale


@pytest.mark.parametrize("fmt", ["i8", "i4", "mx"])
@pytest.mark.parametrize("M,K,b", [(1, 128, 1), (1, 2048, 128), (9, 256, 256), (17, 384, 64), (50, 1024, 32), (10, 1152, 128), (33, 4096, 1),
                                   (8, 4224, 128), (8, 7168, 2), (9, 8192, 64), (5, 16384, 256), (2, 32768, 128), (300, 640, 16)])
@pytest.mark.parametrize("residual", [False, True])
def test_norm(M, K, b, fmt, residual):
    flush(f"norm {fmt} M={M} K={K} b={b} residual={residual}")
    r = np.random.default_rng(K + M)
    w = r.uniform(0.3, 2.0, K).astype(np.float32)
    x = tokens(M, K, M * 31 + K)
    check(x, w, b, fmt, tokens(M, K, 77 + M, special=False) if residual else None)


@pytest.mark.parametrize("fmt", ["i8", "i4", "mx"])
@pytest.mark.parametrize("clip", [1.0, 0.8])
def test_folds_and_clip(fmt, clip):
    if fmt == "mx" and clip != 1.0:
        pytest.skip("no clip ratio")
    r = np.random.default_rng(4)
    K = 896
    check(tokens(20, K, 1), r.uniform(0.3, 2.0, K).astype(np.float32), 64, fmt, tokens(20, K, 2), r.uniform(0.2, 4.0, K).astype(np.float32), clip)


@pytest.mark.parametrize("fmt", ["i8", "mx"])
@pytest.mark.parametrize("which", ["x", "residual"])
def test_the_sum_in_place(fmt, which):
    K = 1024
    x, res = tokens(37, K, 5), tokens(37, K, 6)
    w = np.ones(K, dtype=np.float32)
    a, b = strided(x), strided(res, 8)
    place = a if which == "x" else b
    check(x, w, 64, fmt, res, residual=b, sum_out=place, into=a)
    assert torch.equal(place, dev_bf16(mx.bf16(x + res)))


@pytest.mark.parametrize("fmt", ["i8", "i4", "mx"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38])
def test_rows_that_are_not_finite(fmt, value):
    """NaN, infinity, or a sum of two large values that overflows, in one row; its neighbours are as they were."""
    K = 512
    x, res = tokens(5, K, 8, special=False), tokens(5, K, 9, special=False)
    x[2, 100] = res[2, 100] = mx.bf16(np.array([value], np.float32))[0]
    w = np.ones(K, dtype=np.float32)
    codes, scale = check(x, w, 64, fmt, res)
    s = mx.rows(scale.cpu().numpy()) if fmt == "mx" else scale.cpu().numpy()
    assert (s[2] == 255).any() if fmt == "mx" else np.isnan(s[2])
    assert not (s[[0, 1, 3, 4]] == 255).any() if fmt == "mx" else np.isfinite(s[[0, 1, 3, 4]]).all()


def test_gains_that_are_zero_tiny_or_not_finite():
    K = 256
    x = tokens(4, K, 3, special=False)
    for g in (0.0, 1e-40, 1e-37, float("nan"), float("inf")):
        check(x, np.full(K, g, np.float32), 64, "i8")
        check(x, np.full(K, g, np.float32), 64, "mx")
    w = np.ones(K, np.float32)
    w[3] = np.nan
    check(x, w, 1, "i8")
    check(x, w, 1, "mx")


@pytest.mark.parametrize("eps", [1e-12, 1e-5, 1.0])
def test_eps(eps):
    K = 384
    x = tokens(9, K, 12) * np.float32(1e-3)
    check(mx.bf16(x), np.ones(K, np.float32), 128, "i8", eps=eps)


def test_against_the_definition_in_64_bits():
    """Values within half a step of the definition's, plus the fp32 roundings of the rotation and the norm."""
    M, K, b = 20, 1024, 64
    r = np.random.default_rng(0)
    x, w = tokens(M, K, 1, special=False), r.uniform(0.5, 2, K).astype(np.float32)
    codes, delta, _ = fq().norm_quant(dev_bf16(x), dev(w), b, 8)
    got = fq().read_codes(codes, delta, 8).float().cpu().numpy().astype(np.float64)
    from scipy.linalg import hadamard
    y = x.astype(np.float64) / np.sqrt((x.astype(np.float64) ** 2).mean(axis=1, keepdims=True) + np.float64(np.float32(EPS))) * w
    want = (y.reshape(-1, b) @ hadamard(b) / np.sqrt(b)).reshape(M, K)
    step = np.abs(want).max(axis=1, keepdims=True) / 127
    # half a step; a few fp32 roundings (s, two products, 6 stages) of at most sqrt(b) |y|max; the bf16 of the value
    slack = 2.0 ** -24 * 12 * np.abs(y).max(axis=1, keepdims=True) * np.sqrt(b) + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(got - want) <= 0.5 * step * (1 + 1e-5) + slack + 2.0 ** -8 * step)


def test_codes_are_the_projections_codes():
    """norm_quant's codes and deltas through the integer GEMM, against the norm in fp32 rounded to bf16 and fq.linear: the
    same projection up to that rounding (2^-8) and the two roundings to 8 bits."""
    f = fq()
    M, K, N, b = 60, 1024, 256, 64
    r = np.random.default_rng(2)
    x, res = tokens(M, K, 1, special=False), tokens(M, K, 2, special=False)
    w = (r.standard_normal((N, K)) * 0.02).astype(np.float32)
    gain = np.ones(K, np.float32)
    lin = f.QuantLinear(dev(w), b, 8)
    codes, delta, total = f.norm_quant(dev_bf16(x), dev(gain), b, 8, dev_bf16(res))
    y = f.gemm(codes, delta, lin.w_packed, lin.w_scale, N, K, 8).float().cpu().numpy()
    _, yn = mx.norm(x, gain, EPS, res)
    ref = lin(dev_bf16(yn)).float().cpu().numpy()
    # each side's tokens are within half a step of delta, or bf16's half step, of the same values; weights of |w| sum
    size = np.abs(w).sum(axis=1)[None]
    d = delta.cpu().numpy()[:, None]
    bound = size * np.sqrt(b) * (1.2 * d + 2.0 ** -8 * np.abs(yn).max(axis=1, keepdims=True)) + 2.0 ** -7 * np.abs(ref)
    assert np.all(np.abs(y - ref) <= bound)


def test_no_rows():
    x = torch.zeros((0, 256), dtype=torch.bfloat16, device=DEV)
    codes, delta, total = fq().norm_quant(x, torch.ones(256, device=DEV), 64, 8, x)
    assert codes.shape == (0, 256) and delta.shape == (0,) and total.shape == (0, 256)
