"""Shared inputs and bounds of the microscaled operators' tests."""
import numpy as np
import torch

from oracle import microscaled as mx
from tests.gpu_util import DEV

HALF_BF16 = 2.0 ** -8  # a bf16 rounding, relative to the value


def fq():
    from paper_2609_24433_amd import fq as _fq
    return _fq


def tokens(M, K, seed, special=True):
    """bf16 rows as fp32, heavy in a few channels; the first rows, where there are enough, are special ones."""
    r = np.random.default_rng(seed)
    x = r.standard_normal((M, K)).astype(np.float32)
    x[:, r.choice(K, max(1, K // 128), replace=False)] *= 20
    if special and M >= 8:
        x[0] = 0
        x[1] = 0
        x[1, K // 3] = -3.0
        x[2] = np.tile(np.array([6, 7, 7.5, 8, 5, 2.5, 3.5, 1.25, 0.25, 0.75, -0.25, -5, -7.75, 0, 1, -1], dtype=np.float32), K // 16)
        x[3] *= 1e-38   # subnormals among them
        x[4] *= 3e36
        x[5] = 2.0 ** -133 * (np.arange(K) % 5)  # the smallest bf16 values
        x[6] = 1.0
    return mx.bf16(x)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def dev_bf16(a):
    return dev(a).to(torch.bfloat16)


def strided(a, extra=24):
    """bf16 rows on the GPU with a row stride of K + extra and NaN between them."""
    M, K = a.shape
    t = torch.full((M, K + extra), float("nan"), dtype=torch.bfloat16, device=DEV)
    t[:, :K] = dev_bf16(a)
    return t[:, :K]


def operands(M, K, seed, spread=6):
    """Random codes and scale bytes of rows: (nibbles [M, K], bytes [M, K/32])."""
    r = np.random.default_rng(seed)
    n = r.integers(0, 16, (M, K)).astype(np.uint8)
    return n, r.integers(127 - spread, 127 + spread, (M, K // 32)).astype(np.uint8)


def product_bound(a, w, y):
    """Values a [M, K], w [N, K] and the exact y = a w^T (+ bias): the most that bf16 outputs may be off.  A block's sum of
    32 products is exact in fp32 (multiples of 1/4 up to 32 * 36 under one scale); K/32 of them, a bias and at most 7 joins are
    added with an error of a step of fp32 (2^-23) each of the largest partial sum, at most sum |a w| (+ |bias|, in y's slack);
    one rounding to bf16."""
    K = a.shape[1]
    return np.abs(a) @ np.abs(w).T * 2.0 ** -23 * (K // 32 + 8) + np.abs(y) * (HALF_BF16 + 2.0 ** -22)


def assert_product(y, a, w, bias=None):
    want = a @ w.T
    bound = None
    if bias is not None:
        bound = np.abs(bias.astype(np.float64)) * 2.0 ** -22
        want = want + bias
    got = y.float().cpu().numpy().astype(np.float64)
    most = product_bound(a, w, want) + (0 if bound is None else bound)
    off = np.abs(got - want)
    assert np.all(off <= most), (np.argwhere(off > most)[:4], float((off / np.maximum(most, 1e-300)).max()))
