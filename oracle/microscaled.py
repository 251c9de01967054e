"""Microscaled 4-bit codes, the norm before a projection and their products, plainly (numpy; test infrastructure).

The rounding and the norm follow the library's numerical contract (fp32 operations in its order, the norm's sum and root
in fp64), so codes compare bit for bit; products and values are fp64."""
from __future__ import annotations

import numpy as np
import torch

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x: np.ndarray) -> np.ndarray:
    """fp32 rounded to bf16, as fp32."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def butterfly(x: np.ndarray, b: int) -> np.ndarray:
    """Unnormalized block Hadamard, fp32, stages 1, 2, .. b/2."""
    x = x.astype(np.float32)
    shape, h = x.shape, 1
    with np.errstate(all="ignore"):
        while h < b:
            y = x.reshape(-1, 2, h)
            x = np.stack((y[:, 0] + y[:, 1], y[:, 0] - y[:, 1]), axis=1).reshape(shape)
            h *= 2
    return x


def root(b: int) -> np.float32:
    return np.float32(1.0 / np.sqrt(np.float64(b)))


def fold(x: np.ndarray, b: int, pre=None, post=None) -> np.ndarray:
    """fp32 rows through multiplier, butterfly, 1/sqrt(b) and multiplier."""
    with np.errstate(all="ignore"):
        u = x.astype(np.float32)
        if pre is not None:
            u = u * pre
        u = butterfly(u, b) * root(b)
        return u * post if post is not None else u


def encode(u: np.ndarray):
    """fp32 rows [M, K] -> (nibbles uint8 [M, K], scale bytes uint8 [M, K/32]); zero codes are positive."""
    M, K = u.shape
    v = u.reshape(M, K // 32, 32).astype(np.float64)
    fine = np.isfinite(v).all(axis=2)
    top = np.where(fine, np.abs(np.where(np.isfinite(v), v, 0.0)).max(axis=2), 1.0)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127).clip(-127, 127)
    t = np.where(fine[:, :, None], v, 0.0) * np.exp2(-e.astype(np.float64))[:, :, None]
    a = np.abs(t)[..., None]
    d = np.abs(a - MAGNITUDES)
    best = d.min(axis=-1, keepdims=True)
    near = d == best
    # the nearest; of two, the even one (neighbours have codes of either parity)
    low = near.argmax(axis=-1)
    high = 7 - near[..., ::-1].argmax(axis=-1)
    code = np.where(low % 2 == 0, low, high)
    code = np.where((t < 0) & (code > 0), code + 8, code)
    return code.reshape(M, K).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def decode(nibbles: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """fp64 values of nibbles [M, K] under scale bytes [M, K/32]."""
    M, K = nibbles.shape
    v = MAGNITUDES[nibbles & 7] * np.where(nibbles & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1).reshape(M, K)


def pack_nibbles(n: np.ndarray) -> np.ndarray:
    return (n[:, 0::2] | (n[:, 1::2] << 4)).astype(np.uint8)


def split_nibbles(c: np.ndarray) -> np.ndarray:
    """Bytes [M, K/2] -> nibbles [M, K] with the sign of zeros dropped."""
    n = np.stack((c & 15, c >> 4), axis=2).reshape(c.shape[0], -1)
    return np.where(n == 8, 0, n).astype(np.uint8)


def steps(scale: np.ndarray) -> np.ndarray:
    """Scale bytes [M, K/32] in the library's order [K/128, M, 4]."""
    M, n = scale.shape
    return np.ascontiguousarray(scale.reshape(M, n // 4, 4).transpose(1, 0, 2))


def rows(scale: np.ndarray) -> np.ndarray:
    return np.ascontiguousarray(scale.transpose(1, 0, 2)).reshape(scale.shape[1], -1)


def tiles(codes: np.ndarray) -> np.ndarray:
    """Codes [N, K/2] in the product's order [N/16, K/128, 4, 16, 16]."""
    N, half = codes.shape
    return np.ascontiguousarray(codes.reshape(N // 16, 16, half // 64, 4, 16).transpose(0, 2, 3, 1, 4))


def norm(x: np.ndarray, weight: np.ndarray, eps: float, residual=None):
    """(h, y): the bf16 residual stream and the fp32 normed rows."""
    with np.errstate(all="ignore"):
        h = x.astype(np.float32)
        if residual is not None:
            h = bf16(h + residual.astype(np.float32))
        mean = (h.astype(np.float64) ** 2).sum(axis=1, keepdims=True) / h.shape[1]
        s = (1.0 / np.sqrt(mean + np.float64(np.float32(eps)))).astype(np.float32)
        return h, (h * s) * weight


def codes(u: np.ndarray, b: int, bits: int, r: float = 1.0):
    """Eq. (5) on rotated fp32 rows: (codes int8 [M, K], delta fp32 [M])."""
    q = np.float32(127 if bits == 8 else 7)
    with np.errstate(all="ignore"):
        fine = np.isfinite(u).all(axis=1)
        top = np.abs(np.where(fine[:, None], u, np.float32(0))).max(axis=1)
        rA = np.float32(r) * top
        inv = q / rA
        some = fine & np.isfinite(inv)
        t = np.where(some[:, None], u, np.float32(0)) * np.where(some, inv, np.float32(0))[:, None]
        c = np.clip(np.rint(t), -q, q).astype(np.int8)
        delta = np.where(some, (rA * root(b)) / q, np.where(fine, np.float32(0), np.float32(np.nan)))
    return c, delta.astype(np.float32)
