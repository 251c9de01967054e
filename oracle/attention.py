"""Attention operators from their definitions, numpy in 64 bits (appends: the fp32 rounding contract)."""
from __future__ import annotations

import numpy as np


def norm_rotate(x, table=None, positions=None, weight=None, eps=1e-6, interleaved=False):
    """x [T, H, D] -> fp64; table [length, R/2, 2] (positions clamped into it)."""
    y = np.asarray(x, dtype=np.float64).copy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    if table is None or table.shape[1] == 0:
        return y
    half = table.shape[1]
    cs = np.asarray(table, dtype=np.float64)[np.clip(positions, 0, table.shape[0] - 1)][:, None]
    i = np.arange(half)
    one, two = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = y[..., one].copy(), y[..., two].copy()
    y[..., one] = a * cs[..., 0] - b * cs[..., 1]
    y[..., two] = b * cs[..., 0] + a * cs[..., 1]
    return y


def append_page(new, codes, scale, held, growth=0):
    """One page of one head: `new` fp32 [n, D] goes behind `held` earlier tokens of codes int8 [P, D] under
    fp32 `scale`, which grows by `growth` percent at least where it has to.  Returns (codes, scale) after the append, in
    fp32 arithmetic; slots beyond are as they were."""
    f = np.float32
    codes = codes.copy()
    if len(new) == 0:
        return codes, scale
    a = np.abs(new.astype(f)).max()
    if not np.isfinite(a) or np.isnan(new).any() or (held and np.isnan(scale)):
        codes[held:held + len(new)] = 0
        return codes, f(np.nan)
    s = f(a / f(127))
    if held:
        s = f(scale) if f(scale) >= s else max(s, f(f(scale) * f(f(1) + f(growth) / f(100))))
    if s < np.finfo(f).tiny:
        s = f(0)
    if held and s != f(scale) and s > 0:
        codes[:held] = np.rint(codes[:held].astype(f) * f(f(scale) / s)).astype(np.int8)
    inv = f(f(1) / s) if s > 0 else f(0)
    codes[held:held + len(new)] = np.clip(np.rint(new.astype(f) * inv), -127, 127).astype(np.int8)
    return codes, s


def attention(q, k, v, seen, scale):
    """q [R, D], k and v [S, D], seen bool [R, S] -> (out [R, D], the rows' sum of p |v|, [R, 1] the largest
    scale * sum |q k| over the seen keys).  Rows that see nothing give zeros."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    R, D = q.shape
    if k.shape[0] == 0:
        return np.zeros((R, D)), np.zeros((R, D)), np.zeros((R, 1))
    any_seen = seen.any(axis=0)
    k, v = np.where(any_seen[:, None], k, 0.0), np.where(any_seen[:, None], v, 0.0)
    s = np.where(seen, q @ k.T * scale, -np.inf)
    top = s.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        p = np.exp(s - np.where(np.isneginf(top), 0.0, top))
    p = np.where(seen, p, 0.0)
    total = p.sum(axis=1, keepdims=True)
    total = np.where(seen.any(axis=1, keepdims=True), total, 1.0)
    reach = np.where(seen, np.abs(q) @ np.abs(k).T * scale, 0.0).max(axis=1, keepdims=True)
    return p @ v / total, p @ np.abs(v) / total, reach


def tolerance(out, spread, reach, D, keys, vmax):
    """How far a bf16 result may be from `out`: the output's rounding and the weights' (2^-8, half a step of 8 significant bits, of |out| and of
    sum p |v|), the fp32 scores (D + 16 roundings of sum |q k|, twice: numerator and denominator) and the fp32 sums.  Weights
    under 2^-126 of the row's largest are outside fp32's range and may be lost, at most vmax = max |v| times that each."""
    u = 2.0 ** -24
    return 1.01 * 2.0 ** -8 * (np.abs(out) + spread) + spread * (2 * (D + 16) * u * reach + (keys + 32) * 2 * u) + keys * 2.0 ** -126 * vmax + 1e-37
