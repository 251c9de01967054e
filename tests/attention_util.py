"""Inputs and references shared by the tests of the attention operators."""
import numpy as np
import torch

from oracle import attention as ref
from tests.gpu_util import DEV


def bf16(x):
    """numpy -> the nearest bf16 values (fp64) and their tensor on the device."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.double().numpy(), t.to(DEV)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def make_table(length, R):
    a = np.arange(length)[:, None] * (10000.0 ** (-np.arange(0, R, 2) / R))[None]
    return np.stack([np.cos(a), np.sin(a)], axis=-1).astype(np.float32)


def pages_for(rng, lens, P, spare=3, wide=2):
    """A shuffled page table for the lengths; entries that no token needs are outside the pool."""
    need = [-(-n // P) for n in lens]
    pool = sum(need) + spare
    perm = rng.permutation(pool)
    table = np.full((len(lens), max(need + [0]) + wide), 10 ** 9, dtype=np.int64)
    table[:, -1] = -7
    used = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[used:used + n]
        used += n
    return table, pool


def make_cache(rng, lens, P, H, D, spread=6.0):
    """Random pages: scales over many octaves, the unused pages' NaN, unused slots with any codes."""
    table, pool = pages_for(rng, lens, P)
    kc = rng.integers(-127, 128, (pool, H, P, D)).astype(np.int8)
    vc = rng.integers(-127, 128, (pool, H, P, D)).astype(np.int8)
    ks = (2.0 ** rng.uniform(-7.5, -5.5, (pool, H))).astype(np.float32)
    vs = (2.0 ** rng.uniform(-spread, spread, (pool, H))).astype(np.float32)
    used = np.zeros(pool, dtype=bool)
    for b, n in enumerate(lens):
        used[table[b, :-(-n // P)]] = True
    ks[~used], vs[~used] = np.nan, np.nan
    return table, kc, ks, vc, vs


def native_v(vc):
    """[pool, H, P, D] -> the cache's [pool, H, P/16, D, 16]."""
    pool, H, P, D = vc.shape
    return np.ascontiguousarray(vc.reshape(pool, H, P // 16, 16, D).transpose(0, 1, 2, 4, 3))


def plain_v(native):
    pool, H, g, D, _ = native.shape
    return np.ascontiguousarray(native.transpose(0, 1, 2, 4, 3).reshape(pool, H, g * 16, D))


def to_device(kc, ks, vc, vs):
    from paper_2609_24433_amd import fq
    return fq.KVCache(torch.from_numpy(kc).to(DEV), torch.from_numpy(ks).to(DEV), torch.from_numpy(native_v(vc)).to(DEV),
                      torch.from_numpy(vs).to(DEV))


def sequence(table, codes, scale, b, n, h):
    """Tokens [0, n) of head h of sequence b as fp64 values [n, D]."""
    P, D = codes.shape[2], codes.shape[3]
    page = table[b, :-(-n // P)]
    return (codes[page, h].astype(np.float64) * scale[page, h].astype(np.float64)[:, None, None]).reshape(-1, D)[:n]


def check_rows(got, q, k, v, seen, scale, what):
    """got bf16 [R, D] of one head against the definition within its derived tolerance."""
    out, spread, reach = ref.attention(q, k, v, seen, scale)
    tol = ref.tolerance(out, spread, reach, q.shape[1], k.shape[0], np.abs(v[seen.any(axis=0)]).max(initial=0.0))
    g = got.double().cpu().numpy()
    bad = ~(np.abs(g - out) <= tol)
    if bad.any():
        r, d = np.argwhere(bad)[0]
        raise AssertionError(f"{what}: row {r} dim {d}: {g[r, d]} for {out[r, d]} +- {tol[r, d]} ({bad.sum()} of {bad.size})")
