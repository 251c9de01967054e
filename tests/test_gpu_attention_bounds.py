"""The attention operators where the call's bounds, not its lengths, choose the kernel: max_new and max_kv well above
what the sequences have, and many samples of few queries.  Same definition and derived tolerance as their other tests."""
import numpy as np
import pytest
import torch

from tests.attention_util import bf16, check_rows, ints, make_cache, sequence, to_device
from tests.gpu_util import DEV, flush

pytestmark = pytest.mark.gpu


def fq():
    from paper_2609_24433_amd import fq as _fq
    return _fq


def run(n, lens, Hq, H, D, P, causal, max_new, max_kv, edit=None):
    flush(f"bounds n={n} lens={lens} Hq={Hq} H={H} D={D} P={P} causal={causal} max_new={max_new} max_kv={max_kv}")
    rng = np.random.default_rng(D + P + sum(lens))
    table, kc, ks, vc, vs = make_cache(rng, lens, P, H, D)
    short = -(-max_kv // P) - table.shape[1]
    if short > 0:
        table = np.pad(table, ((0, 0), (0, short)), constant_values=-3)
    if edit:
        edit(table, ks, vs)
    q, qt = bf16(rng.standard_normal((sum(n), Hq, D)) * 1.5)
    out = fq().cache_attention(qt, to_device(kc, ks, vc, vs), ints(table), ints(np.concatenate(([0], np.cumsum(n)))), ints(lens),
                               max_new, max_kv, None, causal)
    torch.cuda.synchronize()
    row = 0
    for b, m in enumerate(lens):
        j, i = np.arange(m)[None, :], np.arange(n[b])[:, None]
        seen = (j <= m - n[b] + i) if causal else np.ones((n[b], m), dtype=bool)
        for h in range(Hq):
            k, v = (sequence(table, c, s, b, m, h // (Hq // H)) for c, s in ((kc, ks), (vc, vs)))
            rows = slice(row, row + n[b])
            check_rows(out[rows, h], q[rows, h], k, v, seen, D ** -0.5, f"sequence {b} head {h}")
        row += n[b]
    return out


BOUNDS = [(1100, 4100), (8200, 520)]


@pytest.mark.parametrize("max_new,max_kv", BOUNDS)
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 144, 256])
@pytest.mark.parametrize("n,lens", [([1], [1]), ([3, 40], [200, 130]), ([150, 0, 3], [150, 77, 511])])
def test_few_rows_under_wide_bounds(D, n, lens, max_new, max_kv):
    run(n, lens, 4, 2, D, 32, True, max_new, max_kv)


@pytest.mark.parametrize("max_new,max_kv", BOUNDS)
@pytest.mark.parametrize("P", [16, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_and_empty_rows_under_wide_bounds(P, causal, max_new, max_kv):
    out = run([0, 4, 6, 1, 70], [20, 0, 2, 129, 257], 6, 2, 128, P, causal, max_new, max_kv)
    assert (out[:4] == 0).all()


@pytest.mark.parametrize("max_new,max_kv", BOUNDS)
def test_silent_and_poisoned_pages_under_wide_bounds(max_new, max_kv):
    def silent(table, ks, vs):
        ks[table[0, 1]] = 0
        vs[table[0, 2]] = 0
    run([5], [300], 4, 2, 64, 64, True, max_new, max_kv, edit=silent)
    rng = np.random.default_rng(1)
    n, m = 100, 200
    table, kc, ks, vc, vs = make_cache(rng, [m], 16, 2, 64)
    table = np.pad(table, ((0, 0), (0, 260)), constant_values=-3)
    ks[table[0, 9], 1] = np.nan  # tokens 144 to 159 of head 1
    vs[table[0, 11], 0] = np.nan  # tokens 176 to 191 of head 0
    qt = bf16(rng.standard_normal((n, 4, 64)))[1]
    out = fq().cache_attention(qt, to_device(kc, ks, vc, vs), ints(table), ints([0, n]), ints([m]), max_new, max_kv)
    nan = torch.isnan(out).cpu().numpy()
    assert (nan.any(axis=2) == nan.all(axis=2)).all()
    at = m - n + np.arange(n)
    for h, first in ((0, 176), (1, 144)):
        for g in range(2):
            assert np.array_equal(nan[:, 2 * h + g, 0], at >= first), h


@pytest.mark.parametrize("Sq,Sk", [(50, 201), (130, 129)])
@pytest.mark.parametrize("D", [48, 64, 80, 128, 160, 256])
def test_many_samples_with_masks(Sq, Sk, D):
    B, Hq, H = 40, 4, 2
    flush(f"samples Sq={Sq} Sk={Sk} D={D}")
    rng = np.random.default_rng(Sq + D)
    mask = rng.random((B, Sk)) < 0.6
    mask[1] = False
    mask[3, :120] = False
    lens = np.where(rng.random(B) < 0.5, Sk, rng.integers(0, Sk + 1, B))
    lens[2] = 0
    seen = mask & (np.arange(Sk)[None, :] < lens[:, None])
    q, qt = bf16(rng.standard_normal((B, Sq, Hq, D)) * 1.5)
    kv = rng.standard_normal((B, Sk, 2 * H, D))
    kv[~seen] = rng.choice([np.nan, np.inf, -np.inf, 1e38], kv[~seen].shape)
    kv, kvt = bf16(kv)
    out = fq().cross_attention(qt, kvt[:, :, :H], kvt[:, :, H:], ints(lens), torch.from_numpy(mask).to(DEV))
    assert (out[1] == 0).all() and (out[2] == 0).all()
    for b in range(0, B, 3):
        for h in range(Hq):
            check_rows(out[b, :, h], q[b, :, h], kv[b, :, h // 2], kv[b, :, H + h // 2], np.broadcast_to(seen[b], (Sq, Sk)), D ** -0.5,
                       f"sample {b} head {h}")
