"""Edges of the attention operators on the GPU: rows past a call's bound, values and queries that are not finite."""
import numpy as np
import pytest
import torch

from tests.attention_util import bf16, check_rows, ints, make_cache, make_table, sequence, to_device
from tests.gpu_util import DEV, flush

pytestmark = pytest.mark.gpu


def fq():
    from paper_2609_24433_amd import fq as _fq
    return _fq


@pytest.mark.parametrize("n,lens,most,P", [
    ([6], [6], 4, 16),             # the rows' slots 0 to 3; 4 and 5 stay
    ([40], [70], 17, 16),          # from inside a page over the next
    ([5], [3], 2, 16),             # the rows that are computed lie before slot 0
    ([5], [3], 4, 16),             # two of them do
    ([300, 3, 150], [300, 40, 500], 130, 128),
    ([64, 65], [64, 65], 64, 64),
])
def test_rows_past_the_bound_leave_the_others_where_they_are(n, lens, most, P):
    """More rows than max_new: the first max_new of a sequence go to their slots kv_len - n + i, under their positions, as
    in a call that has only these rows; the others are not computed; attention places the same rows alike."""
    f = fq()
    flush(f"past the bound n={n} lens={lens} most={most} P={P}")
    rng = np.random.default_rng(sum(n) + P)
    Hq, H, D = 4, 2, 64
    table, kc, ks, vc, vs = make_cache(rng, lens, P, H, D, spread=1.0)
    T = sum(n)
    x = bf16(rng.standard_normal((T, Hq + 2 * H, D)))[1]
    rope = torch.from_numpy(make_table(max(lens), D)).to(DEV)
    start = np.concatenate(([0], np.cumsum(n)))
    kept = [min(k, most) for k in n]
    rows = torch.from_numpy(np.concatenate([np.arange(a, a + k) for a, k in zip(start, kept)])).to(DEV)

    def append(cache, x, q_start, kv_len):
        y = torch.full((x.shape[0], Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
        f.cache_append(cache, ints(table), ints(q_start), ints(kv_len), most, x[:, Hq:Hq + H], x[:, Hq + H:], x[:, :Hq], rope, q_out=y)
        return y
    got, want = (to_device(kc, ks, vc, vs) for _ in range(2))
    y = append(got, x, start, lens)
    z = append(want, x[rows].contiguous(), np.concatenate(([0], np.cumsum(kept))), [m - (k - j) for m, k, j in zip(lens, n, kept)])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.nan_to_num(), b.nan_to_num())
    assert torch.equal(y[rows], z)
    rest = torch.ones(T, dtype=torch.bool, device=DEV)
    rest[rows] = False
    assert (y[rest] == 7.0).all()
    out = f.cache_attention(y, got, ints(table), ints(start), ints(lens), most, max(lens))
    torch.cuda.synchronize()
    k_now, v_now = got.k_codes.cpu().numpy(), got.v_codes.cpu().numpy().transpose(0, 1, 2, 4, 3).reshape(kc.shape)
    q = y.double().cpu().numpy()
    for b, m in enumerate(lens):
        seen = np.arange(m)[None, :] <= m - n[b] + np.arange(kept[b])[:, None]
        for h in range(Hq):
            k, v = (sequence(table, c, s.cpu().numpy(), b, m, h // 2) for c, s in ((k_now, got.k_scale), (v_now, got.v_scale)))
            at = slice(start[b], start[b] + kept[b])
            check_rows(out[at, h], q[at, h], k, v, seen, D ** -0.5, f"sequence {b} head {h}")


SIZES = [(1, 100), (1, 1500), (5, 700), (400, 1500)]


@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("Sq,Sk", SIZES)
def test_an_infinite_value_is_an_infinite_mean(Sq, Sk, D):
    f = fq()
    flush(f"infinite values Sq={Sq} Sk={Sk} D={D}")
    rng = np.random.default_rng(Sq + D)
    Hq, H = 4, 2
    q, qt = bf16(rng.standard_normal((1, Sq, Hq, D)) * 0.5)
    k, kt = bf16(rng.standard_normal((1, Sk, H, D)) * 0.5)
    v = rng.standard_normal((1, Sk, H, D))
    v[0, 7, 0, 3], v[0, 40, 0, 9], v[0, Sk - 1, 1, 5] = np.inf, -np.inf, -np.inf
    v, vt = bf16(v)
    out = f.cross_attention(qt, kt, vt)
    want = torch.zeros((H, D))
    want[0, 3], want[0, 9], want[1, 5] = np.inf, -np.inf, -np.inf
    for h in range(Hq):
        w = want[h // 2]
        there = torch.isinf(w)
        assert (out[0, :, h].float().cpu()[:, there] == w[there]).all()
        finite = np.where(np.isfinite(v[0, :, h // 2]), v[0, :, h // 2], 0.0)
        got = out[0, :, h].clone()
        got[:, there.to(DEV)] = 0
        other = finite.copy()
        other[:, there.numpy()] = 0
        check_rows(got, q[0, :, h], k[0, :, h // 2], other, np.ones((Sq, Sk), dtype=bool), D ** -0.5, f"head {h}")


@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("Sq,Sk", SIZES)
def test_a_sample_that_sees_nothing_is_zeros_whatever_its_queries_hold(Sq, Sk, D):
    f = fq()
    flush(f"nothing seen Sq={Sq} Sk={Sk} D={D}")
    rng = np.random.default_rng(Sq + D)
    B, Hq, H = 3, 4, 2
    q = rng.standard_normal((B, Sq, Hq, D))
    q[1, 0] = rng.choice([np.nan, np.inf, -np.inf], (Hq, D))
    q[1, Sq - 1, 2, 3] = np.nan
    q[2, Sq // 2, 1, 0] = np.nan
    kv = bf16(rng.standard_normal((B, Sk, 2 * H, D)))[1]
    mask = rng.random((B, Sk)) < 0.5
    mask[1] = False
    out = f.cross_attention(bf16(q)[1], kv[:, :, :H], kv[:, :, H:], None, torch.from_numpy(mask).to(DEV))
    assert (out[1] == 0).all()
    nan = torch.isnan(out).cpu().numpy()
    assert nan[2, Sq // 2, 1].all() and nan.any(axis=3).sum() == 1
