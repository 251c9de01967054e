"""What repeated appends to a page cost: bounds that follow from the roundings, on the oracle's page (CPU) and the
library's (GPU)."""
import numpy as np
import pytest
import torch

from oracle import attention as ref
from paper_2609_24433_amd import fq
from tests.attention_util import bf16, ints, native_v, plain_v
from tests.gpu_util import flush

D = 64


def tokens(kind, P, seed=0):
    """[P, D] values that bf16 holds: normal, or each token's largest a little above the last one's."""
    rng = np.random.default_rng(seed + P)
    x = rng.standard_normal((P, D))
    if kind == "rising":
        x = x / np.abs(x).max(axis=1, keepdims=True) * (1.008 ** np.arange(P))[:, None]
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def half_sums(scales):
    """Per token of a page filled one at a time, its bound from the page's scale after every append: half of the scale it
    was written under and of every scale that rose after it."""
    s = np.asarray(scales, dtype=np.float64)
    rose = np.concatenate(([0.0], np.where(s[1:] != s[:-1], s[1:], 0.0)))
    later = rose[::-1].cumsum()[::-1] - rose
    return 0.5 * (s + later)


def geometric(growth, last):
    g = 1 + growth / 100
    return 0.5 * g / (g - 1) * last


EPS = 1 + 2.0 ** -13  # fp32 on the way: a ratio, a reciprocal and a product, each 2^-24 of up to 127 steps


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", ["normal", "rising"])
@pytest.mark.parametrize("growth", [0, 10, 25, 100])
def test_a_page_filled_token_by_token(P, kind, growth):
    x = tokens(kind, P)
    codes, scale, scales = np.zeros((P, D), np.int8), np.float32(0), []
    for i in range(P):
        codes, scale = ref.append_page(x[i:i + 1].astype(np.float32), codes, scale, i, growth)
        scales.append(scale)
    err = np.abs(codes * np.float64(scale) - x).max(axis=1)
    assert (err <= EPS * half_sums(scales)).all()
    need = np.abs(x).max() / 127
    if growth:
        assert err.max() <= EPS * geometric(growth, float(scale)) and scale <= EPS * need * (1 + growth / 100)
    else:
        assert abs(scale / need - 1) < 1e-6
        # what the bound is for: small raises add up
        assert err.max() > (P / 8 if kind == "rising" else 0.5) * scale
    # the same page at once, and again from its first slot
    once, s = ref.append_page(x.astype(np.float32), codes, scale, 0, growth)
    assert np.abs(once * np.float64(s) - x).max() <= EPS * 0.5 * s


@pytest.mark.parametrize("value", [-1, 101, 1 << 20])
def test_growth_outside_its_range_is_refused(value, monkeypatch):
    """(through the C ABI: nothing is launched)"""
    A = 0x100000
    cache = fq._CACHE(A, 2 * A, 3 * A, 4 * A, 8, 2, 64, 64, value)
    batch = fq._BATCH(5 * A, 6 * A, 7 * A, 4, 2, 3, 200)
    heads = fq._HEADS(8 * A, 0, 512, 64)
    assert fq.LIB.fq_cache_append(cache, batch, heads, heads, None, 0, None, 5, None, None) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("kind", ["normal", "rising"])
@pytest.mark.parametrize("growth", [0, 25])
def test_the_librarys_page_filled_token_by_token(P, kind, growth):
    """Bit for bit the oracle's page, and within the bounds, for keys and values; then appended again from its first slot."""
    flush(f"token by token P={P} {kind} growth={growth}")
    cache = fq.kv_cache(3, 2, P, D)
    table = ints([[1]])
    k, v = tokens(kind, P), tokens(kind, P, 7)
    kt, vt = (bf16(np.stack((t, -2 * t), axis=1))[1] for t in (k, v))
    want = [[np.zeros((P, D), np.int8), np.float32(0)] for _ in range(4)]
    values = [k, -2 * k, v, -2 * v]
    scales = [[] for _ in range(4)]
    for i in range(P):
        fq.cache_append(cache, table, ints([0, 1]), ints([i + 1]), 1, kt[i:i + 1], vt[i:i + 1], growth=growth)
        for j in range(4):
            want[j] = ref.append_page(values[j][i:i + 1].astype(np.float32), *want[j], i, growth)
            scales[j].append(want[j][1])
    codes = [*cache.k_codes[1].cpu().numpy(), *plain_v(cache.v_codes.cpu().numpy())[1]]
    got = [*cache.k_scale[1].cpu().numpy(), *cache.v_scale[1].cpu().numpy()]
    for j in range(4):
        assert got[j] == want[j][1] and np.array_equal(codes[j], want[j][0])
        err = np.abs(codes[j] * np.float64(got[j]) - values[j]).max(axis=1)
        assert (err <= EPS * half_sums(scales[j])).all()
        if growth:
            assert err.max() <= EPS * geometric(growth, float(got[j]))
    fq.cache_append(cache, table, ints([0, P]), ints([P]), P, kt, vt, growth=growth)
    codes = [*cache.k_codes[1].cpu().numpy(), *plain_v(cache.v_codes.cpu().numpy())[1]]
    got = [*cache.k_scale[1].cpu().numpy(), *cache.v_scale[1].cpu().numpy()]
    for j in range(4):
        assert np.abs(codes[j] * np.float64(got[j]) - values[j]).max() <= EPS * 0.5 * got[j]


@pytest.mark.gpu
def test_growth_on_a_page_in_use_is_the_contract_bit_for_bit():
    flush("growth on pages in use")
    rng = np.random.default_rng(5)
    P, H, m = 32, 2, 50
    codes = [rng.integers(-127, 128, (2, H, P, D)).astype(np.int8) for _ in range(2)]
    for growth, factor in ((25, 1.1), (25, 1.4), (25, 0.9), (100, 1.01), (7, 1.0001), (0, 1.1)):
        x = rng.standard_normal((10, H, D))
        xt = bf16(x)[1]
        x = xt.double().cpu().numpy()  # [10, H, D]: slots 40 to 49 of the second page
        old = (np.abs(x).max(axis=(0, 2)) / 127 / factor).astype(np.float32)
        scale = np.stack((np.ones(H, np.float32), old))
        cache = fq.KVCache(*(torch.from_numpy(a).to(xt.device) for a in (codes[0], scale.copy(), native_v(codes[1]), scale.copy())))
        fq.cache_append(cache, ints([[0, 1]]), ints([0, 10]), ints([m]), 10, xt, xt, growth=growth)
        kc, vc = cache.k_codes.cpu().numpy(), plain_v(cache.v_codes.cpu().numpy())
        ks, vs = cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()
        for got_c, got_s, c in ((kc, ks, codes[0]), (vc, vs, codes[1])):
            for h in range(H):
                want_c, want_s = ref.append_page(x[:, h].astype(np.float32), c[1, h], scale[1, h], 8, growth)
                assert got_s[1, h] == want_s and np.array_equal(got_c[1, h, :18], want_c[:18]), (growth, factor)
            assert np.array_equal(got_c[0], c[0])
