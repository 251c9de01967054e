"""fq_cache_attention and fq_cross_attention on the GPU against the definition in 64 bits, within a tolerance derived
from the roundings (oracle.attention.tolerance)."""
import numpy as np
import pytest
import torch

from tests.attention_util import bf16, check_rows, ints, make_cache, make_table, native_v, sequence, to_device
from tests.gpu_util import DEV, flush

pytestmark = pytest.mark.gpu


def fq():
    from paper_2609_24433_amd import fq as _fq
    return _fq


def run_cached(n, lens, Hq, H, D, P, causal, seed=0, scale=None, qscale=1.5, spread=1.0, edit=None):
    f = fq()
    flush(f"cached n={n} lens={lens} Hq={Hq} H={H} D={D} P={P} causal={causal}")
    rng = np.random.default_rng(seed + D + P + sum(lens))
    table, kc, ks, vc, vs = make_cache(rng, lens, P, H, D, spread)
    T = sum(n)
    q, qt = bf16(rng.standard_normal((T, Hq, D)) * qscale)
    if edit:
        edit(table, kc, ks, vc, vs, q)
        q, qt = bf16(q)
    cache = to_device(kc, ks, vc, vs)
    out = f.cache_attention(qt, cache, ints(table), ints(np.concatenate(([0], np.cumsum(n)))), ints(lens), max(n), max(lens + [1]),
                            scale, causal)
    torch.cuda.synchronize()
    G, row = Hq // H, 0
    for b, m in enumerate(lens):
        j, i = np.arange(m)[None, :], np.arange(n[b])[:, None]
        seen = (j <= m - n[b] + i) if causal else np.ones((n[b], m), dtype=bool)
        for h in range(H):
            k, v = sequence(table, kc, ks, b, m, h), sequence(table, vc, vs, b, m, h)
            for g in range(G):
                check_rows(out[row:row + n[b], h * G + g], q[row:row + n[b], h * G + g], k, v, seen, scale or D ** -0.5,
                           f"sequence {b} head {h * G + g}")
        row += n[b]
    return out


@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 128, 144, 192, 240, 256])
@pytest.mark.parametrize("n,lens", [([1], [1]), ([1, 1, 1], [17, 64, 200]), ([40], [130]), ([150, 3], [150, 99])])
def test_head_sizes(D, n, lens):
    run_cached(n, lens, 4, 2, D, 32, True)


@pytest.mark.parametrize("Hq,H", [(1, 1), (5, 1), (6, 2), (16, 2), (33, 1), (8, 8), (40, 1)])
@pytest.mark.parametrize("n,lens", [([1, 1], [63, 65]), ([3, 2], [129, 31]), ([70], [100])])
def test_groups_of_heads(Hq, H, n, lens):
    run_cached(n, lens, Hq, H, 64, 64, True)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,lens", [([1, 1, 1, 1, 1], [1, 15, 16, 17, 129]), ([2, 64, 31], [128, 127, 33]), ([257], [300])])
def test_pages_that_end_anywhere(P, causal, n, lens):
    run_cached(n, lens, 8, 2, 128, P, causal)


@pytest.mark.parametrize("causal", [True, False])
def test_empty_sequences_and_rows_that_see_nothing(causal):
    # no rows; rows but no tokens; fewer tokens than rows (causal: the first rows see nothing)
    out = run_cached([0, 4, 6, 1], [20, 0, 2, 5], 4, 2, 64, 16, causal)
    assert (out[:4] == 0).all()
    if causal:
        assert (out[4:8] == 0).all() and (out[8:] != 0).any()


@pytest.mark.parametrize("n,lens,Hq,H,D", [([1], [5003], 8, 2, 128), ([1, 1], [4096, 777], 8, 1, 256), ([2], [9001], 4, 4, 64),
                                           ([20], [3001], 8, 1, 256), ([1] * 3, [2050, 1, 700], 16, 2, 80)])
@pytest.mark.parametrize("causal", [True, False])
def test_long_contexts_for_few_rows(n, lens, Hq, H, D, causal):
    run_cached(n, lens, Hq, H, D, 64, causal, spread=3.0)


@pytest.mark.parametrize("n,lens,Hq,H,D,P", [([513], [1029], 8, 2, 128, 64), ([300, 90], [300, 700], 8, 1, 256, 32),
                                             ([260], [1500], 4, 4, 64, 16), ([129], [640], 6, 2, 96, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows(n, lens, Hq, H, D, P, causal):
    run_cached(n, lens, Hq, H, D, P, causal)


def test_scales_of_pages_over_many_octaves_and_scores_far_apart():
    run_cached([1, 30], [700, 300], 4, 2, 128, 16, True, spread=20.0)
    run_cached([1, 30], [700, 300], 4, 2, 128, 16, True, qscale=60.0)
    run_cached([1, 30, 200], [700, 300, 500], 4, 2, 64, 32, True, scale=0.7, qscale=8.0)

    def grow(table, kc, ks, vc, vs, q):  # scores rise along the sequence: the running maximum moves at every step
        for w in range(table.shape[1] - 2):
            for b in range(2):
                if table[b, w] < len(ks):
                    ks[table[b, w]] = 2.0 ** (-8 + 0.25 * w)
    run_cached([1, 140], [900, 900], 4, 2, 64, 16, False, edit=grow)

    def silent(table, kc, ks, vc, vs, q):  # pages of zeros
        ks[table[0, 1]] = 0
        vs[table[0, 2]] = 0
    run_cached([1], [300], 4, 2, 64, 64, True, edit=silent)


def test_a_poisoned_page_reaches_those_that_see_it():
    f = fq()
    rng = np.random.default_rng(1)
    for n in (1, 5, 100):
        P, H, D, m = 16, 2, 64, 200
        table, kc, ks, vc, vs = make_cache(rng, [m], P, H, D)
        ks[table[0, 9], 1] = np.nan  # tokens 144 to 159 of head 1
        vs[table[0, 11], 0] = np.nan  # tokens 176 to 191 of head 0
        qt = bf16(rng.standard_normal((n, 4, D)))[1]
        out = f.cache_attention(qt, to_device(kc, ks, vc, vs), ints(table), ints([0, n]), ints([m]), n, m)
        nan = torch.isnan(out).cpu().numpy()
        assert (nan.any(axis=2) == nan.all(axis=2)).all()
        at = m - n + np.arange(n)
        for h, first in ((0, 176), (1, 144)):
            for g in range(2):
                assert np.array_equal(nan[:, 2 * h + g, 0], at >= first), (n, h)


def test_a_query_that_is_not_finite_stays_alone():
    f = fq()
    rng = np.random.default_rng(2)
    for n, m in ((1, 100), (50, 60), (300, 400)):
        table, kc, ks, vc, vs = make_cache(rng, [m], 32, 2, 64)
        q = rng.standard_normal((n, 4, 64))
        q[n // 2, 3, 5] = np.nan
        out = f.cache_attention(bf16(q)[1], to_device(kc, ks, vc, vs), ints(table), ints([0, n]), ints([m]), n, m)
        nan = torch.isnan(out).any(dim=2).cpu().numpy()
        assert nan[n // 2, 3] and nan.sum() == 1


def test_a_pool_beyond_32_bit_offsets():
    f = fq()
    rng = np.random.default_rng(6)
    H, P, D, m = 8, 128, 128, 300
    pages = (1 << 32) // (H * P * D) + 40  # 4 GiB of codes and some
    cache = f.kv_cache(pages, H, P, D)
    table = np.array([[pages - 1, pages - 33, 3]])
    kc, vc = (rng.integers(-127, 128, (3, H, P, D)).astype(np.int8) for _ in range(2))
    ks, vs = (rng.uniform(0.01, 0.02, (3, H)).astype(np.float32) for _ in range(2))
    at = torch.from_numpy(table[0]).to(DEV)
    for t, x in zip(cache, (kc, ks, native_v(vc), vs)):
        t[at] = torch.from_numpy(x).to(DEV)
    for n in (1, 200):
        q, qt = bf16(rng.standard_normal((n, H, D)))
        out = f.cache_attention(qt, cache, ints(table), ints([0, n]), ints([m]), n, m)
        local = np.array([[0, 1, 2]])
        seen = np.arange(m)[None, :] <= m - n + np.arange(n)[:, None]
        for h in (0, H - 1):
            check_rows(out[:, h], q[:, h], sequence(local, kc, ks, 0, m, h), sequence(local, vc, vs, 0, m, h), seen, D ** -0.5, f"n={n} h={h}")
    x, xt = bf16(rng.standard_normal((5, H, D)))
    f.cache_append(cache, ints(table[:, :1]), ints([0, 5]), ints([5]), 5, xt, xt)
    k, v = f.cache_read(cache, ints(table[:, :1]), ints([0]), ints([5]), 5)
    # a value is within half a step of its page and head, and bf16's rounding
    step = np.abs(x).max(axis=(0, 2), keepdims=True) / 127
    for t in (k, v):
        assert (np.abs(t[0].double().cpu().numpy() - x) <= 0.501 * step + 2.0 ** -8 * np.abs(x)).all()


# ---------------------------------------------------------------- cross attention

def run_cross(B, Sq, Sk, Hq, H, D, lens=None, mask=None, layout="packed", junk=False, seed=0):
    f = fq()
    flush(f"cross B={B} Sq={Sq} Sk={Sk} Hq={Hq} H={H} D={D} lens={lens} mask={mask is not None} {layout}")
    rng = np.random.default_rng(seed + B + Sq + Sk + D)
    seen = np.ones((B, Sk), dtype=bool) if mask is None else mask.copy()
    if lens is not None:
        seen &= np.arange(Sk)[None, :] < np.asarray(lens)[:, None]
    q, qt = bf16(rng.standard_normal((B, Sq, Hq, D)) * 1.5)
    kv = rng.standard_normal((B, Sk, 2 * H, D))
    if junk:  # what lies in unseen places
        kv[~seen] = rng.choice([np.nan, np.inf, -np.inf, 1e38], kv[~seen].shape)
    kv, kvt = bf16(kv)
    k, v, kt, vt = kv[:, :, :H], kv[:, :, H:], kvt[:, :, :H], kvt[:, :, H:]
    if layout == "heads":  # [B, H, S, D] in memory
        qt = qt.transpose(1, 2).contiguous().transpose(1, 2)
        kt, vt = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kt, vt))
    elif layout == "shared":  # one sample's states for the whole batch, one head for all
        kt, vt = (t[:1, :, :1].expand(B, Sk, H, D) for t in (kt, vt))
        k, v = (np.broadcast_to(t[:1, :, :1], t.shape) for t in (k, v))
    m = None if mask is None else torch.from_numpy(mask).to(DEV)
    out = f.cross_attention(qt, kt, vt, None if lens is None else ints(lens), m)
    torch.cuda.synchronize()
    G = Hq // H
    for b in range(B):
        for h in range(Hq):
            rows = np.broadcast_to(seen[b], (Sq, Sk))
            check_rows(out[b, :, h], q[b, :, h], k[b, :, h // G], v[b, :, h // G], rows, D ** -0.5, f"sample {b} head {h}")
    return out


@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 112, 128, 160, 192, 256])
@pytest.mark.parametrize("Sq,Sk", [(1, 1), (1, 333), (50, 816), (77, 65)])
def test_cross_head_sizes(D, Sq, Sk):
    run_cross(2, Sq, Sk, 4, 2, D)


@pytest.mark.parametrize("Sq,Sk", [(1, 1500), (3, 64), (16, 63), (17, 128), (33, 127), (130, 129), (300, 1000), (1, 6001)])
@pytest.mark.parametrize("Hq,H", [(4, 4), (8, 2), (6, 1)])
def test_cross_lengths(Sq, Sk, Hq, H):
    run_cross(1, Sq, Sk, Hq, H, 64)


@pytest.mark.parametrize("Sq", [1, 5, 40, 200])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_cross_masks_lengths_and_what_lies_in_unseen_places(Sq, D):
    rng = np.random.default_rng(Sq)
    B, Sk = 5, 201
    mask = rng.random((B, Sk)) < 0.6
    mask[1] = False  # sees nothing
    mask[3, :130] = False  # whole steps masked before the first seen key
    lens = [Sk, Sk, 0, 190, 1]
    mask[4, 0] = True
    out = run_cross(B, Sq, Sk, 4, 2, D, lens, mask, junk=True)
    assert (out[1] == 0).all() and (out[2] == 0).all()
    run_cross(B, Sq, Sk, 4, 2, D, lens, None, junk=True)
    run_cross(B, Sq, Sk, 4, 2, D, None, mask, junk=True)


@pytest.mark.parametrize("layout", ["packed", "heads", "shared"])
@pytest.mark.parametrize("Sq", [1, 30, 150])
def test_cross_layouts(layout, Sq):
    run_cross(3, Sq, 270, 8, 4, 64, layout=layout)


def test_cross_broadcast_mask_and_no_states():
    f = fq()
    rng = np.random.default_rng(11)
    q, qt = bf16(rng.standard_normal((3, 4, 2, 64)))
    k, kt = bf16(rng.standard_normal((3, 90, 2, 64)))
    mask = rng.random(90) < 0.5
    m = torch.from_numpy(mask).to(DEV)[None].expand(3, 90)
    out = f.cross_attention(qt, kt, kt, None, m)
    for b in range(3):
        check_rows(out[b, :, 1], q[b, :, 1], k[b, :, 1], k[b, :, 1], np.broadcast_to(mask, (4, 90)), 0.125, "broadcast")
    empty = torch.empty((3, 0, 2, 64), dtype=torch.bfloat16, device=DEV)
    assert (f.cross_attention(qt, empty, empty) == 0).all()
    assert f.cross_attention(qt[:0], kt[:0], kt[:0]).shape == (0, 4, 2, 64)


# ---------------------------------------------------------------- streams, graphs, workspaces

def test_on_another_stream_and_in_a_graph():
    """Appends and attention of a decoding step on a side stream, then captured and replayed between eager work: every
    replay equals the eager results."""
    f = fq()
    rng = np.random.default_rng(12)
    B, Hq, H, D, P = 3, 8, 2, 128, 64
    lens = [2000, 65, 513]
    table, kc, ks, vc, vs = make_cache(rng, lens, P, H, D)
    cache = to_device(kc, ks, vc, vs)
    x = bf16(rng.standard_normal((B, Hq + 2 * H, D)))[1]
    enc = bf16(rng.standard_normal((B, 700, 2 * H, D)))[1]
    rope = torch.from_numpy(make_table(2000, D)).to(DEV)
    pt, qs, kl = ints(table), ints([0, 1, 2, 3]), ints(lens)
    ws = f.workspace(max(f.cache_attention_workspace_bytes(B, Hq, H, D, B, 1, 2000),
                         f.cross_attention_workspace_bytes(B, 1, 700, Hq, H, D)), DEV)

    def step():
        q = f.cache_append(cache, pt, qs, kl, 1, x[:, Hq:Hq + H], x[:, Hq + H:], x[:, :Hq], rope)
        a = f.cache_attention(q, cache, pt, qs, kl, 1, 2000, ws=ws)
        return a, f.cross_attention(a[:, None], enc[:, :, :H], enc[:, :, H:], ws=ws)
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            held = step()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    for _ in range(4):
        for t in held:
            t.fill_(7.0)
        ws.fill_(255)  # a workspace needs no initialization
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, held):
            assert torch.equal(a, b)


def test_a_call_repeats_bit_for_bit_with_any_workspace():
    f = fq()
    rng = np.random.default_rng(13)
    for n, m in ((1, 6000), (60, 900), (400, 1200)):
        table, kc, ks, vc, vs = make_cache(rng, [m], 64, 2, 128)
        cache = to_device(kc, ks, vc, vs)
        qt = bf16(rng.standard_normal((n, 8, 128)))[1]
        args = (qt, cache, ints(table), ints([0, n]), ints([m]), n, m)
        need = f.cache_attention_workspace_bytes(n, 8, 2, 128, 1, n, m)
        want = f.cache_attention(*args)
        for fill in (0, 255):
            ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device=DEV)
            assert torch.equal(f.cache_attention(*args, ws=ws[:max(need, 256)]), want)
            assert (ws[max(need, 256):] == fill).all()


def test_bounds_beyond_the_lengths_change_nothing():
    """max_new and max_kv are bounds: larger ones give the same rows, within the tolerance of another split."""
    f = fq()
    rng = np.random.default_rng(14)
    lens, n = [300, 40], [2, 3]
    table, kc, ks, vc, vs = make_cache(rng, lens, 16, 2, 64)
    table = np.concatenate([table, np.full((2, 600), -1)], axis=1)
    q, qt = bf16(rng.standard_normal((5, 4, 64)))
    cache = to_device(kc, ks, vc, vs)
    for max_new, max_kv in ((3, 300), (50, 300), (3, 9000), (200, 9000)):
        out = f.cache_attention(qt, cache, ints(table), ints([0, 2, 5]), ints(lens), max_new, max_kv)
        row = 0
        for b in range(2):
            seen = np.arange(lens[b])[None, :] <= lens[b] - n[b] + np.arange(n[b])[:, None]
            for h in range(4):
                check_rows(out[row:row + n[b], h], q[row:row + n[b], h], sequence(table, kc, ks, b, lens[b], h // 2),
                           sequence(table, vc, vs, b, lens[b], h // 2), seen, 0.125, f"{max_new} {max_kv}")
            row += n[b]
