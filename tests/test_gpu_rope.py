"""fq_rope_table and fq_qk_rope on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import attention as ref
from tests.attention_util import bf16, ints, make_table
from tests.gpu_util import DEV, flush

pytestmark = pytest.mark.gpu


def fq():
    from paper_2609_24433_amd import fq as _fq
    return _fq


def check(got, x, table, pos, w, eps, inter, what):
    """One bf16 rounding of the result (half a step of 8 significant bits: 2^-8), and fp32 arithmetic: the norm's sum of D squares, and a rotation of two
    products, each a few units of 2^-24 of the pair's size."""
    want = ref.norm_rotate(x, table, pos, w, eps, inter)
    plain = np.abs(ref.norm_rotate(x, None, None, w, eps, inter))
    D = x.shape[-1]
    size = plain.copy()
    if table is not None:
        half = table.shape[1]
        i = np.arange(half)
        one, two = (2 * i, 2 * i + 1) if inter else (i, i + half)
        size[..., one] = size[..., two] = plain[..., one] + plain[..., two]
    tol = 1.01 * 2.0 ** -8 * np.abs(want) + (D + 16) * 2.0 ** -24 * size + 1e-38
    g = got.double().cpu().numpy()
    assert g.shape == want.shape
    assert (np.abs(g - want) <= tol).all(), (what, np.abs(g - want).max())


@pytest.mark.parametrize("T,Hq,Hk,D,R,inter,norm", [
    (1, 1, 1, 16, 16, False, True), (1, 32, 8, 128, 128, False, True), (7, 3, 1, 48, 32, False, True),
    (50, 8, 1, 256, 256, False, False), (33, 5, 5, 80, 80, True, True), (65, 12, 4, 96, 48, True, False),
    (130, 4, 2, 240, 16, False, True), (3, 2, 1, 32, 0, False, True), (3, 2, 1, 64, 0, False, False),
    (1000, 32, 8, 128, 64, True, True), (2049, 9, 3, 112, 96, False, True), (17, 1, 0, 144, 144, False, True),
])
def test_qk_rope(T, Hq, Hk, D, R, inter, norm):
    f = fq()
    flush(f"qk_rope T={T} Hq={Hq} Hk={Hk} D={D} R={R} inter={inter} norm={norm}")
    rng = np.random.default_rng(T * 7 + D)
    x, xt = bf16(rng.standard_normal((T, Hq + 2 * Hk, D)) * np.exp(rng.standard_normal((T, Hq + 2 * Hk, 1))))
    q, k = xt[:, :Hq], xt[:, Hq:Hq + Hk]  # columns of one packed projection
    table = make_table(3 * T + 2, R) if R else None
    pos = rng.permutation(3 * T + 2)[:T]
    w = [rng.uniform(0.5, 2.0, D).astype(np.float32) if norm else None for _ in range(2)]
    dev = [None if a is None else torch.from_numpy(a).to(DEV) for a in (table, *w)]
    yq, yk = f.qk_rope(q, k if Hk else None, dev[0], ints(pos), dev[1], dev[2], eps=1e-5, interleaved=inter)
    torch.cuda.synchronize()
    check(yq, x[:, :Hq], table, pos, w[0], 1e-5, inter, "q")
    if Hk:
        check(yk, x[:, Hq:Hq + Hk], table, pos, w[1], 1e-5, inter, "k")


def test_rows_of_other_strides_and_default_positions():
    f = fq()
    rng = np.random.default_rng(3)
    T, Hq, Hk, D = 21, 4, 2, 64
    q, qt = bf16(rng.standard_normal((Hq, T, D)))  # heads first
    k, kt = bf16(rng.standard_normal((T, Hk, 2, D)))
    table = make_table(T, D)
    yq, yk = f.qk_rope(qt.transpose(0, 1), kt[:, :, 1], torch.from_numpy(table).to(DEV))
    torch.cuda.synchronize()
    check(yq, q.transpose(1, 0, 2), table, np.arange(T), None, 0.0, False, "heads first")
    check(yk, k[:, :, 1], table, np.arange(T), None, 0.0, False, "every other")


def test_positions_outside_the_table_are_clamped_and_long_tables_keep_their_angle():
    f = fq()
    rng = np.random.default_rng(4)
    L, R = 200001, 64
    inv, mag = f.rope_frequencies(R, scaling="by_parts", factor=8.0, original_length=4096)
    table = f.rope_table(L, inv, mag)
    a = np.arange(L)[:, None] * inv.numpy()[None]
    want = mag * np.stack([np.cos(a), np.sin(a)], axis=-1)
    # one rounding of a value up to `mag` to fp32, and the fp64 angle's own: 2e5 * 2^-52
    assert np.abs(table.cpu().numpy() - want).max() <= mag * (2.0 ** -24 + 1e-10)
    x, xt = bf16(rng.standard_normal((4, 2, R)))
    pos = np.array([-5, L + 10, 2 ** 31 - 1, L - 1])
    yq, _ = f.qk_rope(xt, None, table, ints(pos))
    check(yq, x, table.cpu().numpy(), pos, None, 0.0, False, "clamped")


def test_zero_and_non_finite_rows_stay_alone():
    f = fq()
    T, H, D = 5, 3, 128
    x = np.random.default_rng(5).standard_normal((T, H, D))
    x[1, 1] = 0.0
    x[2, 0, 7] = np.nan
    x[3, 2, 9] = np.inf
    _, xt = bf16(x)
    w = torch.ones(D, device=DEV)
    y, _ = f.qk_rope(xt, None, torch.from_numpy(make_table(T, D)).to(DEV), q_weight=w)
    fine = torch.isfinite(y).all(dim=-1).cpu()
    assert (y[1, 1] == 0).all()
    want = torch.ones((T, H), dtype=torch.bool)
    want[2, 0] = want[3, 2] = False
    assert torch.equal(fine, want)


def test_no_tokens_is_no_call():
    f = fq()
    y, _ = f.qk_rope(torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV), None, None)
    assert y.shape == (0, 4, 64)
