"""Microscaled 4-bit quantization and products on the GPU against the plain reference: codes and scales bit for bit, values
exactly, products within the bound of their sums."""
import numpy as np
import pytest
import torch

from oracle import microscaled as mx
from tests.gpu_util import DEV, flush
from tests.mx_util import HALF_BF16, assert_product, dev, dev_bf16, fq, operands, strided, tokens

pytestmark = pytest.mark.gpu


def check_codes(codes, scales, u):
    want, ws = mx.encode(u)
    got, gs = mx.split_nibbles(codes.cpu().numpy()), mx.rows(scales.cpu().numpy())
    assert np.array_equal(gs, ws), np.argwhere(gs != ws)[:4]
    assert np.array_equal(got, want), np.argwhere(got != want)[:4]


@pytest.mark.parametrize("M,K", [(1, 128), (3, 256), (17, 384), (8, 1024), (50, 1152), (9, 4096), (5, 16384), (2, 32768), (257, 640)])
@pytest.mark.parametrize("b", [1, 2, 4, 8, 16, 32, 64, 128, 256])
def test_tokens(M, K, b):
    if K % b:
        pytest.skip("b does not divide K")
    flush(f"mx_quant M={M} K={K} b={b}")
    x = tokens(M, K, 100 + M + K)
    codes, scales = fq().mx_quant(strided(x), b)
    check_codes(codes, scales, mx.fold(x, b))
    got = fq().mx_read(codes, scales).float().cpu().numpy().astype(np.float64)
    assert np.array_equal(got, mx.decode(*mx.encode(mx.fold(x, b))), equal_nan=True)  # sums of large rows overflow


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("pre,post", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("M,K,b", [(1, 128, 1), (40, 896, 64), (16, 2048, 256), (33, 384, 128)])
def test_folds(M, K, b, pre, post, f32):
    r = np.random.default_rng(M + K)
    x = (r.standard_normal((M, K)) * 0.02).astype(np.float32) if f32 else tokens(M, K, 7)
    p = r.uniform(0.3, 3.0, K).astype(np.float32) if pre else None
    q = r.uniform(0.3, 3.0, K).astype(np.float32) if post else None
    t = dev(x) if f32 else strided(x)
    codes, scales = fq().mx_quant(t, b, None if p is None else dev(p), None if q is None else dev(q))
    check_codes(codes, scales, mx.fold(x, b, p, q))


@pytest.mark.parametrize("b", [1, 64])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_value_that_is_not_finite_spoils_its_block_only(b, value):
    x = tokens(3, 512, 5, special=False)
    x[1, 200] = value
    codes, scales = fq().mx_quant(dev_bf16(x), b)
    check_codes(codes, scales, mx.fold(x, b))
    bad = mx.rows(scales.cpu().numpy()) == 255
    assert bad[1, 200 // 32] and bad.sum() == max(1, b // 32) and not bad[0].any() and not bad[2].any()
    values = fq().mx_read(codes, scales).float().cpu().numpy()
    assert np.array_equal(np.isnan(values), np.repeat(bad, 32, axis=1))
    w, sw = operands(16, 512, 1)
    y = fq().mx_gemm(codes, scales, fq().mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw))).float().cpu().numpy()
    assert np.isnan(y[1]).all() and np.isfinite(y[[0, 2]]).all()


def test_sums_that_overflow_in_the_rotation_are_not_finite():
    x = np.zeros((2, 128), dtype=np.float32)
    x[1, :64] = 3e38
    codes, scales = fq().mx_quant(dev_bf16(x), 128)
    assert (mx.rows(scales.cpu().numpy())[1] == 255).any() and (mx.rows(scales.cpu().numpy())[0] == 0).all()


def test_every_code_and_scale_as_values():
    """All bytes under all scales, into rows of a longer stride."""
    n = np.tile(np.arange(16, dtype=np.uint8), 8)
    s = np.arange(256, dtype=np.uint8).repeat(4).reshape(256, 4)
    codes = np.repeat(mx.pack_nibbles(n[None]), 256, axis=0)
    out = torch.full((256, 160), 7.0, dtype=torch.bfloat16, device=DEV)
    fq().mx_read(dev(codes), dev(mx.steps(s)), out[:, :128])
    want = torch.from_numpy(mx.decode(np.repeat(n[None], 256, axis=0), s)).to(torch.bfloat16)  # the largest overflow
    assert torch.equal(out[:, :128].cpu().isnan(), want.isnan()) and bool((out[:, 128:] == 7).all())
    assert torch.equal(out[:, :128].cpu().nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("M,K", [(1, 128), (7, 896), (300, 256), (3, 32768)])
def test_codes_with_a_token_scale_as_values(M, K, bits):
    q = 127 if bits == 8 else 7
    r = np.random.default_rng(K)
    c = r.integers(-q, q + 1, (M, K)).astype(np.int8)
    d = r.uniform(0.01, 2.0, M).astype(np.float32)
    raw = c.view(np.uint8) if bits == 8 else mx.pack_nibbles((c & 15).astype(np.uint8))
    got = fq().read_codes(dev(raw), dev(d), bits)
    assert torch.equal(got.cpu(), torch.from_numpy(c.astype(np.float32) * d[:, None]).to(torch.bfloat16))


@pytest.mark.parametrize("N,K", [(16, 128), (48, 896), (272, 2048), (16, 32768)])
def test_packing(N, K):
    n, _ = operands(N, K, N)
    codes = mx.pack_nibbles(n)
    packed = fq().mx_pack(dev(codes))
    assert np.array_equal(packed.cpu().numpy(), mx.tiles(codes))
    assert np.array_equal(fq().mx_unpack(packed).cpu().numpy(), codes)


ROWS = [1, 2, 15, 16, 17, 33, 50, 64, 65, 100, 129, 257]


@pytest.mark.parametrize("N,K", [(16, 128), (48, 256), (80, 384), (272, 1152), (1040, 640), (64, 4224), (32, 16384), (16, 32768)])
@pytest.mark.parametrize("M", ROWS)
def test_product(M, N, K):
    flush(f"mx_gemm M={M} N={N} K={K}")
    a, sa = operands(M, K, M + K)
    w, sw = operands(N, K, N + K + 1)
    bias = np.random.default_rng(3).standard_normal(N).astype(np.float32) * 100 if M % 2 else None
    out = torch.full((M + 1, N + 16), 5.0, dtype=torch.bfloat16, device=DEV)
    args = (dev(mx.pack_nibbles(a)), dev(mx.steps(sa)), fq().mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw)), None if bias is None else dev(bias))
    fq().mx_gemm(*args, out=out[:M, :N])
    assert_product(out[:M, :N], mx.decode(a, sa), mx.decode(w, sw), bias)
    assert bool((out[M:] == 5).all()) and bool((out[:, N:] == 5).all())
    assert torch.equal(fq().mx_gemm(*args), out[:M, :N])  # the same bits again, into rows of another stride


# every kernel and way of splitting K that the sizes choose: tiles of 64 x 64 to 256 x 256, one a workgroup and several, K
# ending inside a step, whole and in slices with a short last one
@pytest.mark.parametrize("M,N,K", [(300, 512, 512), (513, 784, 1024), (1000, 272, 4096), (700, 2048, 384), (2049, 1040, 256),
                                   (260, 16384, 128), (816, 16384, 640), (2100, 8208, 384), (1500, 4112, 896), (4100, 4112, 1152),
                                   (300, 256, 16384), (520, 2048, 8320), (816, 2048, 16384), (390, 272, 32768), (260, 1024, 7552),
                                   (3000, 16384, 2176), (129, 32768, 256), (1338, 64, 12032), (620, 752, 12928), (1100, 80, 32640),
                                   (116, 1504, 2944), (240, 928, 8064), (287, 2112, 4736), (75, 5728, 1920), (344, 2320, 384), (704, 1600, 2688),
                                   (1165, 176, 10368), (1113, 1872, 27264), (170, 5616, 28288)])
def test_product_of_many_rows(M, N, K):
    flush(f"mx_gemm M={M} N={N} K={K}")
    a, sa = operands(M, K, M)
    w, sw = operands(N, K, N)
    bias = np.random.default_rng(3).standard_normal(N).astype(np.float32) * 100 if M % 2 else None
    out = torch.full((M + 1, N + 16), 5.0, dtype=torch.bfloat16, device=DEV)
    args = (dev(mx.pack_nibbles(a)), dev(mx.steps(sa)), fq().mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw)), None if bias is None else dev(bias))
    fq().mx_gemm(*args, out=out[:M, :N])
    av, wv = dev(mx.decode(a, sa)), dev(mx.decode(w, sw))
    want, size = av @ wv.t(), av.abs() @ wv.abs().t()  # fp64
    slack = 0.0
    if bias is not None:
        want, slack = want + dev(bias).double(), dev(bias).double().abs() * 2.0 ** -22
    off = (out[:M, :N].double() - want).abs()
    assert bool((off <= size * 2.0 ** -23 * (K // 32 + 8) + want.abs() * (HALF_BF16 + 2.0 ** -22) + slack).all())
    assert bool((out[M:] == 5).all()) and bool((out[:, N:] == 5).all())
    assert torch.equal(fq().mx_gemm(*args), out[:M, :N])


def test_some_of_those_split_k():
    assert all(fq().mx_gemm_workspace_bytes(M, N, K) > 0 for M, N, K in ((816, 2048, 16384), (1100, 80, 32640)))


@pytest.mark.parametrize("M", [1, 40, 300])
def test_product_is_exact_where_its_sums_are(M):
    """Integers under one scale: sums below 2^24, outputs that bf16 holds."""
    K, N = 2048, 96
    r = np.random.default_rng(M)
    a = r.choice([0, 2, 10], (M, K), p=[0.9, 0.05, 0.05]).astype(np.uint8)  # 0, 1, -1
    w = np.zeros((N, K), dtype=np.uint8)
    w[np.arange(N), r.integers(0, K, N)] = 4  # 2, once a row: every output is one product
    sa, sw = np.full((M, K // 32), 127, np.uint8), np.full((N, K // 32), 125, np.uint8)
    y = fq().mx_gemm(dev(mx.pack_nibbles(a)), dev(mx.steps(sa)), fq().mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw)))
    assert np.array_equal(y.float().cpu().numpy(), mx.decode(a, sa) @ mx.decode(w, sw).T)


@pytest.mark.parametrize("M", [1, 50, 200])
def test_scales_far_apart(M):
    """Blocks of one row between 2^-60 and 2^60: each enters with its own scale."""
    K, N = 1024, 64
    a, sa = operands(M, K, 1, spread=60)
    w, sw = operands(N, K, 2, spread=2)
    y = fq().mx_gemm(dev(mx.pack_nibbles(a)), dev(mx.steps(sa)), fq().mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw)))
    assert_product(y, mx.decode(a, sa), mx.decode(w, sw))


@pytest.mark.parametrize("M,K,N,b", [(1, 128, 16, 1), (1, 2048, 1024, 128), (16, 1024, 80, 64), (50, 16384, 64, 128), (70, 640, 272, 128),
                                     (300, 2048, 512, 256), (5, 384, 48, 32)])
@pytest.mark.parametrize("folds", [False, True])
def test_projection_is_its_two_halves(M, K, N, b, folds):
    flush(f"mx_linear M={M} K={K} N={N} b={b}")
    f, r = fq(), np.random.default_rng(9)
    x = strided(tokens(M, K, 3, special=False))
    pre, post = (dev(r.uniform(0.5, 2, K).astype(np.float32)) for _ in range(2)) if folds else (None, None)
    w = dev((r.standard_normal((N, K)) * 0.02).astype(np.float32))
    bias = dev(r.standard_normal(N).astype(np.float32)) if folds else None
    lin = f.MXLinear(w, b, None if pre is None else 1 / pre, bias, None if post is None else 1 / post)
    y = lin(x, pre, post)
    codes, scales = f.mx_quant(x, b, pre, post)
    assert torch.equal(y, lin.product(codes, scales))
    a = f.mx_read(codes, scales).double().cpu().numpy()
    wc, ws = f.mx_quant(w, b, None if pre is None else 1 / pre, None if post is None else 1 / post)
    assert_product(y, a, f.mx_read(wc, ws).double().cpu().numpy(), None if bias is None else bias.cpu().numpy())


@pytest.mark.parametrize("M,K,N,b", [(1, 128, 16, 128), (2, 384, 80, 128), (2, 640, 2064, 64), (1, 1280, 16384, 256), (2, 1792, 16, 256),
                                     (1, 2048, 32768, 128), (2, 2432, 5008, 1), (1, 4096, 4096, 32), (2, 2048, 16400, 2), (2, 7680, 48, 16)])
@pytest.mark.parametrize("folds", [False, True])
def test_tokens_one_by_one_or_many(M, K, N, b, folds):
    """A token's outputs do not depend on how the rounding and the product are launched, nor on its neighbour."""
    flush(f"mx_linear M={M} K={K} N={N} b={b}")
    f, r = fq(), np.random.default_rng(K + N)
    x = strided(tokens(M, K, 3, special=False))
    pre, post = (dev(r.uniform(0.5, 2, K).astype(np.float32)) for _ in range(2)) if folds else (None, None)
    w, sw = operands(N, K, 7)
    packed, sw = f.mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw))
    bias = dev(r.standard_normal(N).astype(np.float32)) if folds else None
    y = f.mx_linear(x, packed, sw, b, pre, post, bias)
    assert torch.equal(y, f.mx_gemm(*f.mx_quant(x, b, pre, post), packed, sw, bias))
    bad = x.clone()
    bad[M - 1, K // 3] = float("inf")
    y_bad = f.mx_linear(bad, packed, sw, b, pre, post, bias)
    assert torch.equal(y_bad[:M - 1], y[:M - 1]) and torch.isnan(y_bad[M - 1]).all()


def test_no_rows():
    f = fq()
    x = torch.zeros((0, 256), dtype=torch.bfloat16, device=DEV)
    codes, scales = f.mx_quant(x, 64)
    w, sw = operands(32, 256, 0)
    packed, sw = f.mx_pack(dev(mx.pack_nibbles(w))), dev(mx.steps(sw))
    assert f.mx_gemm(codes, scales, packed, sw).shape == (0, 32) and f.mx_linear(x, packed, sw, 64).shape == (0, 32)
    assert f.mx_read(codes, scales).shape == (0, 256)
