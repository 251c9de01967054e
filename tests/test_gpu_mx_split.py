"""Projections and products whose K is split: partial sums behind codes and scales in a workspace of just the size that is asked for,
eagerly and in a graph."""
import numpy as np
import pytest
import torch

from tests.gpu_util import DEV, flush
from tests.mx_plan_util import plan
from tests.mx_util import HALF_BF16, dev, dev_bf16, fq, strided, tokens

pytestmark = pytest.mark.gpu

# (M, N, K): two slices of 128 x 128 tiles, four, eight of 64 x 64, four of 128 x 256 and of 256 x 256
SPLIT = [(816, 2048, 16384), (2198, 208, 13952), (1100, 80, 32640), (866, 1200, 24192), (1927, 1040, 27008)]
BEHIND = 4096


def weights(f, N, K, b, seed):
    r = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randn((N, K), generator=g, device=DEV) * 0.02
    return f.MXLinear(w, b, None, dev(r.standard_normal(N).astype(np.float32)))


def room(size):
    """A workspace of `size` bytes that begin as NaN, and the bytes behind it."""
    whole = torch.full((size + BEHIND,), 0xA5, dtype=torch.uint8, device=DEV)
    whole[:size] = 0xFF
    return whole[:size], whole[size:]


def assert_near(y, a, lin):
    """The bound of a product's outputs (products are exact, K/32 + 8 sums of fp32, a bf16 rounding), in fp64 on the GPU."""
    f = fq()
    w = f.mx_read(f.mx_unpack(lin.w_packed), lin.w_scales).double()
    bias = lin.bias.double()
    want, size = a @ w.t() + bias, a.abs() @ w.abs().t()
    most = size * 2.0 ** -23 * (a.shape[1] // 32 + 8) + want.abs() * (HALF_BF16 + 2.0 ** -22) + bias.abs() * 2.0 ** -22
    off = (y.double() - want).abs()
    assert bool((off <= most).all()), float((off / most).max())


@pytest.mark.parametrize("b", [1, 128])
@pytest.mark.parametrize("M,N,K", SPLIT)
def test_projection(M, N, K, b):
    flush(f"mx_linear M={M} N={N} K={K} b={b}")
    f = fq()
    assert plan(M, N, K).splits > 1 and f.mx_gemm_workspace_bytes(M, N, K) == plan(M, N, K).splits * M * N * 4
    lin, x = weights(f, N, K, b, M), strided(tokens(M, K, 3, special=False))
    ws, behind = room(f.mx_linear_workspace_bytes(M, N, K))
    out = torch.full((M + 1, N + 16), 5.0, dtype=torch.bfloat16, device=DEV)
    lin(x, ws=ws, out=out[:M, :N])
    assert bool((behind == 0xA5).all()) and bool((out[M:] == 5).all()) and bool((out[:, N:] == 5).all())
    codes, scales = f.mx_quant(x, b)
    partial, behind = room(f.mx_gemm_workspace_bytes(M, N, K))
    assert torch.equal(lin.product(codes, scales, ws=partial), out[:M, :N])
    assert bool((behind == 0xA5).all())
    # the workspace's parts: the codes, the scales, the partial sums, each from a multiple of 256 bytes
    parts, at = [codes, scales, partial], 0
    for t in parts:
        n = t.numel() * t.element_size()
        assert torch.equal(ws[at:at + n], t.reshape(-1).view(torch.uint8))
        at += -(-n // 256) * 256
    assert at == ws.numel() + (-ws.numel()) % 256
    assert_near(out[:M, :N], f.mx_read(codes, scales).double(), lin)


def test_one_byte_less_is_refused():
    f = fq()
    M, N, K = SPLIT[1]
    lin, x = weights(f, N, K, 1, 1), dev_bf16(tokens(M, K, 3, special=False))
    for size, call in ((f.mx_linear_workspace_bytes(M, N, K), lambda ws: lin(x, ws=ws)),
                       (f.mx_gemm_workspace_bytes(M, N, K), lambda ws: lin.product(*f.mx_quant(x), ws=ws))):
        with pytest.raises(f.FQError, match="WORKSPACE"):
            call(room(size)[0][:-1])


@pytest.mark.parametrize("M,N,K", SPLIT[:3])
def test_captured_and_replayed(M, N, K):
    """Two products with partial sums of one workspace, one behind the other in a graph; every replay, with fresh inputs and eager
    calls in the same workspace between, equals eager calls bit for bit."""
    flush(f"graph M={M} N={N} K={K}")
    f = fq()
    one, two = weights(f, N, K, 128, 1), weights(f, N, K, 128, 2)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device=DEV)
    ws, behind = room(f.mx_linear_workspace_bytes(M, N, K))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one(x, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a, b = one(x, ws=ws), two(x, ws=ws)
        c = one(x)  # with a workspace of the graph's own pool
    for k in range(4):
        t = dev_bf16(tokens(M, K, 40 + k, special=False))
        want = one(t), two(t)
        ws.fill_(0xFF)
        x.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and torch.equal(c, want[0]), k
        assert torch.equal(one(t, ws=ws), want[0])
    assert bool((behind == 0xA5).all())
