"""The microscaled operators as a layer uses them: the norm's codes shared by two projections, a gated unit, the down
projection and the next norm; eagerly against the plain reference, on another stream, captured in a graph, and in place."""
import numpy as np
import pytest
import torch

from oracle import microscaled as mx
from tests.gpu_util import DEV, flush
from tests.mx_util import HALF_BF16, dev, dev_bf16, fq, strided, tokens

pytestmark = pytest.mark.gpu


class Layer:
    """hidden -> norm -> gate, up -> silu(gate) up -> down -> next norm (8-bit codes), b = 64."""

    def __init__(self, width, inner, seed, b=64):
        f, r = fq(), np.random.default_rng(seed)
        self.b, self.width = b, width
        self.gain = dev(r.uniform(0.5, 1.5, width).astype(np.float32))
        self.gain2 = dev(r.uniform(0.5, 1.5, width).astype(np.float32))
        mat = lambda n, k: dev((r.standard_normal((n, k)) * k ** -0.5).astype(np.float32))  # noqa: E731
        self.gate, self.up, self.down = f.MXLinear(mat(inner, width), b), f.MXLinear(mat(inner, width), b), f.MXLinear(mat(width, inner), b)

    def __call__(self, x, residual, sums=None):
        f = fq()
        codes, scales, h = f.norm_mx_quant(x, self.gain, self.b, residual)
        g, u = self.gate.product(codes, scales), self.up.product(codes, scales)
        mid = torch.nn.functional.silu(g) * u
        y = self.down(mid)
        c8, d8, total = f.norm_quant(y, self.gain2, self.b, 8, h, sum_out=sums)
        return {"codes": codes, "scales": scales, "h": h, "g": g, "u": u, "mid": mid, "y": y, "c8": c8, "d8": d8, "total": total}


def weights_of(lin):
    """fp64 values of a projection's packed weights."""
    f = fq()
    return f.mx_read(f.mx_unpack(lin.w_packed), lin.w_scales).double()


def near(got, a, w):
    want, size = a @ w.t(), a.abs() @ w.abs().t()
    return bool(((got.double() - want).abs() <= size * 2.0 ** -23 * (a.shape[1] // 32 + 8) + want.abs() * (HALF_BF16 + 2.0 ** -22)).all())


@pytest.mark.parametrize("M,width,inner", [(1, 1024, 4096), (50, 1024, 4096), (300, 512, 1152), (816, 1024, 2048)])
def test_layer(M, width, inner):
    flush(f"layer M={M} width={width} inner={inner}")
    f, lay = fq(), Layer(width, inner, M)
    x, res = tokens(M, width, 1, special=False), tokens(M, width, 2, special=False)
    o = lay(strided(x), dev_bf16(res))
    h, y = mx.norm(x, lay.gain.cpu().numpy(), 1e-6, res)
    n, s = mx.encode(mx.butterfly(y, 64) * mx.root(64))
    assert np.array_equal(o["h"].float().cpu().numpy(), h)
    assert np.array_equal(mx.rows(o["scales"].cpu().numpy()), s) and np.array_equal(mx.split_nibbles(o["codes"].cpu().numpy()), n)
    a = f.mx_read(o["codes"], o["scales"]).double()
    assert near(o["g"], a, weights_of(lay.gate)) and near(o["u"], a, weights_of(lay.up))
    mid = o["mid"].float().cpu().numpy()
    n, s = mx.encode(mx.fold(mid, 64))
    assert near(o["y"], dev(mx.decode(n, s)), weights_of(lay.down))
    h2, y2 = mx.norm(o["y"].float().cpu().numpy(), lay.gain2.cpu().numpy(), 1e-6, h)
    c, d = mx.codes(mx.butterfly(y2, 64), 64, 8)
    assert np.array_equal(o["total"].float().cpu().numpy(), h2)
    assert np.array_equal(o["d8"].cpu().numpy(), d) and np.array_equal(o["c8"].cpu().numpy().view(np.int8), c)


@pytest.mark.parametrize("M", [1, 50, 520])
def test_captured_and_replayed(M):
    """Every replay, with fresh inputs and eager work between, equals an eager call bit for bit."""
    lay = Layer(1024, 2048, 3)
    x, res, sums = (torch.zeros((M, 1024), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lay(x, res, sums)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = lay(x, res, sums)
    for k in range(4):
        a, b = dev_bf16(tokens(M, 1024, 10 + k, special=False)), dev_bf16(tokens(M, 1024, 20 + k, special=False))
        want = lay(a, b)
        x.copy_(a)
        res.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(o[name], want[name]), (k, name)


def test_another_stream():
    """A call works on torch's current stream, behind what that stream holds already."""
    f, lay = fq(), Layer(1024, 2048, 5)
    a, b = dev_bf16(tokens(200, 1024, 1, special=False)), dev_bf16(tokens(200, 1024, 2, special=False))
    want = lay(a, b)
    torch.cuda.synchronize()
    x, busy = torch.zeros_like(a), torch.randn(4096, 4096, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):
            busy = busy @ busy * 1e-3
        x.copy_(a)
        o = lay(x, b)
    torch.cuda.current_stream().wait_stream(side)
    for name in want:
        assert torch.equal(o[name], want[name]), name
    assert f._gpu_stream(0) == torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("split", [False, True])
def test_two_streams_at_once_with_workspaces_of_their_own(split):
    """Products on two streams, many times over, the split ones each with its own partial sums."""
    f, K, N = fq(), 32768, 64
    M = next(m for m in range(37, 2000, 97) if (f.mx_gemm_workspace_bytes(m, N, K) > 0) == split)
    r = np.random.default_rng(0)
    lin = f.MXLinear(dev((r.standard_normal((N, K)) * 0.02).astype(np.float32)), 128)
    xs = [f.mx_quant(dev_bf16(tokens(M, K, s, special=False)), 128) for s in (1, 2)]
    want = [lin.product(*c) for c in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(lin.product(*xs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_the_residual_stream_in_place():
    """A decoder's residual stream updated where it lies, step after step."""
    f = fq()
    M, K = 37, 1024
    gain = torch.ones(K, device=DEV)
    stream = dev_bf16(tokens(M, K, 1, special=False))
    plain = stream.float().cpu().numpy()
    for k in range(5):
        x = tokens(M, K, 30 + k, special=False)
        codes, delta, total = f.norm_quant(dev_bf16(x), gain, 64, 8, stream, sum_out=stream)
        assert total is stream
        plain, y = mx.norm(x, np.ones(K, np.float32), 1e-6, plain)
        c, d = mx.codes(mx.butterfly(y, 64), 64, 8)
        assert np.array_equal(stream.float().cpu().numpy(), plain) and np.array_equal(codes.cpu().numpy().view(np.int8), c)
        assert np.array_equal(delta.cpu().numpy(), d)


def test_a_workspace_that_is_too_small_is_refused():
    f = fq()
    x = dev_bf16(tokens(40, 512, 1, special=False))
    lin = f.MXLinear(dev(np.ones((64, 512), np.float32)), 64)
    ws = torch.empty(f.mx_linear_workspace_bytes(40, 64, 512) - 16, dtype=torch.uint8, device=DEV)
    with pytest.raises(f.FQError, match="WORKSPACE"):
        lin(x, ws=ws)
