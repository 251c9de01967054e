"""Refusals of the microscaled operators and of the norm (CPU: every call here fails a check or has nothing to do, so no
kernel is launched), through the C ABI and the Python binding."""
import pytest
import torch

from paper_2609_24433_amd import fq

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ALIAS = 1, 2, 3, 4, 5, 7
A = 0x100000  # addresses that are never dereferenced, 256 MB apart


def at(i, off=0):
    return A + i * 0x10000000 + off


def norm(x=at(1), ldx=512, r=at(2), ldr=512, w=at(3), eps=1e-6, post=None, M=4, K=512, b=64, bits=8, clip=1.0, sum_=at(4), lds=512,
         codes=at(5), delta=at(6)):
    return fq.LIB.fq_norm_quant(x, ldx, r, ldr, w, eps, post, M, K, b, bits, clip, sum_, lds, codes, delta, None)


def norm_mx(x=at(1), ldx=512, r=at(2), ldr=512, w=at(3), eps=1e-6, post=None, M=4, K=512, b=64, sum_=at(4), lds=512, codes=at(5),
            scales=at(6)):
    return fq.LIB.fq_norm_mx_quant(x, ldx, r, ldr, w, eps, post, M, K, b, sum_, lds, codes, scales, None)


def quant(x=at(1), f32=0, ldx=512, pre=None, post=None, M=4, K=512, b=64, codes=at(5), scales=at(6)):
    return fq.LIB.fq_mx_quant(x, f32, ldx, pre, post, M, K, b, codes, scales, None)


def read(codes=at(1), scale=at(2), M=4, K=512, bits=8, out=at(3), ld=512):
    return fq.LIB.fq_read_codes(codes, scale, M, K, bits, out, ld, None)


def mx_read(codes=at(1), scale=at(2), M=4, K=512, out=at(3), ld=512):
    return fq.LIB.fq_mx_read(codes, scale, M, K, out, ld, None)


def pack(codes=at(1), N=32, K=512, out=at(2)):
    return fq.LIB.fq_mx_pack(codes, N, K, out, None)


def gemm(a=at(1), sa=at(2), w=at(3), sw=at(4), bias=None, y=at(5), ldy=64, M=4, N=64, K=512, ws=at(6), n=1 << 27):
    return fq.LIB.fq_mx_gemm(a, sa, w, sw, bias, y, ldy, M, N, K, ws, n, None)


def linear(x=at(1), ldx=512, pre=None, post=None, M=4, K=512, N=64, b=64, w=at(3), sw=at(4), bias=None, y=at(5), ldy=64, ws=at(6),
           n=1 << 27):
    return fq.LIB.fq_mx_linear(x, ldx, pre, post, M, K, N, b, w, sw, bias, y, ldy, ws, n, None)


@pytest.mark.parametrize("call,want", [
    (lambda: norm(x=None), NULL), (lambda: norm(w=None), NULL), (lambda: norm(codes=None), NULL), (lambda: norm(delta=None), NULL),
    (lambda: norm(r=None), NULL), (lambda: norm(M=-1), SHAPE), (lambda: norm(M=1 << 25), UNSUPPORTED), (lambda: norm(K=0), UNSUPPORTED),
    (lambda: norm(K=192), UNSUPPORTED), (lambda: norm(K=32896), UNSUPPORTED), (lambda: norm(b=0), UNSUPPORTED), (lambda: norm(b=48), UNSUPPORTED),
    (lambda: norm(b=512), UNSUPPORTED), (lambda: norm(K=384, b=256), SHAPE), (lambda: norm(bits=6), UNSUPPORTED),
    (lambda: norm(clip=0.0), UNSUPPORTED), (lambda: norm(clip=1.5), UNSUPPORTED), (lambda: norm(clip=float("nan")), UNSUPPORTED),
    (lambda: norm(eps=0.0), UNSUPPORTED), (lambda: norm(eps=-1.0), UNSUPPORTED), (lambda: norm(eps=float("nan")), UNSUPPORTED),
    (lambda: norm(eps=float("inf")), UNSUPPORTED), (lambda: norm(ldx=504), SHAPE), (lambda: norm(ldr=516), ALIGN),
    (lambda: norm(lds=256), SHAPE), (lambda: norm(ldx=1 << 33), UNSUPPORTED), (lambda: norm(x=at(1, 8)), ALIGN),
    (lambda: norm(post=at(7, 4)), ALIGN), (lambda: norm(sum_=at(1, 1024)), ALIAS), (lambda: norm(sum_=at(2), lds=1024), ALIAS),
    (lambda: norm(codes=at(1)), ALIAS), (lambda: norm(delta=at(5, 1024)), ALIAS), (lambda: norm(delta=at(3, 16)), ALIAS),
    (lambda: norm(sum_=at(5, 512)), ALIAS), (lambda: norm(sum_=at(2), r=at(2), x=at(2, 1024)), ALIAS),
    (lambda: norm(M=0, x=None, codes=None), 0),
    (lambda: norm_mx(scales=None), NULL), (lambda: norm_mx(K=200), UNSUPPORTED), (lambda: norm_mx(scales=at(5, 512)), ALIAS),
    (lambda: norm_mx(eps=0.0), UNSUPPORTED), (lambda: norm_mx(M=0), 0),
])
def test_norm(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("call,want", [
    (lambda: quant(x=None), NULL), (lambda: quant(codes=None), NULL), (lambda: quant(scales=None), NULL), (lambda: quant(M=-1), SHAPE),
    (lambda: quant(M=(1 << 24) + 1), UNSUPPORTED), (lambda: quant(K=64), UNSUPPORTED), (lambda: quant(K=160), UNSUPPORTED),
    (lambda: quant(b=3), UNSUPPORTED), (lambda: quant(K=128, b=256), SHAPE), (lambda: quant(ldx=508), SHAPE), (lambda: quant(ldx=516), ALIGN),
    (lambda: quant(f32=1, ldx=514), ALIGN), (lambda: quant(pre=at(7, 4)), ALIGN), (lambda: quant(scales=at(6, 4)), ALIGN),
    (lambda: quant(codes=at(1, 4080)), ALIAS), (lambda: quant(f32=1, codes=at(1, 8176)), ALIAS), (lambda: quant(scales=at(5, 1008)), ALIAS),
    (lambda: quant(pre=at(5, 1008)), ALIAS), (lambda: quant(M=0, x=None), 0),
    (lambda: read(codes=None), NULL), (lambda: read(bits=0), UNSUPPORTED), (lambda: read(bits=16), UNSUPPORTED), (lambda: read(ld=500), SHAPE),
    (lambda: read(ld=516), ALIGN), (lambda: read(out=at(1, 2032)), ALIAS), (lambda: read(scale=at(3)), ALIAS), (lambda: read(M=0), 0),
    (lambda: mx_read(scale=None), NULL), (lambda: mx_read(K=96), UNSUPPORTED), (lambda: mx_read(out=at(2)), ALIAS), (lambda: mx_read(M=0), 0),
    (lambda: pack(codes=None), NULL), (lambda: pack(N=24), UNSUPPORTED), (lambda: pack(N=-16), SHAPE), (lambda: pack(K=0), UNSUPPORTED),
    (lambda: pack(out=at(1, 8176)), ALIAS), (lambda: pack(out=at(2, 8)), ALIGN), (lambda: pack(N=0), 0),
])
def test_quantization(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("call,want", [
    (lambda: gemm(a=None), NULL), (lambda: gemm(sw=None), NULL), (lambda: gemm(y=None), NULL), (lambda: gemm(M=-1), SHAPE),
    (lambda: gemm(N=-16), SHAPE), (lambda: gemm(N=40, ldy=40), UNSUPPORTED), (lambda: gemm(K=32896), UNSUPPORTED), (lambda: gemm(K=130), UNSUPPORTED),
    (lambda: gemm(M=1 << 24, N=1 << 20, ldy=1 << 20), UNSUPPORTED), (lambda: gemm(M=1 << 25), UNSUPPORTED), (lambda: gemm(ldy=48), SHAPE),
    (lambda: gemm(ldy=68), ALIGN), (lambda: gemm(bias=at(7, 8)), ALIGN), (lambda: gemm(y=at(1, 512)), ALIAS), (lambda: gemm(y=at(4, 16)), ALIAS),
    (lambda: gemm(bias=at(5, 128)), ALIAS), (lambda: gemm(M=0, a=None), 0), (lambda: gemm(N=0, ldy=0), 0),
    (lambda: linear(x=None), NULL), (lambda: linear(w=None), NULL), (lambda: linear(N=8, ldy=8), UNSUPPORTED), (lambda: linear(b=512), UNSUPPORTED),
    (lambda: linear(ldx=256), SHAPE), (lambda: linear(pre=at(7, 4)), ALIGN), (lambda: linear(ws=None), WORKSPACE), (lambda: linear(n=64), WORKSPACE),
    (lambda: linear(ws=at(6, 8)), ALIGN), (lambda: linear(ws=at(1, 256)), ALIAS), (lambda: linear(y=at(6, 16)), ALIAS),
    (lambda: linear(post=at(6)), ALIAS), (lambda: linear(M=0), 0), (lambda: linear(N=0, ldy=0), 0),
])
def test_product(call, want):
    assert call() == want, fq.LIB.fq_last_error()


def test_sizes():
    assert fq.LIB.fq_mx_packed_bytes(48, 256) == 48 * 128 and fq.LIB.fq_mx_packed_bytes(-1, 256) == 0
    for M, N, K in ((0, 64, 256), (4, 0, 256), (4, 64, 0), (-3, 64, 256)):
        assert fq.LIB.fq_mx_gemm_workspace_bytes(M, N, K) == 0 and fq.LIB.fq_mx_linear_workspace_bytes(M, N, K) == 0
    assert fq.LIB.fq_mx_linear_workspace_bytes(5, 64, 256) >= 5 * 128 + 5 * 8


M, K, N = 4, 256, 32


def tensors():
    return dict(x=torch.zeros((M, K), dtype=torch.bfloat16), res=torch.zeros((M, K), dtype=torch.bfloat16), weight=torch.ones((K,)),
                codes=torch.zeros((M, K // 2), dtype=torch.uint8), scales=torch.zeros((K // 128, M, 4), dtype=torch.uint8),
                delta=torch.zeros((M,)), i8=torch.zeros((M, K), dtype=torch.uint8), w=torch.zeros((N // 16, K // 128, 4, 16, 16), dtype=torch.uint8),
                sw=torch.zeros((K // 128, N, 4), dtype=torch.uint8), bias=torch.zeros((N,)), y=torch.zeros((M, N), dtype=torch.bfloat16))


CALLS = {
    "norm_quant": (lambda t: fq.norm_quant(t["x"], t["weight"], 64, 8, t["res"]), ("x", "weight", "res")),
    "norm_mx_quant": (lambda t: fq.norm_mx_quant(t["x"], t["weight"], 64, t["res"], out_codes=t["codes"], out_scales=t["scales"]),
                      ("x", "weight", "res", "codes", "scales")),
    "read_codes": (lambda t: fq.read_codes(t["i8"], t["delta"], 8), ("i8", "delta")),
    "mx_quant": (lambda t: fq.mx_quant(t["x"], 64, t["weight"], t["weight"], t["codes"], t["scales"]), ("x", "weight", "codes", "scales")),
    "mx_read": (lambda t: fq.mx_read(t["codes"], t["scales"]), ("codes", "scales")),
    "mx_pack": (lambda t: fq.mx_pack(t["codes"]), ("codes",)),
    "mx_unpack": (lambda t: fq.mx_unpack(t["w"]), ("w",)),
    "mx_gemm": (lambda t: fq.mx_gemm(t["codes"], t["scales"], t["w"], t["sw"], t["bias"], out=t["y"]),
                ("codes", "scales", "w", "sw", "bias", "y")),
    "mx_linear": (lambda t: fq.mx_linear(t["x"], t["w"], t["sw"], 64, t["weight"], t["weight"], t["bias"], out=t["y"]),
                  ("x", "w", "sw", "weight", "bias", "y")),
}


@pytest.mark.parametrize("name", CALLS)
def test_the_binding_refuses_host_tensors(name):
    with pytest.raises(ValueError, match="host"):
        CALLS[name][0](tensors())


@pytest.mark.parametrize("name", CALLS)
def test_the_binding_refuses_other_types_and_layouts(name):
    call, names = CALLS[name]
    for n in names:
        t = tensors()
        t[n] = t[n].double()
        with pytest.raises(ValueError, match="contiguous|unit column stride"):
            call(t)
        t = tensors()
        t[n] = torch.stack((t[n], t[n]), dim=-1)[..., 0]  # a stride of 2
        with pytest.raises(ValueError, match="contiguous|unit column stride"):
            call(t)
    if name in ("mx_gemm", "mx_linear"):
        for n, wrong in (("sw", tensors()["scales"]), ("y", torch.zeros((M, N + 16), dtype=torch.bfloat16)), ("bias", torch.zeros((N + 1,)))):
            with pytest.raises(ValueError):
                call({**tensors(), n: wrong})


def test_a_sum_needs_a_residual():
    t = tensors()
    with pytest.raises(ValueError, match="residual"):
        fq.norm_quant(t["x"], t["weight"], 64, 8, sum_out=t["res"])


def test_another_device_than_the_current_one_is_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 77, raising=False)
    assert fq._gpu_stream(0) == 77
    with pytest.raises(ValueError, match="GPU 1, the current device is GPU 0"):
        fq._gpu_stream(1)
