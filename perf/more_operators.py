"""Microscaled 4-bit projections and the norm before them, as measured cases: inputs, one pass, the least work of a
pass, the plain form of the same pass in elementary operations, and the definition in 64 bits.

Kinds of case (sizes are the library's own workloads or generic, ragged ones):

  norm    `fq.norm_quant` (`fmt` "i8" or "i4": codes with a scale per token) or `fq.norm_mx_quant` (`fmt` "mx"): the
          residual's addition, the root-mean-square norm with its gain, the block Hadamard, the rounding to codes; then
          `fq.read_codes` / `fq.mx_read`, the codes as values
  quant   `fq.mx_quant`: tokens in bf16 or weights in fp32 through the folds and the block Hadamard into microscaled
          4-bit codes; then `fq.mx_read`
  prod    `fq.mx_gemm`: microscaled codes times packed microscaled weights
  linear  `fq.mx_linear`: the projection from bf16 tokens to bf16 outputs

Microscaled codes: E2M1 nibbles uint8 [M, K/2] (channel 2i in the low half of byte i) and E8M0 bytes [K/128, M, 4], byte
(s, t, j) the scale of channels 128 s + 32 j .. + 31 of row t.  Packed weights: the nibbles of 16 x 128 tiles, uint8
[N/16, K/128, 4, 16, 16], byte (n, s, j, i, c) channels 128 s + 32 j + 2 c and + 1 of output 16 n + i.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_EPS = float(np.float32(1e-6))


def listed():
    return [
        # the norm before the first projection of a decoding step: one token, call and launch latency
        {"name": "norm_token", "kind": "norm", "fmt": "i8", "M": 1, "K": 2048, "b": 128, "residual": True, "post": False},
        # the norm of one language layer at prefill, into microscaled codes
        {"name": "norm_prefix", "kind": "norm", "fmt": "mx", "M": 816, "K": 2048, "b": 128, "residual": True, "post": False},
        # a long prompt into 8 bits without a rotation
        {"name": "norm_long", "kind": "norm", "fmt": "i8", "M": 16383, "K": 4096, "b": 1, "residual": True, "post": False},
        # the action tokens of one denoising step
        {"name": "quant_chunk", "kind": "quant", "M": 50, "K": 1024, "b": 64, "f32": False, "pre": False, "post": False},
        # the widest rows of a long batch (the input of a down projection)
        {"name": "quant_long", "kind": "quant", "M": 4095, "K": 16384, "b": 128, "f32": False, "pre": False, "post": False},
        # offline: a gate projection's weights, with the norm's gain folded in
        {"name": "quant_weights", "kind": "quant", "M": 16384, "K": 2048, "b": 128, "f32": True, "pre": True, "post": False},
        # one token through a wide projection: the stream of its weights
        {"name": "prod_token", "kind": "prod", "M": 1, "K": 2048, "N": 16384, "bias": False},
        # the action tokens through the long rows of a down projection
        {"name": "prod_chunk", "kind": "prod", "M": 50, "K": 16384, "N": 2048, "bias": False},
        # a prefix through a wide projection, with a bias
        {"name": "prod_prefix", "kind": "prod", "M": 816, "K": 2048, "N": 16384, "bias": True},
        # many rows: the matrix cores
        {"name": "prod_large", "kind": "prod", "M": 8191, "K": 4096, "N": 16384, "bias": False},
        # the smallest whole projection: the action expert's gate site
        {"name": "linear_chunk", "kind": "linear", "M": 50, "K": 1024, "N": 4096, "b": 64, "pre": False, "post": False, "bias": False},
        # a prefix through the down projection with a fold, bf16 to bf16
        {"name": "linear_prefix", "kind": "linear", "M": 816, "K": 16384, "N": 2048, "b": 128, "pre": True, "post": False, "bias": False},
    ]


# ---------------------------------------------------------------- drawn cases

def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def _mult(rng, lo, hi, m):
    return max(1, _log(rng, lo, hi) // m) * m


def _block(rng, K):
    return rng.choice([b for b in (1, 1, 16, 32, 64, 64, 128, 128, 256) if K % b == 0])


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "quant", "quant", "prod", "prod", "prod", "prod", "linear", "linear"])
    if kind in ("norm", "quant"):
        f32 = kind == "quant" and rng.random() < 0.3
        while True:
            M, K = _log(rng, 1, 16383), _mult(rng, 128, 16384, 128)
            if M * K <= (1 << 25 if f32 else 1 << 26) - (1 << 16):
                break
        b = _block(rng, K)
        if kind == "norm":
            return {"kind": kind, "fmt": rng.choice(["i8", "i8", "i4", "mx"]), "M": M, "K": K, "b": b,
                    "residual": rng.random() < 0.7, "post": rng.random() < 0.3}
        return {"kind": kind, "M": M, "K": K, "b": b, "f32": f32, "pre": rng.random() < 0.4, "post": rng.random() < 0.3}
    while True:
        M = rng.choice([1, _log(rng, 2, 64), _log(rng, 16, 8191), _log(rng, 64, 8191)])
        K, N = _mult(rng, 128, 16384, 128), _mult(rng, 16, 32768, 16)
        if M * K * N <= 8191 * 4096 * 16384 and K * N <= 1 << 26 and M * N <= 1 << 27 and M * K <= 1 << 26:
            break
    if kind == "prod":
        return {"kind": kind, "M": M, "K": K, "N": N, "bias": rng.random() < 0.3}
    return {"kind": kind, "M": M, "K": K, "N": N, "b": _block(rng, K), "pre": rng.random() < 0.4, "post": rng.random() < 0.3,
            "bias": rng.random() < 0.3}


# ---------------------------------------------------------------- inputs

class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(1000003 * (int(seed) + 1))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def uniform(self, n, lo, hi):
        return torch.rand((n,), generator=self.g, device="cuda", dtype=torch.float32) * (hi - lo) + lo

    def tokens(self, M, K):
        """Rows with a few channels much larger than the rest, as hidden states have them."""
        x = self.normal(M, K)
        x[:, torch.randperm(K, generator=self.g, device="cuda")[:max(1, K // 128)]] *= 20.0
        return x.to(torch.bfloat16)


def prepare(case, seed):
    d, kind, M, K = _Draws(seed), case["kind"], case["M"], case["K"]
    st = {"case": case, "pre": None, "post": None, "bias": None, "residual": None}
    if kind == "norm":
        st["x"] = d.tokens(M, K)
        if case["residual"]:
            st["residual"] = (d.normal(M, K) * 3.0).to(torch.bfloat16)
        st["weight"] = d.uniform(K, 0.5, 1.5)
    elif kind == "quant":
        st["x"] = d.normal(M, K) * 0.02 if case["f32"] else d.tokens(M, K)
    elif kind == "linear":
        st["x"] = d.tokens(M, K)
    else:
        st["a"], st["a_scale"] = _mx_codes(d.tokens(M, K).float())
    if case.get("pre"):
        st["pre"] = d.uniform(K, 0.5, 2.0)
    if case.get("post"):
        st["post"] = d.uniform(K, 0.5, 2.0)
    if kind in ("prod", "linear"):
        N = case["N"]
        w, st["w_scale"] = _mx_codes(d.normal(N, K) * 0.02)
        st["w"] = w.reshape(N // 16, 16, K // 128, 4, 16).permute(0, 2, 3, 1, 4).contiguous()
        if case["bias"]:
            st["bias"] = d.normal(N)
    return st


# ---------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


def _run_own(st):
    from paper_2609_24433_amd import fq
    c = st["case"]
    if c["kind"] == "norm":
        if c["fmt"] == "mx":
            codes, scale, total = fq.norm_mx_quant(st["x"], st["weight"], c["b"], residual=st["residual"], eps=_EPS, post_inv=st["post"])
            values = fq.mx_read(codes, scale)
        else:
            bits = 8 if c["fmt"] == "i8" else 4
            codes, scale, total = fq.norm_quant(st["x"], st["weight"], c["b"], bits, residual=st["residual"], eps=_EPS, post_inv=st["post"])
            values = fq.read_codes(codes, scale, bits)
        return {"sum": total, "values": values} if c["residual"] else {"values": values}
    if c["kind"] == "quant":
        codes, scale = fq.mx_quant(st["x"], c["b"], pre_mult=st["pre"], post_mult=st["post"])
        return fq.mx_read(codes, scale)
    if c["kind"] == "prod":
        return fq.mx_gemm(st["a"], st["a_scale"], st["w"], st["w_scale"], bias=st["bias"])
    return fq.mx_linear(st["x"], st["w"], st["w_scale"], c["b"], smooth_inv=st["pre"], post_inv=st["post"], bias=st["bias"])


# the plain forms: fp32, sums that decide a rounding in 64 bits, one rounding at the end

def _root(b):
    """The float nearest 1 / sqrt(b)."""
    return float(np.float32(1.0 / math.sqrt(b)))


def _rotated(x, b):
    """The block Hadamard without its factor: pairs (a, c) at distance h = 1, 2, .., b/2 become (a + c, a - c)."""
    h = 1
    while h < b:
        y = x.reshape(-1, 2, h)
        x = torch.stack((y[:, 0] + y[:, 1], y[:, 0] - y[:, 1]), dim=1).reshape(x.shape)
        h *= 2
    return x


def _mx_exponents(u):
    """Per block of 32: floor(log2 max) - 2, biased by 127."""
    top = u.reshape(u.shape[0], -1, 32).abs().amax(dim=2)
    e = torch.frexp(top).exponent.to(torch.int32) - 1 - 2 + 127
    return torch.where(top > 0, e, torch.zeros_like(e)).clamp(0, 254)


def _power(n):
    """2^(n - 127) in fp32 for n = 0 .. 254 (the lowest is subnormal)."""
    return torch.where(n > 0, n << 23, torch.full_like(n, 1 << 22)).view(torch.float32)


def _rounded(a):
    """Magnitudes to the nearest of 0 .5 1 1.5 2 3 4 6, ties to the even pattern."""
    step = torch.where(a < 2, torch.full_like(a, 0.5), torch.where(a < 4, torch.ones_like(a), torch.full_like(a, 2.0)))
    return (torch.round(a / step) * step).clamp(max=6.0)


def _mx_values(u):
    """fp32 rows as the values that their microscaled codes stand for."""
    blocks = u.reshape(u.shape[0], -1, 32)
    e = _mx_exponents(u)[:, :, None]
    t = blocks * _power(254 - e)
    return (_rounded(t.abs()) * torch.sign(t) * _power(e)).reshape(u.shape)


def _mx_codes(u):
    """fp32 rows to nibbles [M, K/2] and scale bytes [K/128, M, 4]."""
    M, K = u.shape
    e = _mx_exponents(u)
    t = u.reshape(M, -1, 32) * _power(254 - e)[:, :, None]
    m = _rounded(t.abs())
    n = torch.where(m < 2, m * 2, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8) + 8 * (t < 0).to(torch.uint8)
    n = n.reshape(M, K // 2, 2)
    return n[:, :, 0] + 16 * n[:, :, 1], e.to(torch.uint8).reshape(M, K // 128, 4).permute(1, 0, 2).contiguous()


def _mx_decoded(codes, scale):
    """The values of nibbles [M, K/2] and scale bytes [K/128, M, 4], fp32."""
    M = codes.shape[0]
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device=codes.device)
    n = torch.stack((codes & 15, codes >> 4), dim=2).reshape(M, -1, 32).to(torch.int32)
    e = scale.permute(1, 0, 2).reshape(M, -1, 1).to(torch.int32)
    return (table[n] * _power(e)).reshape(M, -1)


def _unpacked(w):
    return w.permute(0, 3, 1, 2, 4).reshape(w.shape[0] * 16, -1)


def _plain_norm(st):
    c = st["case"]
    h = st["x"].float()
    if st["residual"] is not None:
        h = (h + st["residual"].float()).to(torch.bfloat16).float()
    mean = (h.double() * h.double()).sum(dim=1, keepdim=True) / c["K"]
    s = (torch.ones_like(mean) / torch.sqrt(mean + _EPS)).float()
    u = _rotated(h * s * st["weight"], c["b"])
    root = _root(c["b"])
    if c["fmt"] == "mx":
        u = u * root
    if st["post"] is not None:
        u = u * st["post"]
    if c["fmt"] == "mx":
        values = _mx_values(u)
    else:
        q = 127.0 if c["fmt"] == "i8" else 7.0
        top = u.abs().amax(dim=1, keepdim=True)
        inv = torch.full_like(top, q) / top
        values = torch.round(u * inv).clamp(-q, q) * (top * root / q)
    values = values.to(torch.bfloat16)
    return {"sum": h.to(torch.bfloat16), "values": values} if c["residual"] else {"values": values}


def _folded(st):
    """Tokens or weights through the folds and the rotation, fp32."""
    u = st["x"].float()
    if st["pre"] is not None:
        u = u * st["pre"]
    u = _rotated(u, st["case"]["b"]) * _root(st["case"]["b"])
    return u * st["post"] if st["post"] is not None else u


def _plain_quant(st):
    return _mx_values(_folded(st)).to(torch.bfloat16)


def _product(a, st):
    y = torch.matmul(a, _mx_decoded(_unpacked(st["w"]), st["w_scale"]).t())
    return (y if st["bias"] is None else y + st["bias"]).to(torch.bfloat16)


def _plain_prod(st):
    return _product(_mx_decoded(st["a"], st["a_scale"]), st)


def _plain_linear(st):
    return _product(_mx_values(_folded(st)), st)


_PLAIN = {"norm": _plain_norm, "quant": _plain_quant, "prod": _plain_prod, "linear": _plain_linear}


# ---------------------------------------------------------------- the least work of a pass

def work(case):
    kind, M, K = case["kind"], case["M"], case["K"]
    mx = 17 / 32  # bytes of a microscaled value
    if kind == "norm":
        code = {"i8": 1.0, "i4": 0.5, "mx": mx}[case["fmt"]]
        by = M * K * (2 + 4 * case["residual"] + 2 * code + 2) + 4 * K * (1 + case["post"]) + (0 if case["fmt"] == "mx" else 8 * M)
        return {"bytes": by, "flops": M * K * (6 + case["residual"] + math.log2(case["b"]))}
    if kind == "quant":
        by = M * K * ((4 if case["f32"] else 2) + 2 * mx + 2) + 4 * K * (case["pre"] + case["post"])
        return {"bytes": by, "flops": M * K * (3 + case["pre"] + case["post"] + math.log2(case["b"]))}
    N = case["N"]
    by = mx * N * K + 2 * M * N + 4 * N * case["bias"]
    if kind == "prod":
        return {"bytes": by + mx * M * K, "flops": 2 * M * N * K}
    return {"bytes": by + 2 * M * K + 4 * K * (case["pre"] + case["post"]), "flops": 2 * M * N * K}


# ---------------------------------------------------------------- the definitions in 64 bits

def _hadamard64(x, b):
    """Rows times the block Hadamard matrix: entry (i, j) is (-1)^(bits that i and j share) / sqrt(b)."""
    i = torch.arange(b, device=x.device)
    both = i[:, None] & i[None, :]
    sign = sum(((both >> k) & 1) for k in range(8)) % 2
    return ((x.reshape(-1, b) @ (1.0 - 2.0 * sign.double())) / math.sqrt(b)).reshape(x.shape)


def _grid64(u):
    """Blocks of 32 on the microscaled grid."""
    v = u.reshape(-1, 32)
    top = v.abs().max(dim=1, keepdim=True).values
    unit = torch.exp2(torch.floor(torch.log2(top)) - 2)
    r = torch.where(top > 0, v / unit, torch.zeros_like(v))
    places = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=u.device)
    middle = (places[1:] + places[:-1]) / 2
    a = r.abs()
    # a value on a middle goes to the even place: searchsorted from the left keeps the lower, the odd lower ones go up
    at = torch.searchsorted(middle, a.contiguous())
    at = at + ((at % 2 == 1) & (a == middle[at.clamp(max=6)])).long()
    return (places[at] * torch.sign(r) * torch.where(top > 0, unit, torch.zeros_like(unit))).reshape(u.shape)


def _values64(codes, scale):
    n = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(1).long()
    exponent, half = (n >> 1) & 3, (n & 1).double()
    size = torch.where(exponent == 0, half / 2, (1 + half / 2) * torch.exp2(exponent.double() - 1))
    unit = torch.exp2(scale.double() - 127).transpose(0, 1).flatten(1).repeat_interleave(32, dim=1)
    return size * (1 - 2 * (n >> 3)).double() * unit


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    K = case["K"]
    if kind == "norm":
        h = st["x"].double()
        total = h
        if st["residual"] is not None:
            total = h + st["residual"].double()
            h = total.to(torch.bfloat16).double()  # the norm is that of the residual stream as it is kept
        u = h / torch.sqrt(h.pow(2).mean(dim=1, keepdim=True) + _EPS) * st["weight"].double()
        u = _hadamard64(u, case["b"])
        if st["post"] is not None:
            u = u * st["post"].double()
        if case["fmt"] == "mx":
            values = _grid64(u)
        else:
            step = u.abs().max(dim=1, keepdim=True).values / (127 if case["fmt"] == "i8" else 7)
            values = torch.round(u / step) * step
        return {"sum": total, "values": values} if case["residual"] else {"values": values}
    if kind == "prod":
        a = _values64(st["a"], st["a_scale"])
    else:
        u = st["x"].double()
        if st["pre"] is not None:
            u = u * st["pre"].double()
        u = _hadamard64(u, case["b"])
        if st["post"] is not None:
            u = u * st["post"].double()
        a = _grid64(u)
        if kind == "quant":
            return a
    w = st["w"].permute(0, 3, 1, 2, 4).reshape(case["N"], K // 2)
    y = a @ _values64(w, st["w_scale"]).t()
    return y if st["bias"] is None else y + st["bias"].double()
