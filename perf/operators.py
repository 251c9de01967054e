"""The operators between a layer's quantized projections, as measured cases: inputs, one pass, the least work of a
pass, the plain form of the same pass in elementary 32-bit operations, and the definition in 64 bits.

Kinds of case (sizes are the library's own workloads or generic, ragged ones):

  rope    `fq.qk_rope`: the norms of queries and keys per head and the position rotation, one pass over both
  append  `fq.cache_append`: the same for a packed q|k|v projection, with keys and values rounded to 8 bits into a
          paged cache (one scale per page and head), then `fq.cache_read`, the touched pages as values
  cached  `fq.cache_attention`: queries of a ragged batch over that cache
  cross   `fq.cross_attention`: queries over an encoder's bf16 states of another length

A cache is four tensors: key codes int8 [pages, heads, P, D], key scales fp32 [pages, heads], value codes int8
[pages, heads, P/16, D, 16] (the tokens of a group of 16 adjacent), value scales fp32 [pages, heads].
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False


def listed():
    return [
        # the shortest chunk of action tokens through the norm and the rotation: launch and call latency
        {"name": "rope_chunk", "kind": "rope", "T": 50, "Hq": 8, "Hk": 1, "D": 256, "R": 256, "norm": True, "inter": False,
         "scale": 1.0, "packed": True},
        # a long prefill: adjacent pairs rotated, a quarter of the head left alone, positions compressed by 4
        {"name": "rope_long", "kind": "rope", "T": 16385, "Hq": 32, "Hk": 8, "D": 128, "R": 96, "norm": True, "inter": True,
         "scale": 4.0, "packed": True},
        # one decoding step of a ragged batch: a token a sequence, most of them into a page in use
        {"name": "append_step", "kind": "append", "B": 32, "new": 1, "kv": 2048, "ragged": True, "Hq": 32, "Hk": 8, "D": 128,
         "P": 64, "R": 128, "norm": True, "inter": False, "scale": 1.0, "lseed": 1},
        # a long prompt into an empty cache
        {"name": "append_prompt", "kind": "append", "B": 1, "new": 16383, "kv": 16383, "ragged": False, "Hq": 32, "Hk": 8, "D": 128,
         "P": 64, "R": 128, "norm": True, "inter": False, "scale": 4.0, "lseed": 2},
        # one token of one sequence over the 816-token prefix of the language width 2048 (8 heads of 256 on one key head)
        {"name": "decode_one", "kind": "cached", "B": 1, "new": 1, "kv": 877, "ragged": False, "Hq": 8, "Hk": 1, "D": 256, "P": 64,
         "causal": True, "lseed": 3},
        # a decoding step of a full batch, lengths from a few tokens to 8192
        {"name": "decode_batch", "kind": "cached", "B": 64, "new": 1, "kv": 8192, "ragged": True, "Hq": 32, "Hk": 8, "D": 128, "P": 64,
         "causal": True, "lseed": 4},
        # a decoding step over two long contexts, where only a split of the length fills the card; small pages
        {"name": "decode_long", "kind": "cached", "B": 2, "new": 1, "kv": 131071, "ragged": False, "Hq": 16, "Hk": 2, "D": 128, "P": 16,
         "causal": True, "lseed": 5},
        # the 50 action tokens of a denoising step over the prefix and themselves, every token seeing every other
        {"name": "expert_chunk", "kind": "cached", "B": 1, "new": 50, "kv": 866, "ragged": False, "Hq": 8, "Hk": 1, "D": 256, "P": 64,
         "causal": False, "lseed": 6},
        # the second half of a long prompt, causal
        {"name": "prefill_chunk", "kind": "cached", "B": 1, "new": 4096, "kv": 8190, "ragged": False, "Hq": 32, "Hk": 8, "D": 128, "P": 64,
         "causal": True, "lseed": 7},
        # the action tokens of one denoising step over the backbone's 816 states (width 1024 as 16 heads of 64)
        {"name": "cross_chunk", "kind": "cross", "B": 1, "Sq": 50, "Sk": 816, "Hq": 16, "Hk": 16, "D": 64, "mask": False, "ragged": False,
         "lseed": 8},
        # one query a sample over encoder states of ragged lengths
        {"name": "cross_token", "kind": "cross", "B": 24, "Sq": 1, "Sk": 1500, "Hq": 16, "Hk": 16, "D": 128, "mask": False, "ragged": True,
         "lseed": 9},
        # many queries over long states with padded places masked out and one sample without any state
        {"name": "cross_masked", "kind": "cross", "B": 4, "Sq": 1031, "Sk": 4099, "Hq": 16, "Hk": 8, "D": 128, "mask": True, "ragged": True,
         "lseed": 10},
    ]


# ---------------------------------------------------------------- drawn cases

def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


#: query heads, key heads, head size
_HEADS = [(8, 1, 256), (32, 8, 128), (16, 2, 128), (12, 12, 64), (12, 4, 80), (8, 8, 96), (20, 4, 128), (16, 4, 64), (4, 2, 256), (14, 2, 64)]


def draw(rng):
    kind = rng.choice(["rope", "append", "append", "cached", "cached", "cached", "cached", "cross", "cross"])
    Hq, Hk, D = rng.choice(_HEADS)
    lseed = rng.randint(100, 1 << 30)
    if kind == "rope":
        return {"kind": kind, "T": _log(rng, 1, 12000), "Hq": Hq, "Hk": Hk, "D": D, "R": rng.choice([D, D, D // 32 * 16]),
                "norm": rng.random() < 0.6, "inter": rng.random() < 0.5, "scale": rng.choice([1.0, 1.0, 2.5]), "packed": rng.random() < 0.7}
    if kind == "append":
        B = _log(rng, 1, 48)
        new = rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 16, max(17, 12000 // B))])
        kv = new + rng.choice([0, _log(rng, 1, 3000)])
        return {"kind": kind, "B": B, "new": new, "kv": kv, "ragged": rng.random() < 0.6, "Hq": Hq, "Hk": Hk, "D": D,
                "P": rng.choice([16, 32, 64, 128]), "R": rng.choice([D, D, 0, D // 32 * 16]), "norm": rng.random() < 0.5,
                "inter": rng.random() < 0.3, "scale": rng.choice([1.0, 2.5]), "lseed": lseed}
    if kind == "cached":
        while True:
            B = _log(rng, 1, 64)
            new = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 17, 2048)])
            kv = max(new, _log(rng, 32, 100000))
            # at most a prefill chunk's products and a long decode's bytes
            if B * new * kv * Hq * D <= 1 << 36 and B * kv * Hk * D <= 1 << 28 and B * new * kv * Hq <= 1 << 29:
                break
        return {"kind": kind, "B": B, "new": new, "kv": kv, "ragged": rng.random() < 0.6, "Hq": Hq, "Hk": Hk, "D": D,
                "P": rng.choice([16, 32, 64, 64, 128]), "causal": rng.random() < 0.7, "lseed": lseed}
    while True:
        B, Sq, Sk = _log(rng, 1, 32), rng.choice([1, _log(rng, 2, 2000), _log(rng, 16, 2000)]), _log(rng, 16, 6000)
        if B * Sq * Sk * Hq * D <= 1 << 35 and B * Sk * Hk * D <= 1 << 26 and B * Sq * Sk * Hq <= 1 << 29:
            break
    return {"kind": kind, "B": B, "Sq": Sq, "Sk": Sk, "Hq": Hq, "Hk": Hk, "D": D, "mask": rng.random() < 0.5,
            "ragged": rng.random() < 0.6, "lseed": lseed}


# ---------------------------------------------------------------- lengths (part of a case)

def _lengths(case):
    """Per sequence: (new tokens, tokens in the cache with them)."""
    B, new, kv = case["B"], case["new"], case["kv"]
    if not case["ragged"]:
        return [new] * B, [kv] * B
    r = random.Random(case["lseed"])
    n = [new] + [r.randint(max(1, new // 2), new) for _ in range(B - 1)]
    return n, [kv] + [n[i] + int((kv - new) * r.random() ** 2) for i in range(1, B)]


def _key_lengths(case):
    """Per sample: the encoder's states in use; where they are ragged, the last of several samples has none."""
    B, Sk = case["B"], case["Sk"]
    if not case["ragged"]:
        return [Sk] * B
    r = random.Random(case["lseed"])
    return [Sk] + [r.randint(1, Sk) for _ in range(B - 2)] + ([0] if B > 1 else [])


def _window(case):
    """Tokens in the pages that the new ones of a sequence can touch."""
    return (case["new"] + 2 * case["P"] - 2) // case["P"] * case["P"]


# ---------------------------------------------------------------- inputs

class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(1000003 * (int(seed) + 1))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def uniform(self, shape, lo, hi):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32) * (hi - lo) + lo

    def heads(self, T, H, D, outliers=True):
        """Rows of H heads with a few channels of each head larger than the rest, as keys have them."""
        x = self.normal(T, H, D)
        if outliers:
            x[:, :, torch.randperm(D, generator=self.g, device="cuda")[:max(1, D // 32)]] *= 4.0
        return x


def _table(length, R, scale):
    """cos and sin of position / scale * 10000^(-2 i / R), fp32 [length, R/2, 2]."""
    if not R:
        return None
    f = 10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R) / scale
    a = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * f[None, :]
    return torch.stack((a.cos(), a.sin()), dim=-1).float()


def _pages(d, case, lens):
    """A page table [B, most] over a shuffled pool with some pages to spare."""
    P = case["P"]
    need = [-(-n // P) for n in lens]
    pool = sum(need) + 3
    perm = torch.randperm(pool, generator=d.g, device="cuda").to(torch.int32)
    most = max(need)
    at = np.zeros((len(lens), most), dtype=np.int64)
    used = 0
    for b, n in enumerate(need):
        at[b, :n] = np.arange(used, used + n)
        used += n
    return perm[torch.from_numpy(at).cuda()].contiguous(), pool


def _cache(d, pool, Hk, P, D):
    """A pool of pages that hold rounded keys and values; pages differ in their scales."""
    kc = d.normal(pool, Hk, P, D)
    kc[..., torch.randperm(D, generator=d.g, device="cuda")[:max(1, D // 32)]] *= 4.0
    vc = d.normal(pool, Hk, P // 16, D, 16)
    ks = kc.abs().amax(dim=(2, 3)) / 127
    vs = vc.abs().amax(dim=(2, 3, 4)) / 127
    kc = (kc / ks[:, :, None, None]).round_().clamp_(-127, 127).to(torch.int8)
    vc = (vc / vs[:, :, None, None, None]).round_().clamp_(-127, 127).to(torch.int8)
    spread = d.uniform((pool, Hk), 0.5, 1.5)
    return kc, ks, vc, vs * spread


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def prepare(case, seed):
    d, kind = _Draws(seed), case["kind"]
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    st = {"case": case}
    if kind == "rope":
        T = case["T"]
        if case["packed"]:  # queries and keys are columns of one q|k|v projection
            x = d.heads(T, Hq + 2 * Hk, D).to(torch.bfloat16)
            st["q"], st["k"] = x[:, :Hq], x[:, Hq:Hq + Hk]
        else:
            st["q"], st["k"] = d.heads(T, Hq, D).to(torch.bfloat16), d.heads(T, Hk, D).to(torch.bfloat16)
        length = 2 * T + 5
        st["positions"] = torch.randperm(length, generator=d.g, device="cuda")[:T].sort().values.to(torch.int32)
        st["table"] = _table(length, case["R"], case["scale"])
        st["qw"], st["kw"] = (d.uniform((D,), 0.5, 2.0), d.uniform((D,), 0.5, 2.0)) if case["norm"] else (None, None)
        return st
    if kind == "cross":
        B, Sq, Sk = case["B"], case["Sq"], case["Sk"]
        st["q"] = (d.normal(B, Sq, Hq, D) * 1.5).to(torch.bfloat16)
        kv = d.normal(B, Sk, 2 * Hk, D).to(torch.bfloat16)  # keys and values are columns of one projection
        st["k"], st["v"] = kv[:, :, :Hk], kv[:, :, Hk:]
        st["kv_len"] = _ints(_key_lengths(case)) if case["ragged"] else None
        st["mask"] = (d.uniform((B, Sk), 0.0, 1.0) < 0.8) if case["mask"] else None
        return st
    n, lens = _lengths(case)
    T = sum(n)
    st["q_start"], st["kv_len"] = _ints(np.concatenate(([0], np.cumsum(n))).tolist()), _ints(lens)
    st["pages"], pool = _pages(d, case, lens)
    st["cache"] = _cache(d, pool, Hk, case["P"], D)
    if kind == "append":
        x = d.heads(T, Hq + 2 * Hk, D).to(torch.bfloat16)
        st["q"], st["k"], st["v"] = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
        st["table"] = _table(case["kv"], case["R"], case["scale"])
        st["qw"], st["kw"] = (d.uniform((D,), 0.5, 2.0), d.uniform((D,), 0.5, 2.0)) if case["norm"] else (None, None)
        st["first"] = _ints([(m - k) // case["P"] * case["P"] for k, m in zip(n, lens)])
        return st
    st["q"] = (d.normal(T, Hq, D) * 1.5).to(torch.bfloat16)
    return st


# ---------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["kind"]](state)


def _run_own(st):
    from paper_2609_24433_amd import fq
    c = st["case"]
    if c["kind"] == "rope":
        return fq.qk_rope(st["q"], st["k"], st["table"], st["positions"], st["qw"], st["kw"], interleaved=c["inter"])
    if c["kind"] == "cross":
        return fq.cross_attention(st["q"], st["k"], st["v"], st["kv_len"], st["mask"])
    cache = fq.KVCache(*st["cache"])
    if c["kind"] == "append":
        q = fq.cache_append(cache, st["pages"], st["q_start"], st["kv_len"], c["new"], st["k"], st["v"], st["q"], st["table"],
                            q_weight=st["qw"], k_weight=st["kw"], interleaved=c["inter"])
        k, v = fq.cache_read(cache, st["pages"], st["first"], st["kv_len"], _window(c))
        return {"q": q, "k": k, "v": v}
    return fq.cache_attention(st["q"], cache, st["pages"], st["q_start"], st["kv_len"], c["new"], c["kv"], causal=c["causal"])


# the plain forms: fp32 throughout, one rounding at the end

def _norm_rotate(x, table, positions, weight, inter):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * weight
    if table is None:
        return x
    half = table.shape[1]
    cs = table[positions.long()][:, None]
    c, s = cs[..., 0], cs[..., 1]
    if inter:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y = torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y = torch.cat((a * c - b * s, b * c + a * s), dim=-1)
    return torch.cat((y, x[..., 2 * half:]), dim=-1)


def _plain_rope(st):
    inter = st["case"]["inter"]
    return (_norm_rotate(st["q"], st["table"], st["positions"], st["qw"], inter).to(torch.bfloat16),
            _norm_rotate(st["k"], st["table"], st["positions"], st["kw"], inter).to(torch.bfloat16))


def _sequence_of(q_start, T):
    """Per token of the ragged batch: its sequence and its place in it."""
    t = torch.arange(T, device=q_start.device)
    b = (t[:, None] >= q_start[None, 1:].long()).sum(dim=1)
    return b, t - q_start.long()[b]


def _rounded(new, there, codes, scale, before):
    """New values into pages [B, W, P, H, D]: `there` marks them, `before` the slots in use. The pages' values."""
    amax = torch.where(there, new.abs(), torch.zeros_like(new)).amax(dim=(2, 4))
    old = before[:, :, :1, 0, 0].any(dim=2)[..., None]
    s = torch.where(old, torch.maximum(scale, amax / 127), amax / 127)
    wide = s[:, :, None, :, None]
    inv = torch.where(s > 0, 1 / s, torch.zeros_like(s))[:, :, None, :, None]
    kept = torch.round(codes.float() * torch.where(s > 0, scale / s, torch.zeros_like(s))[:, :, None, :, None])
    got = torch.where(there, torch.clamp(torch.round(new * inv), -127, 127), torch.where(before, kept, torch.zeros_like(kept)))
    return (got * wide).to(torch.bfloat16)


def _plain_append(st):
    case = st["case"]
    P, Hk, D = case["P"], case["Hk"], case["D"]
    kc, ks, vc, vs = st["cache"]
    q_start, kv_len, pages, first = st["q_start"], st["kv_len"].long(), st["pages"], st["first"].long()
    B, T, W = pages.shape[0], st["k"].shape[0], _window(case) // P
    seq, i = _sequence_of(q_start, T)
    n = (q_start[1:] - q_start[:-1]).long()
    slot = (kv_len - n)[seq] + i
    q = _norm_rotate(st["q"], st["table"], slot, st["qw"], case["inter"]).to(torch.bfloat16)
    k = _norm_rotate(st["k"], st["table"], slot, st["kw"], case["inter"])
    v = st["v"].float()
    at = first[:, None] + torch.arange(W * P, device=first.device)[None, :]  # a sequence's slots from its first touched page on
    begin = (kv_len - n)[:, None]
    there = ((at >= begin) & (at < kv_len[:, None])).reshape(B, W, P, 1, 1)
    before = (at < begin).reshape(B, W, P, 1, 1)
    token = (q_start[:-1].long()[:, None] + (at - begin)).clamp(0, T - 1)
    page = torch.gather(pages.long(), 1, (at[:, ::P] // P).clamp(max=pages.shape[1] - 1))
    knew, vnew = (x[token].reshape(B, W, P, Hk, D) for x in (k, v))
    kv = _rounded(knew, there, kc[page].permute(0, 1, 3, 2, 4), ks[page], before)
    vv = _rounded(vnew, there, vc[page].permute(0, 1, 3, 5, 2, 4).reshape(B, W, P, Hk, D), vs[page], before)
    return {"q": q, "k": kv.reshape(B, W * P, Hk, D), "v": vv.reshape(B, W * P, Hk, D)}


def _softmax_product(q, k, v, seen, scale):
    """q [B, H, R, D], k and v [B, H, S, D], seen [B, 1, R, S]: rows that see nothing give zeros."""
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))


def _plain_cached(st):
    case = st["case"]
    Hq, Hk, D, P, n_max = case["Hq"], case["Hk"], case["D"], case["P"], case["new"]
    G = Hq // Hk
    kc, ks, vc, vs = st["cache"]
    q, q_start, kv_len, pages = st["q"], st["q_start"].long(), st["kv_len"].long(), st["pages"].long()
    B, W, T = pages.shape[0], pages.shape[1], q.shape[0]
    k = (kc[pages].float() * ks[pages][..., None, None]).permute(0, 2, 1, 3, 4).reshape(B, Hk, W * P, D)
    v = (vc[pages].float() * vs[pages][..., None, None, None]).permute(0, 2, 1, 3, 5, 4).reshape(B, Hk, W * P, D)
    n = q_start[1:] - q_start[:-1]
    i = torch.arange(n_max, device=q.device)
    rows = q.float()[(q_start[:-1, None] + i[None, :]).clamp(max=T - 1)]  # [B, n_max, Hq, D]
    rows = rows.reshape(B, n_max, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, n_max * G, D)
    j = torch.arange(W * P, device=q.device)
    last = (kv_len - n)[:, None] + i[None, :] if case["causal"] else (kv_len - 1)[:, None].expand(B, n_max)
    seen = (j[None, None, :] <= last[:, :, None]) & (j[None, None, :] < kv_len[:, None, None])
    seen = seen[:, None, :, None, :].expand(B, 1, n_max, G, W * P).reshape(B, 1, n_max * G, W * P)
    o = _softmax_product(rows, k, v, seen, 1 / math.sqrt(D))
    o = o.reshape(B, Hk, n_max, G, D).permute(0, 2, 1, 3, 4).reshape(B, n_max, Hq, D)
    seq, at = _sequence_of(q_start, T)
    return o[seq, at].to(torch.bfloat16)


def _plain_cross(st):
    case = st["case"]
    Hq, Hk, D, Sq, Sk, B = case["Hq"], case["Hk"], case["D"], case["Sq"], case["Sk"], case["B"]
    G = Hq // Hk
    rows = st["q"].float().reshape(B, Sq, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, Sq * G, D)
    k, v = st["k"].float().permute(0, 2, 1, 3).contiguous(), st["v"].float().permute(0, 2, 1, 3).contiguous()
    seen = torch.ones((B, Sk), dtype=torch.bool, device=k.device)
    if st["kv_len"] is not None:
        seen = seen & (torch.arange(Sk, device=k.device)[None, :] < st["kv_len"].long()[:, None])
    if st["mask"] is not None:
        seen = seen & st["mask"]
    o = _softmax_product(rows, k, v, seen[:, None, None, :].expand(B, 1, Sq * G, Sk), 1 / math.sqrt(D))
    return o.reshape(B, Hk, Sq, G, D).permute(0, 2, 1, 3, 4).reshape(B, Sq, Hq, D).to(torch.bfloat16)


_PLAIN = {"rope": _plain_rope, "append": _plain_append, "cached": _plain_cached, "cross": _plain_cross}


# ---------------------------------------------------------------- the least work of a pass

def work(case):
    kind, Hq, Hk, D = case["kind"], case["Hq"], case["Hk"], case["D"]
    if kind == "rope":
        T = case["T"]
        by = 2 * 2 * T * (Hq + Hk) * D + 4 * T + 4 * T * case["R"] + 8 * D * case["norm"]
        return {"bytes": by, "flops": T * (Hq + Hk) * (3 * case["R"] + 4 * D * case["norm"])}
    if kind == "cross":
        B, Sq = case["B"], case["Sq"]
        keys = sum(_key_lengths(case))
        return {"bytes": 2 * 2 * B * Sq * Hq * D + 2 * 2 * keys * Hk * D + B * case["Sk"] * case["mask"] + 4 * B * case["ragged"],
                "flops": 4 * Sq * keys * Hq * D * (0.8 if case["mask"] else 1.0)}
    n, lens = _lengths(case)
    T, B = sum(n), case["B"]
    used = sum(-(-m // case["P"]) for m in lens)
    if kind == "append":
        touched = sum(m - (m - k) // case["P"] * case["P"] for k, m in zip(n, lens))
        by = 2 * T * (Hq + 2 * Hk) * D + 2 * T * Hq * D + 2 * T * Hk * D + 4 * T * case["R"] + 8 * D * case["norm"]
        by += 2 * touched * Hk * D + 2 * 2 * B * _window(case) * Hk * D
        return {"bytes": by, "flops": T * (Hq + Hk) * (3 * case["R"] + 4 * D * case["norm"]) + 4 * T * Hk * D}
    seen = sum((k * (m - k) + k * (k + 1) // 2) if case["causal"] else k * m for k, m in zip(n, lens))
    return {"bytes": 2 * 2 * T * Hq * D + 2 * sum(lens) * Hk * D + 4 * used + 8 * used * Hk, "flops": 4 * seen * Hq * D}


# ---------------------------------------------------------------- the definitions in 64 bits

def _rotated64(x, case, positions, weight):
    """One token or rows [T, H, D] at their positions, angles in 64 bits."""
    x = x.double().clone()
    if weight is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * weight.double()
    R = case["R"]
    if not R:
        return x
    pair = torch.arange(R // 2, device=x.device)
    ang = positions.double()[:, None] * torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=x.device), -2.0 * pair / R)[None] / case["scale"]
    one, two = (2 * pair, 2 * pair + 1) if case["inter"] else (pair, pair + R // 2)
    z = torch.complex(x[..., one], x[..., two]) * torch.polar(torch.ones_like(ang), ang)[:, None]
    x[..., one], x[..., two] = z.real, z.imag
    return x


def _pages64(x, n, m, P, codes, scale):
    """Values of the pages that tokens [m - n, m) of one sequence touch: x [n, H, D] new, codes [W, H, P, D] and scale [W, H] old."""
    out = []
    for w in range(codes.shape[0]):
        lo = (m - n) // P * P + w * P
        held, c = min(max(m - n - lo, 0), P), codes[w].double()
        got = torch.zeros_like(c)
        i, j = max(lo, m - n) - (m - n), min(lo + P, m) - (m - n)
        if j > i:
            new = x[i:j].permute(1, 0, 2)
            s = new.abs().amax(dim=(1, 2)) / 127
            if held:
                s = torch.maximum(s, scale[w].double())
                got[:, :held] = torch.round(c[:, :held] * (scale[w].double() / s)[:, None, None]) * s[:, None, None]
            got[:, held:held + j - i] = torch.round(new / s[:, None, None]).clamp(-127, 127) * s[:, None, None]
        out.append(got.permute(1, 0, 2))
    return torch.cat(out)


def _attend64(q, k, v, last, scale):
    """q [n, G, D], k and v [S, D]; query i sees the keys up to last[i]."""
    s = (q.reshape(-1, q.shape[2]) @ k.t().contiguous()).reshape(q.shape[0], q.shape[1], -1) * scale
    s.masked_fill_(torch.arange(k.shape[0], device=k.device)[None, None, :] > last[:, None, None], -math.inf)
    p = torch.nan_to_num(torch.softmax(s, dim=-1), nan=0.0)
    return (p.reshape(-1, k.shape[0]) @ v).reshape(q.shape)


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    G = Hq // Hk
    if kind == "rope":
        return tuple(_rotated64(st[x], case, st["positions"], st[w]) for x, w in (("q", "qw"), ("k", "kw")))
    if kind == "cross":
        out = torch.zeros((case["B"], case["Sq"], Hq, D), dtype=torch.float64, device="cuda")
        for b, m in enumerate(_key_lengths(case)):
            on = torch.arange(m, device="cuda")
            if st["mask"] is not None:
                on = on[st["mask"][b, :m]]
            for h in range(Hk):
                if len(on):
                    last = torch.full((case["Sq"],), len(on), device="cuda")
                    out[b, :, h * G:(h + 1) * G] = _attend64(st["q"][b, :, h * G:(h + 1) * G].double(), st["k"][b, on, h].double(),
                                                             st["v"][b, on, h].double(), last, D ** -0.5)
        return out
    n, lens = _lengths(case)
    P, (kc, ks, vc, vs) = case["P"], st["cache"]
    start = np.concatenate(([0], np.cumsum(n)))
    if kind == "append":
        W = _window(case) // P
        slots = torch.cat([torch.arange(m - k, m, device="cuda") for k, m in zip(n, lens)])
        q, k = _rotated64(st["q"], case, slots, st["qw"]), _rotated64(st["k"], case, slots, st["kw"])
        got = {"q": q, "k": torch.zeros((case["B"], W * P, Hk, D), dtype=torch.float64, device="cuda")}
        got["v"] = got["k"].clone()
        for b, m in enumerate(lens):
            page = st["pages"][b, (m - n[b]) // P:-(-m // P)].long()
            for x, y, c, s in ((k, "k", kc[page], ks[page]),
                               (st["v"].double(), "v", vc[page].permute(0, 1, 2, 4, 3).reshape(len(page), Hk, P, D), vs[page])):
                got[y][b, :len(page) * P] = _pages64(x[start[b]:start[b + 1]], n[b], m, P, c, s)
        return got
    out = torch.zeros((int(start[-1]), Hq, D), dtype=torch.float64, device="cuda")
    for b, m in enumerate(lens):
        page = st["pages"][b, :-(-m // P)].long()
        last = torch.arange(m - n[b], m, device="cuda") if case["causal"] else torch.full((n[b],), m, device="cuda")
        for h in range(Hk):
            k = (kc[page, h].double() * ks[page, h].double()[:, None, None]).reshape(-1, D)[:m]
            v = (vc[page, h].double() * vs[page, h].double()[:, None, None, None]).permute(0, 1, 3, 2).reshape(-1, D)[:m]
            at = slice(int(start[b]), int(start[b + 1]))
            out[at, h * G:(h + 1) * G] = _attend64(st["q"][at, h * G:(h + 1) * G].double(), k, v, last, D ** -0.5)
    return out
