"""Refusals of the attention entry points (CPU: every call here fails a check or has nothing to do, so no kernel is
launched), through the C ABI's descriptors and the Python binding."""
import ctypes

import pytest
import torch

from paper_2609_24433_amd import fq

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, ALIAS = 1, 2, 3, 4, 5, 7
A = 0x100000  # addresses that are never dereferenced, 256 MB apart


def at(i, off=0):
    return A + i * 0x10000000 + off


def heads(p=None, bs=0, ts=512, hs=64):
    return fq._HEADS(at(1) if p is None else p, bs, ts, hs)


def rope(table=0, length=0, positions=0, qw=0, kw=0, eps=1e-6, rot=0, inter=0):
    return fq._ROPE(table, length, positions, qw, kw, eps, rot, inter, 0)


def cache(kc=at(2), ks=at(3), vc=at(4), vs=at(5), pages=8, H=2, P=64, D=64):
    return fq._CACHE(kc, ks, vc, vs, pages, H, P, D, 0)


def batch(qs=at(6), kl=at(7), pt=at(8), width=4, seqs=2, new=3, kv=200):
    return fq._BATCH(qs, kl, pt, width, seqs, new, kv)


def qk_rope(q=heads(), Hq=4, k=heads(at(2)), Hk=2, r=rope(), T=5, D=64, yq=at(3), yk=at(4)):
    return fq.LIB.fq_qk_rope(q, Hq, k, Hk, r, T, D, yq, yk, None)


def append(c=cache(), b=batch(), k=heads(at(9)), v=heads(at(10)), q=heads(at(11)), Hq=4, r=rope(), T=5, y=at(12)):
    return fq.LIB.fq_cache_append(c, b, k, v, q, Hq, r, T, y, None)


def read(c=cache(), pt=at(8), width=4, first=at(6), last=at(7), seqs=2, n=10, k=at(9), v=at(10)):
    return fq.LIB.fq_cache_read(c, pt, width, first, last, seqs, n, k, v, None)


def attend(q=heads(at(9)), Hq=4, T=5, c=cache(), b=batch(), scale=0.125, out=at(12), ws=at(13), n=1 << 28):
    return fq.LIB.fq_cache_attention(q, Hq, T, c, b, scale, 1, out, ws, n, None)


def cross(q=heads(at(1), 4096), k=heads(at(2), 4096), v=heads(at(3), 4096), kl=None, mask=None, ms=0, B=2, Sq=5, Sk=7, Hq=4, Hk=2, D=64,
          scale=0.125, out=at(4), ws=at(13), n=1 << 28):
    return fq.LIB.fq_cross_attention(q, k, v, kl, mask, ms, B, Sq, Sk, Hq, Hk, D, scale, out, ws, n, None)


@pytest.mark.parametrize("call,want", [
    (lambda: qk_rope(q=None), NULL), (lambda: qk_rope(q=heads(0)), NULL), (lambda: qk_rope(k=None), NULL),
    (lambda: qk_rope(r=None), NULL), (lambda: qk_rope(yq=None), NULL), (lambda: qk_rope(yk=None), NULL),
    (lambda: qk_rope(D=72), UNSUPPORTED), (lambda: qk_rope(D=0), UNSUPPORTED), (lambda: qk_rope(D=272), UNSUPPORTED),
    (lambda: qk_rope(T=-1), SHAPE), (lambda: qk_rope(T=1 << 25), UNSUPPORTED), (lambda: qk_rope(Hq=-1), SHAPE),
    (lambda: qk_rope(Hq=1025), UNSUPPORTED), (lambda: qk_rope(q=heads(at(1, 8))), ALIGN), (lambda: qk_rope(q=heads(ts=516)), ALIGN),
    (lambda: qk_rope(q=heads(ts=-512)), SHAPE), (lambda: qk_rope(q=heads(ts=1 << 33)), UNSUPPORTED), (lambda: qk_rope(yq=at(3, 4)), ALIGN),
    (lambda: qk_rope(r=rope(at(5), 10, rot=80)), SHAPE), (lambda: qk_rope(r=rope(at(5), 10, rot=24)), UNSUPPORTED),
    (lambda: qk_rope(r=rope(at(5), 10, rot=-16)), SHAPE), (lambda: qk_rope(r=rope(0, 10, rot=32)), NULL),
    (lambda: qk_rope(r=rope(at(5), 0, rot=32)), SHAPE), (lambda: qk_rope(r=rope(eps=-1.0)), UNSUPPORTED),
    (lambda: qk_rope(r=rope(eps=float("nan"))), UNSUPPORTED), (lambda: qk_rope(r=rope(qw=at(5, 4))), ALIGN),
    (lambda: qk_rope(r=rope(positions=at(5, 2))), ALIGN),
    (lambda: qk_rope(yq=at(1)), ALIAS), (lambda: qk_rope(yk=at(3)), ALIAS), (lambda: qk_rope(yq=at(2, 256)), ALIAS),
    (lambda: qk_rope(r=rope(qw=at(3, 64))), ALIAS),
    (lambda: qk_rope(T=0, q=None, yq=None), 0), (lambda: qk_rope(Hq=0, Hk=0), 0),
])
def test_qk_rope(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("call,want", [
    (lambda: append(c=None), NULL), (lambda: append(c=cache(kc=0)), NULL), (lambda: append(c=cache(vs=0)), NULL),
    (lambda: append(c=cache(P=48)), UNSUPPORTED), (lambda: append(c=cache(P=256)), UNSUPPORTED), (lambda: append(c=cache(D=8)), UNSUPPORTED),
    (lambda: append(c=cache(H=0)), SHAPE), (lambda: append(c=cache(pages=0)), SHAPE), (lambda: append(c=cache(vc=at(4, 8))), ALIGN),
    (lambda: append(b=None), NULL), (lambda: append(b=batch(qs=0)), NULL), (lambda: append(b=batch(pt=0)), NULL),
    (lambda: append(b=batch(seqs=-1)), SHAPE), (lambda: append(b=batch(seqs=70000)), UNSUPPORTED), (lambda: append(b=batch(new=-1)), SHAPE),
    (lambda: append(b=batch(kv=300)), SHAPE), (lambda: append(b=batch(kl=at(7, 2))), ALIGN), (lambda: append(b=batch(kv=1 << 40, width=1 << 27)), UNSUPPORTED),
    (lambda: append(k=None), NULL), (lambda: append(v=heads(0)), NULL), (lambda: append(q=None), NULL), (lambda: append(y=None), NULL),
    (lambda: append(y=at(12, 8)), ALIGN), (lambda: append(k=heads(at(9), hs=12)), ALIGN), (lambda: append(r=rope(at(14), 9, rot=128)), SHAPE),
    (lambda: append(k=heads(at(2))), ALIAS), (lambda: append(y=at(4)), ALIAS), (lambda: append(y=at(11)), ALIAS), (lambda: append(b=batch(pt=at(3))), ALIAS),
    (lambda: append(c=cache(vc=at(2, 256))), ALIAS), (lambda: append(b=batch(seqs=65535, new=1 << 24, kv=0), Hq=1024), UNSUPPORTED),
    (lambda: append(T=0, k=None, v=None), 0), (lambda: append(b=batch(seqs=0, qs=0, kl=0, pt=0)), 0), (lambda: append(b=batch(new=0)), 0),
])
def test_cache_append(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("call,want", [
    (lambda: read(c=None), NULL), (lambda: read(pt=None), NULL), (lambda: read(first=None), NULL), (lambda: read(seqs=-1), SHAPE),
    (lambda: read(n=-1), SHAPE), (lambda: read(n=1 << 31), UNSUPPORTED), (lambda: read(k=at(9, 8)), ALIGN), (lambda: read(last=at(7, 1)), ALIGN),
    (lambda: read(k=at(2)), ALIAS), (lambda: read(v=at(9)), ALIAS), (lambda: read(c=cache(P=17)), UNSUPPORTED),
    (lambda: read(n=0), 0), (lambda: read(seqs=0), 0), (lambda: read(k=None, v=None), 0),
])
def test_cache_read(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("call,want", [
    (lambda: attend(q=None), NULL), (lambda: attend(c=None), NULL), (lambda: attend(b=None), NULL), (lambda: attend(out=None), NULL),
    (lambda: attend(Hq=5), SHAPE), (lambda: attend(Hq=0), SHAPE), (lambda: attend(T=-2), SHAPE), (lambda: attend(scale=0.0), UNSUPPORTED),
    (lambda: attend(scale=float("inf")), UNSUPPORTED), (lambda: attend(scale=float("nan")), UNSUPPORTED), (lambda: attend(scale=-1.0), UNSUPPORTED),
    (lambda: attend(out=at(12, 2)), ALIGN), (lambda: attend(b=batch(kv=257)), SHAPE), (lambda: attend(out=at(9)), ALIAS), (lambda: attend(out=at(5)), ALIAS),
    (lambda: attend(out=at(6)), ALIAS), (lambda: attend(T=0, q=None), 0), (lambda: attend(b=batch(seqs=0, qs=0, kl=0, pt=0)), 0),
    (lambda: attend(b=batch(new=1 << 24), Hq=1024), UNSUPPORTED),
])
def test_cache_attention(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("call,want", [
    (lambda: cross(q=None), NULL), (lambda: cross(k=heads(0, 4096)), NULL), (lambda: cross(v=None), NULL), (lambda: cross(out=None), NULL),
    (lambda: cross(D=40), UNSUPPORTED), (lambda: cross(Hq=3), SHAPE), (lambda: cross(B=-1), SHAPE), (lambda: cross(B=65536), UNSUPPORTED),
    (lambda: cross(Sq=-1), SHAPE), (lambda: cross(Sk=-1), SHAPE), (lambda: cross(Sk=1 << 25), UNSUPPORTED), (lambda: cross(scale=-0.5), UNSUPPORTED),
    (lambda: cross(k=heads(at(2), 4100)), ALIGN), (lambda: cross(out=at(4, 8)), ALIGN), (lambda: cross(kl=at(5, 3)), ALIGN),
    (lambda: cross(mask=at(5), ms=-1), SHAPE), (lambda: cross(out=at(1)), ALIAS), (lambda: cross(out=at(3)), ALIAS),
    (lambda: cross(mask=at(4), ms=7), ALIAS), (lambda: cross(kl=at(4)), ALIAS), (lambda: cross(B=0), 0), (lambda: cross(Sq=0, q=None), 0),
])
def test_cross_attention(call, want):
    assert call() == want, fq.LIB.fq_last_error()


@pytest.mark.parametrize("long,taken,call", [
    (lambda: fq.cache_attention_workspace_bytes(2, 4, 2, 64, 2, 1, 100000), at(9), lambda n, ws: attend(
        b=batch(width=2000, new=1, kv=100000), T=2, ws=ws, n=n)),
    (lambda: fq.cross_attention_workspace_bytes(2, 5, 100000, 4, 2, 64), at(1), lambda n, ws: cross(Sk=100000, ws=ws, n=n)),
])
def test_workspaces(long, taken, call):
    need = long()
    if need:  # the tokens are split: the partial results need room
        assert call(need - 1, at(13)) == WORKSPACE
        assert call(need, None) == WORKSPACE
        assert call(need, at(13, 8)) == ALIGN
        assert call(need, taken) == ALIAS
    assert fq.cache_attention_workspace_bytes(0, 4, 2, 64, 2, 1, 100) == 0
    assert fq.cache_attention_workspace_bytes(5, 4, 3, 64, 2, 1, 100) == 0
    assert fq.cross_attention_workspace_bytes(1, 1, 0, 4, 2, 64) == 0
    assert fq.cross_attention_workspace_bytes(1, 1, 100, 4, 2, 60) == 0


def test_rope_table():
    t = fq.LIB.fq_rope_table
    assert t(at(1), 1.0, -1, 4, at(2), None) == SHAPE and t(at(1), 1.0, 5, 129, at(2), None) == UNSUPPORTED
    assert t(None, 1.0, 5, 4, at(2), None) == NULL and t(at(1), 1.0, 5, 4, at(1, 16), None) == ALIAS
    assert t(at(1), 1.0, 5, 4, at(2, 4), None) == ALIGN and t(None, 1.0, 0, 4, None, None) == 0
    assert ctypes.sizeof(ctypes.c_void_p) == 8 and len(heads()) == 32 and len(rope()) == len(cache()) == len(batch()) == 56


# ---------------------------------------------------------------- the binding

@pytest.fixture
def no_stream(monkeypatch):
    monkeypatch.setattr(fq, "_stream_handle", lambda: 0)


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def host_cache():
    return fq.kv_cache(4, 2, 16, 64, device="cpu")


@pytest.mark.parametrize("call", [
    lambda: fq.qk_rope(bf(5, 4, 64).float(), None, None),
    lambda: fq.qk_rope(bf(5, 64, 4).transpose(1, 2), None, None),
    lambda: fq.qk_rope(bf(5, 4, 64), bf(4, 2, 64), None),
    lambda: fq.qk_rope(bf(5, 4, 64), bf(5, 2, 32), None),
    lambda: fq.qk_rope(bf(5, 4, 64), None, torch.zeros(9, 16)),
    lambda: fq.qk_rope(bf(5, 4, 64), None, torch.zeros(9, 16, 2).double()),
    lambda: fq.qk_rope(bf(5, 4, 64), None, None, i32(1, 2, 3)),
    lambda: fq.qk_rope(bf(5, 4, 64), None, None, torch.zeros(5, dtype=torch.int64)),
    lambda: fq.qk_rope(bf(5, 4, 64), None, None, q_weight=torch.ones(32)),
    lambda: fq.qk_rope(bf(5, 4, 64), None, None, q_out=bf(5, 4, 32)),
    lambda: fq.cache_append(host_cache(), i32(0, 1)[None], i32(0, 1), i32(1), 1, bf(1, 3, 64), bf(1, 3, 64)),
    lambda: fq.cache_append(host_cache(), i32(0, 1)[None], i32(0), i32(1), 1, bf(1, 2, 64), bf(1, 2, 64)),
    lambda: fq.cache_append(host_cache(), i32(0, 1), i32(0, 1), i32(1), 1, bf(1, 2, 64), bf(1, 2, 64)),
    lambda: fq.cache_append(host_cache()._replace(k_scale=torch.zeros(4, 3)), i32(0, 1)[None], i32(0, 1), i32(1), 1, bf(1, 2, 64), bf(1, 2, 64)),
    lambda: fq.cache_append(host_cache()._replace(v_codes=torch.zeros(4, 2, 16, 64, dtype=torch.int8)), i32(0, 1)[None], i32(0, 1), i32(1), 1, bf(1, 2, 64), bf(1, 2, 64)),
    lambda: fq.cache_append(host_cache(), i32(0, 1)[None], i32(0, 1), i32(1), 1, bf(1, 2, 64), bf(1, 2, 64), bf(2, 4, 64)),
    lambda: fq.cache_read(host_cache(), i32(0, 1)[None], i32(0, 0), i32(1), 4),
    lambda: fq.cache_read(host_cache(), i32(0, 1)[None], i32(0), i32(1), 4, k_out=bf(1, 3, 2, 64)),
    lambda: fq.cache_attention(bf(1, 4, 32), host_cache(), i32(0, 1)[None], i32(0, 1), i32(1), 1, 16),
    lambda: fq.cache_attention(bf(1, 4, 64), host_cache(), i32(0, 1)[None], i32(0, 1), i32(1), 1, 16, out=bf(1, 4, 32)),
    lambda: fq.cross_attention(bf(2, 5, 4, 64), bf(2, 7, 2, 64), bf(2, 8, 2, 64)),
    lambda: fq.cross_attention(bf(2, 5, 4, 64), bf(2, 7, 2, 32), bf(2, 7, 2, 32)),
    lambda: fq.cross_attention(bf(2, 5, 4, 64), bf(2, 7, 2, 64), bf(2, 7, 2, 64), i32(1)),
    lambda: fq.cross_attention(bf(2, 5, 4, 64), bf(2, 7, 2, 64), bf(2, 7, 2, 64), None, torch.zeros(2, 7)),
])
def test_the_binding_refuses(call, no_stream):
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("call,status", [
    (lambda: fq.qk_rope(bf(5, 4, 72), None, None), UNSUPPORTED),
    (lambda: fq.qk_rope(bf(5, 4, 68)[:, :, :64], None, None), ALIGN),
    (lambda: fq.cache_attention(bf(1, 3, 64), host_cache(), i32(0, 1)[None], i32(0, 1), i32(1), 1, 16), SHAPE),
    (lambda: fq.cache_attention(bf(1, 4, 64), host_cache(), i32(0, 1)[None], i32(0, 1), i32(1), 1, 33), SHAPE),
    (lambda: fq.cross_attention(bf(2, 5, 3, 64), bf(2, 7, 2, 64), bf(2, 7, 2, 64)), SHAPE),
])
def test_the_librarys_errors_come_through(call, status, no_stream):
    with pytest.raises(fq.FQError) as e:
        call()
    assert e.value.status == status
