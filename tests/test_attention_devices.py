"""The attention entry points take the addresses of tensors of one GPU only: one that lies elsewhere (lengths are often
made on the host) is refused before its address reaches a kernel.  No GPU needed: tensors that claim to be on GPU 0, and a
library that would accept every call."""
import pytest
import torch

from paper_2609_24433_amd import fq


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


def gpu(t):
    return t.as_subclass(OnGpu)


class Lib:
    """Accepts every call; counts those that would launch."""

    def __init__(self):
        self.launched = 0

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda *a: 256

        def call(*a):
            self.launched += 1
            return fq.FQ_OK
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Lib()
    monkeypatch.setattr(fq, "LIB", lib)
    monkeypatch.setattr(fq, "_stream_handle", lambda: 0)
    return lib


def bf(*shape):
    return gpu(torch.zeros(shape, dtype=torch.bfloat16))


def i32(*v):
    return gpu(torch.tensor(v, dtype=torch.int32))


def cache():
    return {f"cache.{n}": gpu(t) for n, t in fq.kv_cache(4, 2, 16, 64, device="cpu")._asdict().items()}


def taken(t):
    return fq.KVCache(*(t[f"cache.{n}"] for n in fq.KVCache._fields))


def rope_inputs():
    return dict(table=gpu(torch.zeros(9, 16, 2)), positions=i32(1, 2, 3), q_weight=gpu(torch.ones(64)), k_weight=gpu(torch.ones(64)))


def batch():
    return dict(page_table=gpu(torch.zeros((2, 3), dtype=torch.int32)), q_start=i32(0, 1, 3), kv_len=i32(5, 6))


CALLS = {
    "qk_rope": (lambda: dict(q=bf(3, 4, 64), k=bf(3, 2, 64), q_out=bf(3, 4, 64), k_out=bf(3, 2, 64), **rope_inputs()),
                lambda t: fq.qk_rope(t["q"], t["k"], t["table"], t["positions"], t["q_weight"], t["k_weight"], q_out=t["q_out"], k_out=t["k_out"])),
    "cache_append": (lambda: dict(k=bf(3, 2, 64), v=bf(3, 2, 64), q=bf(3, 4, 64), q_out=bf(3, 4, 64), **cache(), **batch(), **rope_inputs()),
                     lambda t: fq.cache_append(taken(t), t["page_table"], t["q_start"], t["kv_len"], 2, t["k"], t["v"], t["q"], t["table"],
                                               t["positions"], t["q_weight"], t["k_weight"], q_out=t["q_out"])),
    "cache_read": (lambda: dict(page_table=batch()["page_table"], first=i32(0, 0), last=i32(3, 4), k_out=bf(2, 7, 2, 64), v_out=bf(2, 7, 2, 64), **cache()),
                   lambda t: fq.cache_read(taken(t), t["page_table"], t["first"], t["last"], 7, t["k_out"], t["v_out"])),
    "cache_attention": (lambda: dict(q=bf(3, 4, 64), ws=gpu(torch.zeros(256, dtype=torch.uint8)), out=bf(3, 4, 64), **cache(), **batch()),
                        lambda t: fq.cache_attention(t["q"], taken(t), t["page_table"], t["q_start"], t["kv_len"], 2, 6, ws=t["ws"], out=t["out"])),
    "cross_attention": (lambda: dict(q=bf(2, 5, 4, 64), k=bf(2, 7, 2, 64), v=bf(2, 7, 2, 64), kv_len=i32(3, 4),
                                     key_mask=gpu(torch.ones((2, 7), dtype=torch.bool)), ws=gpu(torch.zeros(256, dtype=torch.uint8)), out=bf(2, 5, 4, 64)),
                        lambda t: fq.cross_attention(t["q"], t["k"], t["v"], t["kv_len"], t["key_mask"], ws=t["ws"], out=t["out"])),
}


@pytest.mark.parametrize("name,which", [(n, w) for n, (make, _) in CALLS.items() for w in make()])
def test_a_tensor_of_another_device_is_refused(name, which, lib):
    make, call = CALLS[name]
    t = make()
    call(t)
    assert lib.launched == 1
    t[which] = t[which].as_subclass(torch.Tensor)
    with pytest.raises(ValueError):
        call(t)
    assert lib.launched == 1


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_with_all_its_tensors_on_the_host_is_refused(name, monkeypatch):
    """(the library's own checks, which launch nothing: they end at an overlap that the binding gives them)"""
    monkeypatch.setattr(fq, "_stream_handle", lambda: 0)
    make, call = CALLS[name]
    with pytest.raises(ValueError, match="on the host"):
        call({k: v.as_subclass(torch.Tensor) for k, v in make().items()})


def test_keys_alone_on_the_host_are_refused(monkeypatch):
    monkeypatch.setattr(fq, "_stream_handle", lambda: 0)
    q, k = (torch.zeros((3, n, 64), dtype=torch.bfloat16) for n in (0, 2))
    with pytest.raises(ValueError, match="on the host"):
        fq.qk_rope(q, k, None)
    with pytest.raises(ValueError):
        fq.rope_table(4, fq.rope_frequencies(64)[0], device="cpu")
