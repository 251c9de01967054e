"""The example that runs the attention operators between quantized projections: its layers against the same projections
around the definition of attention in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import attention as ref
from tests.attention_util import ints, plain_v, sequence
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("policy_attention", os.path.join(
    os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_attention.py"))


def load():
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs():
    flush("policy_attention at its defaults, shorter")
    m = load()
    y, x, caches, pages = m.run(layers=2, steps=2, prefix=130, actions=50)
    assert y.shape == (50, 1024) and torch.isfinite(y).all() and torch.isfinite(x).all()
    y2 = m.run(layers=2, steps=2, prefix=130, actions=50)[0]
    assert torch.equal(y, y2)


def test_a_layer_is_projection_attention_projection():
    m = load()
    from paper_2609_24433_amd import fq
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    layer = m.CachedLayer(1024, 8, 2, 128, gen)
    n, P = 70, 32
    cache = fq.kv_cache(4, 2, P, 128)
    table = np.array([[2, 0, 3]])
    rope = fq.rope_table(n, *fq.rope_frequencies(128))
    x = torch.randn((n, 1024), generator=gen, device="cuda").to(torch.bfloat16)
    got = layer(x, cache, (ints(table), ints([0, n]), ints([n])), rope, n, n, True)
    h = layer.qkv(x).view(n, 12, 128).double().cpu().numpy()
    q = ref.norm_rotate(h[:, :8], rope.cpu().numpy(), np.arange(n), layer.q_norm.cpu().numpy())
    kc, vc = cache.k_codes.cpu().numpy(), plain_v(cache.v_codes.cpu().numpy())
    ks, vs = cache.k_scale.cpu().numpy(), cache.v_scale.cpu().numpy()
    k = ref.norm_rotate(h[:, 8:10], rope.cpu().numpy(), np.arange(n), layer.k_norm.cpu().numpy())
    a = np.zeros((n, 8, 128))
    seen = np.arange(n)[None] <= np.arange(n)[:, None]
    for i in range(8):
        keys, values = sequence(table, kc, ks, 0, n, i // 4), sequence(table, vc, vs, 0, n, i // 4)
        # the cache holds the layer's keys and values within a step of their page
        assert np.abs(keys - k[:, i // 4]).max() <= ks[:, i // 4].max() and np.abs(values - h[:, 10 + i // 4]).max() <= vs[:, i // 4].max()
        a[:, i] = ref.attention(q[:, i], keys, values, seen, 128 ** -0.5)[0]
    want = x.float() + layer.o(torch.from_numpy(a.reshape(n, 1024)).to("cuda", torch.bfloat16)).float()
    # bf16 queries (2^-8 of their size) and attention outputs, then 8-bit codes of the outputs (1/254 of a row's largest): 2 % of a row
    err = (got.float() - want).norm(dim=1) / want.norm(dim=1)
    assert err.max().item() < 0.02
