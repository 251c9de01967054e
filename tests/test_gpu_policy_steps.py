"""The example's denoising steps share a prompt in the cache: they leave it as it was read, and one step knows nothing of
another's actions."""
import importlib.util
import os

import pytest
import torch

from tests.attention_util import ints
from tests.gpu_util import flush

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("policy_attention", os.path.join(
    os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_attention.py"))


def load():
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("prefix,actions,page", [(130, 50, 64), (128, 50, 64), (40, 5, 128)])
def test_steps_leave_the_prompt_as_it_was_read(prefix, actions, page):
    from paper_2609_24433_amd import fq
    flush(f"policy steps prefix={prefix} actions={actions} page={page}")
    m = load()

    def prompt(steps):
        _, _, caches, pages = m.run(layers=1, steps=steps, prefix=prefix, actions=actions, page=page)
        return [t for c in caches for t in fq.cache_read(c, pages, ints([0]), ints([prefix]), prefix)]
    for a, b in zip(prompt(0), prompt(3)):
        assert torch.equal(a, b)


def test_a_step_knows_nothing_of_the_one_before():
    flush("policy steps one after another")
    m = load()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    p = m.Policy(2, 130, 50, 64, gen)
    p.read(torch.randn((130, 2048), generator=gen, device="cuda").to(torch.bfloat16))
    y = torch.randn((50, 1024), generator=gen, device="cuda").to(torch.bfloat16)
    want = p.velocity(y)
    assert torch.isfinite(want).all()
    for other in (64 * y, torch.full_like(y, float("nan")), torch.full_like(y, float("inf"))):
        p.velocity(other)
        assert torch.equal(p.velocity(y), want)
