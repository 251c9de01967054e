"""Which kernel a microscaled product takes (no GPU needed): every one of them is in the lists that the GPU tests go through."""
import math
import random

import pytest

from paper_2609_24433_amd import fq
from tests.mx_plan_util import PRODUCTS, STREAM, TILE, TOKENS, plan, product_kind, projection_kind


@pytest.mark.parametrize("kind", PRODUCTS)
def test_a_size_for_every_product(kind):
    assert product_kind(*PRODUCTS[kind]) == kind


@pytest.mark.parametrize("kind", TOKENS)
def test_a_size_for_every_projection_of_one_launch(kind):
    assert projection_kind(*TOKENS[kind]) == kind


def test_no_size_takes_a_kernel_that_is_not_listed():
    assert len(PRODUCTS) == len(STREAM) + 2 * len(TILE)
    r = random.Random(3)
    seen = set()
    for _ in range(60000):
        log = lambda lo, hi: int(math.exp(r.uniform(math.log(lo), math.log(hi))))  # noqa: E731
        M = r.choice([1, 2, log(2, 64), log(16, 8192), log(64, 4096)])
        N, K = max(1, log(16, 40000) // 16) * 16, max(1, log(128, 32768) // 128) * 128
        seen.add(product_kind(M, N, K))
        if plan(M, N, K).token:
            seen.add(projection_kind(M, N, K))
    assert seen == set(PRODUCTS) | set(TOKENS)


def test_scratch_is_that_of_the_kernel():
    for M, N, K in [*PRODUCTS.values(), *TOKENS.values()]:
        p = plan(M, N, K)
        partial = p.splits * M * N * 4 if p.splits > 1 else 0
        assert fq.mx_gemm_workspace_bytes(M, N, K) == partial
        up = lambda n: -(-n // 256) * 256  # noqa: E731
        assert fq.mx_linear_workspace_bytes(M, N, K) == (0 if p.token else up(M * K // 2) + up(M * K // 32) + partial)
