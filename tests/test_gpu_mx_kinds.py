"""Every kernel that a microscaled product or projection can take, at a size that takes it: sums that are exact, scales at both
ends, NaN scales; a projection's one launch against its two."""
import pytest

from tests import test_gpu_mx as projections
from tests import test_gpu_mx_edges as edges
from tests.mx_plan_util import PRODUCTS, TOKENS, product_kind, projection_kind

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("test", [edges.test_sums_under_one_scale_are_rounded_once, edges.test_scales_at_both_ends, edges.test_a_scale_that_is_nan])
@pytest.mark.parametrize("kind", PRODUCTS, ids=str)
def test_product(kind, test):
    assert product_kind(*PRODUCTS[kind]) == kind
    test(*PRODUCTS[kind])


@pytest.mark.parametrize("folds", [False, True])
@pytest.mark.parametrize("b", [1, 64, 128])
@pytest.mark.parametrize("kind", TOKENS, ids=str)
def test_projection_in_one_launch(kind, b, folds):
    M, N, K = TOKENS[kind]
    assert projection_kind(M, N, K) == kind
    projections.test_tokens_one_by_one_or_many(M, K, N, b, folds)
