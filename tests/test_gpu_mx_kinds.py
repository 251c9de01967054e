"""Every kernel that a microscaled product can take, at a size that takes it: sums that are exact, scales at both ends, NaN scales."""
import pytest

from tests import test_gpu_mx_edges as edges
from tests.mx_plan_util import PRODUCTS, product_kind

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("test", [edges.test_sums_under_one_scale_are_rounded_once, edges.test_scales_at_both_ends, edges.test_a_scale_that_is_nan])
@pytest.mark.parametrize("kind", PRODUCTS, ids=str)
def test_product(kind, test):
    assert product_kind(*PRODUCTS[kind]) == kind
    test(*PRODUCTS[kind])
