"""The rows in place, scales far apart, queries that are not finite and the page calls' rules in the checked build of the library
(-DAASD_BOUNDS_CHECK): each case ends with a status that holds no AASD_STATUS_INTERNAL."""
import pytest

import test_gpu_kv_not_finite as nan
import test_gpu_kv_share_rules as rules
import test_gpu_kvb_far_scales as far
import test_gpu_kvb_in_place as place
from paper_2505_13204_b200 import binding, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(lib=binding.load_library(build.build(check=True)))
    yield c
    c.close()


@pytest.mark.parametrize("case", place.CASES)
def test_checked_rows_in_place(ctx, case):
    for dtype, rot in (("bf16", "all"), ("f32", "part")):
        place.test_queries_and_keys_in_place(ctx, *case, dtype, rot)


@pytest.mark.parametrize("G,D", [(3, 64), (60, 64), (60, 256), (200, 128)])
def test_checked_scales_far_apart(ctx, G, D):
    far.test_pages_of_small_values_keep_their_weight(ctx, far.SIZES[2], G, D, 1.0)


@pytest.mark.parametrize("shape", nan.SHAPES)
@pytest.mark.parametrize("bits", [4, 8])
def test_checked_rows_with_nan(ctx, shape, bits):
    nan.test_rows_with_nan(ctx, *shape, "one long", bits)


def test_checked_rules_of_the_page_calls(ctx):
    place.test_outputs_over_anything_else_are_refused(ctx)
    rules.test_neighbouring_arrays_and_empty_ones_are_no_overlap(ctx)
    rules.test_compact_looks_at_tables_when_nothing_moves(ctx)
    for B in (4, 40):
        rules.test_a_shared_page_that_is_about_to_be_written_is_reported(ctx, B)
