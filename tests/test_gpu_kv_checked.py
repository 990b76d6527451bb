"""The cache's calls in the checked build of the library (-DAASD_BOUNDS_CHECK): the cases of
test_gpu_kv walk every kernel and launch shape, and each of them ends with a status of 0, which
holds AASD_STATUS_INTERNAL too."""
import pytest

import test_gpu_kv as kv
from paper_2505_13204_b200 import binding, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(lib=binding.load_library(build.build(check=True)))
    yield c
    c.close()


@pytest.mark.parametrize("case", kv.PLANS)
@pytest.mark.parametrize("kind", ["step", "scarce", "churn"])
def test_checked_plan(ctx, case, kind):
    kv.test_plan(ctx, *case, kind)


@pytest.mark.parametrize("case", kv.WRITES)
def test_checked_write(ctx, case):
    kv.test_write(ctx, *case)


@pytest.mark.parametrize("case", kv.ATTENDS)
@pytest.mark.parametrize("tree", [False, True])
def test_checked_attend(ctx, case, tree):
    kv.test_attend(ctx, *case, tree)


@pytest.mark.parametrize("case", [kv.LONG[i] for i in (0, 2, 4, 5, 8, 10)])
def test_checked_attend_long(ctx, case):
    kv.test_attend_long(ctx, *case)


@pytest.mark.parametrize("case", [(6, 9, 200, 2, 128, 3), (3, 70, 64, 1, 256, 5)])
@pytest.mark.parametrize("packed", [False, True])
def test_checked_commit_and_read(ctx, case, packed):
    kv.test_commit(ctx, *case, packed)
    kv.test_read(ctx, case[4], "bf16")


def test_checked_calls_on_what_they_have_to_refuse_or_report(ctx):
    """Bad tables, parents, slots and offsets are found by the calls' own checks, before an index is made of them."""
    for f in (kv.test_plan_leaves_out_packed_tokens_that_do_not_fit, kv.test_plan_reports_inconsistent_books_and_stays_in_bounds,
              kv.test_write_reports_positions_and_slots_out_of_range, kv.test_attend_reports_bad_tables_and_parents,
              kv.test_commit_reports_bad_parents_and_moves_nothing):
        f(ctx)
        assert ctx.poll_status() == 0
