"""The 8-bit cache's and the page operators' calls in the checked build of the library (-DAASD_BOUNDS_CHECK): the cases of
test_gpu_kvb and test_gpu_kv_share walk every kernel and launch shape, and each of them ends with a status of 0, which holds
AASD_STATUS_INTERNAL too."""
import pytest

import test_gpu_kv_share as share
import test_gpu_kvb as kvb
from paper_2505_13204_b200 import binding, build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(lib=binding.load_library(build.build(check=True)))
    yield c
    c.close()


@pytest.mark.parametrize("case", kvb.WRITES)
def test_checked_write(ctx, case):
    kvb.test_write(ctx, *case)


@pytest.mark.parametrize("case", kvb.ATTENDS)
@pytest.mark.parametrize("trees", [False, True])
def test_checked_attend(ctx, case, trees):
    kvb.test_attend(ctx, *case, trees)


@pytest.mark.parametrize("case", [kvb.LONG[i] for i in (0, 2, 4, 5, 8, 10)])
def test_checked_attend_long(ctx, case):
    kvb.test_attend_long(ctx, *case)


@pytest.mark.parametrize("case", kvb.COMMITS)
@pytest.mark.parametrize("packed", [False, True])
def test_checked_commit_and_read(ctx, case, packed):
    kvb.test_commit(ctx, *case, packed)
    kvb.test_read(ctx, case[5], "bf16")


@pytest.mark.parametrize("case", [(8, 3, 300, 20), (40, 10, 1000, 100), (30, 9, 700, 7), (100, 30, 500, 300)])
def test_checked_pages(ctx, case):
    share.test_fork_free_compact(ctx, *case)
    share.test_copy(ctx, 3, 9, 2, 8208, 4)


def test_checked_calls_on_what_they_have_to_refuse_or_report(ctx):
    """Bad tables, parents, slots, books and offsets are found by the calls' own checks, before an index is made of them."""
    for f in (kvb.test_write_reports_bad_pages_and_positions_and_stays_in_bounds, kvb.test_commit_reports_bad_parents_and_moves_nothing,
              share.test_fork_refuses_what_cannot_be, share.test_inconsistent_books_are_reported_and_nothing_outside_is_touched):
        f(ctx)
        assert ctx.poll_status() == 0
    for rows in (5, 60):
        kvb.test_attend_reports_bad_tables_and_parents(ctx, rows)
        assert ctx.poll_status() == 0
