"""Plans over tables and stacks that name pages that are none: a slot that passes 31 bits is not another page's."""

import numpy as np
import pytest

import paper_2602_07721_amd as pk
from pages import ints

pytestmark = pytest.mark.gpu


# Products of page and page size that wrap 32 bits to 0, to a small slot, below 0, or that do not wrap.
@pytest.mark.parametrize("page", [16, 65536, 100000, 2 ** 24])
@pytest.mark.parametrize("count,t", [(1, 8), (5, 64), (5, 5000)])
@pytest.mark.parametrize("popped", [False, True])
def test_rows_of_pages_that_are_none_have_no_slot(page, count, t, popped):
    bad = [2 ** 32 // page, 2 ** 31 // page + 1, 4, -1, 2 ** 31 - 1, -2 ** 31, 3]
    bad = [min(max(x, -2 ** 31), 2 ** 31 - 1) for x in bad]
    print(f"[plan] page {page} counts {count} t {t} popped {popped}", flush=True)
    for x in bad:
        # The second sequence's new rows: in a page that it has, or in one that it takes from the stack.
        table = np.array([[0, 0], [x, 0], [1, 0]])
        free = np.array([x if popped else 2, 0, 0, 0])
        lens = [3, 0 if popped else 2, 4]
        plan = pk.plan_pages(ints(table), ints(free), ints([1]), ints(lens), ints([count] * 3), page, t=t)
        want = np.full(t, -1)
        for b, at in ((0, 0), (1, x), (2, 1)):
            slots = at * page + lens[b] + np.arange(count)
            want[b * count:(b + 1) * count] = np.where((at >= 0) & (slots < 2 ** 31), slots, -1)
        assert np.array_equal(plan.slots.cpu().numpy(), want), f"page {x}"
        assert list(plan.counts.cpu().numpy()) == [count] * 3
        assert list(plan.positions.cpu().numpy()[:3 * count]) == [n + i for n in lens for i in range(count)]
