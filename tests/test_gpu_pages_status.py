"""The pool's status: each thing that does not fit sets its bit by itself, and what fits sets none."""
import pytest
import torch

import paper_2302_01318_b200 as sps
from pages_util import DEV, I32, Device, ints
from test_gpu_pages import grown

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [40, 24577])
@pytest.mark.parametrize("lens,want,bit", [((-1, 9), (0, 9), sps.PAGED_BAD_LENGTH), ((-2 ** 31, 9), (3, 9), sps.PAGED_BAD_LENGTH), ((30, 9), (-1, 9), sps.PAGED_BAD_LENGTH),
                                           ((30, 9), (30, -2 ** 31), sps.PAGED_BAD_LENGTH), ((33, 9), (33, 9), sps.PAGED_BAD_LENGTH), ((30, 9), (49, 9), sps.PAGED_BAD_LENGTH),
                                           ((32, 16), (0, 48), 0), ((0, 0), (0, 0), 0)])
def test_reserve_tells_of_each_count_outside_its_row(n_pages, lens, want, bit):
    m, d = grown(n_pages, 8, [30, 9], ld=6)
    d.t.lens.copy_(ints(lens))
    d.reserve(list(want))
    assert int(d.pool.status) == bit
    assert d.t.lens.tolist() == [min(max(n, 0), 8 * len(r), max(w, 0)) for n, r, w in zip(lens, m.rows, want)]


@pytest.mark.parametrize("parents,bit", [((0, 1, -1), 0), ((0, 1, -2), sps.PAGED_BAD_ROW), ((-2 ** 31, 1, 0), sps.PAGED_BAD_ROW), ((0, 3, 1), sps.PAGED_BAD_ROW),
                                         ((0, 1, 2 ** 31 - 1), sps.PAGED_BAD_ROW)])
def test_fork_tells_of_each_parent_outside_the_table(parents, bit):
    m, d = grown(40, 8, [30, 9, 17])
    m.fork([p if 0 <= p < 3 else -1 for p in parents])
    d.fork(list(parents))
    d.check(m, bit)


@pytest.mark.parametrize("parents", [(0, 1, 2), (2, 0, 1), (0, 0, 0), (1, 1, 2), (-1, -1, -1)])
@pytest.mark.parametrize("page", [40, -1, 2 ** 31 - 1])
@pytest.mark.parametrize("row,entry", [(0, 0), (0, 3), (2, 1)])
def test_fork_tells_of_a_page_outside_the_pool_however_many_children_its_row_has(parents, page, row, entry):
    m, d = grown(40, 8, [30, 9, 17])
    d.t.pages[row, entry] = page
    d.fork(list(parents))
    assert int(d.pool.status) == sps.PAGED_BAD_PAGE
    for i, p in enumerate(parents):
        if p == row:
            assert int(d.t.pages[i, entry]) == page


def test_fork_and_compact_hand_a_length_on_as_it_is():
    m, d = grown(40, 8, [30, 9, 17])
    d.t.lens.copy_(ints([-5, 1000, 17]))
    d.fork([2, 1, 0])
    assert d.t.lens.tolist() == [17, 1000, -5] and int(d.pool.status) == 0
    d.compact()
    assert d.t.lens.tolist() == [17, 1000, -5] and int(d.pool.status) == 0


def test_a_pool_without_a_status_takes_what_does_not_fit_just_so():
    m, d = grown(40, 8, [30, 9, 17])
    d.pool._c.status = None
    d.t.pages[0, 0] = 41
    d.fork([0, -7, 9])
    d.reserve([31, -3, 2 ** 31 - 1])
    assert int(d.pool.status) == 0 and d.t.held.tolist()[:2] == [4, 0]
