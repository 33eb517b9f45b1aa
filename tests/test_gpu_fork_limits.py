"""Forks of what should not be there, by the cluster and by the two launches: lengths behind the table's end, page ids outside the pool."""
import pytest
import torch

from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV
from paper_2609_07306_b200.pages import PagePool

pytestmark = pytest.mark.gpu

PAGE = 4


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(batch, width, pages):
    table, status = torch.full((batch, width), -1, dtype=torch.int32, device="cuda"), ints([0])
    kv = PagedKV(*(torch.zeros((pages, 1, PAGE, 8), device="cuda") for _ in range(2)), table, status)
    return PagePool.empty([kv], status)


SHAPES = [(4, 5), (40, 1700)]                              # 20 entries, and 68000: two launches


@pytest.mark.parametrize("batch,width", SHAPES)
def test_lengths_behind_the_table(batch, width):
    """Each is taken as the nearest that the table holds, whether its row stays or is forked, and reported."""
    cap = PAGE * width
    for over in (cap + 1, 0x7FFFFFFF):
        pool = make(batch, width, 3 * width)
        pool.reserve(ints([0] * batch), ints([cap, 7] + [0] * (batch - 2)))
        assert pool.status.item() == 0
        table, refs, new = pool.page_table.clone(), pool.refs.clone(), ints([-9] * batch)
        pool.fork(ints([0, 1, 0] + [-1] * (batch - 3)), ints([over, 7] + [0] * (batch - 2)), new)
        assert new.tolist() == [cap, 7, cap] + [0] * (batch - 3) and pool.status.item() == B.RR_STATUS_BAD_INDEX
        table[2] = table[0]
        refs[table[0].long()] += 1
        assert torch.equal(pool.page_table, table) and torch.equal(pool.refs, refs)
        assert pool.held.tolist() == [width, 2, width] + [0] * (batch - 3)
    pool.status.zero_()
    pool.fork(ints([0, 1, 0] + [-1] * (batch - 3)), ints([cap, 7, cap] + [0] * (batch - 3)), new)     # as long as the table: nothing to report
    assert new.tolist() == [cap, 7, cap] + [0] * (batch - 3) and pool.status.item() == 0


@pytest.mark.parametrize("batch,width", SHAPES)
@pytest.mark.parametrize("bad", [-1, -5, "pages", 0x7FFFFFFF])
def test_ids_outside_the_pool(batch, width, bad):
    """They are left out of the rows that are forked, reported, and held by nobody; the row that has one stays as it is."""
    pages = 3 * width
    bad = pages if bad == "pages" else bad
    pool = make(batch, width, pages)
    pool.reserve(ints([0] * batch), ints([11, 5, 9] + [0] * (batch - 3)))          # pages 0 1 2, 3 4, 5 6 7
    pool.page_table[0, 1] = bad
    pool.page_table[1, 1] = bad
    new = ints([0] * batch)
    pool.fork(ints([0, 0, 0] + [-1] * (batch - 3)), ints([11, 5, 9] + [0] * (batch - 3)), new)
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and new.tolist()[:3] == [11] * 3 and pool.held.tolist()[:3] == [3] * 3
    assert pool.page_table[:3, :4].tolist() == [[0, bad, 2, -1], [0, -1, 2, -1], [0, -1, 2, -1]]
    # page 1 was row 0's before its entry went wrong, page 4 row 1's: nobody has taken them off
    assert pool.refs.tolist()[:9] == [3, 1, 3, 0, 1, 0, 0, 0, 0] and pool.free.item() == pages - 4
