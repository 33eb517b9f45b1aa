"""What making a pool and asking it for room refuse: nothing is written by a call that is refused."""
import numpy as np
import pytest
import torch

from paper_2609_07306_b200.paged import PagedKV
from paper_2609_07306_b200.pages import PagePool

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def cache(table, pages=12, page=4):
    return PagedKV(*(torch.zeros((pages, 1, page, 8), device="cuda") for _ in range(2)), table)


@pytest.mark.parametrize("other", [dict(pages=11), dict(page=8)])
def test_a_refused_pool_leaves_the_table(other):
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    was = table.clone()
    with pytest.raises(ValueError):
        PagePool.empty([cache(table), cache(table, **other)])
    assert torch.equal(table, was)
    with pytest.raises(ValueError):
        PagePool.empty([cache(table)], status=ints([0, 0]))
    assert torch.equal(table, was)
    assert (PagePool.empty([cache(table)]).page_table == -1).all() and (table == -1).all()


def test_room_for_a_number_that_is_whole():
    table = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    pool = PagePool.empty([cache(table)])
    for new in (2.5, 2.0, "2", None, np.float32(1)):
        with pytest.raises(TypeError):
            pool.reserve(ints([0] * 3), new)
    assert (pool.refs == 0).all()
    pool.reserve(ints([0] * 3), np.int64(5))
    assert pool.held.tolist() == [2] * 3
