"""Where compaction says that each page is now: pools of one round and of several, with and without moves; without new_ids nothing but the pool is written."""
import random

import pytest
import torch

from pages_oracle import Pages
from paper_2609_07306_b200.paged import PagedKV
from paper_2609_07306_b200.pages import PagePool

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("pages,kept", [(1, 0.5), (33, 0.5), (4097, 0.3), (40000, 0.97), (131072, 0.5), (131073, 0.5), (300001, 0.02), (524288, 0.6)])
def test_new_ids(pages, kept):
    batch, width = 5, 12
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(pages)
    k, v = (torch.randn((pages, 1, 2, 4), generator=g, device="cuda") for _ in range(2))
    pool, want = PagePool.empty([PagedKV(k, v, table)]), Pages(batch, width, pages, 2, [k, v])
    rng = random.Random(pages)
    want.outside = {p: 1 for p in range(pages) if rng.random() < kept}
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[list(want.outside)] = 1
    pool.refs.copy_(refs)
    free = pages - len(want.outside)
    pool.free.fill_(free)
    new = [min(2 * width, 2 * (free // batch))] * batch    # the lowest free pages, two tokens each
    pool.reserve(ints([0] * batch), ints(new))
    assert want.reserve([0] * batch, new)
    for call in range(3):
        ids = torch.full((pages + 2,), -9, dtype=torch.int32, device="cuda")
        pool.compact(ids[1:-1])
        assert ids.tolist() == [-9] + want.compact() + [-9]
        want.check(pool, [k, v])
        if call == 0:                                      # every second page of the rows and every third of the caller's is given up
            new = [2 * ((n // 2 + 1) // 2) for n in new]
            pool.reserve(ints(new), 0)
            want.reserve(new, [0] * batch)
            drop = [p for p in want.outside if rng.random() < 0.3]
            for p in drop:
                del want.outside[p]
            if drop:
                pool.refs[drop] -= 1
            pool.free.add_(len(drop))
        if call == 1:
            before = pool.page_table.clone()
            pool.compact()                                 # nothing moves
            assert torch.equal(before, pool.page_table)
