"""The page pool against lists: forks, room, copies on writing, compaction, in long runs of calls and at the sizes where the kernels change their
ways (more rows than warps, than threads, pools of several rounds); strides, layers of unlike caches, refusals of what is not there, graphs, streams."""
import random

import pytest
import torch

from pages_oracle import Pages
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV
from paper_2609_07306_b200.pages import PagePool

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def cache(kind, pages, page, seed):
    """(keys, values) of one layer; kind: type, heads, width, layout."""
    dtype, KH, dh, layout = kind
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)
    if layout == "tokens":                               # heads of a token side by side
        return n(pages, page, KH, dh).transpose(1, 2), n(pages, page, KH, dh).transpose(1, 2)
    if layout == "pair":                                 # keys and values in one pool
        both = n(pages, 2, KH, page, dh)
        return both[:, 0], both[:, 1]
    if layout == "wide":                                 # rows with something behind them
        return n(pages, KH, page, dh + 3)[..., :dh], n(pages, KH, page, dh + 3)[..., :dh]
    return n(pages, KH, page, dh), n(pages, KH, page, dh)


BF, F32 = torch.bfloat16, torch.float32
SMALL = [(BF, 1, 8, "plain")]


def make(batch, width, pages, page, kinds=SMALL, table_pad=0, shift=0):
    table = torch.full((batch, width + table_pad), -1, dtype=torch.int32, device="cuda")[:, :width]
    status = ints([0])
    layers = [cache(k, pages, page, i) for i, k in enumerate(kinds)]
    kvs = [PagedKV(k, v, table, status) for k, v in layers]
    refs = torch.zeros(pages + shift, dtype=torch.int32, device="cuda")[shift:]
    pool = PagePool(table, page, refs, ints([0] * batch), None, kvs, status)
    flat = [c for layer in layers for c in layer]
    return pool, flat, Pages(batch, width, pages, page, flat)


def run(pool, flat, want, steps, seed, every=1):
    """Random calls on both; lens are what a program would have."""
    rng = random.Random(seed)
    batch, page, width = pool.batch, pool.page_tokens, want.width
    lens = [0] * batch
    for i in range(steps):
        kind = rng.choice(("step", "step", "fork", "beams", "roll", "end", "compact", "admit"))
        if kind in ("fork", "beams"):
            p = list(range(batch))
            for b in range(batch):
                if kind == "beams" or rng.random() < 0.3:
                    p[b] = rng.randrange(-1 if rng.random() < 0.2 else 0, batch)
            out = ints([-9] * batch)
            pool.fork(ints(p), ints(lens), out)
            lens = want.fork(p, lens)
            assert out.tolist() == lens
        elif kind == "compact":
            ids = ints([-1] * pool.num_pages)
            pool.compact(ids if rng.random() < 0.5 else None)
            to = want.compact()
            assert ids.tolist() in (to, [-1] * pool.num_pages)
        else:
            new = [rng.randint(0, 3) for _ in range(batch)]
            if kind == "roll":
                lens = [max(0, x - rng.randint(0, 2 * page)) for x in lens]
            elif kind == "end":
                lens = [0 if rng.random() < 0.3 else x for x in lens]
                new = [0] * batch
            elif kind == "admit":
                new = [rng.randint(1, max(1, width * page // 2)) if x == 0 else 1 for x in lens]
            new = [min(n, width * page - x) for x, n in zip(lens, new)]
            if rng.random() < 0.3 and len(set(new)) == 1:
                pool.reserve(ints(lens), new[0])
            else:
                pool.reserve(ints(lens), ints(new))
            ok = want.reserve(lens, new)
            assert pool.status.item() == (0 if ok else B.RR_STATUS_NO_PAGES), (i, kind)
            pool.status.zero_()
            if ok:
                lens = [x + n for x, n in zip(lens, new)]
        if i % every == 0:
            want.check(pool, flat)
    want.check(pool, flat)


KINDS = [(BF, 2, 64, "plain"), (F32, 3, 40, "tokens"), (BF, 1, 7, "wide"), (BF, 4, 16, "pair"), (F32, 2, 6, "wide"), (F32, 1, 64, "tokens"), (BF, 5, 24, "tokens")]


@pytest.mark.parametrize("batch,width,pages,page,kinds", [
    (1, 6, 7, 4, KINDS), (5, 9, 60, 16, KINDS), (7, 12, 50, 1, KINDS), (6, 5, 23, 5, KINDS[:2]), (40, 20, 500, 3, SMALL), (300, 6, 1500, 2, SMALL),
    (3, 70, 130, 8, KINDS[2:5]), (4, 200, 900, 1, SMALL)])
@pytest.mark.parametrize("seed", [1, 2])
def test_runs_of_calls(batch, width, pages, page, kinds, seed):
    run(*make(batch, width, pages, page, kinds, table_pad=seed - 1, shift=seed - 1), steps=40, seed=seed)


@pytest.mark.parametrize("batch,width,pages", [(1100, 3, 2600), (2100, 2, 4300), (20, 30, 40000), (9, 40, 300001), (3, 9, 524288)])
def test_many_rows_and_pages(batch, width, pages):
    """More rows than warps and than threads of a CTA; pages of several CTAs and of several rounds."""
    pool, flat, want = make(batch, width, pages, 2)
    # far pages are in use, the first ones are not: a caller keeps most of the pool
    keep = {p: 1 for p in range(pages - batch * width // 2) if p % 97}
    want.outside = dict(keep)
    ref = torch.zeros(pages, dtype=torch.int32)
    ref[list(keep)] = 1
    pool.refs.copy_(ref)
    pool.free.copy_((ref == 0).sum())
    run(pool, flat, want, steps=14, seed=batch, every=4)


def test_more_layers_than_one_launch():
    pool, flat, want = make(3, 6, 25, 4, [(BF, 1, 8, "plain")] * 64 + [(F32, 2, 4, "tokens"), (BF, 1, 16, "pair")])
    run(pool, flat, want, steps=25, seed=4, every=5)


def test_the_first_of_all_writers_keeps_the_page():
    pool, flat, want = make(4, 4, 20, 8)
    pool.reserve(ints([0, 0, 0, 0]), ints([11, 0, 0, 0]))
    lens = ints([11, 0, 0, 0])
    out = ints([0] * 4)
    pool.fork(ints([0, 0, 0, 0]), lens, out)
    assert out.tolist() == [11] * 4 and pool.refs.tolist()[:3] == [4, 4, 0] and pool.free.item() == 18
    pool.reserve(out, 1)                                  # all write: row 0 keeps page 1
    assert pool.page_table[:, :2].tolist() == [[0, 1], [0, 2], [0, 3], [0, 4]] and pool.refs.tolist()[:5] == [4, 1, 1, 1, 1]
    for c in flat:
        assert all(torch.equal(c[p, :, :3], c[1, :, :3]) for p in (2, 3, 4)) and not torch.equal(c[2, :, 3:], c[1, :, 3:])
    pool.fork(ints([0, 0, 2, 2]), out, lens)
    pool.reserve(lens, ints([1, 0, 0, 1]))                # not all who hold them write: the writers copy
    assert pool.page_table[:, 1].tolist() == [2, 1, 3, 4]
    assert pool.status.item() == 0


def test_taking_tokens_back_below_a_fork():
    """A row that goes on writing inside pages that others hold, and behind tokens that it has given up."""
    pool, flat, want = make(2, 5, 20, 4)
    for args in (([0, 0], [18, 0]),):
        pool.reserve(ints(args[0]), ints(args[1]))
        want.reserve(*args)
    out = ints([0, 0])
    pool.fork(ints([0, 0]), ints([18, 0]), out)
    want.fork([0, 0], [18, 0])
    pool.reserve(ints([6, 18]), ints([9, 0]))             # row 0: 6 tokens stay, 9 new ones: column 1 copied, 2 and 3 replaced, 4 released
    assert want.reserve([6, 18], [9, 0])
    want.check(pool, flat)
    assert pool.page_table[1].tolist() == [0, 1, 2, 3, 4] and pool.page_table[0].tolist() == [0, 5, 6, 7, -1]


def test_too_few_pages():
    """Nothing is given, rows are shortened; the next call that fits goes through."""
    pool, flat, want = make(3, 10, 12, 4)
    for lens, new, ok in (([0, 0, 0], [40, 7, 0], True), ([40, 7, 0], [0, 0, 1], False), ([36, 7, 0], [0, 0, 8], False), ([36, 7, 0], [0, 1, 4], True),
                          ([20, 8, 0], [3, 30, 40], False), ([0, 0, 0], [0, 0, 40], True)):
        pool.status.zero_()
        pool.reserve(ints(lens), ints(new))
        assert want.reserve(lens, new) == ok
        assert pool.status.item() == (0 if ok else B.RR_STATUS_NO_PAGES)
        want.check(pool, flat)


def test_too_few_pages_leaves_shared_ones():
    pool, flat, want = make(2, 5, 6, 4)
    pool.reserve(ints([0, 0]), ints([18, 0]))
    out = ints([0, 0])
    pool.fork(ints([0, 0]), ints([18, 0]), out)
    before = [x.clone() for x in (pool.page_table, pool.refs, pool.held, pool.free, *flat)]
    pool.reserve(ints([7, 18]), ints([13, 0]))            # a copy and three new ones, where one is free
    assert pool.status.item() == B.RR_STATUS_NO_PAGES
    assert all(torch.equal(a, b) for a, b in zip(before, (pool.page_table, pool.refs, pool.held, pool.free, *flat)))


def test_bad_ids_and_lengths():
    pool, flat, want = make(4, 4, 12, 4)
    pool.reserve(ints([0] * 4), ints([9, 5, 3, 0]))       # pages 0-2, 3-4, 5
    assert pool.status.item() == 0
    pool.page_table[0, 1], pool.page_table[1, 1] = 12, -7
    pool.reserve(ints([9, 5, -3, 0]), ints([0, 0, 2, 0])) # a negative length is 0
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and pool.refs.tolist() == [1] * 6 + [0] * 6
    pool.status.zero_()
    pool.reserve(ints([0, 0, 0, 0]), 0)                   # bad ids are left out: pages 1 and 4 are not released
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and pool.refs.tolist() == [0, 1, 0, 0, 1] + [0] * 7 and pool.free.item() == 10
    assert (pool.page_table == -1).all() and (pool.held == 0).all()
    pool.status.zero_()
    pool.reserve(ints([0, 0, 0, 17]), 0)                  # behind the table's end: as much as it holds
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and pool.held.tolist() == [0, 0, 0, 4]
    pool.status.zero_()
    pool.reserve(ints([0, 3, 0, 16]), ints([0x7FFFFFFF, 1, -5, 0]))
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and pool.held.tolist() == [4, 1, 0, 4] and pool.free.item() == 12 - 2 - 9
    pool.status.zero_()
    out = ints([0] * 4)
    pool.fork(ints([4, 1, -2, 0]), ints([2, 3, -4, 16]), out)
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and out.tolist() == [2, 3, 0, 2]
    assert pool.held.tolist()[3] == 1 and pool.page_table[3, 0] == pool.page_table[0, 0]


def test_a_bad_page_is_replaced_where_it_will_be_written():
    pool, flat, want = make(1, 4, 10, 4)
    pool.reserve(ints([0]), 16)
    pool.page_table[0, 2] = 77
    pool.reserve(ints([8]), 8)
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX and pool.page_table.tolist() == [[0, 1, 4, 3]] and pool.refs.tolist()[:6] == [1, 1, 1, 1, 1, 0]


def test_compaction_moves_what_the_caller_keeps():
    pool, flat, want = make(3, 6, 30, 4, KINDS[:3])
    pool.reserve(ints([0] * 3), ints([20, 24, 16]))       # 0-4, 5-10, 11-14
    prefix = pool.page_table[2, :2].clone()
    pool.refs[11:13] += 1                                 # the caller keeps two pages of the last one
    want.rows, want.outside = [list(range(5)), list(range(5, 11)), list(range(11, 15))], {11: 1, 12: 1}
    for lens in ([20, 0, 16], [20, 0, 0]):
        pool.reserve(ints(lens), 0)
        want.reserve(lens, [0] * 3)
    kept = [c[11:13].clone() for c in flat]
    ids = ints([0] * 30)
    pool.compact(ids)
    assert ids.tolist() == want.compact()
    want.check(pool, flat)
    now = ids[prefix.long()].long()
    assert now.tolist() == [5, 6] and all(torch.equal(c[now], k) for c, k in zip(flat, kept))
    pool.compact()                                        # nothing moves
    want.check(pool, flat)


def test_pages_behind_32_bit_offsets():
    pages, page, dh = 270000, 64, 128
    k, v = (torch.empty((pages, 1, page, dh), device="cuda", dtype=BF) for _ in range(2))
    table = torch.full((2, 3), -1, dtype=torch.int32, device="cuda")
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[-5:] = 0
    pool = PagePool(table, page, refs, ints([0, 0]), None, [PagedKV(k, v, table)])
    pool.reserve(ints([0, 0]), ints([100, 0]))
    assert table[0].tolist() == [pages - 5, pages - 4, -1]
    for c in (k, v):
        c[-5:].normal_()
    out = ints([0, 0])
    pool.fork(ints([0, 0]), ints([100, 0]), out)
    pool.reserve(out, ints([0, 1]))
    assert table[1].tolist() == [pages - 5, pages - 3, -1]
    assert all(torch.equal(c[-3, :, :36], c[-4, :, :36]) and not torch.equal(c[-3, :, 36:], c[-4, :, 36:]) for c in (k, v))
    refs[:pages - 5] = 0
    pool.reserve(ints([0, 100]), 0)
    was = [c[[-5, -3]].clone() for c in (k, v)]
    pool.compact()
    assert table[1].tolist() == [0, 1, -1] and all(torch.equal(c[:2], w) for c, w in zip((k, v), was)) and pool.free.item() == pages - 2


def test_captured_and_replayed():
    """A step of beam search as a graph: each replay goes on from where the last one ended."""
    pool, flat, want = make(6, 8, 60, 4, KINDS[:2])
    lens, out, parents, new = ints([9] * 6), ints([0] * 6), ints([0] * 6), ints([1] * 6)
    pool.reserve(ints([0] * 6), 9)
    want.reserve([0] * 6, [9] * 6)

    def step():
        pool.fork(parents, lens, out)
        pool.reserve(out, new)
        lens.copy_(out + new)

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step()
    now, rng = [9] * 6, random.Random(3)
    for _ in range(15):
        p = [rng.randrange(6) for _ in range(6)]
        parents.copy_(ints(p))
        graph.replay()
        now = want.fork(p, now)
        assert want.reserve(now, [1] * 6)
        now = [x + 1 for x in now]
        assert lens.tolist() == now
        want.check(pool, flat)
    pool.compact()
    want.compact()
    want.check(pool, flat)


def test_another_stream():
    pool, flat, want = make(5, 9, 60, 4, KINDS[:2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(pool, flat, want, steps=20, seed=8, every=4)
    torch.cuda.current_stream().wait_stream(side)


def test_the_same_call_gives_the_same_bits():
    outs = []
    for _ in range(3):
        pool, flat, _ = make(300, 10, 2500, 3)
        rng = random.Random(5)
        out = ints([0] * 300)
        pool.reserve(ints([0] * 300), ints([rng.randint(1, 20) for _ in range(300)]))
        pool.fork(ints([rng.randrange(300) for _ in range(300)]), pool.held * 3 - 1, out)
        pool.reserve(out, 2)
        pool.reserve(out * (ints([rng.random() < 0.6 for _ in range(300)])), 0)
        pool.compact()
        outs.append([x.clone() for x in (pool.page_table, pool.refs, pool.held, pool.free, *flat)])
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))


def test_what_the_wrapper_refuses():
    pool, flat, want = make(3, 4, 12, 4)
    table, kv = pool.page_table, pool.caches[0]
    good = lambda: ints([0] * 3)
    for call, kind in ((lambda: PagePool(table, 5, pool.refs, pool.held, None, [kv]), ValueError), (lambda: PagePool(table, 4, pool.refs[:5], pool.held, None, [kv]), ValueError),
                       (lambda: PagePool(table.cpu(), 4, pool.refs, pool.held), ValueError), (lambda: PagePool(table, 4, pool.refs.float(), pool.held), TypeError),
                       (lambda: PagePool(table, 4, pool.refs, pool.held[:2]), ValueError), (lambda: PagePool(table, 4, pool.refs, pool.held, good()), ValueError),
                       (lambda: PagePool(table.t(), 4, pool.refs, pool.held), ValueError), (lambda: PagePool.empty([]), ValueError),
                       (lambda: pool.fork(good()[:2], good(), good()), ValueError), (lambda: pool.fork(good().long(), good(), good()), TypeError),
                       (lambda: pool.fork(good(), good(), good().cpu()), ValueError), (lambda: pool.reserve(good(), -1), ValueError),
                       (lambda: pool.reserve(good(), 1 << 31), ValueError), (lambda: pool.reserve(good(), good()[:1]), ValueError),
                       (lambda: pool.reserve(good().view(3, 1)), ValueError), (lambda: pool.compact(good()), ValueError),
                       (lambda: PagePool(table, 4, pool.refs, pool.held).compact(), ValueError),
                       (lambda: PagePool(table, 4, pool.refs, pool.held).reserve(good()), ValueError)):
        with pytest.raises(kind):
            call()
    same = good()
    with pytest.raises(B.RouteRelayError):
        pool.fork(good(), same, same)
    for name in ("page_table", "refs", "held", "free", "status", "caches"):
        with pytest.raises(AttributeError):
            setattr(pool, name, None)
    empty = PagePool.empty([kv])
    assert empty.free.item() == 12 and (empty.page_table == -1).all() and empty.page_table is table


@pytest.mark.parametrize("pages", [7000, 140000])
def test_many_pages_at_once(pages):
    """More new pages than a CTA hands out by itself, from the gaps of a pool; copies and replaced pages among them."""
    pool, flat, want = make(12, 900, pages, 2)
    rng = random.Random(pages)
    keep = {p: 1 for p in range(pages) if rng.random() < 0.2}
    want.outside = dict(keep)
    pool.refs[list(keep)] = 1
    pool.free.fill_(pages - len(keep))
    for lens, new, parents in (([0] * 12, [700] * 6 + [0] * 6, [0, 0, 0, 3, 4, 5, 1, 1, 5, 5, 9, -1]),
                               ([700, 301, 401, 700, 3, 99, 1, 0, 1, 700, 0, 0], [900, 1, 1200, 0, 800, 777, 899, 1100, 0, 2, 0, 0], list(range(12)))):
        pool.reserve(ints(lens), ints(new))
        assert want.reserve(lens, new)
        want.check(pool, flat)
        out = ints([0] * 12)
        after = [x + n for x, n in zip(lens, new)]
        pool.fork(ints(parents), ints(after), out)
        assert out.tolist() == want.fork(parents, after)
        want.check(pool, flat)
    pool.compact()
    want.compact()
    want.check(pool, flat)
    assert pool.status.item() == 0


@pytest.mark.parametrize("batch,width", [(33, 2000), (700, 97), (2200, 31)])
def test_forks_of_long_tables(batch, width):
    """Tables that take all SMs, forked one call behind the other, with rows that end and parents that there are not."""
    pool, flat, want = make(batch, width, batch * width + 9, 2)
    rng = random.Random(width)
    lens = [rng.randint(0, 2 * width - 2) for _ in range(batch)]
    pool.reserve(ints(lens), 1)
    assert want.reserve(lens, [1] * batch)
    now, other = ints(lens), ints([0] * batch)
    for call in range(4):
        p = [rng.randrange(-1, batch) if rng.random() < 0.7 else b for b in range(batch)]
        bad = list(p)
        if call == 2:
            bad[1], bad[5], p[1], p[5] = batch, -2, 1, 5
        pool.fork(ints(bad), now, other)
        now, other = other, now
        lens = want.fork(p, lens)
    assert pool.status.item() == B.RR_STATUS_BAD_INDEX
    assert now.tolist() == lens
    want.check(pool, flat)


@pytest.mark.parametrize("batch,width,pages,page,kinds", [
    (1, 1, 1, 1, [(BF, 1, 1, "plain")]), (1, 1, 2, 1, [(F32, 1, 1, "tokens")]), (2, 1, 3, 7, [(BF, 3, 1, "pair")]), (3, 2, 4, 1000, [(BF, 1, 256, "plain")]),
    (2, 2, 5, 3, [(F32, 1, 3, "tokens")]), (4, 600, 2500, 1, [(BF, 8, 128, "plain")]), (2, 3, 8, 2048, [(BF, 2, 64, "tokens")]),
    (3, 4, 14, 33, [(BF, 7, 72, "tokens"), (F32, 5, 12, "plain")])])
def test_smallest_and_odd_sizes(batch, width, pages, page, kinds):
    run(*make(batch, width, pages, page, kinds), steps=40, seed=page)
