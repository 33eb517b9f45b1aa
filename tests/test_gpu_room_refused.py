"""A step whose pages could not be given: what is appended behind a refused reserve leaves other sequences' tokens and its own length alone, in the same
graph and without anyone reading the status in between; the verification takes no such token for kept; the next reserve that succeeds opens the rows again."""
import pytest
import torch

from pages_oracle import Pages
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV, inv_freq
from paper_2609_07306_b200.pages import PagePool
from paper_2609_07306_b200.verify import verify_drafts

pytestmark = pytest.mark.gpu

PAGE, WIDTH, KH, DH = 4, 8, 2, 16
BIG = 0x7FFFFFFF


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make(batch, pages, layers=2, status=True, width=WIDTH):
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    bits = ints([0]) if status else None
    g = torch.Generator(device="cuda").manual_seed(batch)
    kvs = [PagedKV(*(torch.randn((pages, KH, PAGE, DH), generator=g, device="cuda") for _ in range(2)), table, bits) for _ in range(layers)]
    return PagePool.empty(kvs, bits), kvs


def tokens(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((n, KH, DH), generator=g, device="cuda") for _ in range(2)]


def append(kvs, lens, new, after, seed=1, axes=False):
    cu = ints([0] + new).cumsum(0).int()
    k, v = tokens(sum(new) + 2, seed)                      # (two of padding)
    more = dict(inv_freq=inv_freq(DH), positions=torch.zeros((1, sum(new) + 2), dtype=torch.int32, device="cuda")) if axes else {}
    for kv in kvs:
        kv.append(k, v, lens, cu=cu, new_lens=after, **more)
    return k, v, cu


def graphed(captured, call):
    if not captured:
        return call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    graph.replay()
    return out


# (rows' tokens of the only sequence, parents, lens and new of the refused call, lengths behind the append)
CASES = {
    # a row has taken back a token that another one still has on the page that it would go on writing
    "shared_page": (6, 18, [0, 0, -1], [18, 17, 0], [0, 8, 0], [18, 17, 0]),
    # all who hold the page want to write, the first one would have kept it
    "all_write": (6, 18, [0, 0, 0], [18, 18, 18], [1, 1, 1], [18, 18, 18]),
    # pages behind a row's tokens that are another one's
    "pages_behind": (6, 20, [0, 0, -1], [20, 8, 0], [0, 8, 0], [20, 8, 0]),
    # nothing shared, pages missing; a row that has them goes on
    "missing": (6, 18, [0, -1, -1], [18, 0, 0], [1, 9, 0], [19, 0, 0]),
    # the page that a row goes on writing is its own, the pages behind it are missing: it gets all of its tokens or none
    "part": (5, 18, [0, -1, -1], [18, 0, 0], [3, 0, 0], [18, 0, 0]),
}


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("axes", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_append_behind_a_refused_reserve(name, axes, captured):
    pages, first, parents, lens, new, want = CASES[name]
    pool, kvs = make(3, pages)
    pool.reserve(ints([0, 0, 0]), ints([first, 0, 0]))
    after = ints([0, 0, 0])
    append(kvs, ints([0, 0, 0]), [first, 0, 0], after, 7)
    out = ints([0, 0, 0])
    pool.fork(ints(parents), after, out)
    assert pool.status.item() == 0
    lists = Pages(3, WIDTH, pages, PAGE)                   # (a refused call shortens rows)
    lists.reserve([0, 0, 0], [first, 0, 0])
    lists.fork(parents, [first, 0, 0])
    assert not lists.reserve(lens, new)
    state = [x for kv in kvs for x in (kv.k_cache, kv.v_cache)]
    before, length, reach, got = [x.clone() for x in state], ints(lens), ints(new), ints([-7] * 3)
    cu, (k, v) = ints([0] + new).cumsum(0).int(), tokens(sum(new) + 2, 1)
    freq, pos = inv_freq(DH), torch.zeros((1, sum(new) + 2), dtype=torch.int32, device="cuda")

    def step():
        pool.reserve(length, reach)
        for kv in kvs:
            kv.append(k, v, length, cu=cu, new_lens=got, **(dict(inv_freq=freq, positions=pos) if axes else {}))

    graphed(captured, step)
    assert pool.status.item() == B.RR_STATUS_NO_PAGES and got.tolist() == want
    # what was written: the tokens of the rows that had room, and nothing else
    at = 0
    for b, n in enumerate(new):
        for i in range(n if want[b] > lens[b] else 0):
            page, place = pool.page_table[b, (lens[b] + i) // PAGE].item(), (lens[b] + i) % PAGE
            for j, x in enumerate((k, v) * len(kvs)):
                assert torch.equal(state[j][page, :, place], x[at + i])
                before[j][page, :, place] = x[at + i]
        at += n
    assert all(torch.equal(a, b) for a, b in zip(before, state))
    lists.check(pool)


@pytest.mark.parametrize("status", [False, True])
def test_rows_are_open_again(status):
    """A refused step that is repeated when another sequence has ended; without a status word as well."""
    pool, kvs = make(3, 6, status=status)
    after, out = ints([0] * 3), ints([0] * 3)
    pool.reserve(ints([0] * 3), ints([18, 0, 0]))
    append(kvs, ints([0] * 3), [18, 0, 0], after, 7)
    pool.fork(ints([0, 0, -1]), after, out)
    for _ in range(2):
        pool.reserve(out, ints([1, 5, 0]))
        append(kvs, out, [1, 5, 0], after)
        assert after.tolist() == out.tolist() == [18, 18, 0]
    pool.reserve(ints([0, 18, 0]), ints([0, 5, 0]))        # the first one ends
    k, v, _ = append(kvs, ints([0, 18, 0]), [0, 5, 0], after)
    assert after.tolist() == [0, 23, 0]
    for kv in kvs:
        for i in range(5):
            page, place = pool.page_table[1, (18 + i) // PAGE].item(), (18 + i) % PAGE
            assert torch.equal(kv.k_cache[page, :, place], k[i]) and torch.equal(kv.v_cache[page, :, place], v[i])


def test_many_rows():
    """More rows than a CTA has threads: every one that shares its page is closed, every one that does not is open."""
    batch = 1300
    pool, kvs = make(batch, batch + 400, layers=1, width=3)
    after, out = ints([0] * batch), ints([0] * batch)
    pool.reserve(after, ints([3] * batch))
    after.fill_(3)
    parents = [b - b % 3 if b < 900 else b for b in range(batch)]      # threes share a page, the others have theirs
    pool.fork(ints(parents), after, out)
    before = kvs[0].k_cache.clone()
    new = [1] * 1299 + [9]                                # 600 copies and two pages, 1000 are free; then a call that needs more than there are
    pool.reserve(out, ints([9] * batch))
    append(kvs, out, [1] * batch, after)
    closed = [3 + (b >= 900) for b in range(batch)]
    assert after.tolist() == closed and pool.status.item() == B.RR_STATUS_NO_PAGES
    shared = sorted({pool.page_table[b, 0].item() for b in range(900)})
    assert torch.equal(kvs[0].k_cache[shared], before[shared])
    pool.status.zero_()
    pool.reserve(out, ints(new))
    append(kvs, out, new, after)
    assert pool.status.item() == 0 and after.tolist() == [3 + n for n in new]


@pytest.mark.parametrize("greedy", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verification_of_tokens_that_had_no_room(greedy, dtype):
    vocab, batch = 300, 4
    lens, rows = [5, 9, 0, 7], [3, 4, 0, 2]
    cu = ints([0] + rows).cumsum(0).int()
    T = sum(rows) + 1
    g = torch.Generator(device="cuda").manual_seed(3)
    target = torch.softmax(torch.randn((T, vocab), generator=g, device="cuda"), 1).to(dtype)
    best = target.float().argmax(1).int()
    toks = torch.cat((best[:1], best[:-1])).contiguous()   # all drafts are their row's best
    u = None if greedy else torch.zeros(T, device="cuda")
    for room, closed in (([BIG] * 4, []), ([8, 13, 0, 9], []), ([7, 13, 0, 9], [0]), ([0, 12, 0, 8], [0, 1, 3])):
        plain, new, in_place = ints([0] * batch), ints([0] * batch), ints(lens)
        out, a = verify_drafts(target, toks, cu, uniform=u, lens=ints(lens), new_lens=plain)
        got, b = verify_drafts(target, toks, cu, uniform=u, lens=ints(lens), new_lens=new, room=ints(room))
        _, c = verify_drafts(target, toks, cu, uniform=u, lens=in_place, new_lens=in_place, room=ints(room))
        _, d = verify_drafts(target, toks, cu, uniform=u, lens=ints(lens), room=ints(room))
        assert plain.tolist() == [8, 13, 0, 9]
        for i in range(batch):
            n = a[i].item()
            assert b[i].item() == c[i].item() == d[i].item() == (-1 if i in closed else n)
            assert new[i].item() == in_place[i].item() == (lens[i] if i in closed else plain[i].item())
            if i not in closed:
                assert torch.equal(out[cu[i]:cu[i + 1]], got[cu[i]:cu[i + 1]])


def test_a_step_as_one_graph():
    """Room, appending, verification, with the lengths in place: replayed until the pool is empty and beyond; the lengths stop where the pages do."""
    pool, kvs = make(2, 7, layers=1)
    lens, after, new = ints([0, 0]), ints([0, 0]), ints([3, 3])
    cu, (k, v) = ints([0, 3, 6]), tokens(6, 2)
    target = torch.zeros((6, 50), device="cuda")
    target[:, 11] = 1.0
    toks = ints([11] * 6)
    pool.reserve(lens, 5)                                 # (so that no launch is the first one in the graph)
    pool.reserve(lens, 0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.reserve(lens, new)
        kvs[0].append(k, v, lens, cu=cu, new_lens=after)
        _, accepted = verify_drafts(target, toks, cu, lens=lens, new_lens=lens, room=pool.room)
    seen = []
    for _ in range(8):
        graph.replay()
        seen.append((lens.tolist(), accepted.tolist(), after.tolist()))
    # pages of 4: 3, 6, 9 and 12 tokens take 2, 4, 6 and 6 of 7 pages; 15 would take 8
    assert seen == [([n, n], [2, 2], [n, n]) for n in (3, 6, 9, 12)] + [([12, 12], [-1, -1], [12, 12])] * 4
    assert pool.status.item() == B.RR_STATUS_NO_PAGES


def test_caches_of_more_rows_than_the_pool():
    pool, kvs = make(3, 9, layers=1)
    table = torch.full((5, WIDTH), -1, dtype=torch.int32, device="cuda")
    table[4, 0] = 8
    other = PagedKV(torch.zeros_like(kvs[0].k_cache), torch.zeros_like(kvs[0].v_cache), table)
    pool = PagePool(pool.page_table, PAGE, pool.refs, pool.held, pool.free, [kvs[0], other], pool.status)
    assert pool.room.shape == (3,) and (pool.room == BIG).all()
    after = ints([0] * 5)
    k, v, _ = append([other], ints([0] * 5), [0, 0, 0, 0, 2], after)
    assert after.tolist() == [0, 0, 0, 0, 2] and torch.equal(other.k_cache[8, :, :2].transpose(0, 1), k[:2])
    with pytest.raises(AttributeError):
        pool.room = None
