"""Infinities and NaN among values that a row may not see, where tiles are multiplied whole: long contexts, every schedule (items apart,
behind a prefix, cut, quartered, whole in turn), rows that see one and share a tile with another."""
import pytest
import torch

import paged_exact as exact
from paged_oracle import assert_within
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
KINDS = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 80), (torch.float32, 64), (torch.float32, 20), (torch.float32, 200)]


def pool(dtype, Bn, KH, dh, page, cap, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-cap // page)
    k, v = (torch.randn((Bn * width, KH, page, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    return g, k, v, torch.randperm(Bn * width, generator=g, device="cuda").view(Bn, width).int()


def put(v, table, b, tok, head, col, x):
    page = v.shape[2]
    v[int(table[b, tok // page]), head, tok % page, col] = x


def shared_call(g, k, v, table, heads, lens, news, prefix=0, causal=True, scale=None):
    dh, cu = k.shape[3], [0]
    for n in news:
        cu.append(cu[-1] + n)
    scale = dh ** -0.5 if scale is None else scale
    q = torch.randn((cu[-1], heads, dh), generator=g, device="cuda").to(k.dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(k, v, table, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), prefix, scale, causal=causal,
                                                     cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    want, bound = exact.shared(q, k, v, table, lens, cu, scale, causal)
    assert status.item() == 0
    assert_within(got, want, bound)
    return got, want


@pytest.mark.parametrize("dtype,dh,heads", [(torch.bfloat16, 128, 4), (torch.bfloat16, 64, 3), (torch.float32, 64, 4)])
def test_a_long_context(dtype, dh, heads):
    """A prompt behind 100000 tokens: one value that all rows see, one that the first half may not, one behind every row but the last; and a
    second sequence beside it that has none of them."""
    n, L = 100, 100000
    g, k, v, table = pool(dtype, 2, 1, dh, 64, L + n, 1)
    put(v, table, 0, 77, 0, 5, NAN)
    put(v, table, 0, L + n // 2, 0, 9, INF)
    put(v, table, 0, L + n // 2 + 3, 0, 9, NAN)
    put(v, table, 0, L + n - 1, 0, 11, -INF)
    got, want = shared_call(g, k, v, table, heads, [L + n, 900], [n, 40])
    hit = torch.zeros(got.shape, dtype=torch.bool)
    hit[:n, :, 5] = True
    hit[n // 2:n, :, 9] = True
    hit[n - 1, :, 11] = True
    assert torch.equal(~got.isfinite().cpu(), hit)
    assert (got[n // 2:n // 2 + 3, :, 9] == INF).all()


def test_many_rows_that_see_one():
    """2000 queries of 8 heads behind a NaN that all of them see: looked at, not computed again, and the same bits beside its column."""
    g, k, v, table = pool(torch.bfloat16, 1, 2, 128, 16, 6000, 2)
    state = g.get_state()
    clean, _ = shared_call(g, k, v, table, 8, [6000], [2000])
    put(v, table, 0, 3, 1, 64, NAN)
    g.set_state(state)
    got, _ = shared_call(g, k, v, table, 8, [6000], [2000])
    assert got[:, 4:, 64].isnan().all()
    got[:, 4:, 64] = clean[:, 4:, 64]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("heads,prefix,lens,news", [
    (4, 300, [400, 500, 340], [64, 64, 64]),           # each sequence by itself
    (4, 300, [400, 500, 340, 301], [3, 40, 7, 1]),     # behind the prefix's tiles
    (40, 300, [400, 120, 30, 0], [2, 1, 1, 1]),        # sequences shorter than the prefix: its later tokens are not theirs
    (8, 0, [700], [1]), (20, 0, [700], [9]), (300, 0, [700], [3])])
def test_every_schedule(dtype, dh, heads, prefix, lens, news):
    for causal in (True, False):
        g, k, v, table = pool(dtype, len(lens), 1, dh, 16, 704, heads)
        if prefix:                                     # the same tokens for all: whole pages shared, the rest copied
            table[:, :prefix // 16] = table[0, :prefix // 16].clone()
            for c in (k, v):
                for b in range(1, len(lens)):
                    c[table[b, prefix // 16].long(), :, :prefix % 16] = c[table[0, prefix // 16].long(), :, :prefix % 16].clone()
        for b, (n, L) in enumerate(zip(news, lens)):
            if L - n >= prefix and n > 2:
                put(v, table, b, L - n // 2, 0, 3 + b, (NAN, INF, -INF, NAN)[b])
                put(v, table, b, L - 1, 0, 3 + b, (INF, NAN, NAN, NAN)[b])
        if prefix:
            put(v, table, 0, 200, 0, 15, INF)
            put(v, table, 0, 31, 0, 15, -INF)
        if heads == 8:
            put(v, table, 0, 600, 0, 15, INF)
        shared_call(g, k, v, table, heads, lens, news, prefix, causal)


def ranges_call(dtype, dh, G, KH, lens, n_q, m, rows, causal, hurt, seed=0, slots=3):
    g, k, v, table = pool(dtype, len(lens), KH, dh, 16, max(lens), seed)
    hurt(v, table)
    rg = torch.full((len(rows), slots, 2), -1, dtype=torch.int32)
    for i, spans in enumerate(rows):
        rg[i, :len(spans)] = torch.tensor(spans, dtype=torch.int32)
    q = torch.randn((len(lens), KH * G, n_q * m, dh), generator=g, device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(k, v, table, status).attend_ranges(q, rg.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), n_q, dh ** -0.5, causal=causal)
    want, bound = exact.ranged(q, k, v, table, lens, rows, n_q, dh ** -0.5, causal)
    assert status.item() == 0
    assert_within(got, want, bound)
    assert not want.isfinite().all() and want.isfinite().any()


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("n_q,m,G", [(6, 64, 4), (6, 16, 1), (4, 3, 3), (6, 33, 10), (6, 3, 8)])
def test_ranges(dtype, dh, n_q, m, G):
    T = n_q * m

    def hurt(v, table):
        put(v, table, 0, T - m // 2 - 1, 0, 7, NAN)
        put(v, table, 0, T - 1, 0, 8, INF)
        put(v, table, 1, 2, 0, 9, -INF)
        put(v, table, 1, m + m // 2, 0, 9, INF)
    rows = [[(0, min(m, 40)), (i * m, i * m + m)] if i else [(0, m)] for i in range(n_q)] * 2
    ranges_call(dtype, dh, G, 1, [T, T], n_q, m, rows, True, hurt, seed=m)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("n_q,m,G", [(2500, 33, 4), (5000, 3, 3), (2500, 40, 7)])
def test_whole_ranges_in_turn(dtype, dh, n_q, m, G):
    """More items than shares: whole rows, nothing to join."""
    n = n_q * m

    def hurt(v, table):
        for i in range(0, n_q, 97):
            put(v, table, 0, i * m + m // 2, 0, i % 16, (NAN, INF, -INF)[i % 3])
            put(v, table, 0, i * m + m - 1, 0, i % 16, NAN)
    rows = [[(max(i - 1, 0) * m, i * m + m)] for i in range(n_q)]
    ranges_call(dtype, dh, G, 1, [n], n_q, m, rows, True, hurt, seed=G, slots=1)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads", [5, 8, 32])
@pytest.mark.parametrize("x", [NAN, INF, -INF])
def test_few_rows_on_the_tensor_cores(dh, heads, x):
    """Up to 32 rows: each quarter's tokens are the others' with weight 0, and what a row sees is its own: an infinity stays one."""
    g, k, v, table = pool(torch.bfloat16, 2, 1, dh, 16, 3000, heads)
    for tok in (5, 20, 40, 63, 1500):
        put(v, table, 0, tok, 0, tok % 7, x)
    put(v, table, 0, 1600, 0, 20, NAN)
    got, want = shared_call(g, k, v, table, heads, [3000, 2500], [1, 1])
    assert got[0, :, [5, 6, 0, 2]].isnan().all() if x != x else (got[0, :, [5, 6, 0, 2]] == x).all()
    assert got[0, :, 20].isnan().all() and got[1].isfinite().all()


@pytest.mark.parametrize("dtype,dh", [(torch.float32, 64), (torch.bfloat16, 80), (torch.bfloat16, 64)])
@pytest.mark.parametrize("m,G", [(65, 4), (33, 8), (1, 260), (1, 9)])
def test_what_the_workspace_held_does_not_matter(dtype, dh, m, G):
    """Rows that leave no marks beside rows that do: the last row tile of an item may have up to eight."""
    n_q = 2400
    n = n_q * m + 20
    g, k, v, table = pool(dtype, 1, 1, dh, 16, n, G)
    lo = torch.arange(n_q, device="cuda") * m
    rg = torch.stack((lo, lo + m + 10), 1)[:, None].int().contiguous()
    for i in range(0, n_q, 5):
        put(v, table, 0, i * m + m + 3, 0, i % 16, NAN)
    q = torch.randn((1, G, n_q * m, dh), generator=g, device="cuda").to(dtype)
    L = torch.tensor([n_q * m], dtype=torch.int32, device="cuda")
    kv, outs = PagedKV(k, v, table), []
    for fill in (0, 255):
        held = [torch.full((size,), fill, dtype=torch.uint8, device="cuda") for size in (1 << 20, 1 << 22, 1 << 24, 1 << 26)]
        del held
        outs.append(kv.attend_ranges(q, rg, L, n_q, 0.1, causal=True))
    ints = [x.view(torch.int16 if dtype == torch.bfloat16 else torch.int32) for x in outs]
    assert torch.equal(*ints)
