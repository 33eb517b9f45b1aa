"""Every kernel of the paged attention with many tiles and many items per CTA: rings that go round, references that follow the maximum behind the first
tile, items cut anywhere, whole items in turn, calls just below and above the number of items from which they are taken so."""
import pytest
import torch

import paged_exact as exact
from paged_oracle import assert_within
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu
KINDS = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 80), (torch.float32, 64), (torch.float32, 20), (torch.float32, 200)]


def pool(dtype, Bn, KH, dh, page, cap, seed, rising=False):
    """rising: keys grow along the sequence, so that the largest logit comes late and often."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-cap // page)
    k, v = (torch.randn((Bn * width, KH, page, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.randperm(Bn * width, generator=g, device="cuda").view(Bn, width).int()
    if rising:
        for b in range(Bn):
            grow = torch.linspace(0.2, 4.0, width, device="cuda").to(dtype)
            k[table[b].long()] *= grow[:, None, None, None]
    return g, k, v, table


def shared_call(dtype, dh, heads, KH, page, lens, news, prefix=0, cu=True, causal=True, rising=False, seed=0, times=20):
    g, k, v, table = pool(dtype, len(lens), KH, dh, page, max(lens), seed, rising)
    if prefix:
        full = prefix // page
        table[:, :full] = table[0, :full].clone()
        if prefix % page:
            for c in (k, v):
                for b in range(1, len(lens)):
                    c[table[b, full].long(), :, :prefix % page] = c[table[0, full].long(), :, :prefix % page].clone()
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(k, v, table, status)
    q = torch.randn((starts[-1], heads, dh), generator=g, device="cuda").to(dtype)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c = torch.tensor(starts, dtype=torch.int32, device="cuda") if cu else None
    got = kv.attend_shared(q, L, prefix, dh ** -0.5, cu=c, causal=causal)
    want, bound = exact.shared(q, k, v, table, lens, starts, dh ** -0.5, causal)
    assert_within(got, want, bound)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(times):
        differ += (kv.attend_shared(q, L, prefix, dh ** -0.5, cu=c, causal=causal) != got).any()
    assert differ.item() == 0 and status.item() == 0


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("heads,KH,page", [(1, 1, 16), (4, 1, 64), (4, 2, 24), (8, 1, 32), (40, 1, 16), (200, 1, 64)])
def test_one_token_of_a_long_sequence(dtype, dh, heads, KH, page):
    shared_call(dtype, dh, heads, KH, page, [200003], [1], seed=heads)
    shared_call(dtype, dh, heads, KH, page, [20003], [1], rising=True, cu=False, seed=heads)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("heads,KH", [(4, 2), (6, 2), (32, 2)])
def test_tokens_of_unlike_sequences_behind_a_prefix(dtype, dh, heads, KH):
    lens = [5000 + x for x in torch.randint(1, 4000, (40,), generator=torch.Generator().manual_seed(heads)).tolist()]
    shared_call(dtype, dh, heads, KH, 16, lens, [1] * 40, prefix=4990, cu=False, seed=1)
    shared_call(dtype, dh, heads, KH, 24, lens, [1, 2, 0, 4, 1] * 8, prefix=4990, rising=True, seed=2)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("heads,KH,prefix,lens,news", [(4, 1, 0, [6000], [3000]), (4, 2, 1000, [5000, 1500, 4000], [900, 333, 64]), (7, 1, 700, [2000] * 9, [31] * 9)])
def test_long_prompts(dtype, dh, heads, KH, prefix, lens, news):
    shared_call(dtype, dh, heads, KH, 32, lens, news, prefix=prefix, rising=True, seed=3, times=5)


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_states_of_another_length(dtype, dh):
    shared_call(dtype, dh, 4, 2, 16, [3001, 17, 9000], [300, 9, 40], causal=False, seed=4, times=5)


def ranges_call(dtype, dh, G, KH, RH, n_q, m, slots, causal, seed, tokens=2000, times=10):
    g, k, v, table = pool(dtype, 2, KH, dh, 16, tokens, seed)
    rows = 2 * RH * n_q
    gen = torch.Generator().manual_seed(seed)
    kinds = []
    for i in range(24):                                # rows without tokens, of one, of 129, of many
        n = (0, 1, 129, 300, 128, 40)[i % 6]
        parts = min(slots, (1, 2, 5)[i % 3], max(n, 1))
        cut = torch.randint(0, tokens - n - 8 * parts, (1,), generator=gen).item()
        spans, left = [], n
        for j in range(parts):
            take = left if j == parts - 1 else left // 2
            spans.append((cut, cut + take) if take else (-1, -1))
            cut, left = cut + take + 7, left - take
        kinds.append(spans)
    pick = torch.randint(0, 24, (rows,), generator=gen).tolist()
    spans = [kinds[i] for i in pick]
    rg = torch.full((24, slots, 2), -1, dtype=torch.int32)
    for i, x in enumerate(kinds):
        rg[i, :len(x)] = torch.tensor(x, dtype=torch.int32)
    rg = rg[torch.tensor(pick)].cuda()
    lens = [tokens, tokens - 300]
    q = torch.randn((2, RH * G, n_q * m, dh), generator=g, device="cuda").to(dtype)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(k, v, table, status)
    got = kv.attend_ranges(q, rg, L, n_q, dh ** -0.5, causal=causal)
    want, bound = exact.ranged(q, k, v, table, lens, spans, n_q, dh ** -0.5, causal)
    assert_within(got, want, bound)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(times):
        differ += (kv.attend_ranges(q, rg, L, n_q, dh ** -0.5, causal=causal) != got).any()
    assert differ.item() == 0 and status.item() == 0


def tensor_cores(dtype, dh):
    return dtype == torch.bfloat16 and dh in (64, 128)


@pytest.mark.parametrize("dtype,dh,G,n_q", [(t, d, G, n) for t, d in KINDS for G in (1, 3, 8, 20, 60, 140, 300) for n in (290, 300, 580, 600, 880, 900, 1200)
                                            if n in (290, 300, 600) or (tensor_cores(t, d) and G <= 8)])
def test_as_many_items_as_are_shared_and_more(dtype, dh, G, n_q):
    """Two sequences of two route heads: 1160 to 4800 items of one row tile (twice as many of 300 rows); whole ones in turn from 1184, 2368, 3552 or 4736 on."""
    ranges_call(dtype, dh, G, 2, 2, n_q, 1, 6, False, seed=G, times=5)


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_single_queries_in_turn(dtype, dh):
    ranges_call(dtype, dh, 2, 1, 1, 2400, 1, 6, False, seed=9)
    ranges_call(dtype, dh, 4, 1, 2, 1300, 1, 6, True, seed=10)


@pytest.mark.parametrize("slots", [257, 1024])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("G,n_q", [(5, 120), (33, 90), (129, 320), (300, 170), (2, 150), (2, 1900)])
def test_many_slots(slots, dh, G, n_q):
    ranges_call(torch.bfloat16, dh, G, 1, 2, n_q, 1, slots, False, seed=G)
