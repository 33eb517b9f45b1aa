"""Attention over token ranges through a page table against the definition in 64 bits."""
import pytest
import torch

from paged_oracle import assert_within, ranged
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.ledger import attend_token_ranges
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu
NAN = float("nan")
KINDS = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64), (torch.float32, 20), (torch.bfloat16, 80), (torch.float32, 256)]


def pool(dtype, Bn, KH, dh, page, lens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = max(1, max(-(-n // page) for n in lens))
    k, v = (torch.full((Bn * width + 1, KH, page, dh), NAN, device="cuda", dtype=dtype) for _ in range(2))
    table = torch.randperm(Bn * width + 1, generator=g, device="cuda")[:Bn * width].view(Bn, width).int()
    for b, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        for c in (k, v):
            c[table[b].long()[t // page], :, t % page] = torch.randn((n, KH, dh), generator=g, device="cuda").to(dtype)
    return g, k, v, table


def check(dtype, dh, H, RH, KH, page, lens, n_q, m, rg, causal=False, seed=0, hurt=None):
    Bn = len(lens)
    g, k, v, table = pool(dtype, Bn, KH, dh, page, lens, seed)
    if hurt:
        hurt(k, v, table)
    q = torch.randn((Bn, n_q * m, H, dh), generator=g, device="cuda").to(dtype).transpose(1, 2)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(k, v, table, status)
    out = kv.attend_ranges(q, rg.cuda(), L, n_q, dh ** -0.5, causal=causal)
    want, bound = ranged(q, k, v, table, lens, rg, n_q, dh ** -0.5, causal)
    assert_within(out, want, bound)
    assert status.item() == 0
    return kv, q, L, out


def slots_of(spans, rows, slots, seed):
    gen = torch.Generator().manual_seed(seed)
    rg = torch.full((rows, slots, 2), -1, dtype=torch.int32)
    for r in range(rows):
        sp = spans[r % len(spans)]
        at = torch.randperm(slots, generator=gen)[:len(sp)].sort().values.tolist() if r % 2 else range(len(sp))
        for s, (lo, hi) in zip(at, sp):
            rg[r, s] = torch.tensor([lo, hi])
    return rg


SPANS = [[], [(3, 4)], [(0, 127)], [(0, 128)], [(5, 134)], [(0, 127), (200, 201)], [(10, 20), (30, 300), (699, 700)], [(650, 900)], [(0, 700)],
         [(0, 1), (2, 3), (4, 5), (6, 7), (698, 705)], [(500, 600), (100, 228)], [(40, 40), (60, 50), (7, 9)]]


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("H,RH,KH", [(2, 2, 2), (8, 2, 1), (10, 2, 2)])
def test_one_query_per_row(dtype, dh, H, RH, KH):
    n_q = len(SPANS)
    check(dtype, dh, H, RH, KH, 16, [700, 433], n_q, 1, slots_of(SPANS, 2 * RH * n_q, 6, 1), seed=H)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("m,G,page", [(16, 3, 24), (64, 2, 64), (33, 8, 7)])
def test_chunks_of_queries_causal(dtype, dh, m, G, page):
    """A prompt of n_q chunks: each chunk's queries share its ranges, the last one cut inside by the mask; 48, 128 and 264 rows."""
    n_q = 6
    n = n_q * m
    spans = [[(c * m, c * m + m) for c in range(i + 1) if (c * 7 + i) % 3 != 1 or c == i] for i in range(n_q)]
    rg = slots_of(spans, 2 * n_q, n_q, 3)
    check(dtype, dh, G, 1, 1, page, [n, n], n_q, m, rg, causal=True, seed=m)


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_queries_before_the_first_token(dtype, dh):
    """A sequence shorter than the queries of the call: those before its first token see nothing."""
    rg = slots_of([[(0, 30), (32, 64)]], 2, 2, 3)
    kv, q, L, out = check(dtype, dh, 2, 1, 1, 16, [20, 64], 1, 32, rg, causal=True)
    assert (out[0, :, :12] == 0).all()


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), NAN])
def test_values_that_a_row_may_not_see(dtype, dh, bad):
    def hurt(k, v, table):
        v[int(table[0, 70 // 16]), 0, 70 % 16, 5] = bad
    rg = slots_of([[(0, 64)], [(0, 20), (64, 128)]], 2, 3, 0)
    kv, q, L, out = check(dtype, dh, 3, 1, 1, 16, [128], 2, 64, rg, causal=True, hurt=hurt)
    hit = torch.zeros(out.shape, dtype=torch.bool)
    hit[0, :, 70:, 5] = True
    assert torch.equal(~out.isfinite().cpu(), hit)


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_per_slot_and_merged_ranges_give_the_same_bits(dtype, dh):
    g, k, v, table = pool(dtype, 1, 1, dh, 16, [640], 5)
    kv, L = PagedKV(k, v, table), torch.tensor([640], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 4, 1, dh), generator=g, device="cuda").to(dtype)
    per_slot = torch.tensor([[[64 * c, 64 * c + 64] for c in (0, 1, 2, 5, 8, 9)]], dtype=torch.int32, device="cuda")
    merged = torch.tensor([[[0, 192], [320, 384], [512, 640], [-1, -1], [-1, -1], [-1, -1]]], dtype=torch.int32, device="cuda")
    a, b = (kv.attend_ranges(q, r, L, 1, 0.1) for r in (per_slot, merged))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.float32, 64)])
def test_as_the_consumer_of_contiguous_keys(dtype, dh):
    """Pages in order are contiguous keys: the same outputs as attend_token_ranges, within both bounds."""
    P, n_q, tokens = 4, len(SPANS), 704
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((P, tokens, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((P * n_q, dh), generator=g, device="cuda").to(dtype)
    rg = slots_of(SPANS, P * n_q, 6, 1).cuda()
    pages = [x.view(P, 1, tokens // 16, 16, dh).transpose(1, 2).reshape(P * tokens // 16, 1, 16, dh) for x in (k, v)]
    table = torch.arange(P * tokens // 16, dtype=torch.int32, device="cuda").view(P, -1)
    L = torch.full((P,), tokens, dtype=torch.int32, device="cuda")
    got = PagedKV(*pages, table).attend_ranges(q.view(P, 1, n_q, dh), rg, L, n_q, 0.125)
    plain = attend_token_ranges(rg, n_q, q, k, v, 0.125)
    want, bound = ranged(q.view(P, 1, n_q, dh), *pages, table, [tokens] * P, rg, n_q, 0.125, False)
    assert_within(got, want, bound)
    assert_within(plain.view(P, 1, n_q, dh), want, bound)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("slots", [1, 33, 1024])
def test_slot_counts(dtype, dh, slots):
    spans = [[((37 * s) % 900, (37 * s) % 900 + 1 + s % 3) for s in range(slots)]]
    check(dtype, dh, 2, 1, 1, 16, [1000], 1, 1, slots_of(spans, 1, slots, 0))


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.float32, 64)])
def test_absent_sequences_and_bad_pages(dtype, dh):
    rg = slots_of([[(0, 50)]], 3, 1, 0)
    kv, q, L, out = check(dtype, dh, 2, 1, 1, 16, [60, 0, 20], 1, 1, rg)
    assert (out[1] == 0).all()
    table = kv.page_table.clone()
    table[0, 2] = 1 << 30
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(kv.k_cache, kv.v_cache, table, status).attend_ranges(q, rg.cuda(), L, 1, dh ** -0.5)
    assert status.item() == B.RR_STATUS_BAD_INDEX
    rg2 = torch.tensor([[[0, 32], [48, 50]], [[0, 50], [-1, -1]], [[0, 50], [-1, -1]]], dtype=torch.int32)
    want, bound = ranged(q, kv.k_cache, kv.v_cache, kv.page_table, [60, 0, 20], rg2, 1, dh ** -0.5, False)
    assert_within(got, want, bound)
