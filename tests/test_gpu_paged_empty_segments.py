"""Segments without tokens behind one whose last tile is no full run of a page: rows of absent sequences, empty ranges, more queries than
tokens.  The tensor cores' kernel walks several of them per CTA; copies of the segment before must not stay unannounced."""
import pytest
import torch

import paged_exact as exact
from paged_oracle import assert_within
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu


def pool(Bn, KH, dh, page, cap, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-cap // page)
    k, v = (torch.randn((Bn * width, KH, page, dh), generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(Bn * width, generator=g, device="cuda").view(Bn, width).int()
    return g, k, v, table


def ranges_call(lens, RH, G, n_q, m, dh, rows, slots, causal=False, page=16, seed=0):
    g, k, v, table = pool(len(lens), RH, dh, page, max(lens), seed)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rg = torch.full((len(rows), slots, 2), -1, dtype=torch.int32)
    for i, spans in enumerate(rows):
        if spans:
            rg[i, :len(spans)] = torch.tensor(spans, dtype=torch.int32)
    q = torch.randn((len(lens), RH * G, n_q * m, dh), generator=g, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    PagedKV(k, v, table, status).attend_ranges(q, rg.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), n_q, dh ** -0.5, causal=causal, out=out)
    assert status.item() == 0
    want, bound = exact.ranged(q, k, v, table, lens, rows, n_q, dh ** -0.5, causal)
    assert_within(out, want, bound)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("m,G", [(1, 5), (1, 33), (33, 4), (64, 4)])
@pytest.mark.parametrize("n_q", [1036, 2100])
def test_empty_ranges_behind_a_partial_tile(dh, m, G, n_q):
    """Seven rows per CTA in shares, fourteen taken in turn: one row of 1 to 261 tokens, then rows without any."""
    spans = ([(0, 133)], [(3, 4)], [(7, 90), (100, 278)])
    rows = [list(spans[i // 7 % 3]) if i % 7 == 0 else [] for i in range(n_q)]
    if n_q > 1184:                                     # in turn: CTA c has rows c, c + 148, ...
        rows = [list(spans[i % 3]) if i < 200 else [] for i in range(n_q)]
    ranges_call([300], 1, G, n_q, m, dh, rows, 2, seed=m)


@pytest.mark.parametrize("m,G", [(1, 8), (33, 2), (64, 4)])
@pytest.mark.parametrize("n_q", [200, 400])
def test_absent_sequences(m, G, n_q):
    """Sequences without tokens, whose ranges are as long as the others'."""
    spans = ([(0, 133)], [(5, 70), (100, 129)])
    ranges_call([150, 0, 0, 0, 131], 1, G, n_q, m, 64, [list(spans[i % 2]) for i in range(5 * n_q)], 2, seed=G)


@pytest.mark.parametrize("slots", [257, 1024])
@pytest.mark.parametrize("m,G,n_q", [(1, 5, 150), (1, 33, 700), (33, 4, 160), (60, 5, 1300)])
def test_many_slots_and_few_tokens(slots, m, G, n_q):
    """More than 256 slots: two segments under way, not four; shares of an item that have no tile."""
    rows = [[(0, 5)], [(0, 133)], [(2 * s, 2 * s + 1) for s in range(130)]]
    ranges_call([300], 1, G, n_q, m, 128, [rows[i % 3] for i in range(n_q)], slots, seed=slots)


@pytest.mark.parametrize("dh", [64, 128])
def test_queries_before_the_first_token(dh):
    """A sequence of many more queries than tokens: row tiles that see nothing, in turn behind one that does."""
    g, k, v, table = pool(3, 1, dh, 16, 100, 5)
    lens, cu = [100, 90, 70], [0, 5, 40005, 40105]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.randn((cu[-1], 8, dh), generator=g, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    PagedKV(k, v, table, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), 0, 0.1,
                                               cu=torch.tensor(cu, dtype=torch.int32, device="cuda"), out=out)
    assert status.item() == 0
    want, bound = exact.shared(q, k, v, table, lens, cu, 0.1)
    assert_within(out, want, bound)
