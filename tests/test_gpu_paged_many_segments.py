"""Segments behind one another on the tensor cores while the cache comes from memory: tiles arrive in any order, and what the two streams take
from the ring of tiles changes hands from segment to segment.  The outputs are the definition's, and the same bits every time."""
import pytest
import torch

import paged_exact as exact
from paged_oracle import assert_within
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu


def pool(Bn, KH, dh, page, cap, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-cap // page)
    k, v = (torch.randn((Bn * width, KH, page, dh), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    return g, k, v, torch.randperm(Bn * width, generator=g, device="cuda").view(Bn, width).int()


@pytest.mark.parametrize("Bn,L,dh,G,page", [(64, 8192, 128, 8, 64), (64, 8192, 64, 8, 16), (40, 4000, 128, 24, 32), (40, 5000, 128, 40, 64), (24, 3333, 128, 100, 24),
                                            (300, 700, 128, 8, 64), (300, 900, 64, 130, 64)])
def test_single_tokens_of_many_sequences(Bn, L, dh, G, page):
    """All row counts of an item: quartered, split and paired; whole tiles and ragged ones."""
    KH = 8 if L > 1000 else 2
    g, k, v, table = pool(Bn, KH, dh, page, L, G)
    lens = [L] * 4 + torch.randint(L // 2, L + 1, (Bn - 4,), generator=torch.Generator().manual_seed(1)).tolist()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(k, v, table, status)
    q = torch.randn((Bn, KH * G, dh), generator=g, device="cuda").bfloat16()
    Lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    first = kv.attend_shared(q, Lt, 0, dh ** -0.5)
    want, bound = exact.shared(q, k, v, table, lens, list(range(Bn + 1)), dh ** -0.5)
    assert_within(first, want, bound)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(150):
        differ += (kv.attend_shared(q, Lt, 0, dh ** -0.5) != first).any()
    assert differ.item() == 0 and status.item() == 0


@pytest.mark.parametrize("m,G,causal", [(1, 8, False), (1, 60, False), (16, 7, True), (33, 5, True), (64, 4, True)])
@pytest.mark.parametrize("n_q", [100, 900])
def test_ranges_of_many_rows(m, G, causal, n_q):
    chunk = 64
    tokens = 64 * chunk
    g, k, v, table = pool(2, 2, 128, 64, tokens, m)
    score = torch.rand((2 * 2 * n_q, 64), generator=g, device="cuda")
    ids = score.topk(11, dim=1).indices.sort(1).values * chunk
    rg = torch.stack((ids, ids + chunk), -1).int()
    rg[::3, -1, 1] -= 17
    rg[::5, 3:] = -1
    lens = [tokens, tokens - 5]
    q = torch.randn((2, 2 * G, n_q * m, 128), generator=g, device="cuda").bfloat16()
    Lt = torch.tensor(lens, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(k, v, table, status)
    first = kv.attend_ranges(q, rg, Lt, n_q, 0.088, causal=causal)
    want, bound = exact.ranged(q, k, v, table, lens, rg.tolist(), n_q, 0.088, causal)
    assert_within(first, want, bound)
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(50):
        differ += (kv.attend_ranges(q, rg, Lt, n_q, 0.088, causal=causal) != first).any()
    assert differ.item() == 0 and status.item() == 0
