"""Where the tokens of a shared prefix come from: pages of its own, whatever the table's width, for sequences that attend by themselves and
for those that share the prefix's tiles."""
import pytest
import torch

import paged_exact as exact
from paged_oracle import assert_within
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu
KINDS = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 80), (torch.float32, 64)]


def pool(dtype, Bn, KH, dh, page, cap, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = -(-cap // page)
    k, v = (torch.randn((Bn * width, KH, page, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    return g, k, v, torch.randperm(Bn * width, generator=g, device="cuda").view(Bn, width).int()


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("lens,news,heads", [
    ([500], [64], 4), ([500, 500], [64, 64], 4),       # filled row tiles: each sequence by itself
    ([500, 500, 500], [64, 3, 1], 4),                  # the same first sequence among others
    ([500, 431, 1], [1, 1, 1], 4), ([500, 431, 60], [1, 1, 1], 40), ([500], [1], 1)])
def test_a_table_shorter_than_the_prefix(dtype, dh, lens, news, heads):
    """500 tokens of prefix in pages of their own, a table with 64 places (of no page at all): the same outputs whoever the neighbours are,
    and nothing to report."""
    g, k, v, pages = pool(dtype, 1, 1, dh, 16, 512, 3)
    table = torch.full((len(lens), 4), -9, dtype=torch.int32, device="cuda")
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    q = torch.randn((cu[-1], heads, dh), generator=g, device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(k, v, table, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), 500, 0.1, prefix_pages=pages[0],
                                                     cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    want, bound = exact.shared(q, k, v, pages.expand(len(lens), -1), lens, cu, 0.1)
    assert_within(got, want, bound)
    assert status.item() == 0


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("lens,news", [([530], [64]), ([530, 530], [64, 64]), ([530, 530, 40], [1, 5, 2])])
def test_lengths_behind_both(dtype, dh, lens, news):
    """Tokens behind the prefix that the table has no places for: left out and reported."""
    g, k, v, pages = pool(dtype, 1, 1, dh, 16, 512, 4)
    table = torch.zeros((len(lens), 4), dtype=torch.int32, device="cuda")
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    q = torch.randn((cu[-1], 4, dh), generator=g, device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(k, v, table, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), 500, 0.1, prefix_pages=pages[0],
                                                     cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    out = []
    for b, n in enumerate(news):                       # query i sees lens - n + i + 1 tokens, of which the first 500 have places
        kk, vv = (exact.tokens(c, pages[0], min(lens[b], 500)) for c in (k, v))
        seen = torch.arange(kk.shape[0], device="cuda") < lens[b] - n + torch.arange(n, device="cuda")[:, None] + 1
        rows = q[cu[b]:cu[b + 1]].reshape(n * 4, dh)
        out.append([x.view(n, 4, dh).cpu() for x in exact.attend_rows(rows, kk[:, 0], vv[:, 0], seen.repeat_interleave(4, 0), 0.1, dtype == torch.bfloat16)])
    assert_within(got, torch.cat([o for o, _ in out]), torch.cat([e for _, e in out]))
    assert status.item() == B.RR_STATUS_BAD_INDEX


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("lens,news,heads", [
    ([0, 200, 230], [1, 1, 1], 2), ([0, 200, 230], [1, 1, 1], 8), ([90, 100, 231, 160], [3, 64, 64, 0], 8),
    ([16, 164], [0, 64], 4), ([0, 300], [64, 64], 4), ([0] * 40 + [170, 190], [1] * 42, 4)])
def test_rows_of_the_table_behind_their_lengths(dtype, dh, lens, news, heads):
    """A free place in the batch, or a short sequence, in front: what its row holds behind its length (other sequences' pages, no pages)
    is nobody's prefix."""
    g, k, v, table = pool(dtype, len(lens), 1, dh, 16, 304, 7)
    long = next(b for b, n in enumerate(lens) if n >= 100)
    stale, sane = table.clone(), table.clone()
    stale[:, :6] = table[long, :6]
    sane[:, :6] = table[long, :6]                      # 96 of the 100 tokens in shared pages, the others in copies
    for c in (k, v):
        for b in range(len(lens)):
            c[table[b, 6].long(), :, :4] = c[table[long, 6].long(), :, :4].clone()
    for b, n in enumerate(lens):
        stale[b, -(-n // 16):] = torch.arange(-3, 300, device="cuda")[:19 - -(-n // 16)].int() if b % 2 else table[(b + 1) % len(lens), 0]
    cu = [0]
    for n in news:
        cu.append(cu[-1] + n)
    q = torch.randn((cu[-1], heads, dh), generator=g, device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(k, v, stale, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), 100, 0.1,
                                                     cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
    want, bound = exact.shared(q, k, v, sane, lens, cu, 0.1)
    assert_within(got, want, bound)
    assert status.item() == 0


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("lens,heads", [([5, 40, 33], 1), ([5, 40, 33], 8), ([0, 0, 0], 8)])
def test_every_sequence_shorter_than_the_prefix(dtype, dh, lens, heads):
    """Places of the prefix that no sequence has are not looked up."""
    g, k, v, table = pool(dtype, 3, 1, dh, 16, 320, 8)
    for b, n in enumerate(lens):
        table[b, :-(-n // 16)] = table[1, :-(-n // 16)]
        table[b, -(-n // 16):] = -7
    q = torch.randn((3, heads, dh), generator=g, device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = PagedKV(k, v, table, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), 300, 0.1)
    want, bound = exact.shared(q, k, v, table, lens, [0, 1, 2, 3], 0.1)
    assert_within(got, want, bound)
    assert status.item() == 0
