"""Appending to a paged cache: positions across page ends, ragged and padded batches, both pairings of the rotation, widths
and strides with and without 16-byte pieces, far positions, bad pages, graphs, streams."""
import pytest
import torch

from paged_oracle import BF, U
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV, inv_freq

pytestmark = pytest.mark.gpu


def make(dtype, KH, dh, page, width, B_, extra=0, token_major=False):
    g = torch.Generator(device="cuda").manual_seed(dh * page + KH)
    pages = B_ * width + extra
    shape = (pages, page, KH, dh) if token_major else (pages, KH, page, dh)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    table = torch.randperm(pages, generator=g, device="cuda")[:B_ * width].view(B_, width).int()
    return g, k, v, table


def turned(x, pos, freq, interleaved):
    """x [heads, dh] at position pos in 64 bits, and the error bound: the angle is rounded to 2^-26 of a turn (2 pi 2^-26
    radians), sine and cosine are off by at most 2 steps, the two products and their sum by one rounding each."""
    x = x.double().cpu()
    rot = 2 * freq.numel()
    a = pos * freq.double().cpu()
    c, s = a.cos(), a.sin()
    i = torch.arange(rot // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y, bound = x.clone(), torch.zeros_like(x)
    y[:, p] = x[:, p] * c - x[:, q] * s
    y[:, q] = x[:, q] * c + x[:, p] * s
    mag = x[:, p].abs() + x[:, q].abs()
    each = mag * (6.2832 * 2.0 ** -26 + 4 * U + 2 * U)
    bound[:, p] = each
    bound[:, q] = each
    return y, bound


def check(got, x, pos, freq, interleaved, msg):
    if freq is None:
        assert torch.equal(got, x), msg
        return
    want, bound = turned(x, pos, freq, interleaved)
    if got.dtype == torch.bfloat16:
        bound = bound + (want.abs() + bound) * BF
        rest = slice(2 * freq.numel(), None)
        assert torch.equal(got[:, rest], x[:, rest]), msg
    assert ((got.double().cpu() - want).abs() <= bound).all(), msg


@pytest.mark.parametrize("dtype,dh,rot,interleaved,page,token_major,sliced", [
    (torch.bfloat16, 128, 128, False, 16, False, True),
    (torch.bfloat16, 64, 32, True, 24, True, False),
    (torch.bfloat16, 40, 20, False, 7, False, False),      # 10 pairs: no 16-byte pieces
    (torch.bfloat16, 64, 64, False, 1, True, True),
    (torch.float32, 64, 64, True, 16, False, True),
    (torch.float32, 128, 64, False, 5, True, False),
    (torch.float32, 7, 6, True, 3, False, False),
    (torch.float32, 256, 0, False, 64, False, False),
])
@pytest.mark.parametrize("ragged", [False, True])
def test_cache_and_queries(dtype, dh, rot, interleaved, page, token_major, sliced, ragged):
    KH, H = 2, 6
    news = [3, 0, 1, 33, 2] if ragged else [1] * 5
    lens = [0, 5, page - 1, page, 3 * page + 1]
    g, kc, vc, table = make(dtype, KH, dh, page, (3 * page + 40) // page + 1, 5, token_major=token_major)
    pad = 4 if ragged else 0
    T = sum(news) + pad
    if sliced:
        qkv = torch.randn((T, (H + 2 * KH) * dh), generator=g, device="cuda").to(dtype)
        q, k, v = (x.view(T, -1, dh) for x in (qkv[:, :H * dh], qkv[:, H * dh:(H + KH) * dh], qkv[:, (H + KH) * dh:]))
    else:
        q, k, v = (torch.randn((T, n, dh), generator=g, device="cuda").to(dtype) for n in (H, KH, KH))
    freq = inv_freq(rot, 10000.0) if rot else None
    cu = torch.tensor([0] + news, device="cuda").cumsum(0).int() if ragged else None
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    nl = torch.full_like(L, -7)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(kc, vc, table, status)
    want_k, want_v = kc.clone(), vc.clone()
    q_out = torch.full((T, H, dh), 9.0, device="cuda", dtype=dtype)
    got = kv.append(k, v, L, cu=cu, q=q, q_out=q_out, inv_freq=freq, interleaved=interleaved, new_lens=nl)
    assert got is q_out and status.item() == 0
    assert nl.tolist() == [a + n for a, n in zip(lens, news)]
    t = 0
    for b in range(5):
        for i in range(news[b]):
            p = lens[b] + i
            pg, off = int(table[b, p // page]), p % page
            check(kc[pg, :, off], k[t], p, freq, interleaved, (b, i))
            check(q_out[t], q[t], p, freq, interleaved, (b, i, "q"))
            assert torch.equal(vc[pg, :, off], v[t])
            want_k[pg, :, off], want_v[pg, :, off] = kc[pg, :, off], vc[pg, :, off]
            t += 1
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)            # nothing else was written
    assert (q_out[t:] == 9.0).all()                                      # padding rows as they were


@pytest.mark.parametrize("pos", [0, 1, 8191, 1 << 20, (1 << 31) - 70])
def test_far_positions(pos):
    dh, page = 64, 1 << 21                                                # (a table of 1024 pages, all the same one)
    kc, vc = (torch.zeros((1, 1, page, dh), device="cuda") for _ in range(2))
    kv = PagedKV(kc, vc, torch.zeros((1, 1024), dtype=torch.int32, device="cuda"))
    k = torch.randn((1, 1, dh), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    freq = inv_freq(dh, 500000.0)
    kv.append(k, k, torch.tensor([pos], dtype=torch.int32, device="cuda"), inv_freq=freq)
    check(kc[0, :, pos % page], k[0], pos, freq, False, pos)


def test_many_sequences_and_in_place_queries():
    g, kc, vc, table = make(torch.bfloat16, 1, 64, 4, 3, 2500)
    news = torch.randint(0, 3, (2500,), generator=torch.Generator().manual_seed(3))
    cu = torch.cat((torch.zeros(1, dtype=torch.long), news.cumsum(0))).int()
    T = int(cu[-1])
    k, v, q = (torch.randn((T, 1, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
    lens = torch.arange(2500, dtype=torch.int32) % 9
    freq = inv_freq(64)
    apart = PagedKV(kc.clone(), vc.clone(), table).append(k, v, lens.cuda(), cu=cu.cuda(), q=q, inv_freq=freq)
    got = PagedKV(kc, vc, table).append(k, v, lens.cuda(), cu=cu.cuda(), q=q, q_out=q, inv_freq=freq)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, apart)
    seq = torch.repeat_interleave(torch.arange(2500), news)
    pos = lens.long()[seq] + torch.arange(T) - cu.long()[seq]
    at = table.cpu().long()[seq, pos // 4]
    assert torch.equal(vc[at.cuda(), :, (pos % 4).cuda()], v)


def test_bad_pages_and_table_ends():
    """Ids outside the pool, positions behind the table, a negative length: left out, reported, queries rotated all the same."""
    g, kc, vc, table = make(torch.float32, 2, 32, 4, 2, 5)
    table[0, 1] = kc.shape[0]
    table[1, 0] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(kc, vc, table, status)
    k, v, q = (torch.randn((5, 2, 32), generator=g, device="cuda") for _ in range(3))
    before_k, before_v = kc.clone(), vc.clone()
    lens = torch.tensor([4, 0, 8, -3, 7], dtype=torch.int32, device="cuda")
    q_out = kv.append(k, v, lens, q=q, inv_freq=inv_freq(32))
    at = int(table[4, 1]), 3
    assert not torch.equal(kc[at[0], :, at[1]], before_k[at[0], :, at[1]])
    before_k[at[0], :, at[1]], before_v[at[0], :, at[1]] = kc[at[0], :, at[1]], v[4]
    assert torch.equal(kc, before_k) and torch.equal(vc, before_v)
    assert status.item() == B.RR_STATUS_BAD_INDEX
    check(q_out[2], q[2], 8, inv_freq(32), False, "behind the table")
    check(q_out[0], q[0], 4, inv_freq(32), False, "bad page")


def test_captured_steps_advance_the_lengths():
    g, kc, vc, table = make(torch.bfloat16, 2, 64, 4, 4, 3)
    kv = PagedKV(kc, vc, table)
    k, v, q = (torch.randn((3, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
    lens, nl = torch.tensor([0, 3, 9], dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    freq, out = inv_freq(64), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            kv.append(k, v, lens, q=q, q_out=out, inv_freq=freq, new_lens=nl)
            lens.copy_(nl)
    torch.cuda.synchronize()
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for b, p in enumerate((step, 3 + step, 9 + step)):
            check(kc[int(table[b, p // 4]), :, p % 4], k[b], p, freq, False, (step, b))
    assert lens.tolist() == [3, 6, 12]


def test_no_tokens():
    g, kc, vc, table = make(torch.float32, 1, 8, 2, 1, 2)
    nl = torch.zeros(2, dtype=torch.int32, device="cuda")
    e = torch.empty((0, 1, 8), device="cuda")
    PagedKV(kc, vc, table).append(e, e, torch.tensor([1, 2], dtype=torch.int32, device="cuda"),
                                  cu=torch.zeros(3, dtype=torch.int32, device="cuda"), q=e, new_lens=nl)
    assert nl.tolist() == [1, 2]
