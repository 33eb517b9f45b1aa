"""The paged cache's operators as a serving program uses them, with the routes of RouteLedger; and what they have in common: far pages,
outputs and inputs off 16 bytes, lengths behind the table, graphs."""
import pytest
import torch

from paged_oracle import assert_within, ranged, shared
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.ledger import RouteLedger
from paper_2609_07306_b200.paged import PagedKV, inv_freq

pytestmark = pytest.mark.gpu


def rotated(x, pos, freq):
    """x [tokens, heads, dh] rotated by halves in 64 bits."""
    a = pos.double()[:, None] * freq.double()
    c, s = a.cos()[:, None], a.sin()[:, None]
    h = freq.numel()
    x = x.double()
    return torch.cat((x[..., :h] * c - x[..., h:2 * h] * s, x[..., h:2 * h] * c + x[..., :h] * s, x[..., 2 * h:]), -1)


def test_a_routed_prompt_and_steps_after_it():
    """A prompt of 8 chunks of 64 tokens: appended with its rotation, routed chunk by chunk (an anchor with token ranges), attended to
    over the routes' ranges; then three single tokens, appended and attending to everything."""
    heads, dh, chunk, n, page = 2, 64, 64, 8, 16
    T = n * chunk
    g = torch.Generator(device="cuda").manual_seed(11)
    kc, vc = (torch.full((60, heads, page, dh), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.randperm(60, generator=g, device="cuda")[:T // page + 1].view(1, -1).int()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(kc, vc, table, status)
    q, k, v = (torch.randn((T, heads, dh), generator=g, device="cuda").bfloat16() for _ in range(3))
    freq, pos = inv_freq(dh), torch.arange(T, device="cuda")
    lens, after = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    qr = kv.append(k, v, lens, cu=torch.tensor([0, T], dtype=torch.int32, device="cuda"), q=q, inv_freq=freq, new_lens=after)
    # one step of bf16 (2^-7) beside the rounding's half
    torch.testing.assert_close(qr.double(), rotated(q, pos, freq), rtol=2 ** -7, atol=1e-6)
    cfg = B.rr_config(batch=1, heads=heads, n_q=n, n_k=n, d=dh, k=4, m=1, r=1, dtype=B.RR_BF16, causal=1, causal_offset=0, seed=5,
                      chunk_tokens=chunk)
    led = RouteLedger(cfg)
    qc = q.view(n, chunk, heads, dh).float().mean(1).transpose(0, 1).contiguous().bfloat16()
    kcn = k.view(n, chunk, heads, dh).float().mean(1).transpose(0, 1).contiguous().bfloat16()
    led.route_anchor(qc.view(1, heads, n, dh), kcn.view(1, heads, n, dh), 0)
    out = kv.attend_ranges(qr.transpose(0, 1).unsqueeze(0), led.token_ranges, after, n, dh ** -0.5, causal=True)
    want, bound = ranged(qr.transpose(0, 1).unsqueeze(0), kc, vc, table, [T], led.token_ranges, n, dh ** -0.5, True)
    assert_within(out, want, bound)
    now = T
    for step in range(3):
        q1, k1, v1 = (torch.randn((1, heads, dh), generator=g, device="cuda").bfloat16() for _ in range(3))
        lens, after = after, lens
        q1 = kv.append(k1, v1, lens, q=q1, inv_freq=freq, new_lens=after)
        now += 1
        got = kv.attend_shared(q1, after, 256, dh ** -0.5)
        want, bound = shared(q1, kc, vc, table, [now], [0, 1], dh ** -0.5, True)
        assert_within(got, want, bound)
    assert after.item() == now and status.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pages_behind_32_bit_offsets(dtype):
    """A pool of more than 2^31 entries, the pages in use at its end; every kernel (1, 8, 40 and 200 rows)."""
    pages, page, dh = 270000, 64, 128
    kc, vc = (torch.empty((pages, 1, page, dh), device="cuda", dtype=dtype) for _ in range(2))
    table = torch.arange(pages - 6, pages, device="cuda").view(2, 3).int()
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = PagedKV(kc, vc, table)
    k, v = (torch.randn((340, 1, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")
    full = torch.zeros(2, dtype=torch.int32, device="cuda")
    kv.append(k, v, lens, cu=torch.tensor([0, 180, 340], dtype=torch.int32, device="cuda"), new_lens=full)
    assert torch.equal(kc[-6, 0], k[:64, 0]) and torch.equal(vc[-3, 0], v[180:244, 0])
    small = [c[-6:] for c in (kc, vc)]                                   # (for the 64-bit form)
    for G in (1, 8, 40, 200):
        q = torch.randn((2, G, dh), generator=g, device="cuda").to(dtype)
        got = kv.attend_shared(q, full, 0, 0.1)
        want, bound = shared(q, *small, table - (pages - 6), [180, 160], [0, 1, 2], 0.1, True)
        assert_within(got, want, bound)
    rg = torch.tensor([[[3, 100], [130, 180]], [[0, 160], [-1, -1]]], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 3, 1, dh), generator=g, device="cuda").to(dtype)
    got = kv.attend_ranges(q, rg, full, 1, 0.1)
    want, bound = ranged(q, *small, table - (pages - 6), [180, 160], rg, 1, 0.1, False)
    assert_within(got, want, bound)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.float32, 64)])
@pytest.mark.parametrize("G", [2, 40])
def test_rows_off_16_bytes(dtype, dh, G):
    """Queries, pages and outputs that start off their 16-byte boundaries, with strides that no vector divides."""
    g = torch.Generator(device="cuda").manual_seed(G)
    pool = [torch.randn((9, 1, 16, dh + 3), generator=g, device="cuda").to(dtype)[..., 1:dh + 1] for _ in range(2)]
    table = torch.randperm(9, generator=g, device="cuda")[:8].view(1, 8).int()
    kv = PagedKV(*pool, table)
    q = torch.randn((5, G, dh + 5), generator=g, device="cuda").to(dtype)[..., 3:dh + 3]
    cu = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    L = torch.tensor([120], dtype=torch.int32, device="cuda")
    hold = torch.full((5, G, dh + 7), 3.0, device="cuda", dtype=dtype)
    out = kv.attend_shared(q, L, 0, 0.1, cu=cu, out=hold[..., 5:dh + 5])
    want, bound = shared(q, *pool, table, [120], [0, 5], 0.1, True)
    assert_within(out, want, bound)
    assert (hold[..., :5] == 3.0).all() and (hold[..., dh + 5:] == 3.0).all()
    k, v, fresh = (torch.randn((1, 1, dh + 1), generator=g, device="cuda").to(dtype)[..., 1:] for _ in range(3))
    kv.append(k, v, L, q=fresh, inv_freq=inv_freq(dh))
    assert torch.equal(pool[1][int(table[0, 7]), 0, 8], v[0, 0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G", [1, 8, 200])
def test_outputs_into_a_slice(dtype, G):
    """An output with the strides of a wider matrix, written whole or joined."""
    g = torch.Generator(device="cuda").manual_seed(G)
    pool = [torch.randn((40, 1, 16, 64), generator=g, device="cuda").to(dtype) for _ in range(2)]
    table = torch.randperm(40, generator=g, device="cuda").view(2, 20).int()
    kv = PagedKV(*pool, table)
    L = torch.tensor([320, 100], dtype=torch.int32, device="cuda")
    q = torch.randn((2, G, 64), generator=g, device="cuda").to(dtype)
    wide = torch.full((2, 3 * G, 64), 5.0, device="cuda", dtype=dtype)
    kv.attend_shared(q, L, 0, 0.1, out=wide[:, G:2 * G])
    assert torch.equal(wide[:, G:2 * G], kv.attend_shared(q, L, 0, 0.1))
    assert (wide[:, :G] == 5.0).all() and (wide[:, 2 * G:] == 5.0).all()


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_lengths_behind_the_table(dtype, dh):
    """A length for which the table has no places: reported, and what the table has is attended to."""
    g = torch.Generator(device="cuda").manual_seed(3)
    pool = [torch.randn((4, 1, 16, dh), generator=g, device="cuda").to(dtype) for _ in range(2)]
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    q = torch.randn((2, 2, dh), generator=g, device="cuda").to(dtype)
    for over in (33, 5000, 2 ** 31 - 1):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kv = PagedKV(*pool, table, status)
        L = torch.tensor([over, 20], dtype=torch.int32, device="cuda")
        got = kv.attend_shared(q, L, 0, 0.1)
        want, bound = shared(q, *pool, table, [32, 20], [0, 1, 2], 0.1, False)
        assert_within(got, want, bound)
        assert status.item() == B.RR_STATUS_BAD_INDEX
        status.zero_()
        rg = torch.tensor([[[0, 2 ** 31 - 1]], [[4, 9]]], dtype=torch.int32, device="cuda")
        got = kv.attend_ranges(q.unsqueeze(2), rg, L, 1, 0.1, causal=True)
        rg[0, 0, 1] = 32
        want, bound = ranged(q.unsqueeze(2), *pool, table, [32, 20], rg, 1, 0.1, False)
        assert_within(got, want, bound)
        assert status.item() == B.RR_STATUS_BAD_INDEX


@pytest.mark.parametrize("dtype,m,G", [(torch.bfloat16, 1, 1), (torch.bfloat16, 1, 8), (torch.bfloat16, 40, 4), (torch.float32, 1, 2), (torch.float32, 40, 4)])
def test_ranges_captured_and_replayed_with_others(dtype, m, G):
    g = torch.Generator(device="cuda").manual_seed(m)
    pool = [torch.randn((16, 1, 16, 64), generator=g, device="cuda").to(dtype) for _ in range(2)]
    table = torch.randperm(16, generator=g, device="cuda").view(1, 16).int()
    kv = PagedKV(*pool, table)
    q = torch.randn((1, G, 2 * m, 64), generator=g, device="cuda").to(dtype)
    L = torch.tensor([256], dtype=torch.int32, device="cuda")
    rg = torch.tensor([[[0, 64], [100, 130]], [[5, 6], [-1, -1]]], dtype=torch.int32, device="cuda")
    out = kv.attend_ranges(q, rg, L, 2, 0.1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.attend_ranges(q, rg, L, 2, 0.1, out=out)
    for spans, n in (([[[0, 64], [100, 130]], [[5, 6], [-1, -1]]], 256), ([[[-1, -1], [-1, -1]], [[0, 200], [200, 256]]], 256), ([[[7, 90], [90, 91]], [[50, 250], [-1, -1]]], 120)):
        rg.copy_(torch.tensor(spans, dtype=torch.int32))
        L.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        want, bound = ranged(q, *pool, table, [n], rg, 2, 0.1, False)
        assert_within(out, want, bound)


def test_refusals_of_the_wrapper():
    pool = [torch.zeros((4, 2, 16, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    table = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    kv = PagedKV(*pool, table)
    q, L = torch.zeros((3, 4, 64), device="cuda", dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32, device="cuda")
    k = q[:, :2]
    bad = [
        lambda: PagedKV(pool[0], pool[1][:, :1], table), lambda: PagedKV(pool[0].half(), pool[1].half(), table),
        lambda: PagedKV(pool[0], pool[1].transpose(0, 1).contiguous().transpose(0, 1), table), lambda: PagedKV(*pool, table.long()),
        lambda: PagedKV(*pool, table.cpu()), lambda: PagedKV(pool[0].cpu(), pool[1].cpu(), table.cpu()),
        lambda: PagedKV(*pool, table, torch.zeros(2, dtype=torch.int32, device="cuda")),
        lambda: kv.append(k.float(), k.float(), L), lambda: kv.append(k, k[:2], L), lambda: kv.append(k, k, L.cpu()), lambda: kv.append(k, k, L[:2]),
        lambda: kv.append(k, k, L, cu=L), lambda: kv.append(k, k, L, q_out=q), lambda: kv.append(k, k, L, inv_freq=torch.zeros(32, device="cuda").double()),
        lambda: kv.append(k, k, L, inv_freq=torch.zeros(33, device="cuda")), lambda: kv.append(k, k, L, new_lens=L),
        lambda: kv.append(k[:2], k[:2], L), lambda: kv.append(k[:0], k[:0], L),
        lambda: kv.attend_shared(q[:, :3], L, 0, 0.1), lambda: kv.attend_shared(q, L, 33, 0.1), lambda: kv.attend_shared(q, L, -1, 0.1),
        lambda: kv.attend_shared(q, L, 0, float("nan")), lambda: kv.attend_shared(q[..., :32], L, 0, 0.1), lambda: kv.attend_shared(q[:2], L, 0, 0.1),
        lambda: kv.attend_shared(q, L, 40, 0.1, prefix_pages=torch.zeros(2, dtype=torch.int32, device="cuda")),
        lambda: kv.attend_shared(q, L, 0, 0.1, out=q[:2]),
        lambda: kv.attend_ranges(q.unsqueeze(2), torch.zeros((5, 1, 2), dtype=torch.int32, device="cuda"), L, 1, 0.1),
        lambda: kv.attend_ranges(q.unsqueeze(2), torch.zeros((6, 1, 3), dtype=torch.int32, device="cuda"), L, 1, 0.1),
        lambda: kv.attend_ranges(q.unsqueeze(2), torch.zeros((9, 1, 2), dtype=torch.int32, device="cuda"), L, 1, 0.1),
        lambda: kv.attend_ranges(q.unsqueeze(2), torch.zeros((6, 1025, 2), dtype=torch.int32, device="cuda"), L, 1, 0.1),
        lambda: kv.attend_ranges(q, torch.zeros((6, 1, 2), dtype=torch.int32, device="cuda"), L, 1, 0.1),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError, B.RouteRelayError)):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
