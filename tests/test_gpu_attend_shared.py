"""Attention behind a shared prefix against the per-sequence definition in 64 bits: every type and kernel, tile and page
ends, ragged, empty, short and padded sequences, masks, values that a row may not see."""
import pytest
import torch

from paged_oracle import assert_within, shared
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu
NAN = float("nan")


def build(dtype, KH, dh, page, prefix, lens, seed, token_major=False, fill=NAN, own_tail=True):
    """A pool whose unused places hold `fill`; sequences share the whole pages of the prefix and copy its tail."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    Bn, width = len(lens), max(1, max(-(-max(n, prefix) // page) for n in lens))
    full = prefix // page
    pages = full + Bn * (width - full) + 2
    shape = (pages, page, KH, dh) if token_major else (pages, KH, page, dh)
    k, v = (torch.full(shape, fill, device="cuda", dtype=dtype) for _ in range(2))
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    perm = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.empty((Bn, width), dtype=torch.int32, device="cuda")
    table[:, :full] = perm[:full]
    table[:, full:] = perm[full:full + Bn * (width - full)].view(Bn, width - full)
    base = [torch.randn((max(prefix, 1), KH, dh), generator=g, device="cuda").to(dtype) for _ in range(2)]
    for b, n in enumerate(lens):
        t = torch.arange(max(n, prefix if b == 0 else 0), device="cuda")
        for c, p in zip((k, v), base):
            x = torch.randn((t.numel(), KH, dh), generator=g, device="cuda").to(dtype)
            x[:min(prefix, t.numel())] = p[:min(prefix, t.numel())]
            c[table[b].long()[t // page], :, t % page] = x
    return g, k, v, table


def run(dtype, H, KH, dh, page, prefix, lens, news, seed=0, causal=True, cu=True, pad=0, token_major=False, scale=None, hurt=None):
    g, k, v, table = build(dtype, KH, dh, page, prefix, lens, seed, token_major)
    if hurt:
        hurt(k, v, table)
    T = sum(news) + pad
    q = torch.randn((H, T, dh), generator=g, device="cuda").to(dtype).transpose(0, 1)      # head-major strides
    scale = dh ** -0.5 if scale is None else scale
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv = PagedKV(k, v, table, status)
    out = torch.full((T, H, dh), 7.0, device="cuda", dtype=dtype)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kv.attend_shared(q, L, prefix, scale, cu=torch.tensor(starts, dtype=torch.int32, device="cuda") if cu else None, causal=causal, out=out)
    want, bound = shared(q, k, v, table, lens, starts, scale, causal)
    assert (out[starts[-1]:] == 7.0).all()
    assert_within(out[:starts[-1]], want[:starts[-1]], bound[:starts[-1]])
    assert status.item() == 0
    again = kv.attend_shared(q, L, prefix, scale, cu=torch.tensor(starts, dtype=torch.int32, device="cuda") if cu else None, causal=causal)
    assert torch.equal(again[:starts[-1]].view(torch.int16 if dtype == torch.bfloat16 else torch.int32),
                       out[:starts[-1]].view(torch.int16 if dtype == torch.bfloat16 else torch.int32))
    return out


KINDS = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64), (torch.float32, 20), (torch.bfloat16, 80), (torch.float32, 256)]


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("prefix", [0, 1, 127, 128, 129, 700])
def test_single_tokens(dtype, dh, prefix):
    run(dtype, 4, 2, dh, 16, prefix, [prefix + x for x in (1, 2, 128, 130, 300)], [1] * 5, seed=prefix, cu=False)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("H,KH,page,prefix", [(5, 1, 24, 261), (7, 7, 7, 40), (16, 2, 64, 256), (6, 3, 128, 0)])
def test_prompts(dtype, dh, H, KH, page, prefix):
    """Several query tokens, causal: row tiles of one and of several sequences, sequences without queries, padding."""
    news = [1, 40, 0, 17, 90]
    run(dtype, H, KH, dh, page, prefix, [prefix + n + x for n, x in zip(news, (0, 5, 9, 130, 1))], news, seed=H, pad=3)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
def test_rows_beyond_one_item(dtype, dh):
    run(dtype, 8, 1, dh, 32, 200, [200 + 150, 200 + 3], [150, 3], seed=5)


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_short_and_absent_sequences(dtype, dh):
    """Sequences with no token, with fewer than the prefix, with as many; fewer tokens than queries."""
    out = run(dtype, 4, 2, dh, 16, 200, [200, 0, 90, 3, 201, 0], [1, 1, 2, 5, 1, 2], seed=9)
    assert (out[1] == 0).all() and (out[4:6] == 0).all()


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("prefix", [0, 150])
def test_states_of_another_length(dtype, dh, prefix):
    """No causal mask: every query sees all tokens."""
    run(dtype, 4, 4, dh, 16, prefix, [prefix + 77, prefix + 1, prefix, prefix + 260], [9, 3, 2, 1], seed=2, causal=False)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.float32, 32)])
def test_token_major_pages_and_large_logits(dtype, dh):
    run(dtype, 4, 2, dh, 16, 130, [200, 131, 400], [2, 1, 3], seed=4, token_major=True, scale=1.5)
    run(dtype, 4, 2, dh, 16, 130, [200, 131, 400], [2, 1, 3], seed=4, scale=-0.3)
    run(dtype, 4, 2, dh, 16, 130, [200, 131, 400], [2, 1, 3], seed=4, scale=0.0)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("bad", [float("inf"), NAN])
def test_values_that_a_prompt_may_not_see(dtype, dh, bad):
    """The same for one sequence alone, and for few rows."""
    for n, G in ((64, 4), (20, 1), (3, 5)):
        def hurt(k, v, table):
            p = int(table[0, (100 + n // 2) // 16])
            v[p, 0, (100 + n // 2) % 16, 7] = bad
        out = run(dtype, G, 1, dh, 16, 100, [100 + n], [n], seed=6, hurt=hurt)
        seen = torch.zeros((n, G, dh), dtype=torch.bool)
        seen[n // 2:, :, 7] = True
        assert torch.equal(~out.isfinite().cpu(), seen)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("bad", [float("inf"), NAN])
def test_values_that_a_row_may_not_see(dtype, dh, bad):
    """An infinity or NaN at a token reaches the queries that see it and no other, in its column only."""
    lens, news = [100 + 60, 100 + 20], [50, 20]

    def hurt(k, v, table):
        p = int(table[0, (100 + 30) // 16])
        v[p, 1, (100 + 30) % 16, 3] = bad
    out = run(dtype, 4, 2, dh, 16, 100, lens, news, seed=6, hurt=hurt)
    seen = torch.zeros((70, 4, dh), dtype=torch.bool)
    seen[20:50, 2:, 3] = True                          # query i of 50 stands at 110 + i
    assert torch.equal(~out.isfinite().cpu(), seen)


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_keys_at_minus_infinity(dtype, dh):
    """Logits of -inf weigh nothing; a query with no other has no softmax."""
    def hurt(k, v, table):
        for c in (table[0].long(),):
            k[c, 0, :, 0] = float("-inf")
    g, k, v, table = build(dtype, 1, dh, 16, 0, [40, 40], 3)
    k[table[0, :1].long(), 0, :, 0] = float("-inf")    # 16 of the 40 tokens
    k[table[1].long(), 0, :, 0] = float("-inf")        # all
    q = (torch.rand((2, 1, dh), generator=g, device="cuda") + 0.5).to(dtype)
    out = PagedKV(k, v, table).attend_shared(q, torch.tensor([40, 40], dtype=torch.int32, device="cuda"), 0, 0.1)
    k2, v2 = (c[table[0, 1:].long()][:, 0].reshape(-1, dh)[:24].double().cpu() for c in (k, v))
    from paged_oracle import attend
    want, bound = attend(q[0, 0].double().cpu(), k2, v2, 0.1, dtype == torch.bfloat16)
    assert_within(out[0, 0], want, bound)
    assert out[1].isnan().all()


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.float32, 64)])
def test_bad_pages_are_left_out(dtype, dh):
    g, k, v, table = build(dtype, 2, dh, 16, 64, [150, 150], 8)
    sane = table.clone()
    table[0, 5], table[1, 6] = k.shape[0] + 3, -2
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.randn((2, 4, dh), generator=g, device="cuda").to(dtype)
    out = PagedKV(k, v, table, status).attend_shared(q, torch.tensor([150, 150], dtype=torch.int32, device="cuda"), 64, 0.2)
    assert status.item() == B.RR_STATUS_BAD_INDEX
    from paged_oracle import attend, rows
    for b, gone in ((0, 5), (1, 6)):
        toks = [t for t in range(150) if t // 16 != gone]
        for h in range(4):
            kk, vv = (rows(c.cpu(), sane[b].cpu(), 16, toks)[:, h // 2] for c in (k, v))
            want, bound = attend(q[b, h].double().cpu(), kk, vv, 0.2, dtype == torch.bfloat16)
            assert_within(out[b, h], want, bound)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_prefix_pages_of_their_own(dtype, dh):
    """The prefix from a list of its own: sequence 0 may be absent."""
    g, k, v, table = build(dtype, 2, dh, 16, 80, [0, 100, 130], 12)
    own = table[1, :5].clone().contiguous()
    table[0] = -1
    q = torch.randn((3, 4, dh), generator=g, device="cuda").to(dtype)
    lens = [0, 100, 130]
    out = PagedKV(k, v, table).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), 80, 0.1, prefix_pages=own)
    table[0] = table[1]
    want, bound = shared(q, k, v, table, lens, [0, 1, 2, 3], 0.1, True)
    assert_within(out, want, bound)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("lens,news", [([100 + 70], [70]), ([100 + 64, 100 + 90, 700], [64, 64, 128]), ([40, 100 + 64], [64, 64]), ([0, 164], [64, 64])])
def test_prompts_that_fill_their_row_tiles(dtype, dh, lens, news):
    """Whole row tiles per sequence (and one sequence alone): each attends by itself, also where it is shorter than the prefix."""
    run(dtype, 4, 1, dh, 16, 100, lens, news, seed=len(lens))
    run(dtype, 4, 1, dh, 24, 100, lens, news, seed=7, causal=False)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
@pytest.mark.parametrize("page", [16, 24])
def test_prompts_with_prefix_pages_of_their_own(dtype, dh, page):
    """The sequences' tables hold nothing for the prefix's whole pages; it ends inside a page, whose rest is the sequences' own."""
    lens, news, prefix = [180, 164], [64, 64], 100
    g, k, v, table = build(dtype, 1, dh, page, prefix, lens, 14)
    pages = table[0, :-(-prefix // page)].clone().contiguous()
    bare = table.clone()
    bare[:, :prefix // page] = -5
    q = torch.randn((128, 4, dh), generator=g, device="cuda").to(dtype)
    cu = torch.tensor([0, 64, 128], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = PagedKV(k, v, bare, status).attend_shared(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), prefix, 0.1, cu=cu, prefix_pages=pages)
    want, bound = shared(q, k, v, table, lens, [0, 64, 128], 0.1, True)
    assert_within(out, want, bound)
    assert status.item() == 0


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_captured_and_replayed_with_other_lengths(dtype, dh):
    lens = [300, 170, 260]
    g, k, v, table = build(dtype, 2, dh, 16, 150, lens, 21)
    kv = PagedKV(k, v, table)
    q = torch.randn((3, 4, dh), generator=g, device="cuda").to(dtype)
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    kv.attend_shared(q, L, 150, 0.1, out=out)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    outs = [torch.empty_like(q), torch.empty_like(q)]
    for gr, o in zip(graphs, outs):
        with torch.cuda.graph(gr):
            kv.attend_shared(q, L, 150, 0.1, out=o)
    for now in (lens, [151, 0, 259], [100, 170, 1]):
        L.copy_(torch.tensor(now, dtype=torch.int32))
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        want, bound = shared(q, k, v, table, now, [0, 1, 2, 3], 0.1, True)
        for o in outs:
            assert_within(o, want, bound)


def test_two_streams_at_once():
    g, k, v, table = build(torch.bfloat16, 2, 128, 16, 500, [700, 600], 30)
    kv = PagedKV(k, v, table)
    q = torch.randn((2, 2, 8, 128), generator=g, device="cuda").bfloat16()
    L = torch.tensor([700, 600], dtype=torch.int32, device="cuda")
    alone = [kv.attend_shared(x, L, 500, 0.1) for x in q]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, x in zip(streams, q):
            with torch.cuda.stream(s):
                got.append([kv.attend_shared(x, L, 500, 0.1) for _ in range(3)])
        torch.cuda.synchronize()
        for a, outs in zip(alone, got):
            assert all(torch.equal(a, o) for o in outs)
