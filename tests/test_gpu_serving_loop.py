"""The operators of the serving loop together, as a program uses them: a prompt of patches and text, forked into samples; steps of drafted tokens that are appended,
attended to and verified, and whose rejected tokens are written over; a compaction in between; the end of all sequences."""
import pytest
import torch

from pages_oracle import Pages
from paged_oracle import assert_within, shared
from paper_2609_07306_b200.paged import PagedKV, axis_sections, inv_freq
from paper_2609_07306_b200.pages import PagePool
from paper_2609_07306_b200.verify import verify_drafts

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,greedy", [(torch.bfloat16, False), (torch.float32, True)])
def test_samples_of_a_prompt(dtype, greedy):
    batch, page, width, pages, KH, H, dh, vocab, layers = 5, 8, 16, 70, 2, 4, 64, 500, 2
    g = torch.Generator(device="cuda").manual_seed(17)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    table, status = torch.full((batch, width), -1, dtype=torch.int32, device="cuda"), ints([0])
    kvs = [PagedKV(torch.zeros((pages, KH, page, dh), device="cuda", dtype=dtype), torch.zeros((pages, KH, page, dh), device="cuda", dtype=dtype), table, status)
           for _ in range(layers)]
    pool = PagePool.empty(kvs, status)
    want = Pages(batch, width, pages, page)
    head = randn(H * dh, vocab) * 0.4
    freq, axis_of = inv_freq(dh), axis_sections((8, 12, 12))
    known = [[None] * layers for _ in range(batch)]        # every sequence's keys and values as they were given, by token

    def forward(tokens, place, cu, lens):
        """A layer's keys, values and queries come from the tokens' numbers; two layers, the second one's attention gives the scores."""
        after = torch.zeros_like(lens)
        at = torch.arange(place.numel(), device="cuda")
        pos = torch.stack((place, at % 7, at % 5)).int()
        for l, kv in enumerate(kvs):
            gl = torch.Generator(device="cuda").manual_seed(l)
            emb = torch.randn((vocab, (H + 2 * KH) * dh), generator=gl, device="cuda").to(dtype)
            qkv = emb[tokens.long()]
            q, k, v = (x.view(-1, n, dh) for x, n in ((qkv[:, :H * dh], H), (qkv[:, H * dh:(H + KH) * dh], KH), (qkv[:, (H + KH) * dh:], KH)))
            q = kv.append(k, v, lens, cu=cu, q=q, inv_freq=freq, new_lens=after, positions=pos, axis_of=axis_of)
            o = kv.attend_shared(q, after, 0, dh ** -0.5, cu=cu)
            w, bound = shared(q, kv.k_cache, kv.v_cache, table, after.tolist(), cu.tolist(), dh ** -0.5, True)
            assert_within(o[:cu[-1]], w[:cu[-1]], bound[:cu[-1]])
        return o.reshape(-1, H * dh).float() @ head, after

    # the prompt of sequence 0; the others are empty slots
    prompt = 21
    tokens = torch.randint(0, vocab, (prompt,), generator=g, device="cuda", dtype=torch.int32)
    lens, none = ints([0] * batch), ints([0] * batch)
    new = ints([prompt, 0, 0, 0, 0])
    pool.reserve(lens, new)
    assert want.reserve([0] * batch, new.tolist())
    cu = torch.cat((none[:1], new.cumsum(0).int()))
    _, lens = forward(tokens, torch.arange(prompt, device="cuda"), cu, lens)
    # four samples of it
    parents, out = ints([0, 0, 0, 0, -1]), ints([0] * batch)
    pool.fork(parents, lens, out)
    now = want.fork(parents.tolist(), lens.tolist())
    lens = out
    assert lens.tolist() == now == [prompt] * 4 + [0]
    last = torch.randint(0, vocab, (batch,), generator=g, device="cuda", dtype=torch.int32)
    spoken = [[] for _ in range(batch)]
    for step in range(6):
        drafts = [3, 0, 5, 2, -1] if step % 2 else [1, 4, 2, 3, -1]                 # the last slot has no rows
        rows = [n + 1 for n in drafts]
        cu = ints([0] + rows).cumsum(0).int()
        pool.reserve(lens, ints(rows))
        assert want.reserve(lens.tolist(), rows)
        want.check(pool)
        tokens = torch.randint(0, vocab, (sum(rows),), generator=g, device="cuda", dtype=torch.int32)
        tokens[cu[:4].long()] = last[:4]
        place = torch.cat([torch.arange(r, device="cuda") + lens[b] for b, r in enumerate(rows)])
        if greedy and step < 4:                            # drafts that are right, up to one of them: the target's own, token by token
            for _ in range(max(drafts)):
                scores, _ = forward(tokens, place, cu, lens)
                after, a = verify_drafts(scores, tokens, cu)
                i = torch.arange(sum(rows), device="cuda")
                for b in range(4):
                    n = min(a[b].item(), drafts[b] - 1)
                    if drafts[b] > 0 and n < drafts[b] - (step % 2):
                        tokens[cu[b].item() + n + 1] = after[cu[b].item() + n]
        scores, _ = forward(tokens, place, cu, lens)
        if greedy:
            kept, accepted = verify_drafts(scores, tokens, cu, lens=lens, new_lens=lens)
            best = scores.argmax(1)
        else:
            p, u = torch.softmax(scores, 1), torch.rand(sum(rows), generator=g, device="cuda")
            draft = torch.softmax(scores + randn(*scores.shape), 1)
            kept, accepted = verify_drafts(p, tokens, cu, draft=draft * 0.05, uniform=u, lens=lens, new_lens=lens)
        a = accepted.tolist()
        assert a[4] == 0 and lens.tolist() == [x + y + 1 for x, y in zip(now[:4], a)] + [0]
        now = lens.tolist()
        for b in range(4):
            said = kept[cu[b]:cu[b + 1]].tolist()
            assert said[:a[b]] == tokens[cu[b] + 1:cu[b] + 1 + a[b]].tolist() and all(0 <= x < vocab for x in said[:a[b] + 1])
            assert said[a[b] + 1:] == [-1] * (drafts[b] - a[b])
            if greedy:
                assert said[:a[b] + 1] == best[cu[b]:cu[b] + a[b] + 1].tolist()
            spoken[b] += said[:a[b] + 1]
            last[b] = said[a[b]]
        if step == 3:                                      # one sequence ends, another one's beams take over; then the pool is compacted
            p = [0, 2, 2, -1, 0]
            nl = ints([0] * batch)
            pool.fork(ints(p), lens, nl)
            now = want.fork(p, now)
            q = torch.randn((batch, H, dh), generator=g, device="cuda").to(dtype)
            before = [kv.attend_shared(q, nl, 0, 0.1) for kv in kvs]
            pool.reserve(nl, 0)
            want.reserve(now, [0] * batch)
            pool.compact()
            want.compact()
            want.check(pool)
            assert sorted(set(table[table >= 0].tolist())) == list(range(pages - pool.free.item()))
            assert all(torch.equal(x, kv.attend_shared(q, nl, 0, 0.1)) for x, kv in zip(before, kvs))
            last, spoken = torch.stack([last[max(x, 0)] for x in p]), [list(spoken[max(x, 0)]) for x in p]
            pool.fork(ints([0, 1, 2, 4, -1]), nl, lens)    # slot 4's sequence into slot 3, for the rows of the next steps
            now = want.fork([0, 1, 2, 4, -1], now)
            last, spoken = last[[0, 1, 2, 4, 4]], [spoken[x] for x in (0, 1, 2, 4, 4)]
            assert lens.tolist() == now
    pool.reserve(none)
    assert status.item() == 0 and pool.free.item() == pages and (table == -1).all() and (pool.refs == 0).all() and (pool.held == 0).all()
