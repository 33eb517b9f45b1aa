"""Verification of drafted tokens against the definition in 64 bits: both modes, both types, vocabularies around every block and cluster size, ragged and
padded batches, rows off 16 bytes, weights that are nothing, NaN or infinite, ties, and the distribution of what comes out."""
import math

import numpy as np
import pytest
import torch

from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.verify import verify_drafts

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def weight(x):
    x = x.double().cpu().numpy()
    return np.where((x > 0) & (x <= float(np.finfo(np.float32).max)), x, 0.0)


def pick(w, u):
    """The first entry whose sum is over u times all, with sums that are rounded once (a positive weight where rounding leaves none)."""
    total = math.fsum(w)
    if total == 0:
        return -1
    cum = np.cumsum(w)
    over = np.flatnonzero((cum > max(u, 0.0) * total) & (w > 0))
    return int(over[0]) if len(over) else int(np.flatnonzero(w)[-1])


def oracle(target, tokens, cu, draft, uniform):
    """(next tokens with None behind the sequences, accepted)"""
    rows, V = target.shape
    tokens = tokens.tolist()
    cu = list(range(rows + 1)) if cu is None else cu.tolist()
    u = None if uniform is None else uniform.double().tolist()
    out, accepted = [None] * rows, []
    for b in range(len(cu) - 1):
        lo, n = cu[b], cu[b + 1] - cu[b] - 1
        if n < 0:
            accepted.append(0)
            continue
        x = tokens[lo + 1:lo + 1 + n]
        a, more = n, None
        if u is None:
            for i in range(n + 1):
                z = target[lo + i].double().cpu().numpy()
                z = np.where(np.isnan(z), -np.inf, z)
                nan = torch.isnan(target[lo + i]).cpu().numpy()
                best = int(np.flatnonzero((z == z[~nan].max()) & ~nan)[0]) if (~nan).any() else -1
                if i == n or best != x[i] or not 0 <= x[i] < V:
                    a, more = i, best
                    break
        else:
            for i in range(n):
                q = None if draft is None else weight(draft[lo + i])
                p = weight(target[lo + i])
                ok = 0 <= x[i] < V and p[x[i]] > u[lo + i] * (1.0 if q is None else q[x[i]])
                if not ok:
                    a = i
                    if q is not None:
                        rest = np.maximum(p - q, 0.0)
                    else:
                        rest = p.copy()
                        if 0 <= x[i] < V:
                            rest[x[i]] = 0.0
                    more = pick(rest, u[lo + n])
                    if more < 0:
                        more = pick(p, u[lo + n])
                    break
            if more is None:
                more = pick(weight(target[lo + n]), u[lo + n])
        out[lo:lo + n + 1] = x[:a] + [more] + [-1] * (n - a)
        accepted.append(a)
    return out, accepted


def inputs(rows, vocab, dtype, seed, pad=0, sharp=2.0):
    """Probabilities of target and draft, of rows that lie `pad` entries further apart than they are long."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    p = torch.softmax(torch.randn((rows, vocab), generator=g, device="cuda") * sharp, 1)
    q = torch.softmax(p.log() + torch.randn((rows, vocab), generator=g, device="cuda") * 0.7, 1)
    apart = lambda x: torch.zeros((rows, vocab + pad), device="cuda", dtype=dtype)[:, :vocab].copy_(x)
    target, draft = apart(p), apart(q)
    cum = draft.double().cumsum(1)
    x = torch.searchsorted(cum, torch.rand((rows, 1), generator=g, device="cuda", dtype=torch.float64) * cum[:, -1:], right=True)[:, 0].clamp_max(vocab - 1)
    tokens = torch.cat((x[:1], x[:-1])).int()             # the token behind row t is tokens[t + 1]
    return target, draft, tokens, torch.rand(rows, generator=g, device="cuda")


def check(target, tokens, cu, draft, uniform, lens=None):
    batch = target.shape[0] if cu is None else cu.shape[0] - 1
    lens = ints([(7 * b) % 31 for b in range(batch)])
    new, status = ints([-5] * batch), ints([0])
    got, accepted = verify_drafts(target, tokens, cu, draft=draft, uniform=uniform, lens=lens, new_lens=new, status=status)
    want, a = oracle(target, tokens, cu, draft, uniform)
    assert accepted.tolist() == a
    assert [g for g, w in zip(got.tolist(), want) if w is not None] == [w for w in want if w is not None]
    has = [1] * batch if cu is None else [int(n > 0) for n in (cu[1:] - cu[:-1]).tolist()]
    assert new.tolist() == [x + h * (y + 1) for x, h, y in zip(lens.tolist(), has, a)]
    return got, accepted, status.item()


VOCABS = [1, 2, 31, 255, 256, 257, 1000, 4095, 8191, 8192, 8193, 32768, 40001, 131072]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype,pad", [(torch.float32, 0), (torch.bfloat16, 8), (torch.bfloat16, 3)])
def test_sampled(vocab, dtype, pad):
    rows = [1, 5, 3, 0, 8, 2, 1, 4]
    cu = ints([0] + rows).cumsum(0).int()
    target, draft, tokens, uniform = inputs(sum(rows) + 3, vocab, dtype, vocab + pad, pad)        # three rows of padding
    check(target, tokens, cu, draft, uniform)
    check(target, tokens, cu, None, uniform * 0.2)


@pytest.mark.parametrize("vocab", VOCABS + [150001])
@pytest.mark.parametrize("dtype,pad,shift", [(torch.float32, 0, 0), (torch.float32, 1, 0), (torch.bfloat16, 0, 0), (torch.bfloat16, 8, 8), (torch.bfloat16, 0, 1)])
def test_greedy(vocab, dtype, pad, shift):
    """Scores with many ties in bf16; the drafts are the best tokens, but for one in eight."""
    rows = [4, 1, 0, 19, 2, 40, 1]
    cu = ints([0] + rows).cumsum(0).int()
    g = torch.Generator(device="cuda").manual_seed(vocab)
    T = sum(rows) + 2
    store = torch.randn((T * (vocab + pad) + shift), generator=g, device="cuda").to(dtype)
    target = store[shift:].view(T, vocab + pad)[:, :vocab]
    z = target.float()
    best = torch.where(z == z.amax(1, keepdim=True), torch.arange(vocab, device="cuda"), vocab).amin(1)
    wrong = torch.rand(T, generator=g, device="cuda") < 0.125
    x = torch.where(wrong, (best + 1) % vocab, best)
    tokens = torch.cat((x[:1], x[:-1])).int()
    check(target, tokens, cu, None, None)


def test_large_vocabularies():
    """More blocks than a CTA keeps sums of, in one row of zeros with few weights, the last entry among them."""
    vocab = 8 * 1024 * 256 * 2 + 777
    target = torch.zeros((2, vocab), device="cuda")
    at = [0, 12345, 2097151, 2097152, 3333333, vocab - 1]
    target[:, at] = torch.tensor([0.1, 0.2, 0.3, 0.15, 0.05, 0.2], device="cuda")
    for u in (0.0, 0.0999, 0.1001, 0.35, 0.7, 0.76, 0.79, 0.81, 0.999):
        check(target, ints([3, 12345]), ints([0, 2]), None, torch.tensor([0.1999, u], device="cuda"))
        check(target, ints([3, 12345]), ints([0, 2]), None, torch.tensor([0.2001, u], device="cuda"))
    check(target, ints([3, 2097152]), ints([0, 2]), None, None)


def test_one_row_per_sequence():
    target, _, tokens, uniform = inputs(70, 999, torch.float32, 3)
    got, accepted, _ = check(target, tokens, None, None, uniform)
    assert (accepted == 0).all()
    check(target, tokens, None, None, None)
    assert torch.equal(verify_drafts(target, tokens, ints(list(range(71))), uniform=uniform)[0], got)


def test_many_drafts():
    """More than a warp looks at once, accepted to the end, to the middle, from the first."""
    rows, V = 100, 50
    target = torch.full((3 * rows, V), 1.0 / V, device="cuda")
    draft = target.clone()
    tokens = ints([t % V for t in range(3 * rows)])
    uniform = torch.full((3 * rows,), 0.5, device="cuda")
    draft[rows + 63] = 0.9                                 # p = 0.02 > 0.5 * 0.9 does not hold
    draft[2 * rows] = 0.9
    cu = ints([0, rows, 2 * rows, 3 * rows])
    _, accepted, _ = check(target, tokens, cu, draft, uniform)
    assert accepted.tolist() == [99, 63, 0]


def test_decisions_next_to_a_border():
    """p > u q is decided by the numbers, not by their product's rounding."""
    u = torch.tensor([1 / 3, 0.7, 0.1], device="cuda")
    q = torch.tensor([0.6, 0.3, 0.9], device="cuda")
    exact = u.double() * q.double()
    for step in (-1, 0, 1):
        p = exact.float()
        if step:
            p = torch.nextafter(p, torch.full_like(p, 2.0 if step > 0 else 0.0))
        target, draft = torch.zeros((6, 4), device="cuda"), torch.zeros((6, 4), device="cuda")
        target[::2, 2], draft[::2, 2] = p, q
        target[:, 3] = 0.5
        uniform = torch.zeros(6, device="cuda")
        uniform[::2] = u
        _, accepted, _ = check(target, ints([0, 2] * 3), ints([0, 2, 4, 6]), draft, uniform)
        assert accepted.tolist() == (p.double() > exact).int().tolist()


def test_weights_that_are_none():
    nan, inf = float("nan"), float("inf")
    rows = [
        ([0.2, nan, 0.3, inf, -1.0, 0.5], [0.9, 0.1, nan, 0.2, 0.0, 0.3]),      # NaN, infinite and negative entries count as 0
        ([0.0, 0.0, 0.0, 0.0, 0.0, 0.0], [0.9, 0.1, 0.2, 0.2, 0.0, 0.3]),       # nothing at all: -1
        ([0.1, 0.2, 0.1, 0.2, 0.1, 0.3], [0.5, 0.5, 0.5, 0.5, 0.5, 0.5]),       # the target is below the draft everywhere: the target's own
        ([nan] * 6, [nan] * 6),
        ([0.0, 0.0, 0.0, 0.4, 0.0, 0.0], [0.0, 0.0, 0.0, 0.1, 0.0, 0.0]),
    ]
    for dtype in (torch.float32, torch.bfloat16):
        for p, q in rows:
            for x in range(6):
                for u in ((0.99, 0.0), (0.99, 0.5), (0.0, 0.9999), (1.0, 1.0), (nan, nan), (0.5, -1.0)):
                    target = torch.tensor([p, [0.25, nan, 0.25, 0.0, 0.5, 0.0]], device="cuda", dtype=dtype)
                    draft = torch.tensor([q, [nan] * 6], device="cuda", dtype=dtype)
                    uniform = torch.tensor(u, device="cuda")
                    if math.isnan(u[1]):                   # (a random number that is none is 0 where a token is drawn)
                        want, a = oracle(target, ints([1, x]), ints([0, 2]), draft, torch.tensor([u[0], 0.0]))
                        got, accepted = verify_drafts(target, ints([1, x]), ints([0, 2]), draft=draft, uniform=uniform)
                        assert got.tolist() == want and accepted.tolist() == a
                    else:
                        check(target, ints([1, x]), ints([0, 2]), draft, uniform)
                        check(target, ints([1, x]), ints([0, 2]), None, uniform)


def test_greedy_with_nan_and_infinities():
    nan, inf = float("nan"), float("inf")
    rows = [[nan, 1.0, 2.0, 2.0, nan, -1.0, 0.0, 1.0, 2.0], [nan] * 9, [-inf] * 9, [nan, -inf, -inf, nan, -inf, nan, nan, nan, nan], [inf, nan, inf] * 3,
            [-0.0, 0.0, -0.0, 0.0, -1.0, nan, -0.0, 0.0, -0.0], [-3.0] * 8 + [-2.0]]
    best = [2, -1, 0, 1, 0, 0, 8]
    for dtype in (torch.float32, torch.bfloat16):
        for wide in (9, 16, 40):                           # 16 bytes at a time, and not
            target = torch.full((7, wide), nan, device="cuda", dtype=dtype)
            target[:, :9] = torch.tensor(rows, device="cuda").to(dtype)
            for t in (target, target[:, :9]):
                got, _, _ = check(t, ints([0] * 7), None, None, None)
                assert got.tolist() == best


def test_drafts_outside_the_vocabulary():
    target, draft, tokens, uniform = inputs(6, 100, torch.float32, 1)
    draft[:, :] = 1e-6
    for bad in (-1, 100, 1 << 30, -(1 << 31)):
        tokens[2] = bad
        for q, u in ((draft, uniform), (None, uniform * 0), (None, None)):
            _, accepted, status = check(target, tokens, ints([0, 3, 6]), q, u)
            if u is not None:
                assert accepted.tolist()[0] <= 1
            assert status == B.RR_STATUS_BAD_INDEX or (u is None and accepted.tolist()[0] == 0)


def test_padding_and_empty_sequences():
    target, draft, tokens, uniform = inputs(9, 300, torch.float32, 4)
    cu = ints([0, 0, 4, 4, 6])
    for q, u in ((draft, uniform), (None, None)):
        check(target, tokens, cu, q, u)
    for u in (uniform[:0], None):
        got, accepted = verify_drafts(target[:0], tokens[:0], ints([0, 0, 0]), uniform=u)
        assert got.shape == (0,) and accepted.tolist() == [0, 0]
    # what is padding is not written
    args = B.rr_verify_args(target=target.data_ptr(), tokens=tokens.data_ptr(), cu=cu.data_ptr(), accepted=ints([0] * 4).data_ptr(), target_stride=300,
                            dtype=B.RR_F32, rows=9, batch=4, vocab=300)
    out, acc = ints([77] * 9), ints([0] * 4)
    args.out, args.accepted = out.data_ptr(), acc.data_ptr()
    B.rr_verify_drafts(args, torch.cuda.current_stream().cuda_stream)
    assert out.tolist()[6:] == [77] * 3 and 77 not in out.tolist()[:6]
    # lens in place
    lens = ints([5, 6, 7, 8])
    want = lens + ints([0, 1, 0, 1]) + verify_drafts(target, tokens, cu, draft=draft, uniform=uniform, lens=lens, new_lens=lens)[1]
    assert torch.equal(lens, want.int())


def test_a_malformed_list_of_sequences():
    """Rows outside the arrays are not read, whatever cu says."""
    target, draft, tokens, uniform = inputs(8, 300, torch.float32, 4)
    for cu in ([0, 9, 12], [-3, 4, 8], [0, 5, 2, 8], [8, 8, 1 << 30]):
        for q, u in ((draft, uniform), (None, None)):
            got, accepted = verify_drafts(target, tokens, ints(cu), draft=q, uniform=u)
            assert (accepted >= 0).all() and (accepted < 8).all()


def test_the_tokens_are_the_targets():
    """One draft from q, all combinations of 50 x 40 x 40 evenly spaced random numbers: the first token's shares are the target's.  A share is off by at most
    what an evenly spaced number misses at each of the borders: of the 5 tokens drawn, of the test, of the 5 of the remainder."""
    p, q = [0.05, 0.3, 0.15, 0.4, 0.1], [0.35, 0.2, 0.3, 0.1, 0.05]
    n0, n1, n2 = 50, 40, 40
    grid = lambda n: (torch.arange(n, device="cuda") + 0.5) / n
    u0, u1, u2 = (x.reshape(-1) for x in torch.meshgrid(grid(n0), grid(n1), grid(n2), indexing="ij"))
    N = u0.numel()
    target = torch.tensor(p, device="cuda").expand(2 * N, 5)
    draft = torch.tensor(q, device="cuda").expand(2 * N, 5)
    cum = torch.tensor(q, device="cuda").cumsum(0)
    tokens = torch.zeros((N, 2), dtype=torch.int32, device="cuda")
    tokens[:, 1] = torch.searchsorted(cum, u0, right=True).clamp_max(4).int()
    got, accepted = verify_drafts(target, tokens.view(-1), torch.arange(0, 2 * N + 1, 2, device="cuda").int(), draft=draft, uniform=torch.stack((u1, u2), 1).view(-1))
    share = torch.bincount(got[::2].long(), minlength=5).double() / N
    assert (share.cpu() - torch.tensor(p, dtype=torch.float64)).abs().max() < 2 / n0 + 1 / n1 + 2 / n2
    kept = sum(min(a, b) for a, b in zip(p, q))
    assert abs(accepted.double().mean().item() - kept) < 5 / n0 + 1 / n1


def test_captured_on_another_stream_and_far_rows():
    target, draft, tokens, uniform = inputs(12, 5000, torch.bfloat16, 9)
    cu, lens, new = ints([0, 5, 12]), ints([3, 4]), ints([0, 0])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        got, accepted = verify_drafts(target, tokens, cu, draft=draft, uniform=uniform, lens=lens, new_lens=new)
    for seed in (10, 11, 12):
        for x, y in zip((target, draft, tokens, uniform), inputs(12, 5000, torch.bfloat16, seed)):
            x.copy_(y)
        graph.replay()
        want, a = oracle(target, tokens, cu, draft, uniform)
        assert got.tolist() == want and accepted.tolist() == a and new.tolist() == [x + y + 1 for x, y in zip([3, 4], a)]
    # rows more than 2^31 entries apart
    store = torch.empty(2 * (1 << 31) + 5000, dtype=torch.bfloat16, device="cuda")
    far = store.as_strided((3, 5000), (1 << 31, 1))
    far.copy_(target[:3])
    check(far, tokens[:3], ints([0, 3]), draft[:3], uniform[:3])
    check(far, tokens[:3], ints([0, 3]), None, None)


def test_what_the_wrapper_refuses():
    target, draft, tokens, uniform = inputs(6, 100, torch.float32, 1)
    cu = ints([0, 3, 6])
    two = ints([0, 0])
    for call, kind in ((lambda: verify_drafts(target.half(), tokens, cu), TypeError), (lambda: verify_drafts(target.cpu(), tokens, cu), ValueError),
                       (lambda: verify_drafts(target, tokens[:5], cu), ValueError), (lambda: verify_drafts(target, tokens.long(), cu), ValueError),
                       (lambda: verify_drafts(target, tokens, cu.long()), ValueError), (lambda: verify_drafts(target, tokens, cu[:1]), ValueError),
                       (lambda: verify_drafts(target, tokens, cu, draft=draft), ValueError), (lambda: verify_drafts(target, tokens, cu, draft=draft[:5], uniform=uniform), ValueError),
                       (lambda: verify_drafts(target, tokens, cu, draft=draft.bfloat16(), uniform=uniform), ValueError),
                       (lambda: verify_drafts(target, tokens, cu, uniform=uniform.double()), ValueError), (lambda: verify_drafts(target, tokens, cu, uniform=uniform[::2]), ValueError),
                       (lambda: verify_drafts(target, tokens, cu, new_lens=two), ValueError), (lambda: verify_drafts(target, tokens, cu, lens=two[:1], new_lens=two), ValueError),
                       (lambda: verify_drafts(target.t(), tokens, cu), ValueError), (lambda: verify_drafts(target.clone().requires_grad_(), tokens, cu), ValueError),
                       (lambda: verify_drafts(target[0], tokens, cu), ValueError), (lambda: verify_drafts(target[:0], tokens[:0]), ValueError),
                       (lambda: verify_drafts(target, tokens, cu, status=two), ValueError),
                       (lambda: verify_drafts(target.t().contiguous().t(), tokens, cu), ValueError)):
        with pytest.raises(kind):
            call()
    with torch.no_grad():
        verify_drafts(target.clone().requires_grad_(), tokens, cu)
