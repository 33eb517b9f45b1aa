"""Operators of the serving loop around the paged key/value cache: what comes before and behind its attention in a step.

axes      new tokens into the cache, keys and queries rotated by positions of several axes (time, height, width)
beams     a step of beam search: every beam becomes a copy of the one that it descends from, and gets a page of its own to write to
room      pages for the sequences' next tokens: what is no longer needed goes back, what is missing is handed out
compact   the pages in use move to the front of the pool
verify    drafted tokens against the target's probabilities from given random numbers, or against the target's best tokens

Each operator has a plain form here (elementary torch operations, 32 bits, 64 for angles, long sums and values next to a border) and the
calls that a user of the library makes.  `exact` computes the same from the definitions, in 64 bits and by ordinary lists.
"""
import math
import random

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------------------
def listed():
    return [
        # a decoding step of 64 sequences whose positions count time, height and width, sections of pairs one behind the other
        dict(name="axes_step", op="axes", dtype="bf16", batch=64, heads=32, kv_heads=8, dh=128, rot=128, interleaved=False, axes=3, mixed=False,
             page=16, new=1, ctx=2000, ragged=False),
        # prompts of text and images that enter the cache together, the axes taking turns from pair to pair
        dict(name="axes_images", op="axes", dtype="bf16", batch=9, heads=32, kv_heads=8, dh=128, rot=128, interleaved=False, axes=3, mixed=True,
             page=64, new=4000, ctx=900, ragged=True),
        # fp32, two axes, pairs side by side, half of the head's width rotated, odd page size and counts
        dict(name="axes_f32_pairs", op="axes", dtype="f32", batch=5, heads=6, kv_heads=3, dh=64, rot=32, interleaved=True, axes=2, mixed=False,
             page=24, new=700, ctx=333, ragged=True),
        # four beams of one request, two layers: latency
        dict(name="beams_one", op="beams", dtype="bf16", groups=1, beams=4, kv_heads=8, dh=128, page=16, ctx=1000, layers=2),
        # 32 requests of eight beams each, pages of 64 tokens in eight layers
        dict(name="beams_batch", op="beams", dtype="bf16", groups=32, beams=8, kv_heads=8, dh=128, page=64, ctx=700, layers=8),
        # the steps of 64 sequences with up to five drafted tokens each: few pages come and go
        dict(name="room_step", op="room", dtype="bf16", batch=64, kv_heads=8, dh=64, page=16, ctx=8000, new=6, ended=False, layers=1),
        # half of 512 sequences have ended and prompts of up to 4000 tokens take their places
        dict(name="room_admit", op="room", dtype="bf16", batch=512, kv_heads=1, dh=64, page=16, ctx=4000, new=4000, ended=True, layers=1),
        # a small fp32 pool, odd sizes, strides of a token-major pool
        dict(name="compact_small", op="compact", dtype="f32", batch=7, kv_heads=3, dh=40, page=12, ctx=300, keep=0.6, layers=2),
        # half of the sequences have ended: a quarter of a pool of 2 GB moves
        dict(name="compact_pool", op="compact", dtype="bf16", batch=64, kv_heads=8, dh=128, page=32, ctx=8000, keep=0.5, layers=2),
        # one sequence's step, five drafts of a vocabulary of 32768: latency
        dict(name="verify_one", op="verify", dtype="f32", batch=1, drafts=5, vocab=32768, accept=0.7, greedy=False, ragged=False),
        # the step of a batch, up to four drafts, a vocabulary of odd size
        dict(name="verify_step", op="verify", dtype="f32", batch=64, drafts=4, vocab=131071, accept=0.7, greedy=False, ragged=True),
        # temperature zero: 96 sequences, up to seven drafts against the best tokens of bf16 logits
        dict(name="verify_greedy", op="verify", dtype="bf16", batch=96, drafts=7, vocab=131072, accept=0.8, greedy=True, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    op = rng.choice(("axes", "beams", "room", "compact", "verify", "verify"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    kv, page = rng.choice((1, 2, 3, 4, 8)), rng.choice((8, 12, 16, 24, 32, 64))
    if op == "axes":
        dh, new = rng.choice((32, 64, 80, 128)), _log(rng, 1, 4000)
        return dict(op=op, dtype=dtype, batch=_log(rng, 1, 200), heads=kv * rng.choice((1, 2, 4, 5)), kv_heads=kv, dh=dh, rot=rng.choice((dh, dh // 2)),
                    interleaved=rng.random() < 0.4, axes=rng.choice((2, 3, 4)), mixed=rng.random() < 0.5, page=page, new=new,
                    ctx=_log(rng, 1, 2000), ragged=new > 1)
    dh, layers = rng.choice((40, 64, 128)), rng.choice((1, 2, 3, 8))
    if op == "beams":
        return dict(op=op, dtype=dtype, groups=_log(rng, 1, 64), beams=rng.choice((2, 4, 5, 8)), kv_heads=kv, dh=dh, page=page, ctx=_log(rng, 20, 4000), layers=layers)
    if op == "room":
        ended = rng.random() < 0.5
        return dict(op=op, dtype=dtype, batch=_log(rng, 2, 512), kv_heads=kv, dh=dh, page=page, ctx=_log(rng, 20, 8000), new=_log(rng, 20, 4000) if ended else rng.randint(1, 9),
                    ended=ended, layers=1)
    if op == "compact":
        return dict(op=op, dtype=dtype, batch=_log(rng, 4, 128), kv_heads=kv, dh=dh, page=page, ctx=_log(rng, 50, 8000), keep=rng.choice((0.3, 0.5, 0.8)), layers=layers)
    return dict(op=op, dtype=dtype, batch=_log(rng, 1, 128), drafts=rng.choice((1, 2, 3, 4, 5, 7)), vocab=_log(rng, 500, 150000), accept=rng.choice((0.5, 0.7, 0.9)),
                greedy=rng.random() < 0.4, ragged=rng.random() < 0.7)


def _entries(case):
    """Entries that a state of this case holds on the GPU."""
    if case["op"] == "axes":
        return sum(_lens(case)[1]) * case["dh"] * (case["heads"] + 2 * case["kv_heads"])
    if case["op"] == "verify":
        return 2 * case["batch"] * (case["drafts"] + 1) * case["vocab"]
    return 2 * case["layers"] * _pages(case) * case["page"] * case["kv_heads"] * case["dh"]


def draw(rng):
    top = {}
    for c in listed():
        w = dict(work(c), entries=_entries(c))
        for key in w:
            top[c["op"], key] = max(top.get((c["op"], key), 0), w[key])
    while True:
        c = _draw_one(rng)
        w = dict(work(c), entries=_entries(c))
        if all(w[key] <= top[c["op"], key] for key in w):
            return c


def _lens(case):
    """Tokens per sequence, part of the case.  axes: before, new.  beams: of each group.  room: the two steps' (tokens, new ones).
    compact: tokens.  verify: rows (drafts and the token before them)."""
    rng = random.Random("%s %d" % (case["op"], case["page"] if "page" in case else case["vocab"]))
    if case["op"] == "axes":
        B = case["batch"]
        return ([rng.randint(0, case["ctx"]) for _ in range(B)],
                [rng.randint(1, case["new"]) if case["ragged"] else case["new"] for _ in range(B)])
    if case["op"] == "beams":
        return [rng.randint(max(1, case["ctx"] // 2), case["ctx"]) for _ in range(case["groups"])]
    if case["op"] == "room":
        B, n = case["batch"], case["new"]
        if not case["ended"]:
            a = [rng.randint(case["ctx"] // 2, case["ctx"]) for _ in range(B)]
            return a, [rng.randint(1, n) for _ in range(B)], [x + rng.randint(1, n) for x in a], [rng.randint(1, n) for _ in range(B)]
        first = [rng.randint(1, n) for _ in range(B)]
        second = [rng.randint(1, n) for _ in range(B)]
        even = [b % 2 == 0 for b in range(B)]
        return ([0 if e else s for e, s in zip(even, second)], [f if e else 1 for e, f in zip(even, first)],
                [f if e else 0 for e, f in zip(even, first)], [1 if e else s for e, s in zip(even, second)])
    if case["op"] == "compact":
        return [rng.randint(1, case["ctx"]) for _ in range(case["batch"])]
    return [rng.randint(0, case["drafts"]) + 1 if case["ragged"] else case["drafts"] + 1 for _ in range(case["batch"])]


def _parents(case):
    """The beam that each beam descends from, within its group."""
    rng = random.Random("parents %d" % case["beams"])
    K = case["beams"]
    return [g * K + rng.randrange(K) for g in range(case["groups"]) for _ in range(K)]


def _up(n, page):
    return -(-n // page)


def _width(case):
    """Columns of the page table."""
    a, page = _lens(case), case["page"]
    if case["op"] == "axes":
        return max(_up(x + n, page) for x, n in zip(*a))
    if case["op"] == "beams":
        return _up(max(a) + 1, page)
    if case["op"] == "room":
        return max(_up(x + n, page) for x, n in list(zip(a[0], a[1])) + list(zip(a[2], a[3])))
    return _up(max(a), page)


def _pages(case):
    """Pages of the pool: what its fullest moment needs, and some more."""
    a, page = _lens(case), case["page"]
    if case["op"] == "axes":
        return sum(_up(x + n, page) for x, n in zip(*a))
    if case["op"] == "beams":
        return sum(_up(x, page) + (case["beams"] - 1) * (_up(x, page) - x // 2 // page) for x in a) + case["groups"] * case["beams"] + 3
    if case["op"] == "room":
        n = max(sum(_up(x + y, page) for x, y in zip(a[i], a[i + 1])) for i in (0, 2))
        m = sum(max(_up(x + y, page), _up(u + v, page)) for x, y, u, v in zip(*a))
        return max(n + n // 16, m) + 5
    return sum(_up(x, page) for x in a) + 5


# ---- work -----------------------------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    a = _lens(case)
    if case["op"] == "axes":
        T, H, KH = sum(a[1]), case["heads"], case["kv_heads"]
        return {"bytes": T * case["dh"] * e * 2 * (H + 2 * KH) + 4 * T * case["axes"], "flops": 3 * T * case["rot"] * (H + KH)}
    if case["op"] == "verify":
        if case["greedy"]:
            return {"bytes": sum(a) * case["vocab"] * e, "flops": sum(a) * case["vocab"]}
        # a row of the target's, and one of the draft's where a token was rejected
        rows = sum(2 - case["accept"] ** (n - 1) for n in a)
        return {"bytes": int(rows * case["vocab"]) * e, "flops": int(rows * case["vocab"])}
    page, token = case["page"], 2 * case["layers"] * case["kv_heads"] * case["dh"] * e
    if case["op"] == "beams":
        K, p = case["beams"], _parents(case)
        copies = sum((K - len(set(p[g * K:g * K + K]))) * (a[g] % page) for g in range(case["groups"]))
        entries = sum(K * _up(x, page) for x in a)
        return {"bytes": 2 * copies * token + 4 * entries + 4 * _pages(case), "flops": entries}
    if case["op"] == "room":
        changed = sum(abs(_up(x + y, page) - _up(u + v, page)) for x, y, u, v in zip(*a))
        return {"bytes": 2 * (4 * _pages(case) + 8 * case["batch"] + 12 * changed), "flops": 2 * _pages(case)}
    live = sum(_up(x, page) for x in _kept(case))
    return {"bytes": int(2 * live * (1 - live / _pages(case)) * page * token + 8 * live + 8 * _pages(case)), "flops": live + _pages(case)}


def _kept(case):
    """compact: tokens of the sequences that have not ended."""
    rng = random.Random("kept %d" % case["batch"])
    return [x if b == 0 or rng.random() < case["keep"] else 0 for b, x in enumerate(_lens(case))]


# ---- inputs ---------------------------------------------------------------------------------------------------
class _State:
    pass


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _randn(g, shape, dt):
    return torch.empty(shape, device="cuda", dtype=dt).normal_(generator=g)


def _table(g, case, own_cols, shared=None):
    """A table whose row b holds own_cols[b] pages of its own, scattered over the pool; with `shared` = (first row, columns) of each row, the first
    columns are those of another row.  (table, held, refs)"""
    pages, W, B = _pages(case), _width(case), len(own_cols)
    perm = torch.randperm(pages, generator=g, device="cuda").int()
    mine = torch.tensor(own_cols, device="cuda")
    col = torch.arange(W, device="cuda")
    begin = torch.zeros_like(mine)
    if shared is not None:
        row, begin = torch.tensor(shared[0], device="cuda"), torch.tensor(shared[1], device="cuda")
    at = (torch.cumsum(mine, 0) - mine)[:, None] + col - begin[:, None]
    here = (col >= begin[:, None]) & (col < (begin + mine)[:, None])
    table = torch.where(here, perm[torch.where(here, at, 0)], -1)
    if shared is not None:
        table = torch.where(col < begin[:, None], table[row], table)
    held = (begin + mine).int()
    return table.contiguous(), held, _count(table, pages)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s, dt = _State(), _DT[case["dtype"]]
    s.case = case
    if case["op"] == "verify":
        return _prepare_verify(s, case, g, dt)
    a, page, KH, dh = _lens(case), case["page"], case["kv_heads"], case["dh"]
    # keys and values of all layers, as one allocation; the small fp32 pools keep a token's heads side by side
    shape = (case.get("layers", 1), 2, _pages(case), KH, page, dh)
    if case["dtype"] == "f32":
        s.pool = _randn(g, shape[:3] + (page, KH, dh), dt).transpose(3, 4)
    else:
        s.pool = _randn(g, shape, dt)
    if case["op"] == "axes":
        T, B, H = sum(a[1]), case["batch"], case["heads"]
        s.table, s.held, s.refs = _table(g, case, [_up(x + n, page) for x, n in zip(*a)])
        s.lens, s.new_lens = _ints(a[0]), _ints([0] * B)
        s.cu = None if case["new"] == 1 else _ints([0] + a[1]).cumsum(0).int()
        qkv = _randn(g, (T, (H + 2 * KH) * dh), dt)                          # the projections' output, side by side
        s.q = qkv[:, :H * dh].view(T, H, dh)
        s.k = qkv[:, H * dh:(H + KH) * dh].view(T, KH, dh)
        s.v = qkv[:, (H + KH) * dh:].view(T, KH, dh)
        n = case["rot"] // 2
        s.inv_freq = (10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)).float()
        pair = torch.arange(n, device="cuda")
        s.axis_of = (pair % case["axes"] if case["mixed"] else pair * case["axes"] // n).int()
        # patches of images of 1 to 70 by 1 to 70 behind one another in time
        s.positions = torch.randint(0, 70, (case["axes"], T), generator=g, device="cuda", dtype=torch.int32)
        s.positions[0] += torch.arange(T, device="cuda", dtype=torch.int32) // 50
    elif case["op"] == "beams":
        K = case["beams"]
        lens = [x for x in a for _ in range(K)]
        begin = [0 if b % K == 0 else x // 2 // page for b, x in enumerate(lens)]
        s.table, s.held, s.refs = _table(g, case, [_up(x, page) - y for x, y in zip(lens, begin)], ([b // K * K for b in range(len(lens))], begin))
        s.lens, s.new_lens, s.parents = _ints(lens), _ints([0] * len(lens)), _ints(_parents(case))
    elif case["op"] == "room":
        s.table, s.held, s.refs = _table(g, case, [_up(x + n, page) for x, n in zip(a[2], a[3])])
        s.steps = [(_ints(a[0]), _ints(a[1])), (_ints(a[2]), _ints(a[3]))]
    else:
        kept = torch.tensor(_kept(case), device="cuda") > 0
        table, held, _ = _table(g, case, [_up(x, page) for x in a])
        s.table0, s.held = torch.where(kept[:, None], table, -1), torch.where(kept, held, 0)
        s.refs0 = _count(s.table0, _pages(case))
        s.table, s.refs = s.table0.clone(), s.refs0.clone()
    s.free = (s.refs == 0).sum().int().view(1)
    if own:
        from paper_2609_07306_b200.paged import PagedKV
        from paper_2609_07306_b200.pages import PagePool
        s.kvs = [PagedKV(layer[0], layer[1], s.table) for layer in s.pool]
        if case["op"] != "axes":
            s.pages = PagePool(s.table, page, s.refs, s.held, s.free, s.kvs)
    return s


def _prepare_verify(s, case, g, dt):
    rows, V, B = _lens(case), case["vocab"], case["batch"]
    T = sum(rows)
    s.cu = _ints([0] + rows).cumsum(0).int()
    last = torch.zeros(T, dtype=torch.bool, device="cuda")
    last[(s.cu[1:] - 1).long()] = True
    logits = torch.empty((T, V), device="cuda").normal_(0.0, 2.5, generator=g)
    s.lens, s.new_lens = torch.randint(0, 9000, (B,), generator=g, device="cuda", dtype=torch.int32), _ints([0] * B)
    pick = torch.rand(T, generator=g, device="cuda")
    s.draft = s.uniform = None
    if case["greedy"]:
        s.target = logits.to(dt)
        best = s.target.float().argmax(1)
        after = torch.where(pick < case["accept"], best, (best + 1) % V)
    else:
        p = torch.softmax(logits, 1)
        s.target = p.to(dt)
        # a draft model that agrees with the target by the given share and otherwise draws as for another row
        s.draft = (case["accept"] * p + (1 - case["accept"]) * p.roll((1, V // 3), (0, 1))).to(dt)
        s.uniform = torch.rand(T, generator=g, device="cuda")
        cum = s.draft.double().cumsum(1)
        after = torch.searchsorted(cum, pick.double()[:, None] * cum[:, -1:], right=True)[:, 0].clamp_max(V - 1)
        s.draft[last] = float("nan")                                         # (a sequence's last row drafted nothing)
    # the step's tokens: the last known one of a sequence, then its drafts
    s.tokens = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    s.tokens[1:] = torch.where(last[:-1], s.tokens[1:], after[:-1].int())
    s.most = max(rows)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    op = s.case["op"]
    if op == "axes":
        if own:
            q = s.kvs[0].append(s.k, s.v, s.lens, cu=s.cu, q=s.q, inv_freq=s.inv_freq, interleaved=s.case["interleaved"], new_lens=s.new_lens,
                                positions=s.positions, axis_of=s.axis_of)
        else:
            q = _axes(s)
        return {"q": q, "cache": s.pool, "lens": s.new_lens}
    if op == "verify":
        if own:
            from paper_2609_07306_b200.verify import verify_drafts
            tokens, accepted = verify_drafts(s.target, s.tokens, s.cu, draft=s.draft, uniform=s.uniform, lens=s.lens, new_lens=s.new_lens)
        else:
            tokens, accepted = _verify(s)
        return {"tokens": tokens, "accepted": accepted, "lens": s.new_lens}
    if op == "beams":
        if own:
            s.pages.fork(s.parents, s.lens, s.new_lens)
            s.pages.reserve(s.new_lens, 1)
        else:
            _fork(s)
            _reserve(s, s.new_lens, torch.ones_like(s.lens))
        return {"table": s.table, "refs": s.refs, "held": s.held, "free": s.free, "lens": s.new_lens, "cache": s.pool}
    if op == "room":
        (lens_a, new_a), (lens_b, new_b) = s.steps
        if own:
            s.pages.reserve(lens_a, new_a)
            s.pages.reserve(lens_b, new_b)
        else:
            _reserve(s, lens_a, new_a)
            _reserve(s, lens_b, new_b)
        return {"table": s.table, "refs": s.refs, "held": s.held, "free": s.free}
    # the pool as the ended sequences have left it
    s.table.copy_(s.table0)
    s.refs.copy_(s.refs0)
    if own:
        s.pages.compact()
    else:
        _compact(s)
    return {"table": s.table, "refs": s.refs, "cache": s.pool}


def _rotate(x, cos, sin, interleaved):
    """x [T, heads, dh] in 32 bits; the first 2 * cos.shape[1] entries of a head are rotated."""
    n = cos.shape[1]
    cos, sin, y = cos[:, None], sin[:, None], x.clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _axes(s):
    case, T, page = s.case, s.k.shape[0], s.case["page"]
    t = torch.arange(T, device="cuda")
    if s.cu is None:
        b, i = t, torch.zeros_like(t)
    else:
        b = torch.searchsorted(s.cu[1:].long().contiguous(), t, right=True)
        i = t - s.cu.long()[b]
    place = s.lens.long()[b] + i
    angle = s.positions[s.axis_of.long()].double().T * s.inv_freq.double()
    cos, sin = angle.cos().float(), angle.sin().float()
    at = s.table.long()[b, place // page]
    s.pool[0, 0][at, :, place % page] = _rotate(s.k.float(), cos, sin, case["interleaved"]).to(s.k.dtype)
    s.pool[0, 1][at, :, place % page] = s.v
    s.new_lens.copy_(s.lens + 1 if s.cu is None else s.lens + s.cu[1:] - s.cu[:-1])
    return _rotate(s.q.float(), cos, sin, case["interleaved"]).to(s.q.dtype)


def _count(table, pages):
    """How many entries of the table hold each page."""
    n = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    return n.scatter_add_(0, torch.where(table < 0, pages, table).long().view(-1), torch.ones_like(table).view(-1))[:pages]


def _fork(s):
    col, row = torch.arange(s.table.shape[1], device="cuda"), torch.arange(s.table.shape[0], device="cuda")
    p, page = s.parents.long(), s.case["page"]
    stays = p == row
    from_p = p.clamp_min(0)
    held = torch.where(stays, s.held, torch.where(p < 0, 0, torch.minimum(s.held[from_p], (s.lens[from_p] + page - 1) // page)))
    s.table.copy_(torch.where(col < held[:, None], s.table[from_p], -1))
    s.held.copy_(held)
    s.new_lens.copy_(torch.where(p < 0, 0, s.lens[from_p]))
    s.refs.copy_(_count(s.table, s.refs.shape[0]))
    s.free.copy_((s.refs == 0).sum())


def _reserve(s, lens, new):
    page, (B, W), pages = s.case["page"], s.table.shape, s.refs.shape[0]
    col, row = torch.arange(W, device="cuda"), torch.arange(B, device="cuda")
    c0, part, c1 = lens // page, lens % page, ((lens + new + page - 1) // page).clamp_max(W)
    keep = torch.minimum(s.held, c1)
    table = torch.where(col < keep[:, None], s.table, -1)
    refs = _count(table, pages)
    shared = (table >= 0) & (refs[table.clamp_min(0).long()] > 1)
    behind = shared & (col >= (c0 + (part > 0))[:, None])                    # shared pages without tokens of this sequence
    at = c0.long().clamp_max(W - 1)
    want = torch.where((new > 0) & (part > 0) & (c0 < keep), table[row, at], -1).long()
    there = torch.where(want < 0, pages, want)
    wants = torch.zeros(pages + 1, dtype=torch.int32, device="cuda").scatter_add_(0, there, torch.ones_like(lens))
    first = torch.full((pages + 1,), B, device="cuda").scatter_reduce_(0, there, row, "amin")
    holders = refs[want.clamp_min(0)]
    copied = (want >= 0) & (holders > 1) & ~((wants[there] == holders) & (first[there] == row))
    fresh = behind | ((col == c0[:, None]) & copied[:, None]) | ((col >= keep[:, None]) & (col < c1[:, None]))
    rank = fresh.view(-1).cumsum(0).view(B, W)
    okay = rank[-1, -1] <= (refs == 0).sum()
    fresh &= okay
    ids = torch.argsort((refs > 0).byte(), stable=True)                      # free pages first, ascending
    s.table.copy_(torch.where(fresh, ids[(rank - 1).clamp(0, pages - 1)].int(), table))
    s.held.copy_(torch.where(okay, torch.maximum(keep, c1), keep))
    s.refs.copy_(_count(s.table, pages))
    s.free.copy_((s.refs == 0).sum())
    rows = (copied & okay).nonzero()[:, 0]
    src, dst = want[rows], s.table[rows, at[rows]].long()
    moved = (torch.arange(page, device="cuda") < part[rows, None])[:, None, :, None]
    s.pool[:, :, dst] = torch.where(moved, s.pool[:, :, src], s.pool[:, :, dst])


def _compact(s):
    pages = s.refs.shape[0]
    live = s.refs > 0
    low = torch.arange(pages, device="cuda") < live.sum()
    dst, src = (~live & low).nonzero()[:, 0], (live & ~low).nonzero()[:, 0]
    s.pool[:, :, dst] = s.pool[:, :, src]
    s.refs[dst] = s.refs[src]
    s.refs[src] = 0
    to = torch.arange(pages, device="cuda")
    to[src] = dst
    s.table.copy_(torch.where(s.table < 0, -1, to[s.table.clamp_min(0).long()].int()))


def _verify(s):
    T, V = s.target.shape
    B, most = s.lens.shape[0], s.most
    cu = s.cu.long()
    n = cu[1:] - cu[:-1] - 1                                                 # drafts
    i = torch.arange(most, device="cuda")
    row = (cu[:-1, None] + i).clamp_max(T - 1)                               # [B, most]
    is_draft = i < n[:, None]
    x = torch.where(is_draft, s.tokens.long()[(row + 1).clamp_max(T - 1)], 0)
    if s.uniform is None:
        z = s.target.float()
        best = torch.where(z == z.amax(1, keepdim=True), torch.arange(V, device="cuda"), V).amin(1)
        ok = best[row] == x
    else:
        ok = s.target[row, x].double() > s.uniform.double()[row] * s.draft[row, x].double()
    accepted = (ok & is_draft).int().cumprod(1).sum(1)
    end = cu[:-1] + accepted
    if s.uniform is None:
        token = best[end]
    else:
        p = s.target[end].double()
        cum = torch.where((accepted < n)[:, None], (p - s.draft[end].double()).clamp_min(0.0), p).cumsum(1)
        token = torch.searchsorted(cum, s.uniform.double()[cu[1:] - 1, None] * cum[:, -1:], right=True)[:, 0].clamp_max(V - 1)
    out = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), torch.arange(T, device="cuda"), right=True)
    j = torch.arange(T, device="cuda") - cu[seq]
    after = s.tokens[(torch.arange(T, device="cuda") + 1).clamp_max(T - 1)]
    out = torch.where(j < accepted[seq], after, torch.where(j == accepted[seq], token[seq].int(), out))
    s.new_lens.copy_(s.lens + accepted + 1)
    return out, accepted.int()


# ---- the definitions, in 64 bits and by ordinary lists -----------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "axes":
        return _exact_axes(case, s)
    if case["op"] == "verify":
        return _exact_verify(case, s)
    P = _Pages(case, s)
    if case["op"] == "beams":
        P.fork(s.parents.tolist())
        P.reserve(P.lens, [1] * len(P.lens))
        return {"table": P.out_table(), "refs": _ints(P.refs()), "held": _ints([len(r) for r in P.rows]), "free": _ints([P.refs().count(0)]),
                "lens": _ints(P.lens), "cache": P.cache}
    if case["op"] == "room":
        for lens, new in s.steps:
            P.reserve(lens.tolist(), new.tolist())
        return {"table": P.out_table(), "refs": _ints(P.refs()), "held": _ints([len(r) for r in P.rows]), "free": _ints([P.refs().count(0)])}
    P.compact()
    return {"table": P.out_table(), "refs": _ints(P.refs()), "cache": P.cache}


class _Pages:
    """The pool as lists: a row is the list of its pages, and a page's holders are counted when they are asked for."""

    def __init__(self, case, s):
        self.page, self.pages, self.width = case["page"], _pages(case), s.table.shape[1]
        self.rows = [r[:h] for r, h in zip(s.table.tolist(), s.held.tolist())]
        self.lens = s.lens.tolist() if hasattr(s, "lens") else None
        self.cache = s.pool.double() if case["op"] != "room" else None

    def refs(self):
        n = [0] * self.pages
        for r in self.rows:
            for p in r:
                n[p] += 1
        return n

    def out_table(self):
        return _ints([r + [-1] * (self.width - len(r)) for r in self.rows])

    def fork(self, parents):
        rows, lens = self.rows, self.lens
        self.rows = [rows[b] if p == b else rows[p][:-(-lens[p] // self.page)] for b, p in enumerate(parents)]
        self.lens = [lens[p] for p in parents]

    def reserve(self, lens, new):
        page = self.page
        for b, r in enumerate(self.rows):
            self.rows[b] = r[:-(-(lens[b] + new[b]) // page)]
        n = self.refs()
        writers = {}
        for b, r in enumerate(self.rows):
            if new[b] > 0 and lens[b] % page and lens[b] // page < len(r):
                writers.setdefault(r[lens[b] // page], []).append(b)
        free = iter([p for p in range(self.pages) if n[p] == 0])
        for b, r in enumerate(self.rows):
            first = lens[b] // page
            out = r[:first]
            for c in range(first, -(-(lens[b] + new[b]) // page)):
                used = lens[b] % page if c == first else 0
                if c < len(r) and (n[r[c]] == 1 or used and (not new[b] or writers[r[c]][0] == b and len(writers[r[c]]) == n[r[c]])):
                    out.append(r[c])
                    continue
                p = next(free)
                if used and c < len(r) and self.cache is not None:
                    self.cache[:, :, p, :, :used] = self.cache[:, :, r[c], :, :used]
                out.append(p)
            self.rows[b] = out

    def compact(self):
        n = self.refs()
        live = [p for p in range(self.pages) if n[p]]
        gaps = [p for p in range(len(live)) if n[p] == 0]
        to = dict(zip([p for p in live if p >= len(live)], gaps))
        for p, d in to.items():
            self.cache[:, :, d] = self.cache[:, :, p]
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]


def _exact_axes(case, s):
    page, B, n = case["page"], case["batch"], case["rot"] // 2
    table, lens = s.table.tolist(), s.lens.tolist()
    cu = list(range(B + 1)) if s.cu is None else s.cu.tolist()
    pos = s.positions.double()
    angle = torch.stack([pos[a] * f for a, f in zip(s.axis_of.tolist(), s.inv_freq.double())], 1)
    z = torch.polar(torch.ones_like(angle), angle)[:, None]
    turned = []
    for x in (s.k.double(), s.q.double()):
        part, rest = x[..., :2 * n], x[..., 2 * n:]
        if case["interleaved"]:
            y = torch.view_as_real(torch.view_as_complex(part.unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2)
        else:
            y = torch.complex(part[..., :n].contiguous(), part[..., n:].contiguous()) * z
            y = torch.cat((y.real, y.imag), -1)
        turned.append(torch.cat((y, rest), -1))
    cache = s.pool.double()
    for b in range(B):
        t = list(range(cu[b], cu[b + 1]))
        where = torch.tensor([[table[b][(lens[b] + j) // page], (lens[b] + j) % page] for j in range(len(t))], device="cuda")
        cache[0, 0][where[:, 0], :, where[:, 1]] = turned[0][t[0]:t[-1] + 1]
        cache[0, 1][where[:, 0], :, where[:, 1]] = s.v[t[0]:t[-1] + 1].double()
    return {"q": turned[1], "cache": cache, "lens": None}


def _exact_verify(case, s):
    cu, drafted, lens = s.cu.tolist(), s.tokens.tolist(), s.lens.tolist()
    out, accepted, after = [-1] * cu[-1], [], []
    u = None if s.uniform is None else s.uniform.double().tolist()
    for b in range(case["batch"]):
        first, n = cu[b], cu[b + 1] - cu[b] - 1
        target = s.target[first:first + n + 1].double().cpu().numpy()
        if u is None:
            best = [int(np.flatnonzero(z == z.max())[0]) for z in target]
            a = next((i for i in range(n) if best[i] != drafted[first + 1 + i]), n)
            token = best[a]
        else:
            draft = s.draft[first:first + n].double().cpu().numpy()
            x = drafted[first + 1:first + 1 + n]
            a = next((i for i in range(n) if not target[i][x[i]] > u[first + i] * draft[i][x[i]]), n)
            weight = target[a] if a == n else np.maximum(target[a] - draft[a], 0.0)
            token = int(np.flatnonzero(np.cumsum(weight) > u[first + n] * math.fsum(weight))[0])
        out[first:first + a + 1] = drafted[first + 1:first + 1 + a] + [token]
        accepted.append(a)
        after.append(lens[b] + a + 1)
    return {"tokens": _ints(out), "accepted": _ints(accepted), "lens": _ints(after)}
