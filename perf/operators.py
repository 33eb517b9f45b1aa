"""Operators of a paged key/value cache, as a serving program that routes with this library uses them.

append   the new tokens' keys and values go into the pages of their sequences, keys (and the queries of the same tokens)
         rotated by their positions on the way
shared   attention of a batch whose sequences begin with the same long prefix: the prefix's pages are read once for all
         sequences, each sequence's own pages for itself
ranges   attention over the token ranges that the routing layers write, the tokens read through the page table

Each operator has a plain form here (elementary torch operations, 32 bits, 64 for the angles of the rotation) and the
calls that a user of the library makes.  `exact` computes the same from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------------------
def listed():
    return [
        # a decoding step of 64 sequences: one token each, a few hundred kilobytes, latency
        dict(name="append_step", op="append", dtype="bf16", batch=64, heads=32, kv_heads=8, dh=128, rot=128, interleaved=False,
             page=16, new=1, ctx=2000, ragged=False),
        # prompts of unlike lengths that enter the cache together
        dict(name="append_prompts", op="append", dtype="bf16", batch=13, heads=32, kv_heads=8, dh=128, rot=128, interleaved=False,
             page=64, new=2500, ctx=900, ragged=True),
        # fp32, pairs side by side, half of the head's width rotated, odd page size and counts
        dict(name="append_f32_pairs", op="append", dtype="f32", batch=5, heads=6, kv_heads=3, dh=64, rot=32, interleaved=True,
             page=24, new=700, ctx=333, ragged=True),
        # one interactive sequence's neighbours: four short continuations of one system prompt
        dict(name="shared_small", op="shared", dtype="bf16", batch=4, heads=8, kv_heads=8, dh=64, page=16, prefix=2048, own=200,
             new=1, ragged=True),
        # a decoding step of 64 sequences behind a prefix of 32768 tokens
        dict(name="shared_step", op="shared", dtype="bf16", batch=64, heads=32, kv_heads=8, dh=128, page=64, prefix=32768, own=2000,
             new=1, ragged=True),
        # the sequences' own prompts, read into the cache, attend to the prefix and causally to themselves
        dict(name="shared_prompts", op="shared", dtype="bf16", batch=8, heads=32, kv_heads=8, dh=128, page=32, prefix=8197, own=512,
             new=512, ragged=True),
        # fp32 arithmetic, sizes off every tile
        dict(name="shared_f32", op="shared", dtype="f32", batch=11, heads=8, kv_heads=4, dh=64, page=16, prefix=4001, own=300,
             new=3, ragged=True),
        # one sequence's decoding step: every route row is one group of four heads, 12 chunks of 64 tokens
        dict(name="ranges_one", op="ranges", dtype="bf16", batch=1, heads=32, kv_heads=8, route_heads=8, dh=128, page=64, chunk=64,
             k=12, n_q=1, m=1, ctx=16384, causal=False, coalesce=False),
        # the decoding step of a batch, each head with its own route of 64 chunks
        dict(name="ranges_step", op="ranges", dtype="bf16", batch=16, heads=32, kv_heads=8, route_heads=32, dh=128, page=16, chunk=64,
             k=64, n_q=1, m=1, ctx=32768, causal=False, coalesce=True),
        # a prompt of 128 query chunks of 64 tokens, 32 selected chunks each, causal inside the chunk
        dict(name="ranges_prompt", op="ranges", dtype="bf16", batch=2, heads=32, kv_heads=8, route_heads=8, dh=128, page=64, chunk=64,
             k=32, n_q=128, m=64, ctx=8192, causal=True, coalesce=False),
        # fp32, one query per row, ranges cut by the sequence's end
        dict(name="ranges_f32", op="ranges", dtype="f32", batch=2, heads=8, kv_heads=8, route_heads=8, dh=64, page=48, chunk=33,
             k=12, n_q=128, m=1, ctx=4100, causal=False, coalesce=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_one(rng):
    op = rng.choice(("append", "shared", "shared", "ranges", "ranges"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    kv = rng.choice((1, 2, 3, 4, 8))
    dh = rng.choice((64, 128)) if dtype == "bf16" else rng.choice((32, 64, 80, 128))
    group = rng.choice((1, 2, 4, 5, 7, 8))
    page = rng.choice((8, 16, 24, 32, 64, 128))
    if op == "append":
        new = _log(rng, 1, 2500)
        return dict(op=op, dtype=dtype, batch=_log(rng, 1, 200), heads=kv * group, kv_heads=kv, dh=dh, rot=rng.choice((dh, dh // 2)),
                    interleaved=rng.random() < 0.4, page=page, new=new, ctx=_log(rng, 1, 2000), ragged=new > 1)
    if op == "shared":
        new = rng.choice((1, 1, 1, 2, 5, _log(rng, 6, 512)))
        return dict(op=op, dtype=dtype, batch=_log(rng, 1, 128), heads=kv * group, kv_heads=kv, dh=dh, page=page,
                    prefix=_log(rng, 100, 32768), own=max(new, _log(rng, 1, 2000)), new=new, ragged=True)
    n_q, m = rng.choice(((1, 1), (1, 1), (_log(rng, 2, 128), 1), (_log(rng, 2, 128), rng.choice((16, 33, 64)))))
    chunk = rng.choice((16, 33, 64)) if m == 1 else m
    chunks = n_q if m > 1 else max(n_q, _log(rng, 4, 512))
    return dict(op=op, dtype=dtype, batch=_log(rng, 1, 16), heads=kv * group, kv_heads=kv, route_heads=rng.choice((kv, kv * group)), dh=dh,
                page=page, chunk=chunk, k=min(chunks, _log(rng, 1, 64)), n_q=n_q, m=m, ctx=chunks * chunk, causal=m > 1,
                coalesce=rng.random() < 0.5)


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        for key in ("bytes", "flops"):
            for d in ("bf16", "f32"):
                if c["dtype"] == d:
                    top[c["op"], d, key] = max(top.get((c["op"], d, key), 0), w[key])
    while True:
        c = _draw_one(rng)
        w = work(c)
        if all(w[key] <= top[c["op"], c["dtype"], key] for key in ("bytes", "flops")):
            return c


def _lens(case):
    """Tokens per sequence: {"before", "new"} of append, {"own", "new"} of shared, {"ctx"} of ranges; they are part of the case."""
    rng = random.Random("%s %d %d" % (case["op"], case["batch"], case["dh"]))
    B = case["batch"]
    if case["op"] == "append":
        return ([rng.randint(0, case["ctx"]) for _ in range(B)],
                [rng.randint(1, case["new"]) if case["ragged"] else case["new"] for _ in range(B)])
    if case["op"] == "shared":
        new = [rng.randint((case["new"] + 1) // 2, case["new"]) for _ in range(B)]
        return [max(n, rng.randint(1, case["own"])) for n in new], new
    if case["m"] > 1:
        return [case["ctx"]] * B, None
    return [rng.randint(max(1, case["ctx"] * 7 // 8), case["ctx"]) for _ in range(B)], None


# ---- work -----------------------------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    H, KH, dh, B = case["heads"], case["kv_heads"], case["dh"], case["batch"]
    a, new = _lens(case)
    if case["op"] == "append":
        T = sum(new)
        return {"bytes": T * dh * e * 2 * (H + 2 * KH), "flops": 3 * T * case["rot"] * (H + KH)}
    if case["op"] == "shared":
        P, T = case["prefix"], sum(new)
        seen = sum(n * (P + o - n) + n * (n + 1) // 2 for o, n in zip(a, new))
        return {"bytes": (P + sum(a)) * KH * dh * 2 * e + T * H * dh * 2 * e, "flops": 4 * H * dh * seen}
    RH, n_q, m, k, c = case["route_heads"], case["n_q"], case["m"], case["k"], case["chunk"]
    chunks = -(-case["ctx"] // c)
    visible = [min(k, i + 1) if case["causal"] else min(k, chunks) for i in range(n_q)]
    tokens = sum(visible) * c
    if case["causal"]:
        seen, touched = tokens * m - n_q * m * (m - 1) // 2, chunks * c
    else:
        seen, touched = tokens * m, c * chunks * (1 - (1 - min(1, k / chunks)) ** (n_q * RH // KH))
    return {"bytes": int(B * KH * touched) * dh * 2 * e + B * H * n_q * m * dh * 2 * e + B * RH * n_q * k * 8, "flops": 4 * B * H * dh * seen}


# ---- inputs ---------------------------------------------------------------------------------------------------
class _State:
    pass


def _randn(g, shape, dt, scale=1.0):
    return torch.empty(shape, device="cuda", dtype=dt).normal_(0.0, scale, generator=g)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev, dt, s = "cuda", _DT[case["dtype"]], _State()
    s.case = case
    B, H, KH, dh, page = case["batch"], case["heads"], case["kv_heads"], case["dh"], case["page"]
    a, new = _lens(case)
    if case["op"] == "append":
        total = [x + n for x, n in zip(a, new)]
        shared_pages = 0
    elif case["op"] == "shared":
        total = [case["prefix"] + x for x in a]
        shared_pages = case["prefix"] // page            # whole pages of the prefix are the same memory in every table
    else:
        total, shared_pages = a, 0
    width = max(-(-t // page) for t in total)
    # a sequence holds its own pages behind the shared ones, scattered over the pool; the rest of its table is 0
    need = torch.tensor([-(-t // page) - shared_pages for t in total], device=dev)
    pages = shared_pages + int(sum(-(-t // page) - shared_pages for t in total))
    perm = torch.randperm(pages, generator=g, device=dev).int()
    table = torch.zeros((B, width), dtype=torch.int32, device=dev)
    table[:, :shared_pages] = perm[:shared_pages]
    col = torch.arange(width - shared_pages, device=dev)
    first = shared_pages + torch.cumsum(need, 0) - need
    mine = col < need[:, None]
    table[:, shared_pages:][mine] = perm[(first[:, None] + col)[mine]]
    s.table = table
    s.k_cache = _randn(g, (pages, KH, page, dh), dt)
    s.v_cache = _randn(g, (pages, KH, page, dh), dt)
    s.scale = dh ** -0.5
    if case["op"] == "append":
        T = sum(new)
        s.lens = torch.tensor(a, dtype=torch.int32, device=dev)
        s.new_lens = torch.zeros_like(s.lens)
        s.cu = None if case["new"] == 1 else torch.tensor([0] + new, dtype=torch.int32, device=dev).cumsum(0).int()
        # the projections' output, as one matrix: queries, keys and values of a token side by side
        qkv = _randn(g, (T, (H + 2 * KH) * dh), dt)
        s.q = qkv[:, :H * dh].view(T, H, dh)
        s.k = qkv[:, H * dh:(H + KH) * dh].view(T, KH, dh)
        s.v = qkv[:, (H + KH) * dh:].view(T, KH, dh)
        s.inv_freq = (10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=dev) / case["rot"])).float()
    elif case["op"] == "shared":
        T = sum(new)
        s.lens = torch.tensor(total, dtype=torch.int32, device=dev)
        s.cu = None if case["new"] == 1 else torch.tensor([0] + new, dtype=torch.int32, device=dev).cumsum(0).int()
        s.max_new, s.max_own = max(new), max(a)
        s.q = _randn(g, (T, H, dh), dt, 1.5)
        _share(s, case, page, B)
    else:
        RH, n_q, m, k, c = case["route_heads"], case["n_q"], case["m"], case["k"], case["chunk"]
        s.lens = torch.tensor(a, dtype=torch.int32, device=dev)
        s.q = _randn(g, (B, H, n_q * m, dh), dt, 1.5)
        chunks = -(-case["ctx"] // c)
        score = torch.rand((B * RH, n_q, chunks), generator=g, device=dev)
        i, j = torch.arange(n_q, device=dev)[:, None], torch.arange(chunks, device=dev)
        if case["causal"]:
            score = torch.where(j > i, -1.0, torch.where(j == i, 2.0, score))      # a chunk selects itself, and none behind it
        val, ids = score.view(B * RH * n_q, chunks).topk(k, dim=1)
        ids = torch.where(val < 0, chunks, ids).sort(1).values
        lo, hi = ids * c, ids * c + c
        if case["coalesce"]:
            start = torch.ones_like(ids, dtype=torch.bool)
            start[:, 1:] = ids[:, 1:] != ids[:, :-1] + 1
            run = start.cumsum(1) - 1
            lo = torch.full_like(lo, 1 << 40).scatter_reduce_(1, run, lo, "amin")
            hi = torch.full_like(hi, -1).scatter_reduce_(1, run, hi, "amax")
        gone = (lo >= chunks * c) | (hi < 0)
        s.ranges = torch.stack((torch.where(gone, -1, lo), torch.where(gone, -1, hi)), -1).int().contiguous()
        s.max_tokens = k * c
    if own:
        from paper_2609_07306_b200.paged import PagedKV
        s.kv = PagedKV(s.k_cache, s.v_cache, s.table)
    return s


def _share(s, case, page, B):
    """The tokens of a prefix that ends inside a page stand in every sequence's own page: each holds a copy of them."""
    tail = case["prefix"] % page
    if tail:
        col = case["prefix"] // page
        for c in (s.k_cache, s.v_cache):
            c[s.table[:, col].long(), :, :tail] = c[s.table[0, col].long(), :, :tail].clone()


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    case = s.case
    if case["op"] == "append":
        if own:
            q = s.kv.append(s.k, s.v, s.lens, cu=s.cu, q=s.q, inv_freq=s.inv_freq, interleaved=case["interleaved"], new_lens=s.new_lens)
        else:
            q = _append(s, case)
        return {"q": q, "k_cache": s.k_cache, "v_cache": s.v_cache, "lens": s.new_lens}
    if case["op"] == "shared":
        if own:
            return s.kv.attend_shared(s.q, s.lens, case["prefix"], s.scale, cu=s.cu)
        return _shared(s, case)
    if own:
        return s.kv.attend_ranges(s.q, s.ranges, s.lens, case["n_q"], s.scale, causal=case["causal"])
    return _ranges(s, case)


def _seq(cu, T, B):
    """(sequence, place in it) of each new token."""
    t = torch.arange(T, device="cuda")
    if cu is None:
        return t, torch.zeros_like(t)
    b = torch.searchsorted(cu[1:].long().contiguous(), t, right=True)
    return b, t - cu.long()[b]


def _rotate(x, cos, sin, interleaved):
    """x [T, heads, dh] in 32 bits; the first 2 * cos.shape[1] entries of a head are rotated."""
    n = cos.shape[1]
    cos, sin, y = cos[:, None], sin[:, None], x.clone()
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _append(s, case):
    T, page = s.k.shape[0], case["page"]
    b, i = _seq(s.cu, T, case["batch"])
    pos = s.lens.long()[b] + i
    angle = pos.double()[:, None] * s.inv_freq.double()
    cos, sin = angle.cos().float(), angle.sin().float()
    at = s.table.long()[b, pos // page]
    s.k_cache[at, :, pos % page] = _rotate(s.k.float(), cos, sin, case["interleaved"]).to(s.k.dtype)
    s.v_cache[at, :, pos % page] = s.v
    s.new_lens.copy_(s.lens + 1 if s.cu is None else s.lens + s.cu[1:] - s.cu[:-1])
    return _rotate(s.q.float(), cos, sin, case["interleaved"]).to(s.q.dtype)


def _weights(x):
    """softmax over the last axis; all zero where everything is masked."""
    top = x.amax(-1, keepdim=True)
    w = (x - torch.where(top.isneginf(), 0.0, top)).exp_()
    return w / w.sum(-1, keepdim=True).clamp_min(1e-38)


def _shared(s, case):
    T, H, dh = s.q.shape
    B, KH, P, page = case["batch"], case["kv_heads"], case["prefix"], case["page"]
    b, i = _seq(s.cu, T, B)
    n = torch.ones_like(s.lens) if s.cu is None else s.cu[1:] - s.cu[:-1]
    limit = (s.lens - n).long()[b] + i + 1                               # tokens before this one are seen
    q = s.q.float().view(T, KH, H // KH, dh)
    tp = torch.arange(P, device="cuda")
    at = s.table[0].long()[tp // page]
    kp, vp = s.k_cache[at, :, tp % page].float(), s.v_cache[at, :, tp % page].float()          # [P, KH, dh]
    ts = P + torch.arange(s.max_own, device="cuda")
    at = s.table.long()[:, (ts // page).clamp_max(s.table.shape[1] - 1)]
    there = (ts < s.lens[:, None])[:, :, None, None]
    ks = torch.where(there, s.k_cache[at, :, ts % page].float(), 0.0)                           # [B, own, KH, dh]
    vs = torch.where(there, s.v_cache[at, :, ts % page].float(), 0.0)
    pad = torch.zeros((B, s.max_new, KH, H // KH, dh), device="cuda")
    pad[b, i] = q
    x = torch.cat((torch.einsum("thgd,phd->thgp", q, kp), torch.einsum("bnhgd,bshd->bnhgs", pad, ks)[b, i]), -1) * s.scale
    t = torch.cat((tp, ts))
    x = torch.where((t < limit[:, None])[:, None, None], x, -math.inf)
    w = _weights(x)
    pad = torch.zeros((B, s.max_new, KH, H // KH, s.max_own), device="cuda")
    pad[b, i] = w[..., P:]
    out = torch.einsum("thgp,phd->thgd", w[..., :P], vp) + torch.einsum("bnhgs,bshd->bnhgd", pad, vs)[b, i]
    return out.reshape(T, H, dh).to(s.q.dtype)


def _ranges(s, case):
    B, H, Q, dh = s.q.shape
    KH, RH, n_q, m, page = case["kv_heads"], case["route_heads"], case["n_q"], case["m"], case["page"]
    rows = s.ranges.shape[0]
    lo = s.ranges[..., 0].long()
    size = torch.where(lo < 0, 0, s.ranges[..., 1].long() - lo)
    end = size.cumsum(1)
    j = torch.arange(s.max_tokens, device="cuda")
    slot = torch.searchsorted(end, j.expand(rows, -1).contiguous(), right=True).clamp_max(lo.shape[1] - 1)
    tok = lo.gather(1, slot) + j - (end - size).gather(1, slot)
    row = torch.arange(rows, device="cuda")
    b, h = row // (RH * n_q), row // n_q % RH // (RH // KH)
    there = (j < end[:, -1:]) & (tok < s.lens.long()[b, None])
    tok = torch.where(there, tok, 0)
    at = s.table.long()[b[:, None], tok // page]
    k = torch.where(there[..., None], s.k_cache[at, h[:, None], tok % page].float(), 0.0)      # [rows, tokens, dh]
    v = torch.where(there[..., None], s.v_cache[at, h[:, None], tok % page].float(), 0.0)
    G = H // RH
    q = s.q.float().view(B, RH, G, n_q, m, dh).permute(0, 1, 3, 4, 2, 5).reshape(rows, m, G, dh)
    x = torch.einsum("rmgd,rtd->rmgt", q, k) * s.scale
    seen = there[:, None].expand(rows, m, -1)
    if case["causal"]:
        pos = s.lens.long()[b, None] - Q + (row % n_q)[:, None] * m + torch.arange(m, device="cuda")
        seen = seen & (tok[:, None] <= pos[..., None])
    w = _weights(torch.where(seen[:, :, None], x, -math.inf))
    out = torch.einsum("rmgt,rtd->rmgd", w, v)
    return out.view(B, RH, n_q, m, G, dh).permute(0, 1, 4, 2, 3, 5).reshape(B, H, Q, dh).to(s.q.dtype)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------
def _softmax_rows(q, k, v, seen, scale):
    """q [n, dh], k, v [t, dh], seen [n, t] -> [n, dh]; zero where a query sees nothing."""
    z = (q @ k.T) * scale
    z[~seen] = -math.inf
    p = torch.softmax(z, 1)
    p[~seen.any(1)] = 0.0
    return p @ v


def exact(case, seed):
    s = prepare(case, seed)
    page, B, H, KH, dh = case["page"], case["batch"], case["heads"], case["kv_heads"], case["dh"]
    table, lens = s.table.tolist(), s.lens.tolist()
    if case["op"] == "append":
        cu = list(range(B + 1)) if s.cu is None else s.cu.tolist()
        kc, vc = s.k_cache.double(), s.v_cache.double()
        q = s.q.double()
        new = []
        for b in range(B):
            n = cu[b + 1] - cu[b]
            new.append(lens[b] + n)
            p = torch.arange(lens[b], lens[b] + n, device="cuda", dtype=torch.float64)
            a = torch.outer(p, s.inv_freq.double())
            z = torch.polar(torch.ones_like(a), a)[:, None]
            turned = []
            for x in (s.k[cu[b]:cu[b + 1]].double(), s.q[cu[b]:cu[b + 1]].double()):
                part, rest = x[..., :case["rot"]], x[..., case["rot"]:]
                if case["interleaved"]:
                    y = torch.view_as_real(torch.view_as_complex(part.unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2)
                else:
                    y = torch.complex(part[..., :case["rot"] // 2], part[..., case["rot"] // 2:]) * z
                    y = torch.cat((y.real, y.imag), -1)
                turned.append(torch.cat((y, rest), -1))
            q[cu[b]:cu[b + 1]] = turned[1]
            where = torch.tensor([[table[b][(lens[b] + j) // page], (lens[b] + j) % page] for j in range(n)], device="cuda")
            kc[where[:, 0], :, where[:, 1]] = turned[0]
            vc[where[:, 0], :, where[:, 1]] = s.v[cu[b]:cu[b + 1]].double()
        return {"q": q, "k_cache": kc, "v_cache": vc, "lens": None}
    if case["op"] == "shared":
        cu = list(range(B + 1)) if s.cu is None else s.cu.tolist()
        out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
        G = H // KH
        for b in range(B):
            used = s.table[b, :-(-lens[b] // page)].long()
            k = s.k_cache[used].double().permute(1, 0, 2, 3).reshape(KH, -1, dh)[:, :lens[b]]
            v = s.v_cache[used].double().permute(1, 0, 2, 3).reshape(KH, -1, dh)[:, :lens[b]]
            n = cu[b + 1] - cu[b]
            seen = torch.arange(lens[b], device="cuda") <= torch.arange(lens[b] - n, lens[b], device="cuda")[:, None]
            for h in range(H):
                out[cu[b]:cu[b + 1], h] = _softmax_rows(s.q[cu[b]:cu[b + 1], h].double(), k[h // G], v[h // G], seen, s.scale)
        return out
    RH, n_q, m = case["route_heads"], case["n_q"], case["m"]
    if B * RH * n_q > 8192:
        return None
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    ranges = s.ranges.tolist()
    G, Q = H // RH, n_q * m
    for b in range(B):
        used = s.table[b, :-(-lens[b] // page)].long()
        k = s.k_cache[used].permute(1, 0, 2, 3).reshape(KH, -1, dh)
        v = s.v_cache[used].permute(1, 0, 2, 3).reshape(KH, -1, dh)
        for h in range(RH):
            for i in range(n_q):
                ids = [t for lo, hi in ranges[(b * RH + h) * n_q + i] if lo >= 0 for t in range(lo, min(hi, lens[b]))]
                tok = torch.tensor(ids, device="cuda", dtype=torch.long)
                kk, vv = k[h * KH // RH, tok].double(), v[h * KH // RH, tok].double()
                q = s.q[b, h * G:(h + 1) * G, i * m:(i + 1) * m].double().reshape(G * m, dh)
                seen = torch.ones((m, len(ids)), dtype=torch.bool, device="cuda")
                if case["causal"]:
                    seen = tok <= lens[b] - Q + i * m + torch.arange(m, device="cuda")[:, None]
                out[b, h * G:(h + 1) * G, i * m:(i + 1) * m] = _softmax_rows(q, kk, vv, seen.repeat(G, 1), s.scale).view(G, m, dh)
    return out
