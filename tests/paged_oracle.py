"""Plain 64-bit forms of the paged cache's operators, token by token from their definitions, and how far FP32 arithmetic may
be from them.

Bounds (u = 2^-24, half a step of FP32; a bf16 rounding is off by half a step, 2^-8):
  logit    a dot product of dh terms and two products: |dx| <= (dh + 4) u * scale * sum_e |q_e k_e|
  weight   2^(x log2 e - m): relative error |dx| plus |x| * 2 u of the argument's rounding and 4 u of the function
  output   sum_j w_j v_j / sum_j w_j over n tokens: each side's relative weight error, (n + 8) u of each sum; in all
           |do| <= (2 * weight error + 2 (n + 8) u) * A,  A = sum_j w_j |v_j|
  bf16     the weights are rounded to bf16 before the product with the values: 2^-8 A more; the result once: 2^-8 |o|.
           The tensor cores' FP32 sums may cut instead of round: twice the u of the dot product's terms.
"""
import torch

U = 2.0 ** -24
BF = 2.0 ** -8


def place(table, page, b, tok):
    return int(table[b, tok // page]), tok % page


def rows(cache, table_row, page, toks):
    """[n, kv_heads, dh] of the listed tokens, on the CPU in 64 bits."""
    t = torch.as_tensor(toks, dtype=torch.long)
    if t.numel() == 0:
        return torch.zeros((0, cache.shape[1], cache.shape[3]), dtype=torch.float64)
    return cache[table_row.long()[t // page], :, t % page].double()


def attend(q, k, v, scale, bf16):
    """One query [dh] over [n, dh]: (output, bound of its error)."""
    n, dh = k.shape
    if n == 0:
        z = torch.zeros(dh, dtype=torch.float64)
        return z, z
    x = (k @ q) * scale
    w = torch.softmax(x, 0)
    o, A = w @ v, w @ v.abs()
    finite = torch.where(x.isfinite(), x, 0.0)
    mag = torch.where(x.isfinite(), (k.abs() @ q.abs()) * abs(scale), 0.0).max()
    weight = (dh + 4) * (2 if bf16 else 1) * U * mag + finite.abs().max() * 2 * U + 4 * U
    bound = (2 * weight + 2 * (n + 8) * U) * A
    if bf16:
        bound = bound + BF * A + BF * o.abs()
    return o, bound + 1e-37


def shared(q, k_cache, v_cache, table, lens, cu, scale, causal):
    """Sequence by sequence (nothing shared): outputs and bounds [tokens, heads, dh]; padding rows are NaN."""
    q, k_cache, v_cache, table = q.cpu(), k_cache.cpu(), v_cache.cpu(), table.cpu()
    bf16 = q.dtype == torch.bfloat16
    T, H, dh = q.shape
    page, KH = k_cache.shape[2], k_cache.shape[1]
    out = torch.full((T, H, dh), float("nan"), dtype=torch.float64)
    bound = torch.zeros_like(out)
    for b in range(len(lens)):
        n = cu[b + 1] - cu[b]
        k, v = (rows(c, table[b], page, range(lens[b])) for c in (k_cache, v_cache))
        for i in range(n):
            see = max(0, lens[b] - n + i + 1) if causal else lens[b]
            for h in range(H):
                kh = h // (H // KH)
                out[cu[b] + i, h], bound[cu[b] + i, h] = attend(q[cu[b] + i, h].double(), k[:see, kh], v[:see, kh], scale, bf16)
    return out, bound


def ranged(q, k_cache, v_cache, table, lens, ranges, n_q, scale, causal):
    """Outputs and bounds [batch, heads, n_q * m, dh]."""
    q, k_cache, v_cache, table, ranges = q.cpu(), k_cache.cpu(), v_cache.cpu(), table.cpu(), ranges.cpu().tolist()
    bf16 = q.dtype == torch.bfloat16
    Bn, H, Q, dh = q.shape
    page, KH, m = k_cache.shape[2], k_cache.shape[1], Q // n_q
    RH = len(ranges) // (Bn * n_q)
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.zeros_like(out)
    for b in range(Bn):
        for r in range(RH):
            for i in range(n_q):
                toks = [t for lo, hi in ranges[(b * RH + r) * n_q + i] if lo >= 0 for t in range(lo, min(hi, lens[b]))]
                k, v = (rows(c, table[b], page, toks)[:, r // (RH // KH)] for c in (k_cache, v_cache))
                t = torch.as_tensor(toks, dtype=torch.long)
                for j in range(m):
                    pos = lens[b] - Q + i * m + j
                    sel = t <= pos if causal else torch.ones(len(toks), dtype=torch.bool)
                    for h in range(r * (H // RH), (r + 1) * (H // RH)):
                        out[b, h, i * m + j], bound[b, h, i * m + j] = attend(q[b, h, i * m + j].double(), k[sel], v[sel], scale, bf16)
    return out, bound


def assert_within(got, want, bound):
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan), f"NaN at {(got.isnan() != nan).nonzero()[:5].tolist()}"
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf])
    fine = ~(nan | inf)
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or over.max() <= 0, f"off by {(got - want).abs()[fine].max()} where {bound[fine].max()} is allowed; {int((over > 0).sum())} values"
