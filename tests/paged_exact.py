"""The paged cache's attention in 64 bits for many rows at once, on the GPU: the definitions and error bounds of paged_oracle (which goes
row by row on the CPU), as matrix products."""
import torch

from paged_oracle import BF, U


def attend_rows(q, k, v, seen, scale, bf16):
    """q [n, dh], k and v [t, dh], seen [n, t]: outputs and bounds [n, dh] in 64 bits; zeros where a row sees nothing.  Infinities and NaN
    among the values reach the rows that see them."""
    n, dh = q.shape
    if k.shape[0] == 0:
        z = torch.zeros((n, dh), dtype=torch.float64, device=q.device)
        return z, z
    q, k, v = q.double(), k.double(), v.double()
    x = (q @ k.T) * scale
    mag = ((q.abs() @ k.abs().T) * abs(scale)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
    top = x.abs().masked_fill(~seen, 0.0).amax(1, keepdim=True)
    w = torch.softmax(x.masked_fill(~seen, float("-inf")), 1).masked_fill(~seen, 0.0)
    w = torch.where(seen.any(1, keepdim=True), w, 0.0)
    fine = torch.where(v.isfinite(), v, 0.0)
    o, A = w @ fine, w @ fine.abs()
    s = seen.double()
    nan, up, down = (s @ c.double() > 0 for c in (v.isnan(), v == float("inf"), v == float("-inf")))
    count = s.sum(1, keepdim=True)
    weight = (dh + 4) * (2 if bf16 else 1) * U * mag + top * 2 * U + 4 * U
    bound = (2 * weight + 2 * (count + 8) * U) * A
    if bf16:
        bound = bound + BF * A + BF * o.abs()
    o = torch.where(up, float("inf"), torch.where(down, float("-inf"), o))
    return torch.where(nan | (up & down), float("nan"), o), bound + 1e-37


def tokens(cache, pages, n):
    """[n, kv_heads, dh]: the first n tokens of a page list."""
    t = torch.arange(n, device=cache.device)
    return cache[pages.long()[t // cache.shape[2]], :, t % cache.shape[2]]


def shared(q, k_cache, v_cache, table, lens, cu, scale, causal=True):
    """Each sequence by itself from its own row of the table: outputs and bounds [cu[-1], heads, dh], on the CPU."""
    H, dh, KH, dev = q.shape[1], q.shape[2], k_cache.shape[1], q.device
    out = torch.zeros((cu[-1], H, dh), dtype=torch.float64, device=dev)
    bound = torch.zeros_like(out)
    for b, L in enumerate(lens):
        n, G = cu[b + 1] - cu[b], H // KH
        if n == 0:
            continue
        limit = L - n + torch.arange(n, device=dev) + 1 if causal else torch.full((n,), L, device=dev)
        seen = (torch.arange(L, device=dev) < limit[:, None]).repeat_interleave(G, 0)
        k, v = (tokens(c, table[b], L) for c in (k_cache, v_cache))
        for h in range(KH):
            rows = q[cu[b]:cu[b + 1], h * G:(h + 1) * G].reshape(n * G, dh)
            o, e = attend_rows(rows, k[:, h], v[:, h], seen, scale, q.dtype == torch.bfloat16)
            out[cu[b]:cu[b + 1], h * G:(h + 1) * G] = o.view(n, G, dh)
            bound[cu[b]:cu[b + 1], h * G:(h + 1) * G] = e.view(n, G, dh)
    return out.cpu(), bound.cpu()


def ranged(q, k_cache, v_cache, table, lens, ranges, n_q, scale, causal=False):
    """Outputs and bounds [batch, heads, n_q * m, dh], on the CPU; ranges as a list of rows of (start, end)."""
    Bn, H, Q, dh = q.shape
    dev, KH, m = q.device, k_cache.shape[1], Q // n_q
    RH = len(ranges) // (Bn * n_q)
    G = H // RH
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    bound = torch.zeros_like(out)
    for b in range(Bn):
        if lens[b] == 0:
            continue
        k, v = (tokens(c, table[b], lens[b]) for c in (k_cache, v_cache))
        alike = {}                                     # rows of the same ranges and key head are one product
        for r in range(RH):
            for i in range(n_q):
                alike.setdefault((r * KH // RH, tuple(map(tuple, ranges[(b * RH + r) * n_q + i])), i if causal else 0), []).append((r, i))
        for (kh, spans, _), rows in alike.items():
            ids = [t for lo, hi in spans if lo >= 0 for t in range(lo, min(hi, lens[b]))]
            if not ids:
                continue
            tok = torch.tensor(ids, device=dev)
            x = torch.stack([q[b, r * G:(r + 1) * G, i * m:(i + 1) * m] for r, i in rows]).reshape(-1, dh)
            pos = torch.stack([lens[b] - Q + i * m + torch.arange(m, device=dev) for r, i in rows])[:, None].expand(-1, G, -1).reshape(-1)
            seen = tok <= pos[:, None] if causal else torch.ones((x.shape[0], len(ids)), dtype=torch.bool, device=dev)
            o, e = attend_rows(x, k[tok, kh], v[tok, kh], seen, scale, q.dtype == torch.bfloat16)
            for j, (r, i) in enumerate(rows):
                out[b, r * G:(r + 1) * G, i * m:(i + 1) * m] = o.view(len(rows), G, m, dh)[j]
                bound[b, r * G:(r + 1) * G, i * m:(i + 1) * m] = e.view(len(rows), G, m, dh)[j]
    return out.cpu(), bound.cpu()
