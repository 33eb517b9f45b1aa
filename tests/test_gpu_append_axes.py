"""Appending with positions of several axes, against the rotation in 64 bits: sections and turns of axes, both pairings, types, strides of the positions, far and
negative positions, padding, axes that there are not; and equal bits to the plain append where the positions are the places."""
import pytest
import torch

from paged_oracle import BF, U
from paper_2609_07306_b200 import binding as B
from paper_2609_07306_b200.paged import PagedKV, axis_sections, inv_freq

pytestmark = pytest.mark.gpu


def turned(x, pos, axis_of, freq, interleaved):
    """x [tokens, heads, dh] in 64 bits, and how far FP32 may be off: the angle is rounded to 2^-26 of a turn, sine and cosine are off by at most 2 steps, the two
    products and their sum by one rounding each; bf16 rounds the result once."""
    rot = 2 * freq.numel()
    y = x.double()
    a = pos.double()[axis_of.long()].T[:, None] * freq.double()
    i = torch.arange(rot // 2, device="cuda")
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    out, bound = y.clone(), torch.zeros_like(y)
    out[..., p] = y[..., p] * a.cos() - y[..., q] * a.sin()
    out[..., q] = y[..., q] * a.cos() + y[..., p] * a.sin()
    each = (y[..., p].abs() + y[..., q].abs()) * (6.2832 * 2.0 ** -26 + 6 * U)
    bound[..., p] = each
    bound[..., q] = each
    if x.dtype == torch.bfloat16:
        bound = bound + (out.abs() + bound) * BF
    return out, bound


def setup(dtype, KH, H, dh, page, news, lens, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = max((a + n + page - 1) // page for a, n in zip(lens, news)) + 1
    pages = len(news) * width
    kc, vc = (torch.randn((pages, KH, page, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.randperm(pages, generator=g, device="cuda").view(-1, width).int()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    T = sum(news) + pad
    q, k, v = (torch.randn((T, n, dh), generator=g, device="cuda").to(dtype) for n in (H, KH, KH))
    cu = torch.tensor([0] + news, device="cuda").cumsum(0).int()
    return g, PagedKV(kc, vc, table, status), q, k, v, cu, torch.tensor(lens, dtype=torch.int32, device="cuda")


def places(kv, cu, lens):
    """(page, place) of every new token."""
    out = []
    for b, n in enumerate((cu[1:] - cu[:-1]).tolist()):
        for i in range(n):
            p = lens[b].item() + i
            out.append((kv.page_table[b, p // kv.page_tokens].item(), p % kv.page_tokens))
    return torch.tensor(out, device="cuda").T


@pytest.mark.parametrize("dtype,dh,rot,interleaved,page,axes,sections", [
    (torch.bfloat16, 128, 128, False, 16, 3, (16, 24, 24)),
    (torch.bfloat16, 64, 32, True, 24, 2, None),
    (torch.bfloat16, 40, 20, False, 7, 3, (1, 8, 1)),          # 10 pairs: no 16-byte pieces
    (torch.float32, 64, 64, True, 16, 4, None),
    (torch.float32, 7, 6, False, 3, 3, (1, 1, 1)),
    (torch.float32, 256, 256, False, 5, 2, (100, 28)),
    (torch.bfloat16, 128, 64, False, 16, 1, None),
])
@pytest.mark.parametrize("strided", [False, True])
def test_rotation(dtype, dh, rot, interleaved, page, axes, sections, strided):
    news, lens = [3, 0, 1, 33, 2], [0, 5, page - 1, page, 3 * page + 1]
    g, kv, q, k, v, cu, L = setup(dtype, 2, 6, dh, page, news, lens, dh + axes, pad=4)
    T = q.shape[0]
    freq = inv_freq(rot)
    pos = torch.randint(-50, 100000, (axes, T), generator=g, device="cuda", dtype=torch.int32)
    if strided:                                                # [tokens, axes], as a program may hold them
        pos = torch.empty((T, axes + 2), dtype=torch.int32, device="cuda")[:, :axes].copy_(pos.T).T
    axis_of = axis_sections(sections) if sections else torch.arange(rot // 2, device="cuda").int() % axes
    out, nl = torch.full_like(q, 9.0), torch.zeros_like(L)
    before = kv.k_cache.clone(), kv.v_cache.clone()
    got = kv.append(k, v, L, cu=cu, q=q, q_out=out, inv_freq=freq, interleaved=interleaved, new_lens=nl, positions=pos,
                    axis_of=None if axes == 1 else axis_of)
    n = sum(news)
    assert got is out and kv.status.item() == 0 and nl.tolist() == [a + b for a, b in zip(lens, news)]
    page_at, at = places(kv, cu, L)
    for x, y in ((q, out[:n]), (k, kv.k_cache[page_at, :, at])):
        want, bound = turned(x[:n], pos[:, :n], axis_of, freq, interleaved)
        assert ((y.double() - want).abs() <= bound).all()
        assert torch.equal(y[..., rot:], x[:n, :, rot:])
    assert torch.equal(kv.v_cache[page_at, :, at], v[:n]) and (out[n:] == 9.0).all()
    for c, old in zip((kv.k_cache, kv.v_cache), before):       # nothing else was written
        c[page_at, :, at] = old[page_at, :, at]
        assert torch.equal(c, old)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_positions_that_are_places(dtype):
    news, lens = [5, 1, 40], [1000, 0, 77]
    runs = []
    for axes in (0, 1, 3):
        g, kv, q, k, v, cu, L = setup(dtype, 2, 4, 64, 16, news, lens, 3)
        more = {}
        if axes:
            own = torch.cat([torch.arange(a, a + n) for a, n in zip(lens, news)]).int().cuda()
            more = dict(positions=own.expand(axes, -1), axis_of=torch.arange(32, device="cuda").int() % axes)
        runs.append((kv.append(k, v, L, cu=cu, q=q, inv_freq=inv_freq(64), **more), kv.k_cache, kv.v_cache))
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


@pytest.mark.parametrize("pos", [0, -1, 8191, 1 << 24, (1 << 31) - 1, -(1 << 31)])
def test_far_positions(pos):
    g, kv, q, k, v, cu, L = setup(torch.float32, 1, 1, 64, 16, [1], [3], 5)
    freq = inv_freq(64, 500000.0)
    p = torch.tensor([[pos], [7]], dtype=torch.int32, device="cuda")
    axis = torch.arange(32, device="cuda").int() % 2
    got = kv.append(k, v, L, q=q, inv_freq=freq, positions=p, axis_of=axis)
    want, bound = turned(q, p, axis, freq, False)
    assert ((got.double() - want).abs() <= bound).all()


def test_an_axis_that_there_is_not():
    g, kv, q, k, v, cu, L = setup(torch.float32, 1, 2, 16, 16, [4], [3], 5)
    pos = torch.randint(1, 50, (2, 4), generator=g, device="cuda", dtype=torch.int32)
    axis = torch.tensor([0, 1, 2, -1, 1, 0, 5, 1], dtype=torch.int32, device="cuda")
    freq = inv_freq(16)
    got = kv.append(k, v, L, cu=cu, q=q, inv_freq=freq, positions=pos, axis_of=axis)
    assert kv.status.item() == B.RR_STATUS_BAD_INDEX
    zero = torch.cat((pos, torch.zeros_like(pos[:1])))         # pairs of no axis are not turned
    want, bound = turned(q, zero, torch.where((axis < 0) | (axis > 1), 2, axis), freq, False)
    assert ((got.double() - want).abs() <= bound).all()


def test_what_the_wrapper_refuses():
    g, kv, q, k, v, cu, L = setup(torch.float32, 1, 2, 16, 16, [4], [3], 5)
    pos, axis, freq = torch.zeros((3, 4), dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"), inv_freq(16)
    call = lambda **kw: kv.append(k, v, L, cu=cu, q=q, **{**dict(inv_freq=freq, positions=pos, axis_of=axis), **kw})
    call()
    for kw, kind in ((dict(positions=None), ValueError), (dict(axis_of=None), ValueError), (dict(inv_freq=None), ValueError), (dict(positions=pos.long()), ValueError),
                     (dict(positions=pos[:, :3]), ValueError), (dict(positions=pos[0]), ValueError), (dict(positions=pos.cpu()), ValueError),
                     (dict(axis_of=axis[:7]), ValueError), (dict(axis_of=axis.long()), TypeError), (dict(axis_of=axis.cpu()), ValueError),
                     (dict(positions=pos[:0]), ValueError)):
        with pytest.raises(kind):
            call(**kw)
    none = torch.zeros((0, 1, 16), device="cuda")              # no tokens: lengths only
    new = torch.zeros_like(L)
    kv.append(none, none, L, cu=torch.zeros_like(cu), inv_freq=freq, positions=pos[:, :0], axis_of=axis, new_lens=new)
    assert torch.equal(new, L)
