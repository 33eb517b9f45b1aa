"""Appends of more tokens than there are 32 for each SM, which CTAs of half as many threads take, and of one token fewer; against the rotation in 64 bits, all widths
and types, with places and with several axes as positions."""
import pytest
import torch

from paged_oracle import BF, U
from paper_2609_07306_b200.paged import PagedKV, inv_freq

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def turned(x, angle, interleaved):
    """x [tokens, heads, dh] in 64 bits, and how far FP32 may be off: the angle is rounded to 2^-26 of a turn, sine and cosine are off by at most 2 steps, the two
    products and their sum by one rounding each; bf16 rounds the result once."""
    rot, y = 2 * angle.shape[1], x.double()
    a, i = angle[:, None], torch.arange(angle.shape[1], device="cuda")
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    out, bound = y.clone(), torch.zeros_like(y)
    out[..., p] = y[..., p] * a.cos() - y[..., q] * a.sin()
    out[..., q] = y[..., q] * a.cos() + y[..., p] * a.sin()
    each = (y[..., p].abs() + y[..., q].abs()) * (6.2832 * 2.0 ** -26 + 6 * U)
    bound[..., p], bound[..., q] = each, each
    if x.dtype == torch.bfloat16:
        bound = bound + (out.abs() + bound) * BF
    return out, bound


@pytest.mark.parametrize("dtype,dh,rot,interleaved,pad", [
    (torch.bfloat16, 128, 128, False, 0), (torch.bfloat16, 64, 32, True, 8), (torch.bfloat16, 40, 20, False, 1), (torch.float32, 256, 256, False, 0),
    (torch.float32, 64, 64, True, 4), (torch.float32, 7, 6, False, 0), (torch.float32, 16, 0, False, 0)])
@pytest.mark.parametrize("axes", [0, 3])
@pytest.mark.parametrize("more", [0, 1, 700])
def test_many_tokens(dtype, dh, rot, interleaved, pad, axes, more):
    if axes and not rot:
        axes = 0
    T = 32 * torch.cuda.get_device_properties(0).multi_processor_count + more
    news = [1, T // 2, 0, T - T // 2 - 4, 0, 1]            # two tokens of padding behind them
    lens, page, KH, H = [3, 0, 7, 40, 9, 15], 16, 2, 3
    width = max((a + n + page - 1) // page for a, n in zip(lens, news)) + 1
    g = torch.Generator(device="cuda").manual_seed(T + dh)
    pages = 6 * width
    kc, vc = (torch.zeros((pages, KH, page, dh), device="cuda", dtype=dtype) for _ in range(2))
    table = torch.randperm(pages, generator=g, device="cuda").view(6, width).int()
    kv = PagedKV(kc, vc, table, ints([0]))
    q, k, v = (torch.randn((T, n, dh + pad), generator=g, device="cuda").to(dtype)[..., :dh] for n in (H, KH, KH))
    cu, L, after = ints([0] + news).cumsum(0).int(), ints(lens), ints([0] * 6)
    n = sum(news)
    b = torch.repeat_interleave(torch.arange(6, device="cuda"), torch.tensor(news, device="cuda"))
    place = torch.arange(n, device="cuda") - cu[b] + L[b]
    freq, args = inv_freq(rot) if rot else None, {}
    if axes:
        pos = torch.randint(-9, 5000, (axes, T), generator=g, device="cuda", dtype=torch.int32)
        axis = torch.arange(rot // 2, device="cuda").int() % axes
        args = dict(positions=pos, axis_of=axis)
        at = pos[axis.long(), :n].T
    else:
        at = place[:, None].expand(-1, max(rot // 2, 0))
    out = torch.full((T, H, dh), 9.0, device="cuda", dtype=dtype)
    kv.append(k, v, L, cu=cu, q=q, q_out=out, inv_freq=freq, interleaved=interleaved, new_lens=after, **args)
    assert kv.status.item() == 0 and after.tolist() == [x + y for x, y in zip(lens, news)] and (out[n:] == 9.0).all()
    page_at, in_page = table[b, place // page].long(), place % page
    for x, y in ((q, out[:n]), (k, kc[page_at, :, in_page])):
        if rot:
            want, bound = turned(x[:n], at.double() * freq.double(), interleaved)
            assert ((y.double() - want).abs() <= bound).all()
        else:
            assert torch.equal(x[:n], y)
    assert torch.equal(vc[page_at, :, in_page], v[:n])
    kc[page_at, :, in_page] = 0
    vc[page_at, :, in_page] = 0
    assert not kc.any() and not vc.any()                   # nothing else was written
