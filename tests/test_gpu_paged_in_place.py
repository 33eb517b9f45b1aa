"""Outputs into the queries' own memory: the same outputs as into other memory, also where a row has to be computed again."""
import pytest
import torch

from paper_2609_07306_b200.paged import PagedKV

pytestmark = pytest.mark.gpu
KINDS = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 80), (torch.float32, 64)]


def bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


def cache(dtype, KH, dh, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((120, KH, 16, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    v.view(-1)[torch.randint(0, v.numel(), (40,), generator=g, device="cuda")] = float("nan")
    v.view(-1)[torch.randint(0, v.numel(), (40,), generator=g, device="cuda")] = float("-inf")
    return g, k, v, torch.arange(120, dtype=torch.int32, device="cuda").view(2, 60)


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("heads,prefix,lens,news", [(2, 0, [900, 700], [1, 1]), (16, 0, [900, 700], [1, 1]), (8, 300, [900, 700], [3, 40]),
                                                    (8, 0, [900, 700], [200, 129]), (600, 0, [30, 20], [1, 1])])
def test_shared(dtype, dh, heads, prefix, lens, news):
    g, k, v, table = cache(dtype, 2, dh, heads)
    table[1, :prefix // 16] = table[0, :prefix // 16].clone()
    kv = PagedKV(k, v, table)
    cu = torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device="cuda")
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    wide = torch.randn((sum(news), heads, dh + 16), generator=g, device="cuda").to(dtype)
    before, q = wide.clone(), wide[..., 8:dh + 8]
    want = kv.attend_shared(q, L, prefix, 0.1, cu=cu)
    got = kv.attend_shared(q, L, prefix, 0.1, cu=cu, out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(bits(got), bits(want))
    assert torch.equal(wide[..., :8], before[..., :8]) and torch.equal(wide[..., dh + 8:], before[..., dh + 8:])
    assert lens[0] < 100 or not want.isfinite().all()


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("n_q,m,G", [(12, 1, 1), (12, 16, 5), (12, 40, 8), (2400, 36, 4), (3000, 3, 1), (5000, 3, 1)])
def test_ranges(dtype, dh, n_q, m, G):
    g, k, v, table = cache(dtype, 1, dh, m)
    kv = PagedKV(k, v, table)
    L = torch.tensor([900, 850], dtype=torch.int32, device="cuda")
    lo = torch.randint(0, 700, (2 * n_q, 2, 1), generator=g, device="cuda").sort(1).values
    rg = torch.cat((lo, lo + torch.tensor([[50], [190]], device="cuda")), 2).int()
    q = torch.randn((2, G, n_q * m, dh), generator=g, device="cuda").to(dtype)
    want = kv.attend_ranges(q, rg, L, n_q, 0.1, causal=True)
    assert want[0, :, n_q * m - 1].isfinite().any()
    got = kv.attend_ranges(q, rg, L, n_q, 0.1, causal=True, out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(bits(got), bits(want))


def test_other_strides_are_refused():
    g, k, v, table = cache(torch.bfloat16, 2, 64, 1)
    kv = PagedKV(k, v, table)
    L = torch.tensor([90, 70], dtype=torch.int32, device="cuda")
    hold = torch.zeros(4096, device="cuda", dtype=torch.bfloat16)
    q, out = hold[:1024].view(2, 8, 64), hold.as_strided((2, 8, 64), (1024, 64, 1))
    with pytest.raises(RuntimeError):
        kv.attend_shared(q, L, 0, 0.1, out=out)
    rg = torch.zeros((4, 1, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError):
        kv.attend_ranges(q.unsqueeze(2), rg, L, 1, 0.1, out=out.unsqueeze(2))
