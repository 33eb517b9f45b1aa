"""What PagedKV holds on to, and what it refuses to lose silently."""
import pytest
import torch

from paper_2609_07306_b200.paged import PagedKV, inv_freq

pytestmark = pytest.mark.gpu


def make():
    k, v = (torch.randn((8, 2, 16, 64), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    return k, v, torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)


def test_tensors_are_not_exchanged():
    k, v, table = make()
    kv = PagedKV(k, v, table)
    for name in ("k_cache", "v_cache", "page_table", "status"):
        with pytest.raises(AttributeError):
            setattr(kv, name, getattr(kv, name))
    assert kv.k_cache is k and kv.v_cache is v and kv.page_table is table and kv.status is None
    q, L = torch.randn((2, 2, 64), device="cuda", dtype=torch.bfloat16), torch.tensor([64, 64], dtype=torch.int32, device="cuda")
    a = kv.attend_shared(q, L, 0, 0.1)
    kv.page_table.copy_(kv.page_table.flip(0))         # what is written into them counts
    assert torch.equal(kv.attend_shared(q, L, 0, 0.1), PagedKV(k, v, table.clone()).attend_shared(q, L, 0, 0.1))
    assert not torch.equal(kv.attend_shared(q, L, 0, 0.1), a)


def test_gradients_are_refused():
    k, v, table = make()
    kv = PagedKV(k, v, table)
    q, L = torch.randn((2, 2, 64), device="cuda", dtype=torch.bfloat16), torch.tensor([3, 4], dtype=torch.int32, device="cuda")
    rg = torch.tensor([[[0, 3]]] * 4, dtype=torch.int32, device="cuda")
    w = q.clone().requires_grad_()
    for call in (lambda: kv.attend_shared(w, L, 0, 0.1), lambda: kv.attend_shared(w * 2, L, 0, 0.1), lambda: kv.attend_shared(q, L, 0, 0.1, out=w),
                 lambda: kv.attend_ranges(w.unsqueeze(2), rg, L, 1, 0.1), lambda: kv.append(w, q, L), lambda: kv.append(q, w, L),
                 lambda: kv.append(q, q, L, q=w), lambda: PagedKV(k.clone().requires_grad_(), v, table)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    with torch.no_grad():
        assert torch.equal(kv.attend_shared(w, L, 0, 0.1), kv.attend_shared(q, L, 0, 0.1))
        kv.append(w, w, L, q=w, inv_freq=inv_freq(64))
    with torch.inference_mode():
        assert torch.equal(kv.attend_shared(w, L, 0, 0.1), kv.attend_shared(q, L, 0, 0.1))
