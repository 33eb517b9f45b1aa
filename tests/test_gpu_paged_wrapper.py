"""What PagedKV holds on to, and what it refuses to lose silently."""
import pytest
import torch

from paper_2609_07306_b200.paged import PagedKV

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
