"""What the operators that go by a pool's room refuse, on the host.  No GPU."""
import ctypes as C

import pytest

import __graft_entry__ as entry
from paper_2609_07306_b200 import binding as B
from test_serving_refusals import BIG, append, axes, calls, kv, pool, verify

INVALID = B.RR_ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def test_alignment():
    lib = B.lib()
    assert calls(pool(room=0x70002), [kv()], 1) == (INVALID,) * 3
    assert lib.rr_kv_append(C.byref(kv()), C.byref(append(room=0x70001)), None) == INVALID
    assert lib.rr_kv_append_axes(C.byref(kv()), C.byref(append(room=0x70001)), C.byref(axes()), None) == INVALID
    assert lib.rr_verify_drafts(C.byref(verify(room=0xA0002)), None) == INVALID


def test_room_needs_the_lengths():
    assert B.lib().rr_verify_drafts(C.byref(verify(room=0xA0000, lens=None, new_lens=None)), None) == INVALID


def test_the_workspace_does_not_grow_with_it():
    assert B.rr_pages_workspace(pool(room=0x70000)) == B.rr_pages_workspace(pool())
    assert calls(pool(room=0x70000), [kv()], 1, nbytes=B.rr_pages_workspace(pool()) - 1, lens=0x1000) == (B.RR_ERR_TOO_SMALL,) * 3 and BIG > 0
