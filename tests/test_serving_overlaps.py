"""Results on memory that the same call still reads are refused on the host, before anything is enqueued, also where only some entries coincide.  No GPU."""
import ctypes as C

import pytest

import __graft_entry__ as entry
from paper_2609_07306_b200 import binding as B
from test_serving_refusals import append, kv, pool, verify

INVALID = B.RR_ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


@pytest.mark.parametrize("what", ["lens", "parents", "held", "refs", "free", "table"])
@pytest.mark.parametrize("shift", [-8, -4, 4, 8])
def test_fork(what, shift):
    """Three rows: 12 bytes."""
    at = dict(parents=0x2000, lens=0x1000, held=0x50000, refs=0x40000, free=0x60000, table=0x30000)[what]
    if what in ("free",) and shift > 0:
        return                                             # (behind the one number)
    ws = 0x100
    assert B.lib().rr_pages_fork(C.byref(pool()), 0x2000, 0x1000, at + shift, ws, 1 << 40, None) == INVALID


@pytest.mark.parametrize("what", ["tokens", "cu", "uniform", "lens", "target", "draft"])
@pytest.mark.parametrize("result", ["out", "accepted", "new_lens"])
@pytest.mark.parametrize("shift", [-8, 0, 8])
def test_verify(what, result, shift):
    if what == "lens" and result != "out" and shift == 0:
        return                                             # in the lengths' place
    at = dict(target=0x10000, draft=0x20000, tokens=0x30000, cu=0x40000, uniform=0x50000, lens=0x60000)[what]
    assert B.lib().rr_verify_drafts(C.byref(verify(**{result: at + shift})), None) == INVALID


@pytest.mark.parametrize("a,b", [("out", "accepted"), ("out", "new_lens"), ("accepted", "new_lens")])
@pytest.mark.parametrize("shift", [-8, 0, 8])
def test_results_of_verify(a, b, shift):
    assert B.lib().rr_verify_drafts(C.byref(verify(**{a: 0x70000, b: 0x70000 + shift})), None) == INVALID


@pytest.mark.parametrize("what", ["lens", "cu"])
@pytest.mark.parametrize("shift", [-8, -4, 4, 8])
def test_append(what, shift):
    at = dict(lens=0x30000, cu=0x40000)[what]
    assert B.lib().rr_kv_append(C.byref(kv()), C.byref(append(new_lens=at + shift)), None) == INVALID
