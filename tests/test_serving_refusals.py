"""What appending with axes, the page pool and the verification refuse, on the host: every check returns before anything is enqueued.  No GPU."""
import ctypes as C
import os
import re

import pytest

import __graft_entry__ as entry
from paper_2609_07306_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, TOO_LARGE, TOO_SMALL = B.RR_ERR_INVALID_ARG, B.RR_ERR_UNSUPPORTED, B.RR_ERR_TOO_LARGE, B.RR_ERR_TOO_SMALL


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def kv(**kw):
    d = dict(k=0x10000, v=0x20000, page_table=0x30000, page_stride=4096, head_stride=1024, token_stride=64, table_stride=8,
             dtype=B.RR_BF16, num_pages=10, page_tokens=16, kv_heads=2, dh=64, batch=3, pages_per_seq=8)
    return B.rr_paged_kv(**{**d, **kw})


def append(**kw):
    d = dict(k=0x10000, v=0x20000, lens=0x30000, cu=0x40000, inv_freq=0x50000, k_token_stride=128, k_head_stride=64,
             v_token_stride=128, v_head_stride=64, tokens=5, rot=64)
    return B.rr_append_args(**{**d, **kw})


def axes(**kw):
    return B.rr_axes_args(**{**dict(positions=0x60000, axis_of=0x70000, axis_stride=5, token_stride=1, axes=3), **kw})


def pool(**kw):
    d = dict(page_table=0x30000, refs=0x40000, held=0x50000, free_pages=0x60000, table_stride=8, num_pages=10, page_tokens=16, batch=3, pages_per_seq=8)
    return B.rr_page_pool(**{**d, **kw})


def verify(**kw):
    d = dict(target=0x10000, draft=0x20000, tokens=0x30000, cu=0x40000, uniform=0x50000, lens=0x60000, out=0x70000, accepted=0x80000,
             new_lens=0x90000, target_stride=100, draft_stride=100, dtype=B.RR_F32, rows=9, batch=3, vocab=100)
    return B.rr_verify_args(**{**d, **kw})


@pytest.mark.parametrize("name", ["rr_axes_args", "rr_page_pool", "rr_verify_args"])
def test_structs_match_the_header(name):
    hdr = open(os.path.join(ROOT, "include", "routerelay.h")).read()
    body = re.sub(r"/\*.*?\*/", "", hdr[hdr.index(f"typedef struct {name} {{"):hdr.index(f"}} {name};")], flags=re.S)
    size = {"int32_t": 4, "int64_t": 8, "float": 4}
    want = []
    for decl in body.split("{", 1)[1].split(";"):
        words = decl.replace(",", " ").replace("const ", "").split()
        if words:
            kind = 8 if "*" in decl else size[words[0]]
            want += [(w.replace("*", ""), kind) for w in words[1:] if w != "*"]
    assert want == [(n, C.sizeof(t)) for n, t in getattr(B, name)._fields_]


def test_packed_arguments_match_the_structs():
    from paper_2609_07306_b200 import paged
    from paper_2609_07306_b200 import verify as V
    for packed, st in ((paged._AXES, B.rr_axes_args), (V._VERIFY, B.rr_verify_args)):
        assert packed.size == C.sizeof(st)
        vals = [i + 1 for i in range(len(st._fields_))]
        x = st.from_buffer_copy(packed.pack(*vals))
        assert [getattr(x, f) for f, _ in st._fields_] == vals


@pytest.mark.parametrize("a,x", [({}, dict(positions=None)), ({}, dict(axes=0)), ({}, dict(axis_stride=-1)), ({}, dict(token_stride=-1)),
                                 ({}, dict(positions=0x60002)), ({}, dict(axis_of=0x70001)), (dict(rot=0), {}), (dict(k=None), {}),
                                 (dict(rot=3), {}), (dict(new_lens=0x30000), {}), (dict(q=0x70000), {})])
def test_axes(a, x):
    assert B.lib().rr_kv_append_axes(C.byref(kv()), C.byref(append(**a)), C.byref(axes(**x)), None) == INVALID


def test_axes_null():
    lib = B.lib()
    assert lib.rr_kv_append_axes(C.byref(kv()), C.byref(append()), None, None) == INVALID
    assert lib.rr_kv_append_axes(None, C.byref(append()), C.byref(axes()), None) == INVALID
    assert lib.rr_kv_append_axes(C.byref(kv(dtype=7)), C.byref(append()), C.byref(axes()), None) == UNSUPPORTED
    assert lib.rr_kv_append_axes(C.byref(kv()), C.byref(append(tokens=0)), C.byref(axes()), None) == B.RR_OK


BIG = 1 << 40
POOL = [(dict(page_table=None), INVALID), (dict(refs=None), INVALID), (dict(held=None), INVALID), (dict(free_pages=None), INVALID),
        (dict(num_pages=0), INVALID), (dict(page_tokens=0), INVALID), (dict(batch=0), INVALID), (dict(pages_per_seq=0), INVALID),
        (dict(table_stride=7), INVALID), (dict(table_stride=-1, batch=1), INVALID), (dict(refs=0x40002), INVALID), (dict(status=0x40001), INVALID),
        (dict(num_pages=B.RR_PAGES_MAX_PAGES + 1), TOO_LARGE), (dict(batch=B.RR_PAGES_MAX_BATCH + 1, pages_per_seq=1), TOO_LARGE), (dict(batch=1 << 20, pages_per_seq=1 << 12, table_stride=1 << 12), TOO_LARGE)]


def calls(p, caches, n, ws=0x100, nbytes=BIG, lens=0x1000, arg=0x2000, out=0x3000, each=0, ids=None):
    lib, p = B.lib(), C.byref(p)
    c = (B.rr_paged_kv * max(1, len(caches)))(*caches)
    return (lib.rr_pages_fork(p, arg, lens, out, ws, nbytes, None), lib.rr_pages_reserve(p, lens, arg, each, c, n, ws, nbytes, None),
            lib.rr_pages_compact(p, c, n, ids, ws, nbytes, None))


@pytest.mark.parametrize("kw,code", POOL)
def test_pool(kw, code):
    n = C.c_size_t()
    assert B.lib().rr_pages_workspace(C.byref(pool(**kw)), C.byref(n)) == code
    assert calls(pool(**kw), [kv()], 1) == (code, code, code)


def test_workspace():
    n = B.rr_pages_workspace(pool())
    assert n > 0 and B.lib().rr_pages_workspace(C.byref(pool()), None) == INVALID and B.lib().rr_pages_workspace(None, None) == INVALID
    assert calls(pool(), [kv()], 1, nbytes=n - 1) == (TOO_SMALL,) * 3
    assert calls(pool(), [kv()], 1, ws=None) == (INVALID,) * 3
    assert calls(pool(), [kv()], 1, ws=0x108) == (INVALID,) * 3
    sizes = [B.rr_pages_workspace(pool(num_pages=p, batch=b, pages_per_seq=w, table_stride=w)) for p, b, w in ((10, 3, 8), (1000, 3, 8), (1000, 200, 64))]
    # a number for every entry and page, two for every row, three for every move; each list rounded up to 16 bytes, and 64 bytes in front
    assert sizes == sorted(sizes) and sizes[0] < sizes[2] <= 64 + 4 * (200 * 64 + 2 * 200 + 1000 + 3 * 501 + 4 * 3)


def test_fork():
    lib, p = B.lib(), C.byref(pool())
    for parents, lens, out in ((None, 0x1000, 0x3000), (0x2000, None, 0x3000), (0x2000, 0x1000, None), (0x2000, 0x1000, 0x1000), (0x2000, 0x1000, 0x2000),
                               (0x2001, 0x1000, 0x3000), (0x2000, 0x1002, 0x3000), (0x2000, 0x1000, 0x3003)):
        assert lib.rr_pages_fork(p, parents, lens, out, 0x100, BIG, None) == INVALID


def test_reserve_and_compact():
    for caches, n, code in (([], 0, INVALID), ([kv()], -1, INVALID), ([kv(num_pages=11)], 1, INVALID), ([kv(page_tokens=8)], 1, INVALID),
                            ([kv(), kv(dh=300)], 2, UNSUPPORTED), ([kv(), kv(k=None)], 2, INVALID), ([kv(dtype=3)], 1, UNSUPPORTED)):
        assert calls(pool(), caches, n)[1:] == (code, code)
    huge = dict(page_tokens=1 << 20)
    assert calls(pool(**huge), [kv(**huge, kv_heads=64)], 1)[1:] == (TOO_LARGE, TOO_LARGE)
    lib, c = B.lib(), (B.rr_paged_kv * 1)(kv())
    for lens, new, each in ((None, 0x2000, 0), (0x1002, 0x2000, 0), (0x1000, 0x2001, 0), (0x1000, None, -1)):
        assert lib.rr_pages_reserve(C.byref(pool()), lens, new, each, c, 1, 0x100, BIG, None) == INVALID
    assert lib.rr_pages_reserve(C.byref(pool()), 0x1000, None, 0, None, 1, 0x100, BIG, None) == INVALID
    assert calls(pool(), [kv()], 1, ids=0x5001)[2] == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(target=None), INVALID), (dict(tokens=None), INVALID), (dict(out=None), INVALID), (dict(out=0x30000), INVALID), (dict(accepted=None), INVALID), (dict(lens=None), INVALID),
    (dict(uniform=None), INVALID), (dict(cu=None), INVALID), (dict(rows=-1), INVALID), (dict(batch=0), INVALID), (dict(vocab=0), INVALID),
    (dict(target_stride=-1), INVALID), (dict(draft_stride=-5), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(vocab=(1 << 30) + 1), TOO_LARGE),
    (dict(batch=(1 << 27) + 1), TOO_LARGE), (dict(target=0x10002), INVALID), (dict(draft=0x20001), INVALID), (dict(tokens=0x30001), INVALID),
    (dict(uniform=0x50002), INVALID), (dict(status=0x50002), INVALID), (dict(dtype=B.RR_BF16, target=0x10001), INVALID)])
def test_verify(kw, code):
    assert B.lib().rr_verify_drafts(C.byref(verify(**kw)), None) == code


def test_verify_null():
    assert B.lib().rr_verify_drafts(None, None) == INVALID
