"""What the paged cache's operators refuse, on the host: every check returns before anything is enqueued.  No GPU."""
import ctypes as C
import os
import re

import pytest

import __graft_entry__ as entry
from paper_2609_07306_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


def shared(**kw):
    d = dict(q=0x10000, out=0x20000, lens=0x30000, cu=0x40000, q_token_stride=256, q_head_stride=64, out_token_stride=256,
             out_head_stride=64, tokens=5, heads=4, prefix_tokens=100, causal=1, scale=0.125)
    return B.rr_shared_args(**{**d, **kw})


def ranges(**kw):
    d = dict(q=0x10000, out=0x20000, ranges=0x30000, lens=0x40000, q_batch_stride=1024, q_head_stride=256, q_token_stride=64,
             out_batch_stride=1024, out_head_stride=256, out_token_stride=64, heads=4, route_heads=2, n_q=2, m=2, slots=3, causal=1,
             scale=0.125)
    return B.rr_ranges_args(**{**d, **kw})


@pytest.mark.parametrize("name", ["rr_paged_kv", "rr_append_args", "rr_shared_args", "rr_ranges_args"])
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
    for packed, st in ((paged._APPEND, B.rr_append_args), (paged._SHARED, B.rr_shared_args), (paged._RANGES, B.rr_ranges_args)):
        assert packed.size == C.sizeof(st)
        n = len(st._fields_)
        vals = [i + 1 for i in range(n)]
        x = st.from_buffer_copy(packed.pack(*vals))
        assert [getattr(x, f) for f, _ in st._fields_] == vals


CACHE = [(dict(k=None), B.RR_ERR_INVALID_ARG), (dict(v=None), B.RR_ERR_INVALID_ARG), (dict(page_table=None), B.RR_ERR_INVALID_ARG),
         (dict(num_pages=0), B.RR_ERR_INVALID_ARG), (dict(page_tokens=0), B.RR_ERR_INVALID_ARG), (dict(kv_heads=0), B.RR_ERR_INVALID_ARG),
         (dict(batch=0), B.RR_ERR_INVALID_ARG), (dict(pages_per_seq=0), B.RR_ERR_INVALID_ARG), (dict(page_stride=-1), B.RR_ERR_INVALID_ARG),
         (dict(head_stride=-1), B.RR_ERR_INVALID_ARG), (dict(token_stride=-1), B.RR_ERR_INVALID_ARG), (dict(table_stride=-1), B.RR_ERR_INVALID_ARG),
         (dict(dtype=2), B.RR_ERR_UNSUPPORTED), (dict(dh=0), B.RR_ERR_UNSUPPORTED), (dict(dh=257), B.RR_ERR_UNSUPPORTED),
         (dict(k=0x10001), B.RR_ERR_INVALID_ARG), (dict(page_table=0x30002), B.RR_ERR_INVALID_ARG), (dict(status=0x30002), B.RR_ERR_INVALID_ARG)]


@pytest.mark.parametrize("kw,code", CACHE)
def test_cache_description(kw, code):
    lib, n = B.lib(), C.c_size_t()
    c = kv(**kw)
    assert lib.rr_kv_append(C.byref(c), C.byref(append()), None) == code
    assert lib.rr_attend_shared_workspace(C.byref(c), C.byref(shared()), C.byref(n)) == code
    assert lib.rr_attend_shared(C.byref(c), C.byref(shared()), 0x100, 1 << 40, None) == code
    assert lib.rr_attend_paged_ranges_workspace(C.byref(c), C.byref(ranges()), C.byref(n)) == code
    assert lib.rr_attend_paged_ranges(C.byref(c), C.byref(ranges()), 0x100, 1 << 40, None) == code


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(lens=None), dict(tokens=-1), dict(cu=None), dict(q=0x70000),
                                dict(q=0x70000, q_out=0x80000), dict(rot=-2), dict(rot=66), dict(rot=3), dict(inv_freq=None),
                                dict(interleaved=2), dict(new_lens=0x30000), dict(k_token_stride=-1), dict(v_head_stride=-1),
                                dict(k=0x10001), dict(cu=0x40002), dict(new_lens=0x90001)])
def test_append(kw):
    assert B.lib().rr_kv_append(C.byref(kv()), C.byref(append(**kw)), None) == B.RR_ERR_INVALID_ARG


def test_null_descriptions():
    lib, n = B.lib(), C.c_size_t()
    assert lib.rr_kv_append(None, C.byref(append()), None) == B.RR_ERR_INVALID_ARG
    assert lib.rr_kv_append(C.byref(kv()), None, None) == B.RR_ERR_INVALID_ARG
    assert lib.rr_attend_shared(C.byref(kv()), None, None, 0, None) == B.RR_ERR_INVALID_ARG
    assert lib.rr_attend_paged_ranges(C.byref(kv()), None, None, 0, None) == B.RR_ERR_INVALID_ARG
    assert lib.rr_attend_shared_workspace(C.byref(kv()), C.byref(shared()), None) == B.RR_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), B.RR_ERR_INVALID_ARG), (dict(out=None), B.RR_ERR_INVALID_ARG), (dict(lens=None), B.RR_ERR_INVALID_ARG),
    (dict(tokens=-1), B.RR_ERR_INVALID_ARG), (dict(cu=None), B.RR_ERR_INVALID_ARG), (dict(heads=0), B.RR_ERR_INVALID_ARG),
    (dict(heads=3), B.RR_ERR_INVALID_ARG), (dict(prefix_tokens=-1), B.RR_ERR_INVALID_ARG), (dict(prefix_tokens=129), B.RR_ERR_INVALID_ARG),
    (dict(causal=2), B.RR_ERR_INVALID_ARG), (dict(scale=float("nan")), B.RR_ERR_INVALID_ARG), (dict(scale=float("inf")), B.RR_ERR_INVALID_ARG),
    (dict(q_token_stride=-1), B.RR_ERR_INVALID_ARG), (dict(q=0x10001), B.RR_ERR_INVALID_ARG), (dict(lens=0x30001), B.RR_ERR_INVALID_ARG),
    (dict(tokens=1 << 29), B.RR_ERR_TOO_LARGE)])
def test_shared(kw, code):
    assert B.lib().rr_attend_shared(C.byref(kv()), C.byref(shared(**kw)), 0x100, 1 << 40, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), B.RR_ERR_INVALID_ARG), (dict(out=None), B.RR_ERR_INVALID_ARG), (dict(lens=None), B.RR_ERR_INVALID_ARG),
    (dict(ranges=None), B.RR_ERR_INVALID_ARG), (dict(heads=5), B.RR_ERR_INVALID_ARG), (dict(route_heads=3), B.RR_ERR_INVALID_ARG),
    (dict(route_heads=0), B.RR_ERR_INVALID_ARG), (dict(n_q=0), B.RR_ERR_INVALID_ARG), (dict(m=0), B.RR_ERR_INVALID_ARG),
    (dict(slots=0), B.RR_ERR_INVALID_ARG), (dict(slots=B.RR_MAX_RANGE_SLOTS + 1), B.RR_ERR_TOO_LARGE), (dict(causal=-1), B.RR_ERR_INVALID_ARG),
    (dict(scale=float("nan")), B.RR_ERR_INVALID_ARG), (dict(out_head_stride=-4), B.RR_ERR_INVALID_ARG),
    (dict(n_q=1 << 20, m=1 << 20), B.RR_ERR_TOO_LARGE), (dict(n_q=1 << 28), B.RR_ERR_TOO_LARGE)])
def test_ranges(kw, code):
    assert B.lib().rr_attend_paged_ranges(C.byref(kv()), C.byref(ranges(**kw)), 0x100, 1 << 40, None) == code


def test_sizes_that_pass_32_bits():
    big = kv(page_tokens=1 << 20, pages_per_seq=1 << 12)
    assert B.lib().rr_attend_shared(C.byref(big), C.byref(shared()), 0x100, 1 << 40, None) == B.RR_ERR_TOO_LARGE
    wide = kv(page_tokens=1 << 10, pages_per_seq=1 << 12)
    assert B.lib().rr_attend_paged_ranges(C.byref(wide), C.byref(ranges(slots=1024)), 0x100, 1 << 40, None) == B.RR_ERR_TOO_LARGE


def test_workspaces():
    n = B.rr_attend_shared_workspace(kv(), shared())
    assert n > 0
    lib = B.lib()
    assert lib.rr_attend_shared(C.byref(kv()), C.byref(shared()), None, n, None) == B.RR_ERR_INVALID_ARG
    assert lib.rr_attend_shared(C.byref(kv()), C.byref(shared()), 0x100, n - 1, None) == B.RR_ERR_TOO_SMALL
    assert lib.rr_attend_shared(C.byref(kv()), C.byref(shared()), 0x180, n, None) == B.RR_ERR_INVALID_ARG
    n = B.rr_attend_paged_ranges_workspace(kv(), ranges())
    assert lib.rr_attend_paged_ranges(C.byref(kv()), C.byref(ranges()), 0x100, n - 1, None) == B.RR_ERR_TOO_SMALL
    assert B.rr_attend_shared_workspace(kv(), shared(tokens=0)) >= 0
    # a call without tokens has nothing to do
    assert lib.rr_attend_shared(C.byref(kv()), C.byref(shared(tokens=0)), None, 0, None) == B.RR_OK


def test_outputs_over_the_queries():
    """The same memory with the same strides, or none in common."""
    lib = B.lib()
    ws = lambda **kw: B.rr_attend_shared_workspace(kv(), shared(**kw))
    assert ws(out=0x10000) > 0
    assert ws(out=0x10000, tokens=3, heads=2, out_token_stride=256) > 0
    for kw in (dict(out_token_stride=512), dict(out_head_stride=128)):
        assert lib.rr_attend_shared(C.byref(kv()), C.byref(shared(out=0x10000, **kw)), 0x100, 1 << 40, None) == B.RR_ERR_INVALID_ARG
    assert B.rr_attend_paged_ranges_workspace(kv(), ranges(out=0x10000)) > 0
    for kw in (dict(out_batch_stride=2048), dict(out_head_stride=512), dict(out_token_stride=128)):
        assert lib.rr_attend_paged_ranges(C.byref(kv()), C.byref(ranges(out=0x10000, **kw)), 0x100, 1 << 40, None) == B.RR_ERR_INVALID_ARG


def serving(tokens, batch, heads, prefix, dh=128, dtype=B.RR_BF16):
    c = kv(kv_heads=8, dh=dh, batch=batch, pages_per_seq=8192, page_tokens=64, page_stride=1 << 16, head_stride=64 * dh, token_stride=dh, dtype=dtype)
    return B.rr_attend_shared_workspace(c, shared(q_token_stride=heads * dh, q_head_stride=dh, out_token_stride=heads * dh, out_head_stride=dh,
                                                  tokens=tokens, heads=heads, prefix_tokens=prefix))


def test_workspaces_go_by_what_is_joined():
    """A token of one sequence: some megabytes.  Long prompts: what the SMs cut, whatever the length; less than the outputs.  Rows behind a
    shared prefix: one partial of the prefix and, in tiles of up to 128 rows, two of their own, of FP32."""
    assert serving(1, 1, 32, 0) < 10 << 20 and serving(1, 1, 64, 4096) < 10 << 20
    for n in (4096, 32768, 131072):
        assert serving(n, 1, 32, 0) < 100 << 20 and serving(n, 4, 32, 8192) < 120 << 20
    assert serving(131072, 1, 32, 8192) < 131072 * 32 * 128 * 2
    for n, b in ((3000, 8), (4096, 256), (16384, 2048)):
        assert serving(n, b, 32, 8192) < 3 * n * 32 * (128 * 4 + 8) + (100 << 20)
    for dtype in (B.RR_BF16, B.RR_F32):
        sizes = [serving(n, 2, 32, 0, dtype=dtype) for n in (2, 8, 64, 512, 4096, 32768, 262144)]
        assert sizes == sorted(sizes)
    c = kv(kv_heads=8, dh=128, batch=2, page_stride=1 << 20, head_stride=8192, token_stride=128, page_tokens=64, pages_per_seq=128)
    whole = ranges(heads=32, route_heads=8, n_q=128, m=64, slots=32, q_token_stride=128, q_head_stride=1 << 20, q_batch_stride=1 << 25,
                   out_token_stride=128, out_head_stride=1 << 20, out_batch_stride=1 << 25)
    assert B.rr_attend_paged_ranges_workspace(c, whole) == 2 * 32 * 8192           # a byte a row
