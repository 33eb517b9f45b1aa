"""PagedKV: the paged key/value cache behind the routes (torch tensors) and its three operators -- appending new tokens
with the position rotation, attention of a batch that shares a prefix, attention over the routes' token ranges.  Every
operator runs in the library's kernels; PyTorch is used for device memory and streams only."""
from __future__ import annotations

import torch

from . import binding as B
from .ledger import _raw_stream

_DTYPES = {torch.bfloat16: B.RR_BF16, torch.float32: B.RR_F32}


def _ptr(t):
    return None if t is None else t.data_ptr()


def inv_freq(rot: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """base ** (-2 j / rot) for the rot / 2 pairs, computed in 64 bits."""
    j = torch.arange(0, rot, 2, dtype=torch.float64)
    return (base ** (-j / rot)).float().to(device)


class PagedKV:
    """k_cache, v_cache  [pages, kv_heads, page_tokens, dh], bf16 or fp32, alike in shape and strides; the last dimension is
    contiguous, the others may have any strides (a token-major pool [pages, page_tokens, kv_heads, dh] is passed as
    `pool.transpose(1, 2)`, one that holds keys and values side by side as two slices of it)
    page_table        [batch, pages_per_seq] int32: the page of every page_tokens tokens of a sequence
    status            optional [1] int32: RR_STATUS_* bits are OR-ed into it (RR_STATUS_BAD_INDEX: a page id outside the
                      pool, or a position behind the table's end, was met and left out)

    The object keeps the tensors, checks the descriptions of the arguments and passes addresses on; it keeps no results
    and no workspace, so calls on several streams do not meet (each call's workspace comes from torch's allocator on the
    current stream, and from a graph's pool while one is captured).  Work goes to the current stream of the cache's
    device, whichever device is the current one."""

    def __init__(self, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor,
                 status: torch.Tensor | None = None):
        if k_cache.dim() != 4 or k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype:
            raise ValueError("k_cache and v_cache must be [pages, kv_heads, page_tokens, dh] of one shape and type")
        if k_cache.dtype not in _DTYPES:
            raise TypeError(f"the cache must be bfloat16 or float32, not {k_cache.dtype}")
        if k_cache.stride() != v_cache.stride():
            raise ValueError("k_cache and v_cache must have the same strides")
        if k_cache.shape[3] > 1 and k_cache.stride(3) != 1:
            raise ValueError("the entries of a head must be contiguous")
        self.k_cache, self.v_cache, self.page_table, self.status = k_cache, v_cache, page_table, status
        self.device = k_cache.device
        self._need(page_table, "page_table", torch.int32, 2)
        if page_table.shape[1] > 1 and page_table.stride(1) != 1:
            raise ValueError("the rows of page_table must be contiguous")
        self._need(v_cache, "v_cache", k_cache.dtype, 4)
        if status is not None:
            self._need(status, "status", torch.int32, 1, (1,))
        self.batch = page_table.shape[0]
        pages, self.kv_heads, page_tokens, self.dh = k_cache.shape
        self._kv = B.rr_paged_kv(
            k=k_cache.data_ptr(), v=v_cache.data_ptr(), page_table=page_table.data_ptr(), status=_ptr(status),
            page_stride=k_cache.stride(0), head_stride=k_cache.stride(1), token_stride=k_cache.stride(2),
            table_stride=page_table.stride(0), dtype=_DTYPES[k_cache.dtype], num_pages=pages,
            page_tokens=page_tokens, kv_heads=self.kv_heads, dh=self.dh, batch=self.batch,
            pages_per_seq=page_table.shape[1])

    def _need(self, t, name, dtype, dim, shape=None):
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the cache on {self.device}")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
        if t.dim() != dim or (shape is not None and tuple(t.shape) != tuple(shape)):
            raise ValueError(f"{name} has shape {tuple(t.shape)}" + (f", expected {tuple(shape)}" if shape is not None else ""))

    def _heads(self, t, name, dim, shape=None):
        self._need(t, name, self.k_cache.dtype, dim, shape)
        if t.shape[-1] != self.dh:
            raise ValueError(f"{name} has heads of {t.shape[-1]} entries, the cache of {self.dh}")
        if self.dh > 1 and t.stride(-1) != 1:
            raise ValueError(f"the entries of a head of {name} must be contiguous")

    def _ints(self, t, name, shape):
        self._need(t, name, torch.int32, len(shape), shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")

    def _launch(self, fn, workspace_bytes, args):
        if self.device.index == torch.cuda.current_device():
            return self._launch_here(fn, workspace_bytes, args)
        with torch.cuda.device(self.device):
            return self._launch_here(fn, workspace_bytes, args)

    def _launch_here(self, fn, workspace_bytes, args):
        stream = _raw_stream(self.device)
        if workspace_bytes is None:
            fn(self._kv, args, stream)
            return
        n = workspace_bytes(self._kv, args)
        ws = torch.empty(n, dtype=torch.uint8, device=self.device) if n else None
        fn(self._kv, args, _ptr(ws), n, stream)

    def append(self, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, *, cu: torch.Tensor | None = None,
               q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
               inv_freq: torch.Tensor | None = None, interleaved: bool = False,
               new_lens: torch.Tensor | None = None) -> torch.Tensor | None:
        """Writes the new tokens' keys and values [tokens, kv_heads, dh] (any token and head strides) into the cache, keys
        rotated by their positions; returns the same tokens' queries [tokens, heads, dh], rotated, if they are given
        (in q_out, which may be q itself; else in a new tensor).
        lens      [batch] int32 tokens in the cache before the call: the position of a sequence's first new token
        cu        [batch + 1] int32: sequence b owns the tokens cu[b] .. cu[b + 1] - 1, those behind cu[batch] are padding
                  and written nowhere; None: one token per sequence
        inv_freq  [rot / 2] float32, rotates the first rot entries of a head: the pairs (j, j + rot / 2), or with
                  interleaved=True (2 j, 2 j + 1); None: nothing is rotated
        new_lens  [batch] int32: gets lens + new tokens (another tensor than lens)"""
        self._heads(k, "k", 3, (k.shape[0], self.kv_heads, self.dh))
        self._heads(v, "v", 3, k.shape)
        self._ints(lens, "lens", (self.batch,))
        if cu is not None:
            self._ints(cu, "cu", (self.batch + 1,))
        if new_lens is not None:
            self._ints(new_lens, "new_lens", (self.batch,))
        if inv_freq is not None:
            self._need(inv_freq, "inv_freq", torch.float32, 1)
            if not inv_freq.is_contiguous():
                raise ValueError("inv_freq must be contiguous")
        if q is not None:
            self._heads(q, "q", 3, (k.shape[0], q.shape[1], self.dh))
            if q_out is None:
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            else:
                self._heads(q_out, "q_out", 3, q.shape)
        elif q_out is not None:
            raise ValueError("q_out without q")
        if k.shape[0] == 0:
            k = v = self.k_cache                                       # (an empty tensor has no address)
            args = B.rr_append_args()
            q_in = None
        else:
            q_in = q
            args = B.rr_append_args(k_token_stride=k.stride(0), k_head_stride=k.stride(1),
                                    v_token_stride=v.stride(0), v_head_stride=v.stride(1), tokens=k.shape[0])
        args.k, args.v, args.lens = k.data_ptr(), v.data_ptr(), lens.data_ptr()
        args.cu, args.new_lens = _ptr(cu), _ptr(new_lens)
        if inv_freq is not None:
            args.inv_freq, args.rot = inv_freq.data_ptr(), 2 * inv_freq.shape[0]
        args.interleaved = 1 if interleaved else 0
        if q_in is not None:
            args.q, args.q_out, args.q_heads = q.data_ptr(), q_out.data_ptr(), q.shape[1]
            args.q_token_stride, args.q_head_stride = q.stride(0), q.stride(1)
            args.out_token_stride, args.out_head_stride = q_out.stride(0), q_out.stride(1)
        self._launch(B.rr_kv_append, None, args)
        return q_out

    def attend_shared(self, q: torch.Tensor, lens: torch.Tensor, prefix_tokens: int, scale: float, *,
                      cu: torch.Tensor | None = None, causal: bool = True,
                      prefix_pages: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of the queries [tokens, heads, dh] to their sequences' tokens in the cache, the first prefix_tokens
        of which are the same for all sequences and read once for all (from prefix_pages, or else sequence 0's table).
        lens    [batch] int32 tokens in the cache, the queries' own among them
        cu      as in append; rows of out behind cu[batch] are left as they were
        causal  the queries are their sequence's last tokens, and none sees a token behind its own; False: every query
                sees all lens[b] tokens (attention to states of another length, e.g. an encoder's)
        A query without tokens gets zeros."""
        self._heads(q, "q", 3)
        self._ints(lens, "lens", (self.batch,))
        if cu is not None:
            self._ints(cu, "cu", (self.batch + 1,))
        if prefix_pages is not None:
            page = self.k_cache.shape[2]
            self._ints(prefix_pages, "prefix_pages", prefix_pages.shape[:1])
            if prefix_pages.shape[0] * page < prefix_tokens:
                raise ValueError(f"prefix_pages holds {prefix_pages.shape[0]} pages, {prefix_tokens} tokens need more")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            self._heads(out, "out", 3, q.shape)
        if q.shape[0] == 0 and (cu is not None or self.batch == 0):
            return out
        args = B.rr_shared_args(
            q=q.data_ptr(), out=out.data_ptr(), lens=lens.data_ptr(), cu=_ptr(cu), prefix_pages=_ptr(prefix_pages),
            q_token_stride=q.stride(0), q_head_stride=q.stride(1), out_token_stride=out.stride(0),
            out_head_stride=out.stride(1), tokens=q.shape[0], heads=q.shape[1], prefix_tokens=prefix_tokens,
            causal=1 if causal else 0, scale=scale)
        self._launch(B.rr_attend_shared, B.rr_attend_shared_workspace, args)
        return out

    def attend_ranges(self, q: torch.Tensor, ranges: torch.Tensor, lens: torch.Tensor, n_q: int, scale: float, *,
                      causal: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of the queries [batch, heads, n_q * m, dh] over the routes' token ranges, read through the page table.
        ranges  [batch * route_heads * n_q, slots, 2] int32, as RouteLedger.token_ranges: row (b, r, i) holds the ranges of
                the heads / route_heads query heads of route head r and of the m query tokens of chunk i
        lens    [batch] int32 tokens in the cache: range tokens from there on are left out
        causal  the query tokens are the sequence's last n_q * m, and none sees a token behind its own
        A query without tokens gets zeros."""
        self._heads(q, "q", 4)
        self._ints(lens, "lens", (self.batch,))
        self._need(ranges, "ranges", torch.int32, 3)
        if not ranges.is_contiguous() or ranges.shape[2] != 2:
            raise ValueError("ranges must be contiguous [rows, slots, 2]")
        if q.shape[0] != self.batch or n_q < 1 or q.shape[2] % n_q != 0:
            raise ValueError(f"q has shape {tuple(q.shape)}, expected [{self.batch}, heads, {n_q} * m, {self.dh}]")
        if ranges.shape[0] == 0 or ranges.shape[0] % (self.batch * n_q) != 0:
            raise ValueError(f"ranges has {ranges.shape[0]} rows, not a multiple of batch * n_q = {self.batch * n_q}")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            self._heads(out, "out", 4, q.shape)
        args = B.rr_ranges_args(
            q=q.data_ptr(), out=out.data_ptr(), ranges=ranges.data_ptr(), lens=lens.data_ptr(),
            q_batch_stride=q.stride(0), q_head_stride=q.stride(1), q_token_stride=q.stride(2),
            out_batch_stride=out.stride(0), out_head_stride=out.stride(1), out_token_stride=out.stride(2),
            heads=q.shape[1], route_heads=ranges.shape[0] // (self.batch * n_q), n_q=n_q, m=q.shape[2] // n_q,
            slots=ranges.shape[1], causal=1 if causal else 0, scale=scale)
        self._launch(B.rr_attend_paged_ranges, B.rr_attend_paged_ranges_workspace, args)
        return out
