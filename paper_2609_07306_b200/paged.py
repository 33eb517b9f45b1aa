"""PagedKV: the paged key/value cache behind the routes (torch tensors) and its three operators -- appending new tokens
with the position rotation, attention of a batch that shares a prefix, attention over the routes' token ranges.  Every
operator runs in the library's kernels; PyTorch is used for device memory and streams only."""
from __future__ import annotations

import ctypes as C
import struct

import torch

from . import binding as B

# rr_append_args, rr_shared_args and rr_ranges_args as bytes (a call's arguments in one step; 64-bit alignment throughout)
_APPEND = struct.Struct("@8P8q4i")
_SHARED = struct.Struct("@5P4q4if4x")
_RANGES = struct.Struct("@4P6q6if4x")

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

    Forward only: no operator has a gradient, and a tensor that requires one is refused (but under torch.no_grad()).
    The object keeps the tensors (they are written to, not exchanged: another table is another PagedKV), checks the descriptions of the arguments and passes addresses on; it keeps no results
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
        if k_cache.requires_grad or v_cache.requires_grad:
            raise ValueError("the cache must not require a gradient (its operators have none)")
        self._tensors = (k_cache, v_cache, page_table, status)
        self.device = k_cache.device
        if self.device.type != "cuda":
            raise ValueError("the cache must be on a CUDA device (there is no CPU path)")
        self._index, self._dtype = self.device.index, k_cache.dtype
        self.batch = page_table.shape[0]
        pages, self.kv_heads, self.page_tokens, self.dh = k_cache.shape
        if v_cache.device != self.device:
            raise ValueError(f"v_cache is on {v_cache.device}, the cache on {self.device}")
        if page_table.dim() != 2:
            raise ValueError("page_table must be [batch, pages_per_seq]")
        self._ints(page_table, "page_table", tuple(page_table.shape), rows_apart=True)
        if status is not None:
            self._ints(status, "status", (1,))
        self._kv = B.rr_paged_kv(
            k=k_cache.data_ptr(), v=v_cache.data_ptr(), page_table=page_table.data_ptr(), status=_ptr(status),
            page_stride=k_cache.stride(0), head_stride=k_cache.stride(1), token_stride=k_cache.stride(2),
            table_stride=page_table.stride(0), dtype=_DTYPES[k_cache.dtype], num_pages=pages,
            page_tokens=self.page_tokens, kv_heads=self.kv_heads, dh=self.dh, batch=self.batch,
            pages_per_seq=page_table.shape[1])
        self._at = C.addressof(self._kv)
        self._lib = B.lib()

    # what the description points to: the tensors are written to, not exchanged
    k_cache = property(lambda self: self._tensors[0])
    v_cache = property(lambda self: self._tensors[1])
    page_table = property(lambda self: self._tensors[2])
    status = property(lambda self: self._tensors[3])

    # -- checks: one comparison each for what is right, the reason where it is not ----------------------------
    def _heads(self, t, name, shape):
        """t has the cache's type and device, the given shape (its last entry dh), contiguous heads; its strides."""
        strides = t.stride()
        if t.dtype is self._dtype and t.get_device() == self._index and t.shape == shape and strides[-1] == 1 and not t.requires_grad:
            return strides
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which the cache's operators do not have: call them under torch.no_grad()")
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the cache on {self.device}")
        if t.dtype is not self._dtype:
            raise TypeError(f"{name} must be {self._dtype}, not {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if self.dh > 1 and t.numel() > 0 and strides[-1] != 1:
            raise ValueError(f"the entries of a head of {name} must be contiguous")
        return strides

    def _ints(self, t, name, shape, rows_apart=False):
        if t.dtype is torch.int32 and t.get_device() == self._index and t.shape == shape and t.is_contiguous():
            return
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the cache on {self.device}")
        if t.dtype is not torch.int32:
            raise TypeError(f"{name} must be torch.int32, not {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if not (rows_apart and (t.shape[1] <= 1 or t.stride(1) == 1)):
            raise ValueError(f"{name} must be contiguous")

    def _run(self, name, args, workspace=None):
        """One library call on the current stream of the cache's device."""
        if self._index != torch._C._cuda_getDevice():
            with torch.cuda.device(self.device):
                return self._run(name, args, workspace)
        stream = torch._C._cuda_getCurrentRawStream(self._index)
        if workspace is None:
            rc = getattr(self._lib, name)(self._at, args, stream)
        else:
            n = C.c_size_t()
            rc = getattr(self._lib, workspace)(self._at, args, C.byref(n))
            if rc == B.RR_OK:
                n = n.value
                ws = torch.empty(n, dtype=torch.uint8, device=self.device) if n else None
                rc = getattr(self._lib, name)(self._at, args, _ptr(ws), n, stream)
        if rc != B.RR_OK:
            raise B.RouteRelayError(rc, name)

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
        if k.dim() != 3:
            raise ValueError("k must be [tokens, kv_heads, dh]")
        n = k.shape[0]
        shape = (n, self.kv_heads, self.dh)
        ks = self._heads(k, "k", shape)
        vs = self._heads(v, "v", shape)
        self._ints(lens, "lens", (self.batch,))
        if cu is not None:
            self._ints(cu, "cu", (self.batch + 1,))
        if new_lens is not None:
            self._ints(new_lens, "new_lens", (self.batch,))
        rot = 0
        if inv_freq is not None:
            if inv_freq.dtype is not torch.float32 or inv_freq.get_device() != self._index or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
                raise ValueError(f"inv_freq must be contiguous float32 [rot / 2] on {self.device}")
            rot = 2 * inv_freq.shape[0]
        heads, q_strides = 0, (0, 0, 0, 0)
        if q is not None:
            if q.dim() != 3:
                raise ValueError("q must be [tokens, heads, dh]")
            shape = (n, q.shape[1], self.dh)
            qs = self._heads(q, "q", shape)
            if q_out is None:
                q_out = q.new_empty(shape)
                os = (shape[1] * self.dh, self.dh)
            else:
                os = self._heads(q_out, "q_out", shape)
            heads, q_strides = shape[1], (qs[0], qs[1], os[0], os[1])
        elif q_out is not None:
            raise ValueError("q_out without q")
        if n == 0:                                     # (an empty tensor has no address)
            if cu is None:
                raise ValueError(f"no tokens for {self.batch} sequences")
            k, v, heads = self.k_cache, self.v_cache, 0
        self._run("rr_kv_append", _APPEND.pack(
            k.data_ptr(), v.data_ptr(), q.data_ptr() if heads else 0, q_out.data_ptr() if heads else 0, lens.data_ptr(),
            0 if cu is None else cu.data_ptr(), 0 if new_lens is None else new_lens.data_ptr(),
            0 if rot == 0 else inv_freq.data_ptr(), ks[0], ks[1], vs[0], vs[1], *q_strides, n, heads, rot,
            1 if interleaved else 0))
        return q_out

    def attend_shared(self, q: torch.Tensor, lens: torch.Tensor, prefix_tokens: int, scale: float, *,
                      cu: torch.Tensor | None = None, causal: bool = True,
                      prefix_pages: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of the queries [tokens, heads, dh] to their sequences' tokens in the cache, the first prefix_tokens
        of which are the same for all sequences and read once for all (from prefix_pages [pages] int32, or else from the table's row of
        the first sequence that has as many tokens).
        lens    [batch] int32 tokens in the cache, the queries' own among them
        cu      as in append; rows of out behind cu[batch] are left as they were
        causal  the queries are their sequence's last tokens, and none sees a token behind its own; False: every query
                sees all lens[b] tokens (attention to states of another length, e.g. an encoder's)
        out     as q; may be q itself
        A query without tokens gets zeros."""
        if q.dim() != 3:
            raise ValueError("q must be [tokens, heads, dh]")
        shape = (q.shape[0], q.shape[1], self.dh)
        qs = self._heads(q, "q", shape)
        self._ints(lens, "lens", (self.batch,))
        if cu is not None:
            self._ints(cu, "cu", (self.batch + 1,))
        if prefix_pages is not None:
            self._ints(prefix_pages, "prefix_pages", tuple(prefix_pages.shape[:1]))
            if prefix_pages.shape[0] * self.page_tokens < prefix_tokens:
                raise ValueError(f"prefix_pages holds {prefix_pages.shape[0]} pages, {prefix_tokens} tokens need more")
        if out is None:
            out = q.new_empty(shape)
            os = (shape[1] * self.dh, self.dh)
        else:
            os = self._heads(out, "out", shape)
        if shape[0] == 0 and cu is not None:
            return out
        self._run("rr_attend_shared", _SHARED.pack(
            q.data_ptr(), out.data_ptr(), lens.data_ptr(), 0 if cu is None else cu.data_ptr(),
            0 if prefix_pages is None else prefix_pages.data_ptr(), qs[0], qs[1], os[0], os[1],
            shape[0], shape[1], prefix_tokens, 1 if causal else 0, scale), "rr_attend_shared_workspace")
        return out

    def attend_ranges(self, q: torch.Tensor, ranges: torch.Tensor, lens: torch.Tensor, n_q: int, scale: float, *,
                      causal: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
        """Attention of the queries [batch, heads, n_q * m, dh] over the routes' token ranges, read through the page table.
        ranges  [batch * route_heads * n_q, slots, 2] int32, as RouteLedger.token_ranges: row (b, r, i) holds the ranges of
                the heads / route_heads query heads of route head r and of the m query tokens of chunk i
        lens    [batch] int32 tokens in the cache: range tokens from there on are left out
        causal  the query tokens are the sequence's last n_q * m, and none sees a token behind its own
        out     as q; may be q itself
        A query without tokens gets zeros."""
        if q.dim() != 4:
            raise ValueError("q must be [batch, heads, n_q * m, dh]")
        shape = (self.batch, q.shape[1], q.shape[2], self.dh)
        qs = self._heads(q, "q", shape)
        self._ints(lens, "lens", (self.batch,))
        if ranges.dim() != 3:
            raise ValueError("ranges must be [rows, slots, 2]")
        rows, slots = ranges.shape[0], ranges.shape[1]
        self._ints(ranges, "ranges", (rows, slots, 2))
        if n_q < 1 or shape[2] % n_q != 0 or rows == 0 or rows % (self.batch * n_q) != 0:
            raise ValueError(f"{rows} range rows and {shape[2]} query tokens do not make {n_q} chunks of {self.batch} sequences")
        if out is None:
            out = q.new_empty(shape)
            os = (shape[1] * shape[2] * self.dh, shape[2] * self.dh, self.dh)
        else:
            os = self._heads(out, "out", shape)
        self._run("rr_attend_paged_ranges", _RANGES.pack(
            q.data_ptr(), out.data_ptr(), ranges.data_ptr(), lens.data_ptr(), *qs[:3], *os[:3],
            shape[1], rows // (self.batch * n_q), n_q, shape[2] // n_q, slots, 1 if causal else 0,
            scale), "rr_attend_paged_ranges_workspace")
        return out
