"""PagePool: who owns which page of the paged caches of a model's layers -- forks, room for new tokens, freeing, compaction.  The
bookkeeping and the copies of pages run in the library's kernels; PyTorch is used for device memory and streams only."""
from __future__ import annotations

import ctypes as C
from operator import index

import torch

from . import binding as B
from .paged import PagedKV


class PagePool:
    """page_table  [batch, pages_per_seq] int32: the first held[b] entries of row b are sequence b's pages, the others -1
    page_tokens tokens of a page
    refs        [pages] int32: how many entries of the table hold a page (and how many holders the caller counts besides); 0: free
    held        [batch] int32
    free        [1] int32: how many pages are free; None: counted from refs.  It is kept by differences (compact counts anew): whoever frees or takes a
                page by writing to refs changes it, too
    caches      the layers' caches (PagedKV), all of this pool's number and size of pages, and of this table or one that is kept like it
    status      optional [1] int32: RR_STATUS_* bits are OR-ed into it (RR_STATUS_BAD_INDEX: a page id outside the pool, a negative length or one
                behind the table's end; RR_STATUS_NO_PAGES: fewer free pages than a call of reserve needed, which then gave none)

    room        [batch] int32, made by the pool: up to which place each sequence may be written to, 2^31 - 1 unless the last call of reserve could not give it all of its pages.
                The caches' append goes by the room of the pool that was made over them last (calls that are captured later, not those in an older graph)

    PagePool.empty makes the state of a pool whose pages are all free.  The object keeps the tensors (they are written to, not exchanged) and one
    workspace.  Its calls change the state: order them, and the operators that read the table, on one stream or by events;
    graphs that hold them may not run at the same time.  Keep the object until its work on streams other than the one that it was made on has
    ended.  Work goes to the current stream of the table's device, whichever device is the current one."""

    def __init__(self, page_table: torch.Tensor, page_tokens: int, refs: torch.Tensor, held: torch.Tensor,
                 free: torch.Tensor | None = None, caches: "list[PagedKV] | tuple[PagedKV, ...]" = (), status: torch.Tensor | None = None):
        self.device = page_table.device
        if self.device.type != "cuda":
            raise ValueError("the page table must be on a CUDA device (there is no CPU path)")
        if page_table.dim() != 2 or refs.dim() != 1:
            raise ValueError("page_table must be [batch, pages_per_seq] and refs [pages]")
        self._index, self.batch, self.page_tokens, self.num_pages = self.device.index, page_table.shape[0], page_tokens, refs.shape[0]
        self._ints(page_table, "page_table", tuple(page_table.shape), rows_apart=True)
        self._ints(refs, "refs", (self.num_pages,))
        self._ints(held, "held", (self.batch,))
        if status is not None:
            self._ints(status, "status", (1,))
        if free is None:
            free = (refs == 0).sum(dtype=torch.int32).view(1)
        self._ints(free, "free", (1,))
        caches = tuple(caches)
        for i, kv in enumerate(caches):
            if kv.device != self.device:
                raise ValueError(f"cache {i} is on {kv.device}, the page table on {self.device}")
            if kv.page_tokens != page_tokens or kv.k_cache.shape[0] != self.num_pages:
                raise ValueError(f"cache {i} has {kv.k_cache.shape[0]} pages of {kv.page_tokens} tokens, the pool {self.num_pages} of {page_tokens}")
        # (a cache of a table that is kept like this one may have more rows, which no call closes)
        room = torch.full((max([self.batch] + [kv.batch for kv in caches]),), 0x7FFFFFFF, dtype=torch.int32, device=self.device)
        self._tensors = (page_table, refs, held, free, status, caches, room[:self.batch])
        self._pool = B.rr_page_pool(
            page_table=page_table.data_ptr(), refs=refs.data_ptr(), held=held.data_ptr(), free_pages=free.data_ptr(),
            status=None if status is None else status.data_ptr(), room=room.data_ptr(), table_stride=page_table.stride(0), num_pages=self.num_pages,
            page_tokens=page_tokens, batch=self.batch, pages_per_seq=page_table.shape[1])
        self._caches = (B.rr_paged_kv * max(1, len(caches)))(*[kv._kv for kv in caches])
        self._lib = B.lib()
        self._bytes = B.rr_pages_workspace(self._pool)
        self._ws = torch.empty(self._bytes, dtype=torch.uint8, device=self.device)
        self._at, self._caches_at, self._layers, self._ws_at = C.addressof(self._pool), C.addressof(self._caches), len(caches), self._ws.data_ptr()
        for kv in caches:
            kv._room, kv._p_room = room, room.data_ptr()

    @classmethod
    def empty(cls, caches: "list[PagedKV] | tuple[PagedKV, ...]", status: torch.Tensor | None = None) -> "PagePool":
        """The pool of these layers' caches with every page free: the (common) table is filled with -1."""
        caches = tuple(caches)
        if not caches:
            raise ValueError("a pool needs a cache")
        table, pages = caches[0].page_table, caches[0].k_cache.shape[0]
        if any(kv.page_table.data_ptr() != table.data_ptr() or kv.page_table.shape != table.shape for kv in caches):
            raise ValueError("the caches must have one page table")
        zeros = [torch.zeros(n, dtype=torch.int32, device=table.device) for n in (pages, table.shape[0])]
        pool = cls(table, caches[0].page_tokens, *zeros, torch.full((1,), pages, dtype=torch.int32, device=table.device), caches, status)
        table.fill_(-1)                                # (caches that do not go together have been refused by now)
        return pool

    page_table = property(lambda self: self._tensors[0])
    refs = property(lambda self: self._tensors[1])
    held = property(lambda self: self._tensors[2])
    free = property(lambda self: self._tensors[3])
    status = property(lambda self: self._tensors[4])
    caches = property(lambda self: self._tensors[5])
    room = property(lambda self: self._tensors[6])

    _ints = PagedKV._ints

    def _stream(self):
        """The current stream of the pool's device; None where another device is the current one."""
        return torch._C._cuda_getCurrentRawStream(self._index) if self._index == torch._C._cuda_getDevice() else None

    def _done(self, rc, name):
        if rc != B.RR_OK:
            raise B.RouteRelayError(rc, name)

    def fork(self, parents: torch.Tensor, lens: torch.Tensor, new_lens: torch.Tensor) -> None:
        """Row b becomes what row parents[b] was, all rows at once; parents[b] == b: it stays, -1: its sequence has ended and the
        row is emptied.  A child holds the pages of its parent's tokens together with it; nothing is copied before one of them is written to (reserve).
        parents   [batch] int32
        lens      [batch] int32 tokens of the sequences
        new_lens  [batch] int32: gets lens[parents[b]] (at most what the table holds), 0 for rows that were emptied (memory that neither lens, parents nor the pool has any of)"""
        shape = (self.batch,)
        self._ints(parents, "parents", shape)
        self._ints(lens, "lens", shape)
        self._ints(new_lens, "new_lens", shape)
        stream = self._stream()
        if stream is None:
            with torch.cuda.device(self.device):
                return self.fork(parents, lens, new_lens)
        self._done(self._lib.rr_pages_fork(self._at, parents.data_ptr(), lens.data_ptr(), new_lens.data_ptr(), self._ws_at, self._bytes, stream), "rr_pages_fork")

    def reserve(self, lens: torch.Tensor, new: "torch.Tensor | int" = 0) -> None:
        """Sequence b keeps its first lens[b] tokens and may be appended to by new (or new[b]) tokens: pages behind that are released,
        missing ones given (the lowest free ones first, in the order of the sequences), and a page that will be written and that others hold
        too becomes the sequence's own, its tokens copied in all caches.  reserve(lens) with lens[b] = 0 frees a sequence.
        lens  [batch] int32
        new   an int, or [batch] int32
        If the pool has fewer free pages than the call needs, none is given (RR_STATUS_NO_PAGES) and rows are only shortened; with new / page_tokens + 2 free
        pages per sequence there are always enough.  A sequence that lacks pages, or whose page is another's, too, is closed until a call succeeds: the caches' append
        writes none of its tokens and leaves its length (room; give it to verify_drafts as well), so that a captured step that is not looked at in between harms
        no other sequence.  What else writes to the caches has to go by the status or by room."""
        shape = (self.batch,)
        self._ints(lens, "lens", shape)
        if isinstance(new, torch.Tensor):
            self._ints(new, "new", shape)
            tokens, each = new.data_ptr(), 0
        else:
            tokens, each = None, index(new)                # (a number that is not whole is refused, not cut)
            if not 0 <= each <= 0x7FFFFFFF:
                raise ValueError(f"new must be between 0 and 2^31 - 1, not {new}")
        if not self._layers:
            raise ValueError("reserve copies pages: the pool needs its caches")
        stream = self._stream()
        if stream is None:
            with torch.cuda.device(self.device):
                return self.reserve(lens, new)
        self._done(self._lib.rr_pages_reserve(self._at, lens.data_ptr(), tokens, each, self._caches_at, self._layers, self._ws_at, self._bytes, stream),
                   "rr_pages_reserve")

    def compact(self, new_ids: torch.Tensor | None = None) -> None:
        """The pages in use become the first ones of the pool, in the table, in refs and in all caches: of L pages in use, the i-th of those
        numbered L or higher moves to the i-th free page below L.
        new_ids  [pages] int32: gets where each page is now, for ids kept outside the table (a prefix's pages, for instance)"""
        if new_ids is not None:
            self._ints(new_ids, "new_ids", (self.num_pages,))
        if not self._layers:
            raise ValueError("compact copies pages: the pool needs its caches")
        stream = self._stream()
        if stream is None:
            with torch.cuda.device(self.device):
                return self.compact(new_ids)
        self._done(self._lib.rr_pages_compact(self._at, self._caches_at, self._layers, None if new_ids is None else new_ids.data_ptr(), self._ws_at, self._bytes,
                                              stream), "rr_pages_compact")
