"""Pages of a paged cache, shared between sequences and copied on write.

``PageTable`` is the bookkeeping: which pages a sequence's slots lie in and how
many sequences hold each page.  It owns no device memory; the operations that
need page contents moved return the (source, destination) pairs.  ``PagePool``
adds the device pool of every layer, the device page table, and the copies
(``gs_pages_copy``), and hands out the ``gs_cache`` descriptors that
``gs_rope_append`` and ``gs_decode_attention`` take.

A forked sequence shares every page of the one it came from.  ``prepare`` must
be called before slots are written: it maps their pages and gives a sequence
pages of its own where they were shared, so no write reaches another sequence.
"""
from __future__ import annotations

from typing import Dict, Iterable, List, Sequence, Tuple

import numpy as np

from . import gs

PAGE_TOKENS = 64
Pairs = List[Tuple[int, int]]


class PageTable:
    """Rows of page numbers with reference counts (host only)."""

    def __init__(self, n_pages: int, max_seqs: int, max_ctx: int):
        if n_pages < 1 or max_seqs < 1 or max_ctx < 1:
            raise ValueError("n_pages, max_seqs and max_ctx must be positive")
        self.max_ctx = max_ctx
        self.rows = np.zeros((max_seqs, -(-max_ctx // PAGE_TOKENS)), dtype=np.int32)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self._pages: Dict[int, List[int]] = {}            # open sequence -> its pages
        self._free = list(range(n_pages - 1, -1, -1))
        self._closed = list(range(max_seqs - 1, -1, -1))

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def pages(self, seq: int) -> List[int]:
        return list(self._of(seq))

    def _of(self, seq: int) -> List[int]:
        if seq not in self._pages:
            raise ValueError(f"sequence {seq} is not open")
        return self._pages[seq]

    def open(self) -> int:
        """A new, empty sequence: its row of the table."""
        if not self._closed:
            raise gs.GsError(gs.GS_ERR_OOM, "every sequence row is in use")
        seq = self._closed.pop()
        self._pages[seq] = []
        return seq

    def fork(self, seq: int, count: int = 1) -> List[int]:
        """Sequences that share every page of ``seq``."""
        pages = self._of(seq)
        if count < 0 or count > len(self._closed):
            raise gs.GsError(gs.GS_ERR_OOM, "too few free sequence rows")
        new = []
        for _ in range(count):
            s = self.open()
            self._pages[s] = list(pages)
            self.rows[s, : len(pages)] = pages
            new.append(s)
        for p in pages:
            self.refs[p] += count
        return new

    def prepare(self, spans: Iterable[Tuple[int, int, int]]) -> Pairs:
        """Make slots [first, first + count) of each (seq, first, count) writable.

        Maps missing pages and replaces shared ones that the span touches;
        returns the pages to copy.  Nothing changes if the pool is too small.  Of
        several spans of one sequence, a later one may start where an earlier one
        ends.
        """
        spans = list(spans)
        held: Dict[int, int] = {}                         # pages by then
        for seq, first, count in spans:
            have = held.get(seq, len(self._of(seq)))
            if count < 1 or first < 0 or first + count > self.max_ctx:
                raise gs.GsError(gs.GS_ERR_INVALID_ARG, "slots out of range")
            if first > have * PAGE_TOKENS:
                raise gs.GsError(gs.GS_ERR_INVALID_ARG, "slots start beyond the sequence's pages")
            held[seq] = max(have, -(-(first + count) // PAGE_TOKENS))
        if self._need(spans) > len(self._free):
            raise gs.GsError(gs.GS_ERR_OOM, "page pool exhausted")
        pairs: Pairs = []
        for seq, first, count in spans:
            pages = self._pages[seq]
            for at in range(first // PAGE_TOKENS, -(-(first + count) // PAGE_TOKENS)):
                if at < len(pages) and self.refs[pages[at]] == 1:
                    continue
                new = self._free.pop()
                self.refs[new] = 1
                if at < len(pages):
                    self.refs[pages[at]] -= 1
                    pairs.append((pages[at], new))
                    pages[at] = new
                else:
                    pages.append(new)
                self.rows[seq, at] = new
        return pairs

    def _need(self, spans: Sequence[Tuple[int, int, int]]) -> int:
        """Pages that prepare(spans) takes from the pool."""
        refs: Dict[int, int] = {}
        touched = set()
        need = 0
        for seq, first, count in spans:
            pages = self._pages[seq]
            for at in range(first // PAGE_TOKENS, -(-(first + count) // PAGE_TOKENS)):
                if (seq, at) in touched:
                    continue
                touched.add((seq, at))
                if at >= len(pages):
                    need += 1
                    continue
                left = refs.get(pages[at], int(self.refs[pages[at]]))
                if left > 1:                              # the last holder keeps it
                    refs[pages[at]] = left - 1
                    need += 1
        return need

    def truncate(self, seq: int, length: int) -> None:
        """Give back the pages beyond the first ``length`` slots."""
        pages = self._of(seq)
        keep = -(-length // PAGE_TOKENS)
        if length < 0 or keep > len(pages):
            raise gs.GsError(gs.GS_ERR_INVALID_ARG, "length out of range")
        for p in pages[keep:]:
            self._drop(p)
        del pages[keep:]

    def close(self, seq: int) -> None:
        """Free a sequence: its row, and the pages that it alone held."""
        for p in self._of(seq):
            self._drop(p)
        del self._pages[seq]
        self._closed.append(seq)

    def _drop(self, page: int) -> None:
        self.refs[page] -= 1
        if self.refs[page] == 0:
            self._free.append(page)

    def compact(self) -> Pairs:
        """Move the used pages to the lowest numbers, so that the pool's end is
        free; returns the pages to copy.  No page is both source and destination."""
        used = int((self.refs > 0).sum())
        holes = [p for p in range(used) if self.refs[p] == 0]
        moved = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        pairs = list(zip(moved, holes))
        new = dict(pairs)
        for src, dst in pairs:
            self.refs[dst], self.refs[src] = self.refs[src], 0
        for seq, pages in self._pages.items():
            pages[:] = [new.get(p, p) for p in pages]
            self.rows[seq, : len(pages)] = pages
        self._free = list(range(len(self.refs) - 1, used - 1, -1))
        return pairs


class PagePool:
    """A PageTable with its pages: [n_layers][n_pages][2][n_kv_heads][64 * head_dim].

    All device work is enqueued on ``stream`` (default: the current stream at
    construction), on which the pages' readers and writers run too.
    """

    def __init__(self, *, n_layers: int, n_pages: int, n_kv_heads: int, head_dim: int, dtype,
                 max_seqs: int, max_ctx: int, device: str = "cuda:0", stream=None):
        import torch
        self._torch = torch
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError("dtype must be torch.float16 or torch.bfloat16")
        self.table = PageTable(n_pages, max_seqs, max_ctx)
        self.n_kv_heads, self.head_dim, self.dtype = n_kv_heads, head_dim, dtype
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        with torch.cuda.stream(self.stream):
            self.kv = torch.zeros(n_layers, n_pages, 2, n_kv_heads, PAGE_TOKENS * head_dim,
                                  dtype=dtype, device=self.device)
            self.rows = torch.zeros(self.table.rows.shape, dtype=torch.int32, device=self.device)
            self.err = torch.zeros(1, dtype=torch.int32, device=self.device)
        code = gs.GS_F16 if dtype == torch.float16 else gs.GS_BF16
        self._caches = [gs.gs_cache(self.kv[i].data_ptr(), n_pages, n_kv_heads, head_dim, code,
                                    self.rows.data_ptr(), max_seqs, self.rows.shape[1])
                        for i in range(n_layers)]

    def layer(self, i: int) -> gs.gs_cache:
        """The descriptor of layer ``i`` (valid for the pool's lifetime)."""
        return self._caches[i]

    def open(self) -> int:
        return self.table.open()

    def fork(self, seq: int, count: int = 1) -> List[int]:
        new = self.table.fork(seq, count)
        self._upload()
        return new

    def prepare(self, spans: Iterable[Tuple[int, int, int]]) -> None:
        """Make slots writable (see PageTable.prepare); copies shared pages."""
        before = self.table.rows.copy()
        self._copy(self.table.prepare(spans))
        if not np.array_equal(before, self.table.rows):
            self._upload()

    def truncate(self, seq: int, length: int) -> None:
        self.table.truncate(seq, length)

    def close(self, seq: int) -> None:
        self.table.close(seq)

    def compact(self) -> int:
        """Close the pool's gaps; returns the number of pages in use, which are
        then pages 0 .. that number - 1."""
        self._copy(self.table.compact())
        self._upload()
        return int((self.table.refs > 0).sum())

    def check(self) -> None:
        """Synchronise and raise if a kernel met an index out of range."""
        self.stream.synchronize()
        with self._torch.cuda.stream(self.stream):     # in order with the kernels that raise it
            word = int(self.err.item())
            if word:
                self.err.zero_()
        if word:
            raise gs.GsError(gs.GS_ERR_DEVICE_CHECK, "a kernel's bounds check fired")

    def _upload(self) -> None:
        with self._torch.cuda.stream(self.stream):
            self.rows.copy_(self._torch.from_numpy(self.table.rows))

    def _copy(self, pairs: Pairs) -> None:
        if not pairs:
            return
        layers, n_pages = self.kv.shape[:2]
        page_bytes = self.kv[0, 0].numel() * self.kv.element_size()
        with self._torch.cuda.stream(self.stream):     # (and its device)
            ids = self._torch.tensor(pairs, dtype=self._torch.int32).t().contiguous().to(self.device)
            gs.gs_pages_copy(self.kv.data_ptr(), n_pages, self.kv.data_ptr(), n_pages, layers,
                             page_bytes, ids[0].data_ptr(), ids[1].data_ptr(), len(pairs),
                             self.err.data_ptr(), self.stream.cuda_stream)
